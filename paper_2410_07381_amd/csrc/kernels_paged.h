// A paged cache of keys and values in 8 bits for gfx950: appending to it, and single-token attention over it.
//
// A block is a page's tokens of one K/V head.  Its numbers are e4m3 codes times one power of two: a block that grows
// past its range has its codes shifted to the next exponent, which rounds none of them but those under the smallest
// normal, and a product with the scale is exact wherever it is taken.
//
// Pages consist of units of 16 tokens.  K's lie token by token, V's dim by dim with the 16 tokens of a dim side by side: a
// lane's 8 or 16 bytes are then a fragment of the products' first operand as they come from memory (K's rows
// are tokens, V's rows are dims), and nothing goes through LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/tally.h"
#include "kernels_onepass.h"
#include "kernels_prefix.h"
#include "kernels_rope.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

constexpr uint32_t kUnit = 16;                             // tokens side by side in V's pages

// ---- appending ---------------------------------------------------------------------------
// K/V heads of a logical block: four waves with a unit of a head each.
__host__ __device__ inline uint32_t append_heads(uint32_t page) { return page >= 64 ? 1 : 64 / page; }
inline uint64_t append_blocks(const tally_kv_append_args &a) {
  const uint32_t h = append_heads(a.page);
  return (uint64_t)((a.kv_heads + h - 1) / h) * ((uint64_t)a.total / a.page + 2ull * a.n_seqs);
}

#ifdef __HIP_DEVICE_COMPILE__
// Exponent of a block by the largest of its magnitudes' bits in fp32: the smallest e from 1 on with
// m <= 448 x 2^(e - 127).  448 is 1.75 x 2^8, so a mantissa over 1.75 carries into the exponent.
__device__ __forceinline__ int block_exp(uint32_t top) {
  const int e = (int)((top + 0x1FFFFFu) >> 23) - 8;
  return e < 1 ? 1 : e > 254 ? 254 : e;
}
__device__ __forceinline__ uint32_t magnitude_bits(float x) {   // (none of what is no number)
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
// fp64 to fp32 such that rounding the result to fewer than 20 bits is rounding the number itself: cut after 20
// bits, the last of them set where anything was cut off.
__device__ __forceinline__ float cut(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = (uint32_t)(b >> 32) | ((uint32_t)b != 0u ? 1u : 0u);
  return (float)__builtin_bit_cast(double, (uint64_t)hi << 32);
}
// Four numbers times 2^by to codes.  (fma with 0: infinities become NaN, numbers stay.)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, int by) {
  auto f = [&](float x) { return __builtin_ldexpf(__builtin_fmaf(x, 0.f, x), by); };
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(f(a), f(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f(c), f(d), w, true);
}
__device__ __forceinline__ uint32_t shift_codes(uint32_t w, int by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes4(lo[0], lo[1], hi[0], hi[1], by);
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int by = 32; by; by >>= 1) {
    const uint32_t w = (uint32_t)__shfl_xor((int)v, by);
    v = v > w ? v : w;
  }
  return v;
}
#endif

template <int DIM>
struct AppendBodyT {
  using Args = tally_kv_append_args;
  static constexpr int THREADS = kThreads;
  static constexpr int MIN_WAVES = 2;
  static constexpr unsigned DYN_LDS = 0;
  static constexpr bool END_BARRIER = true;                // (the waves' largest magnitudes)
  static constexpr bool YIELDS = false;
  static constexpr bool RANGE = false;
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) { append<false>(a, bx); }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) { append<true>(a, bx); }

  template <bool NT>
  static __device__ __forceinline__ void append(const Args &a, uint32_t block) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef uint32_t u32x2_nt __attribute__((ext_vector_type(2)));
    constexpr uint32_t PIECES = DIM / 16, ROUNDS = 16 * PIECES / 64;   // pieces of 16 numbers of a token; rounds of a unit
    constexpr uint32_t SIDE = DIM / 2;                       // lanes of V side by side, two dims each
    constexpr int VT = DIM / 8;                              // tokens of such a lane
    constexpr int MORE = 2;                                  // units of a wave, at most
    __shared__ uint32_t s_top[2][4];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t P = a.page, heads = append_heads(P), groups = (a.kv_heads + heads - 1) / heads;
    const uint32_t slot = block / groups, per_head = P >= 64 ? 4u : P / kUnit, units = P / kUnit;
    const uint32_t head = block % groups * heads + wave / per_head, unit0 = wave % per_head;
    // the sequence of this slot: the last one that starts at or before it, 63 candidates at a time; the lane behind
    // the last candidate has where that one ends
    uint32_t seq = 0, first, last;
    for (uint32_t n = a.n_seqs;;) {
      const uint32_t step = (n + 62) / 63, s = lane * step < n ? lane * step : n;
      const int32_t v = a.cu_seqlens[seq + s];
      const uint32_t edge = v < 0 ? 0u : (uint32_t)v < a.total ? (uint32_t)v : a.total;
      const bool ok = s < n && edge / P + 2 * (seq + s) <= slot;
      const uint32_t c = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(ok)), i = c ? c - 1 : 0;
      seq += i * step;
      if (step == 1) {
        first = (uint32_t)__builtin_amdgcn_readlane((int)edge, (int)i);
        last = (uint32_t)__builtin_amdgcn_readlane((int)edge, (int)i + 1);
        break;
      }
      n = n - i * step < step ? n - i * step : step;
    }
    const int32_t count = last > first ? (int32_t)(last - first) : 0;
    const int32_t said = a.lens[seq], len = said < 0 ? 0 : said < (1 << 30) ? said : 1 << 30;
    const int32_t begin = len - count, cap = (int32_t)(a.seq_pages * P);   // (place of the first new token)
    const int32_t lo = begin > 0 ? begin : 0, hi = len < cap ? len : cap;
    const uint32_t nth = slot - (first / P + 2 * seq);
    // (all of it the same for the whole workgroup; slots before the first sequence wrap)
    if (hi <= lo || nth > (uint32_t)(hi - 1) / P - (uint32_t)lo / P) return;
    const uint32_t at = (uint32_t)lo / P + nth;
    const int32_t id = a.table[(uint64_t)seq * (a.ld_table ? a.ld_table : a.seq_pages) + at];
    if (id < 0 || (uint32_t)id >= a.n_pages) return;
    // new tokens of the page: [from, to)
    const int32_t base = (int32_t)(at * P);
    const uint32_t from = (uint32_t)(lo > base ? lo - base : 0), to = hi - base < (int32_t)P ? (uint32_t)(hi - base) : P;
    const uint32_t row0 = first + (uint32_t)(base - begin);   // row of the page's place 0 (wraps where that is an old one)
    const bool mine = head < a.kv_heads;
    const uint64_t block_at = (uint64_t)(uint32_t)id * a.kv_heads + (mine ? head : 0);
    uint8_t *kp = a.k_pages + block_at * P * DIM, *vp = a.v_pages + block_at * P * DIM;
    int old_k = 0, old_v = 0;
    if (from != 0) { old_k = a.k_exps[block_at]; old_v = a.v_exps[block_at]; }
    const uint32_t LDK = a.ld_k ? a.ld_k : a.kv_heads * DIM, LDV = a.ld_v ? a.ld_v : a.kv_heads * DIM;
    const uint32_t turned = a.rot / 16, half = a.rot / 2;
    const bool split = !(a.flags & TALLY_ROPE_INTERLEAVED);
    const double by = a.magnitude > 0.f ? (double)a.magnitude : 1.0;
    const uint32_t piece = lane % PIECES;
    const bool turns = piece < turned, apart = turns && split;
    const uint32_t one = piece * (apart ? 8 : 16), two = one + (apart ? half : 8);   // dims of the piece's halves

    float k[MORE][ROUNDS][16];
    uint32_t v[MORE][VT];
    uint32_t top_k = 0, top_v = 0;
#pragma unroll
    for (int m = 0; m < MORE; ++m) {
      const uint32_t unit = unit0 + m * 4;
      const bool live = mine && unit < units && unit * kUnit < to && unit * kUnit + kUnit > from;
      if (!live) continue;
#pragma unroll
      for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t t = unit * kUnit + r * (64 / PIECES) + lane / PIECES;
#pragma unroll
        for (int e = 0; e < 16; ++e) k[m][r][e] = 0.f;
        if (t < from || t >= to) continue;
        const uint32_t row = row0 + t;
        const uint16_t *x = a.k + (uint64_t)row * LDK + head * DIM;
        const u32x4_nt u = RopeBody::load<NT>(x + one), w = RopeBody::load<NT>(x + two);
        float (&o)[16] = k[m][r];                          // (o[e] and o[8 + e]: a pair)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u0 = bf16_lo(u[e]), u1 = bf16_hi(u[e]), w0 = bf16_lo(w[e]), w1 = bf16_hi(w[e]);
          if (split) o[2 * e] = u0, o[2 * e + 1] = u1, o[8 + 2 * e] = w0, o[9 + 2 * e] = w1;
          else o[e] = u0, o[8 + e] = u1, o[4 + e] = w0, o[12 + e] = w1;
        }
        if (turns) {
          const int32_t position = a.positions ? a.positions[row] : base + (int32_t)t;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const Turn z = turn_of(position, a.freqs[piece * 8 + e]);
            const double c = z.c * by, s = z.s * by, p0 = (double)o[e], q0 = (double)o[8 + e];
            o[e] = cut(__builtin_fma(p0, c, -(q0 * s)));
            o[8 + e] = cut(__builtin_fma(q0, c, p0 * s));
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint32_t b = magnitude_bits(o[e]);
          top_k = top_k > b ? top_k : b;
        }
      }
      const uint32_t t0 = unit * kUnit + lane / SIDE * VT;
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        v[m][i] = 0;
        if (t0 + i < from || t0 + i >= to) continue;
        v[m][i] = *reinterpret_cast<const uint32_t *>(a.v + (uint64_t)(row0 + t0 + i) * LDV + head * DIM + lane % SIDE * 2);
        const uint32_t b = magnitude_bits(bf16_lo(v[m][i])), d = magnitude_bits(bf16_hi(v[m][i]));
        top_v = top_v > b ? top_v : b;
        top_v = top_v > d ? top_v : d;
      }
    }
    top_k = wave_max_u32(top_k);
    top_v = wave_max_u32(top_v);
    if (lane == 0) s_top[0][wave] = top_k, s_top[1][wave] = top_v;
    __syncthreads();
    const uint32_t w0 = wave / per_head * per_head;
    for (uint32_t i = 0; i < per_head; ++i) {
      top_k = top_k > s_top[0][w0 + i] ? top_k : s_top[0][w0 + i];
      top_v = top_v > s_top[1][w0 + i] ? top_v : s_top[1][w0 + i];
    }
    if (!mine) return;                                     // (no barrier behind it)
    int ek = block_exp(top_k), ev = block_exp(top_v);
    if (from != 0) {
      ek = ek > old_k ? ek : old_k;
      ev = ev > old_v ? ev : old_v;
    }
    if (unit0 == 0 && lane == 0) {
      a.k_exps[block_at] = (uint8_t)ek;
      a.v_exps[block_at] = (uint8_t)ev;
    }
#pragma unroll
    for (int m = 0; m < MORE; ++m) {
      const uint32_t unit = unit0 + m * 4, first_token = unit * kUnit;
      if (unit >= units || first_token >= to) continue;
      const bool live = first_token + kUnit > from;
#pragma unroll
      for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t t = first_token + r * (64 / PIECES) + lane / PIECES;
        uint8_t *row = kp + t * DIM;
        if (live && t >= from && t < to) {
          const float (&o)[16] = k[m][r];
          u32x2_nt u, w;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (split) {
              u[e] = codes4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3], 127 - ek);
              w[e] = codes4(o[8 + 4 * e], o[9 + 4 * e], o[10 + 4 * e], o[11 + 4 * e], 127 - ek);
            } else {
              u[e] = codes4(o[2 * e], o[8 + 2 * e], o[2 * e + 1], o[9 + 2 * e], 127 - ek);
              w[e] = codes4(o[4 + 2 * e], o[12 + 2 * e], o[5 + 2 * e], o[13 + 2 * e], 127 - ek);
            }
          }
          *reinterpret_cast<u32x2_nt *>(row + one) = u;
          *reinterpret_cast<u32x2_nt *>(row + two) = w;
        } else if (t < from && ek != old_k) {
          u32x2_nt u = *reinterpret_cast<u32x2_nt *>(row + one), w = *reinterpret_cast<u32x2_nt *>(row + two);
#pragma unroll
          for (int e = 0; e < 2; ++e) u[e] = shift_codes(u[e], old_k - ek), w[e] = shift_codes(w[e], old_k - ek);
          *reinterpret_cast<u32x2_nt *>(row + one) = u;
          *reinterpret_cast<u32x2_nt *>(row + two) = w;
        }
      }
      // V: VT tokens of two dims; a unit that is not all new is put together with what is there
      if (!live && ev == old_v) continue;
      const uint32_t t0 = first_token + lane / SIDE * VT;
      uint8_t *col = vp + first_token * DIM + lane % SIDE * 32 + lane / SIDE * VT;
      const bool whole = first_token >= from && first_token + kUnit <= to;
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        uint32_t w[VT / 4];
#pragma unroll
        for (int i = 0; i < VT / 4; ++i) w[i] = 0;
        if (!whole)
#pragma unroll
          for (int i = 0; i < VT / 4; ++i) w[i] = *reinterpret_cast<const uint32_t *>(col + d * 16 + 4 * i);
#pragma unroll
        for (int i = 0; i < VT / 4; ++i) {
          uint32_t is_new = 0, before = 0;
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t t = t0 + 4 * i + j;
            is_new |= t >= from && t < to ? 0xFFu << (8 * j) : 0u;
            before |= t < from ? 0xFFu << (8 * j) : 0u;
          }
          uint32_t c = 0;
          if (live) {
            auto number = [&](int j) { return d ? bf16_hi(v[m][4 * i + j]) : bf16_lo(v[m][4 * i + j]); };
            c = codes4(number(0), number(1), number(2), number(3), 127 - ev);
          }
          if (ev != old_v) w[i] = (w[i] & ~before) | (shift_codes(w[i], old_v - ev) & before);
          w[i] = (w[i] & ~is_new) | (c & is_new);
        }
        if constexpr (VT == 16) *reinterpret_cast<u32x4_nt *>(col + d * 16) = u32x4_nt{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<u32x2_nt *>(col + d * 16) = u32x2_nt{w[0], w[1]};
      }
    }
#endif
  }
};
using AppendBody = AppendBodyT<128>;
using AppendNarrowBody = AppendBodyT<64>;

// ---- single-token attention ----------------------------------------------------------------
// How a call is cut up.  How long sequences are is known on the device alone, and a batch's lengths may differ by any
// factor, so the parts are dealt out there: all sequences have T strips of 128 tokens together; a part is at most
// c = max(least, ceil(T / parts)) of one sequence, whose parts are then made equal.  So there are
// at most `parts` + batch of them however the tokens are spread, and each workgroup finds its own by counting
// through the lengths, 64 at a time.
//
// A workgroup has 16 query heads at most of one K/V head and a part's tokens, each wave a tile of 32 in turn, with a state
// of its own; the four are merged in LDS at the end.
constexpr uint32_t kPagedStrip = 128, kPagedTile = 32, kPagedRows = 16;
struct PagedPlan {
  uint32_t group, row_tiles;                               // query heads of a K/V head; workgroups that share them
  uint32_t least, parts;                                   // strips of a part at least; parts over all sequences, beside one more for each
  uint32_t slots;                                          // parts that there may be
  uint32_t single;                                         // no sequence can have two: nothing to merge
};
inline PagedPlan paged_plan(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t page, uint32_t seq_pages) {
  PagedPlan p;
  p.group = heads / kv_heads;
  p.row_tiles = (p.group + kPagedRows - 1) / kPagedRows;
  const uint64_t across = (uint64_t)kv_heads * p.row_tiles, strips = ((uint64_t)seq_pages * page + kPagedStrip - 1) / kPagedStrip;
  p.least = strips <= 4 ? 4 : 2;
  p.parts = across >= 1024 ? 1 : (uint32_t)(1024 / across);
  if (p.parts > 256) p.parts = 256;
  const uint64_t most = (strips + p.least - 1) / p.least;  // of one sequence
  p.single = most <= 1;
  const uint64_t all = batch * (most ? most : 1);
  p.slots = (uint32_t)(all < (uint64_t)p.parts + batch ? all : (uint64_t)p.parts + batch);
  return p;
}
// Scratch: (max, sum) of each part's heads, and behind them each one's acc.
__host__ __device__ inline uint64_t paged_acc_at(uint64_t records) { return (records * 2 + 3) / 4 * 4; }   // in floats
inline size_t paged_scratch_bytes(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t page, uint32_t seq_pages) {
  const PagedPlan p = paged_plan(batch, heads, kv_heads, page, seq_pages);
  const uint64_t n = p.single ? 0 : (uint64_t)p.slots * heads;
  return (size_t)(paged_acc_at(n) + n * dim) * sizeof(float);
}

#ifdef __HIP_DEVICE_COMPILE__
// A sequence's parts, and of them one.
struct PagedPart {
  uint32_t seq, len;                                       // len: tokens of the sequence
  uint32_t first, parts;                                   // its parts: first, first + 1, ...
  uint32_t strips;                                         // of each of them (the last may have fewer)
};
__device__ __forceinline__ uint32_t wave_sum_u32(uint32_t v) {
#pragma unroll
  for (int by = 32; by; by >>= 1) v += (uint32_t)__shfl_xor((int)v, by);
  return v;
}
__device__ __forceinline__ uint32_t paged_len(const tally_attn_paged_args &a, uint32_t seq) {
  const int32_t said = a.lens[seq], cap = (int32_t)(a.seq_pages * a.page);
  return said < 0 ? 0u : said < cap ? (uint32_t)said : (uint32_t)cap;
}
// The sequence that has part `part` (or, with `of`, the one that is number `part`).  False where there is none.
__device__ __forceinline__ bool paged_find(const tally_attn_paged_args &a, const PagedPlan &p, uint32_t part, bool of, PagedPart &found) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t sum = 0;
  for (uint32_t i = lane; i < a.batch; i += 64) sum += (paged_len(a, i) + kPagedStrip - 1) / kPagedStrip;
  const uint32_t all = wave_sum_u32(sum), even = (all + p.parts - 1) / p.parts, c = even > p.least ? even : p.least;
  uint32_t before = 0;
  for (uint32_t i0 = 0; i0 < a.batch; i0 += 64) {
    const uint32_t i = i0 + lane, len = i < a.batch ? paged_len(a, i) : 0u;
    const uint32_t strips = (len + kPagedStrip - 1) / kPagedStrip;
    const uint32_t mine = i < a.batch ? (strips ? (strips + c - 1) / c : 1u) : 0u;
    uint32_t upto = mine;                                  // with those of the lanes before
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const uint32_t w = (uint32_t)__shfl_up((int)upto, by);
      if (lane >= (uint32_t)by) upto += w;
    }
    const uint64_t hit = __builtin_amdgcn_ballot_w64(of ? i == part : mine != 0 && part < before + upto);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      found.seq = i0 + l;
      found.len = (uint32_t)__builtin_amdgcn_readlane((int)len, l);
      found.parts = (uint32_t)__builtin_amdgcn_readlane((int)mine, l);
      found.first = before + (uint32_t)__builtin_amdgcn_readlane((int)upto, l) - found.parts;
      const uint32_t n = (found.len + kPagedStrip - 1) / kPagedStrip;
      found.strips = (n + found.parts - 1) / found.parts;
      return true;
    }
    before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  }
  return false;
}
#endif

template <int DIM>
__global__ __launch_bounds__(256, 4) void attn_paged_partial(tally_attn_paged_args a, PagedPlan p, uint32_t urgent) {
#ifdef __HIP_DEVICE_COMPILE__
  if (urgent) __builtin_amdgcn_s_setprio(3);
  typedef OnePass<DIM, 16, 32, 3> F;
  constexpr int KH = DIM / 64, DT = DIM / 16;              // 64-byte pieces of a key; blocks of 16 dims
  __shared__ float2 s_ml[4][16];
  __shared__ __align__(16) float s_acc[4][16][DIM / 2];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t across = a.kv_heads * p.row_tiles, part = blockIdx.x / across, nth = blockIdx.x % across;
  const uint32_t kv = nth / p.row_tiles, row0 = nth % p.row_tiles * kPagedRows;
  const uint32_t rows = p.group - row0 < kPagedRows ? p.group - row0 : kPagedRows;
  PagedPart mine;
  if (!paged_find(a, p, part, false, mine)) return;        // (the same for the whole workgroup)
  const uint32_t s0 = (part - mine.first) * mine.strips, n = mine.len;
  const uint32_t end = s0 * kPagedStrip < n ? (n - s0 * kPagedStrip < mine.strips * kPagedStrip ? n : (s0 + mine.strips) * kPagedStrip) : 0u;
  const uint32_t r = lane % 16, quarter = lane / 16, head = kv * p.group + row0 + r, LDQ = a.ld_q ? a.ld_q : a.heads * DIM;
  // q: fragment 2 h + j has dims 64 h + 16 quarter + 8 j and the seven behind
  bf16x8_t q[2 * KH];
#pragma unroll
  for (int i = 0; i < 2 * KH; ++i) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (r < rows) u = *reinterpret_cast<const uint4 *>(a.q + (uint64_t)mine.seq * LDQ + head * DIM + i / 2 * 64 + quarter * 16 + i % 2 * 8);
    q[i] = __builtin_bit_cast(bf16x8_t, u);
  }
  f32x4_t acc[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = kNothing, l = 0.f;
  bool some = false;                                       // a token of this wave's counts
  const float c = (a.scale > 0.f ? a.scale : DIM == 128 ? 0.08838834764831845f : 0.125f) * kLog2e;
  const int32_t *table = a.table + (uint64_t)mine.seq * (a.ld_table ? a.ld_table : a.seq_pages);
  const uint32_t last_page = n ? (n - 1) / a.page : 0u;
  // a lane's row of K in a tile: token 8 (r / 4) + 4 u + r % 4 for product u, so that it gets the scores of eight
  // neighbours, 8 quarter + 4 u + i, and of V eight neighbours of each dim
  for (uint32_t t0 = s0 * kPagedStrip + wave * kPagedTile; t0 < end; t0 += 4 * kPagedTile) {
    // the two units' pages
    const uint8_t *kb[2], *vb[2];
    uint32_t ke[2], ve[2];
    bool there[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t t = t0 + u * kUnit, at = t / a.page < last_page ? t / a.page : last_page;
      const int32_t id = table[at];
      there[u] = id >= 0 && (uint32_t)id < a.n_pages;
      const uint64_t block = (uint64_t)(there[u] ? (uint32_t)id : 0u) * a.kv_heads + kv;
      const uint64_t byte = block * a.page * DIM + t % a.page * DIM;
      kb[u] = a.k_pages + byte;
      vb[u] = a.v_pages + byte;
      ke[u] = a.k_exps[block];
      ve[u] = a.v_exps[block];
    }
    const uint8_t *k_at = (r >= 8 ? kb[1] : kb[0]) + (r / 4 % 2 * 8 + r % 4) * DIM + quarter * 16;
    const uint8_t *v_at = (quarter >= 2 ? vb[1] : vb[0]) + r * 16 + quarter % 2 * 8;
    uint4 k[2][KH];
    uint2 v[DT];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < KH; ++h) k[u][h] = *reinterpret_cast<const uint4 *>(k_at + u * 4 * DIM + h * 64);
#pragma unroll
    for (int d = 0; d < DT; ++d) v[d] = *reinterpret_cast<const uint2 *>(v_at + d * 256);
    auto wide = [](uint32_t lo, uint32_t hi, float by) {   // eight codes as bf16, times a power of two
      uint4 w;
      w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false));
      w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true));
      w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false));
      w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true));
      return __builtin_bit_cast(bf16x8_t, w);
    };
    f32x4_t s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < KH; ++h) {
        s[u] = F::mma(wide(k[u][h].x, k[u][h].y, 1.f), q[2 * h], s[u]);
        s[u] = F::mma(wide(k[u][h].z, k[u][h].w, 1.f), q[2 * h + 1], s[u]);
      }
    }
    const float by = c * __uint_as_float((quarter >= 2 ? ke[1] : ke[0]) << 23), v_by = __uint_as_float((quarter >= 2 ? ve[1] : ve[0]) << 23);
#pragma unroll
    for (int u = 0; u < 2; ++u) s[u] *= by;
    // tokens of the lane's eight that count
    const uint32_t t = t0 + quarter * 8;
    const uint32_t count = !(quarter >= 2 ? there[1] : there[0]) || t >= end ? 0u : end - t < 8u ? end - t : 8u;
    if (t0 + kPagedTile > end || !there[0] || !there[1]) {
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j)
        if (j >= count) s[j / 4][j % 4] = -INFINITY;
      const uint32_t lo = count >= 4 ? ~0u : (1u << 8 * count) - 1, hi = count >= 8 ? ~0u : count > 4 ? (1u << 8 * (count - 4)) - 1 : 0u;
#pragma unroll
      for (int d = 0; d < DT; ++d) v[d].x &= lo, v[d].y &= hi;
    }
    some |= __builtin_amdgcn_ballot_w64(count != 0) != 0;
    float top = s[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j / 4][j % 4]);
    top = across_rows<MaxOp>(top);
    const float now = fmaxf(m, top), fade = F::exp2(m - now);
    m = now;
    l *= fade;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = F::pack(F::exp2(s[j / 2][j % 2 * 2] - m), F::exp2(s[j / 2][j % 2 * 2 + 1] - m));
      l = F::add_pair(w[j], l);
    }
    const bf16x8_t weights = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      acc[d] *= fade;
      acc[d] = F::mma(wide(v[d].x, v[d].y, v_by), weights, acc[d]);
    }
  }
  // The four waves' states: each row's maximum and sum first, then the weighted acc, half of the dims at a time.
  l = across_rows<AddOp>(l);
  if (lane < 16) s_ml[wave][lane] = make_float2(m, some ? l : kNoTokens);
  __syncthreads();
  auto top_of = [&](uint32_t row) { return fmaxf(fmaxf(s_ml[0][row].x, s_ml[1][row].x), fmaxf(s_ml[2][row].x, s_ml[3][row].x)); };
  const float weight = F::exp2(m - top_of(r));
  constexpr uint32_t PIECES = DIM / 8;                     // of four dims, in half of them
  const uint32_t row = threadIdx.x / PIECES, piece = threadIdx.x % PIECES;
  f32x4_t o[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h) __syncthreads();
#pragma unroll
    for (int d = 0; d < DT / 2; ++d)
      *reinterpret_cast<f32x4_t *>(&s_acc[wave][r][(d * 4 + quarter ^ r % PIECES) * 4]) = acc[h * DT / 2 + d] * weight;
    __syncthreads();
    o[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (row < 16)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[h] += *reinterpret_cast<const f32x4_t *>(&s_acc[i][row][(piece ^ row % PIECES) * 4]);
  }
  if (row >= rows) return;
  const float top = top_of(row);
  float sum = 0.f;
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 w = s_ml[i][row];
    any |= !(w.y < 0.f);
    sum += w.y < 0.f ? 0.f : w.y * F::exp2(w.x - top);
  }
  const uint32_t h0 = kv * p.group + row0 + row;
  if (mine.parts == 1) {
    const float over = any ? 1.f / sum : 0.f;              // (scores of -inf throughout: NaN, as in a prompt)
    uint16_t *out = a.out + (uint64_t)mine.seq * (a.ld_out ? a.ld_out : a.heads * DIM) + h0 * DIM + piece * 4;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<uint2 *>(out + h * (DIM / 2)) =
          make_uint2(F::pack(o[h][0] * over, o[h][1] * over), F::pack(o[h][2] * over, o[h][3] * over));
    return;
  }
  const uint64_t to = (uint64_t)part * a.heads + h0;
  if (piece == 0) reinterpret_cast<float2 *>(a.scratch)[to] = make_float2(top, any ? sum : kNoTokens);
  float *rec = static_cast<float *>(a.scratch) + paged_acc_at((uint64_t)p.slots * a.heads) + to * DIM + piece * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4_t *>(rec + h * (DIM / 2)) = o[h];
#endif
}

// One row per workgroup: the parts' weights exp(m - max), each wave a quarter of the parts, 16 bytes of a part's acc to a lane.
template <int DIM>
__global__ __launch_bounds__(256) void attn_paged_merge(tally_attn_paged_args a, PagedPlan p, uint32_t urgent) {
#ifdef __HIP_DEVICE_COMPILE__
  if (urgent) __builtin_amdgcn_s_setprio(3);
  constexpr uint32_t LANES = DIM / 4, SIDE = 64 / LANES;   // parts side by side in a wave
  __shared__ float s_acc[4][DIM];
  __shared__ float s_sum[4];
  const uint32_t head = blockIdx.x % a.heads, seq = blockIdx.x / a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  PagedPart mine;
  if (!paged_find(a, p, seq, true, mine) || mine.parts == 1) return;
  const uint64_t row = (uint64_t)mine.first * a.heads + head;
  const float2 *ml = reinterpret_cast<const float2 *>(a.scratch) + row;
  const float *rec = static_cast<const float *>(a.scratch) + paged_acc_at((uint64_t)p.slots * a.heads) + row * DIM + lane % LANES * 4;
  float top = kNothing;
  for (uint32_t i = lane; i < mine.parts; i += 64) top = fmaxf(top, ml[(uint64_t)i * a.heads].x);
  top = wave_max(top);
  float sum = 0.f;
  bool any = false;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t i = wave * SIDE + lane / LANES; i < mine.parts; i += 4 * SIDE) {
    const float2 s = ml[(uint64_t)i * a.heads];
    const float w = __builtin_amdgcn_exp2f(s.x - top);
    any |= !(s.y < 0.f);
    sum += s.y < 0.f ? 0.f : s.y * w;
    acc += *reinterpret_cast<const f32x4_t *>(rec + (uint64_t)i * a.heads * DIM) * w;
  }
  if constexpr (SIDE == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = across_rows<AddOp>(acc[e]);
    sum = across_rows<AddOp>(sum);
  } else {
    auto halves = [](float o) {
      float w = o;
      asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(o), "+v"(w));
      return o + w;
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = halves(acc[e]);
    sum = halves(sum);
  }
  if (lane < LANES) *reinterpret_cast<f32x4_t *>(&s_acc[wave][lane * 4]) = acc;
  any = __builtin_amdgcn_ballot_w64(any) != 0;
  if (lane == 0) s_sum[wave] = any ? sum : kNoTokens;
  __syncthreads();
  if (threadIdx.x < DIM) {
    const uint32_t d = threadIdx.x;
    const float o = (s_acc[0][d] + s_acc[1][d]) + (s_acc[2][d] + s_acc[3][d]);
    float all = 0.f;
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      any |= !(s_sum[i] < 0.f);
      all += s_sum[i] < 0.f ? 0.f : s_sum[i];
    }
    const uint32_t LDO = a.ld_out ? a.ld_out : a.heads * DIM;
    a.out[(uint64_t)seq * LDO + head * DIM + d] = f32_to_bf16(any ? o / all : 0.f);
  }
#endif
}

inline PagedPlan paged_plan(const tally_attn_paged_args &a) { return paged_plan(a.batch, a.heads, a.kv_heads, a.page, a.seq_pages); }

template <int DIM>
hipError_t launch_paged_dim(hipStream_t s, const tally_attn_paged_args &a, uint32_t urgent) {
  const PagedPlan p = paged_plan(a);
  const hipError_t e = launch(attn_paged_partial<DIM>, dim3(p.slots * a.kv_heads * p.row_tiles), dim3(256), 0, s, a, p, urgent);
  if (e != hipSuccess || p.single) return e;
  return launch(attn_paged_merge<DIM>, dim3(a.heads * a.batch), dim3(256), 0, s, a, p, urgent);
}
inline hipError_t launch_attn_paged(hipStream_t s, const void *args, uint32_t urgent) {
  tally_attn_paged_args a;
  memcpy(&a, args, sizeof(a));
  return a.dim == 64 ? launch_paged_dim<64>(s, a, urgent) : launch_paged_dim<128>(s, a, urgent);
}

}  // namespace tally
