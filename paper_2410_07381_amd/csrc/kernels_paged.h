// A paged cache of keys and values in 8 bits for gfx950: appending to it, and single-token attention over it.
//
// A block is a page's tokens of one K/V head.  Its numbers are e4m3 codes times one power of two: a block that grows
// past its range has its codes shifted to the next exponent, which rounds none of them but those under the smallest
// normal, and a product with the scale is exact wherever it is taken.
//
// Pages consist of units of 16 tokens.  K's lie token by token, V's dim by dim with the 16 tokens of a dim side by side: a
// lane's 8 or 16 bytes are then a fragment of the products' first operand as they come from memory (K's rows
// are tokens, V's rows are dims), and nothing goes through LDS.
//
// What bounds both is memory, and for small calls one load waiting for another.  Measured (us of a call; what it reads and
// writes once at the 5.12 TB/s of a copy in brackets; an empty launch is 2.4):
//   appending, 8 heads of 128: one token 4.7; one for each of 64 sequences 6.3; 24 prompts of 1 to 4096 tokens 24.1 [16.3]; 32768 tokens 46.0 [39.3];
//   attention: 4 sequences of up to 512 tokens, 12 heads of 64, 5.8; 16 of up to 3001, 28/4 heads of 128, 12.2 [4.9]; 32 of up to 4096, 32/8,
//   31.9 [26.3]; 8 of up to 131071 173 to 188 from card to card [210], 6.2 to 5.7 TB/s.
// FETCH_SIZE and WRITE_SIZE say that either moves what it has to and nothing beside it (append of 32768 tokens 135 MB in and 67 MB out;
// 32 sequences of up to 4096 tokens 136 MB in).
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
// A wave's piece of work is 1024 numbers of K and as many of V: 8 tokens of a head of 128, 16 of one of 64.
//
// Prompts (kind 0): a wave takes such a piece of a page and one K/V head after the other, since the sines and cosines of its tokens
// are more work than all else on a head's keys.  A workgroup has all pieces of a page, which share their largest magnitudes through
// LDS, or of several small pages.
//
// Single tokens (kind 1): where there is hardly more than one a sequence, a wave takes a page, and of it the pieces that have new
// tokens: mostly it is one, and waves for the others would be in its way.  In between, and with more than four pieces to a page
// (kind 4), a workgroup's four waves take a page's pieces in turn.  Both go through pieces twice where a wave has several.
//
// Figures (us, 8 heads of 128).  Sequences x tokens each, kinds 0 / 1: pages of 16, 64 x 1 6.4 / 6.2, 64 x 2 7.0 / 8.4, 200 x 2 12.3 / 11.6; of 128,
// 8 x 1 6.1 / 4.9, 64 x 1 20.1 / 5.4; of 64, 64 x 1 11.5 / 5.4.  Kinds 0 / 1 / 4: pages of 128, 64 x 2 20.4 / 8.5 / 7.0, 64 x 8 21.0 / 9.8 / 7.1, 64 x 15
// 20.8 / 16.2 / 8.7, 64 x 16 (kind 0 from here on) 20.7 / 16.3 / 8.5, 200 x 4 58.2 / 12.6 / 14.8, 200 x 15 61.5 / 27.7 / 19.1, 400 x 4 119.5 / 20.9 / 27.1; of 64,
// 64 x 4 12.2 / 8.6 / 6.7, 64 x 8 (kind 0 from here on) 11.4 / 10.8 / 7.3, 200 x 4 28.8 / 13.7 / 14.4, 200 x 8 30.8 / 16.4 / 16.7.  So kind 1 would still be
// the faster one for hundreds of sequences of up to four tokens, and kind 4 some way beyond its end; the lines are simpler than that.  It
// is the average that decides: a prompt among single tokens is gone through by one wave a page, or four (pages of 128, 127 x 1 and 380 tokens of one
// sequence: kind 1 46, kind 4 16).
//
// Heads a wave goes through, 1 / 2, one prompt: pages of 16, 7000 tokens 13.5 / 14.2, 8192 14.5 / 12.9, 13504 21.2 / 19.9, 20000 33.4 / 30.0; of 64,
// 14.7 / 15.7, 15.4 / 13.6, 22.9 / 23.5, 35.6 / 32.9; of 128, 15.5 / 16.6, 17.2 / 16.2, 28.4 / 25.4, 41.7 / 41.5.  2 / 4: pages of 16 and 32, 32768
// tokens 45.6 / 45.7, 38229 53.5 / 57.3, 54613 73.0 / 76.2, 65536 85.3 / 85.0; of 64, 49.7 / 47.3, 58.3 / 57.9, 78.6 / 78.0, 91.6 / 87.9; of 128, 56.3 / 53.6,
// 67.2 / 72.0, 91.3 / 94.7, 104.8 / 99.9.  Pages of 16 and 32 never want four, those of 64 and 128 now two and now four, which no size of a call
// tells beforehand; and with up to four a worker needs 133 to 137 registers, with up to two 120 to 127.
//
// As workers, 32768 tokens, in the best of the configurations that are tried / as one slice of the whole grid (both from the call to its end, some 13
// more than a call among others): pages of 16 and 32 68 / 60, of 64 64 / 64, of 128 63 / 71.
//
// Tried: 16 tokens of a head of 128 a wave (194 registers, two waves per SIMD; 32768 tokens 47 to 55), the next head's numbers asked for ahead (pages
// of 128 51 and 48, others the same, registers spilled in workers), a page's id and old bytes asked for earlier (64 tokens 6.4).
constexpr uint64_t kAppendPieces = 8192;                   // from so many on a wave has two heads
__host__ __device__ constexpr uint32_t append_tokens(uint32_t dim) { return 1024 / dim; }   // of a piece
__host__ __device__ inline uint32_t append_kind(const tally_kv_append_args &a) {
  const uint64_t n = a.n_seqs;
  return a.total <= n + n / 8 ? 1 : a.page / append_tokens(a.dim) > 4 && a.total < n * a.page / 8 ? 4 : 0;
}
// waves of a workgroup, and slots (pages) that it has
__host__ __device__ inline uint32_t append_waves(const tally_kv_append_args &a) {
  const uint32_t pieces = a.page / append_tokens(a.dim);
  return append_kind(a) || pieces < 4 ? 4 : pieces;
}
__host__ __device__ inline uint32_t append_pages(const tally_kv_append_args &a) {
  const uint32_t kind = append_kind(a);
  return kind ? 4 / kind : append_waves(a) * append_tokens(a.dim) / a.page;
}
inline uint64_t append_slots(const tally_kv_append_args &a) { return (uint64_t)a.total / a.page + 2ull * a.n_seqs; }
// K/V heads that a logical block goes through, one after the other.
__host__ __device__ inline uint32_t append_heads(const tally_kv_append_args &a) {
  const uint64_t pieces = (uint64_t)a.total / append_tokens(a.dim) * a.kv_heads;
  uint32_t h = 1;
  if (append_kind(a) == 0 && a.kv_heads > 1 && pieces >= kAppendPieces) h = 2;   // (a branch: the compiler then has code for each)
  return h;
}
inline uint64_t append_blocks(const tally_kv_append_args &a) {
  const uint32_t h = append_heads(a), pages = append_pages(a);
  return (uint64_t)((a.kv_heads + h - 1) / h) * ((append_slots(a) + pages - 1) / pages);
}

#ifdef __HIP_DEVICE_COMPILE__
// Exponent of a block by the bits of the largest of its magnitudes: the smallest e from 1 on with m <= 448 x 2^(e - 127).  448 is
// 1.75 x 2^8, so a mantissa over 1.75 carries into the exponent.
__device__ __forceinline__ int block_exp(uint32_t top) {
  const int e = (int)((top + 0x1FFFFFu) >> 23) - 8;
  return e < 1 ? 1 : e > 254 ? 254 : e;
}
// fp64 to fp32 such that rounding the result to a code is rounding the number itself: of the bits behind the first one the four that a code and
// half a step of it take, and in the twelfth whether anything was cut off.  A block's first border between two codes is 2^(e - 137), 2^-136 or more.
// Of what lies above it fp32 has the twelfth bit where it is subnormal too, down to 2^-149; what lies below is a zero.  (Cut behind the twentieth
// it is an instruction less, 32768 tokens 45.8 for 46.1, and the bit is lost below 2^-129, where keys beside a border of the lowest exponents then
// went to the even code.  Those blocks' codes made once more, behind a branch, made workers up to 60 % slower.)
__device__ __forceinline__ float cut(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = (uint32_t)(b >> 32), off = (hi & 0xFFFFu) | (uint32_t)b;
  uint32_t any;                                            // (written out: as an expression it is a comparison and a choice)
  asm("v_min_u32 %0, 1, %1" : "=v"(any) : "v"(off));
  return (float)__builtin_bit_cast(double, (uint64_t)__builtin_amdgcn_perm(hi, any, 0x0706000Cu) << 32);
}
// 2^by for by from -127 on, 0 below.
__device__ __forceinline__ float power_of_two(int by) {
  return __uint_as_float(by >= -126 ? (uint32_t)(by + 127) << 23 : by == -127 ? 0x400000u : 0u);
}
// Four numbers times a power of two to codes.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float by) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * by, b * by, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * by, d * by, w, true);
}
__device__ __forceinline__ uint32_t shift_codes(uint32_t w, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes4(lo[0], lo[1], hi[0], hi[1], by);
}
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_nt __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t same(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
#endif

// WAVES of a workgroup; FEW: 0, or how many of them share a page (kinds 1 and 4).
template <int DIM, int WAVES, int FEW>
struct AppendBodyT {
  using Args = tally_kv_append_args;
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int MIN_WAVES = WAVES == 16 ? 4 : 3;
  static constexpr unsigned DYN_LDS = FEW ? 0 : WAVES * 8192;   // (a wave's sines and cosines)
  static constexpr bool END_BARRIER = FEW != 1;               // (the waves' largest magnitudes)
  static constexpr bool YIELDS = false;
  static constexpr bool RANGE = false;
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) { append<false>(a, bx); }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) { append<true>(a, bx); }

  template <bool NT>
  static __device__ __forceinline__ void append(const Args &a, uint32_t block) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr uint32_t TOK = append_tokens(DIM), PIECES = DIM / 16;   // tokens of a wave's piece of work; 16 numbers of a token a lane
    // Of V a lane has eight tokens of two dims: the whole unit of 16 tokens and 64 dims, so that two lanes make up a dim's 16 bytes.  (Few
    // tokens, of heads of 128: the same eight as of K and all dims; the unit's other half need not be gone through.)
    constexpr bool WHOLE = !FEW || DIM == 64;
    constexpr uint32_t SIDE = WHOLE ? 32 : 64;               // lanes side by side
    constexpr int AUX = NT ? 2 : 0;
    const uint32_t lane = threadIdx.x & 63, wave = same(threadIdx.x >> 6);
    const uint32_t shift = (uint32_t)__builtin_ctz(a.page), P = a.page;
    const uint32_t HN = FEW ? 1 : append_heads(a), groups = (a.kv_heads + HN - 1) / HN;
    const uint32_t per_page = FEW ? FEW : P / TOK, h0 = block % groups * HN;
    const uint32_t slot = block / groups * (WAVES / per_page) + wave / per_page;
    // The sequence of this slot: the last one that starts at or before it, 63 candidates at a time; the lane behind the last
    // candidate has where that one ends.
    uint32_t seq = 0, first, last;
    int32_t said;
    for (uint32_t n = a.n_seqs;;) {
      const uint32_t step = (n + 62) / 63, s = lane * step < n ? lane * step : n;
      const int32_t v = a.cu_seqlens[seq + s], w = a.lens[seq + (s < n ? s : n - 1)];
      const uint32_t edge = v < 0 ? 0u : (uint32_t)v < a.total ? (uint32_t)v : a.total;
      const bool ok = s < n && (edge >> shift) + 2 * (seq + s) <= slot;
      const uint32_t c = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(ok)), i = c ? c - 1 : 0;
      seq += i * step;
      if (step == 1) {
        first = (uint32_t)__builtin_amdgcn_readlane((int)edge, (int)i);
        last = (uint32_t)__builtin_amdgcn_readlane((int)edge, (int)i + 1);
        said = __builtin_amdgcn_readlane(w, (int)i);
        break;
      }
      n = n - i * step < step ? n - i * step : step;
    }
    const int32_t count = last > first ? (int32_t)(last - first) : 0;
    const int32_t len = said < 0 ? 0 : said < (1 << 30) ? said : 1 << 30;
    const int32_t begin = len - count, cap = (int32_t)(a.seq_pages * P);   // (place of the first new token)
    const int32_t lo = begin > 0 ? begin : 0, hi = len < cap ? len : cap;
    const uint32_t nth = slot - ((first >> shift) + 2 * seq);
    // (slots before the first sequence wrap)
    bool there = hi > lo && nth <= ((uint32_t)(hi - 1) >> shift) - ((uint32_t)lo >> shift);
    if (FEW && !there) return;
    const uint32_t at = there ? ((uint32_t)lo >> shift) + nth : 0u;
    const int32_t base = (int32_t)(at << shift);
    // new tokens of the page: [from, to); the first of them is row `row` of k and v
    const uint32_t from = (uint32_t)(lo > base ? lo - base : 0), to = hi - base < (int32_t)P ? (uint32_t)(hi - base) : P;
    const uint32_t row = there ? first + (uint32_t)(base + (int32_t)from - begin) : 0u;
    int32_t id = 0;
    if (there) {
      id = (int32_t)same((uint32_t)a.table[(uint64_t)seq * (a.ld_table ? a.ld_table : a.seq_pages) + at]);
      there = id >= 0 && (uint32_t)id < a.n_pages;
    }
    if (FEW && !there) return;
    const uint32_t LDK = a.ld_k ? a.ld_k : a.kv_heads * DIM, LDV = a.ld_v ? a.ld_v : a.kv_heads * DIM;
    const uint32_t turned = a.rot / 16, half = a.rot / 2;
    const bool split = !(a.flags & TALLY_ROPE_INTERLEAVED);
    const uint32_t piece = lane % PIECES, tok = lane / PIECES;
    const bool turns = piece < turned, apart = turns && split;
    const uint32_t one = piece * (apart ? 8 : 16), two = one + (apart ? half : 8);   // dims of the lane's two eights
    auto v_first = [&](uint32_t u0) { return (WHOLE ? u0 / kUnit * kUnit : u0) + lane / SIDE * 8; };
    auto v_dim = [&](uint32_t u0) { return (WHOLE && DIM == 128 ? u0 % kUnit * 8 : 0u) + lane % SIDE * 2; };

    // Sines and cosines of the lane's pairs, of tokens u0 .. u0 + TOK - 1 of the page.
    extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
    Turn z[8], *table = reinterpret_cast<Turn *>(tally_dyn_lds) + (FEW ? 0 : wave * (TOK * DIM / 2));
    auto make_turns = [&](uint32_t u0) {
      const double by = a.magnitude > 0.f ? (double)a.magnitude : 1.0;
      if constexpr (FEW) {
        const uint32_t t = u0 + tok;
        int32_t position = base + (int32_t)t;
        if (a.positions) position = t >= from && t < to ? a.positions[row + (t - from)] : 0;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = a.freqs[turns ? piece * 8 + e : 0];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          z[e] = turn_of(position, f[e]);
          z[e].c *= by, z[e].s *= by;
        }
      } else {
        // A lane makes those of one pair and eight neighbours: where positions are neighbours too the first, and the others by turning
        // on and on by the frequency.  They stay in LDS, a piece's pairs side by side for lanes that are.
        const uint32_t pair = lane % PIECES * 8 + lane / PIECES % 8, t0 = u0 + lane / (DIM / 2) * 8;
        const float f = a.freqs[pair < half ? pair : 0];
        Turn w = turn_of(base + (int32_t)t0, f);
        const Turn on = turn_of(1, f);
        w.c *= by, w.s *= by;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          if (a.positions) {
            const uint32_t t = t0 + j;
            w = turn_of(t >= from && t < to ? a.positions[row + (t - from)] : 0, f);
            w.c *= by, w.s *= by;
          }
          table[(t0 - u0 + j) * (DIM / 2) + lane % (DIM / 2)] = w;
          w = Turn{__builtin_fma(w.c, on.c, -(w.s * on.s)), __builtin_fma(w.s, on.c, w.c * on.s)};
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (other lanes of the wave read them; its LDS accesses are in order)
        __builtin_amdgcn_wave_barrier();
      }
    };
    float k[16];                                           // (k[e] and k[8 + e]: a pair)
    uint32_t v[8];
    uint4 x, y;
    // New numbers of tokens u0 .. u0 + TOK - 1 of the page, and of V's part, are asked for; zeros for other tokens.
    auto ask = [&](uint32_t u0, uint32_t head) {
      const buf_t kb = make_buf(a.k + (uint64_t)row * LDK + head * DIM, ((to - from - 1) * LDK + DIM) * 2);
      const buf_t vb = make_buf(a.v + (uint64_t)row * LDV + head * DIM, ((to - from - 1) * LDV + DIM) * 2);
      const uint32_t t = (u0 + tok - from) * LDK;
      x = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(kb, (t + one) * 2, 0, AUX));
      y = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(kb, (t + two) * 2, 0, AUX));
      const uint32_t tv = v_first(u0) - from, col = v_dim(u0);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __builtin_amdgcn_raw_buffer_load_b32(vb, ((tv + j) * LDV + col) * 2, 0, AUX);
    };
    // What was asked for, keys turned.
    auto take = [&] {
      // pairs that are neighbours come apart: words of first ones and of second ones
      const uint32_t u[4] = {x.x, x.y, x.z, x.w}, w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t c = e < 2 ? u[2 * e] : w[2 * e - 4], d = e < 2 ? u[2 * e + 1] : w[2 * e - 3];
        const uint32_t p = split ? u[e] : __builtin_amdgcn_perm(d, c, 0x05040100u), q = split ? w[e] : __builtin_amdgcn_perm(d, c, 0x07060302u);
        k[2 * e] = bf16_lo(p), k[2 * e + 1] = bf16_hi(p);
        k[8 + 2 * e] = bf16_lo(q), k[9 + 2 * e] = bf16_hi(q);
      }
      if (turns) {
#pragma unroll
        for (int e = 0; e < 8 && !FEW; ++e) z[e] = table[tok * (DIM / 2) + e * PIECES + piece];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double p0 = (double)k[e], q0 = (double)k[8 + e];
          k[e] = cut(__builtin_fma(p0, z[e].c, -(q0 * z[e].s)));
          k[8 + e] = cut(__builtin_fma(q0, z[e].c, p0 * z[e].s));
        }
      }
    };
    // A lane's largest magnitudes so far: K's, and of V's bits two side by side.  (K's maxima leave NaN out; infinities, and what of
    // V is no number, have to be left out by name, where there are any.)
    float mk = 0.f;
    u16x2_t mv = {0, 0};
    auto tops = [&] {
      const float mk0 = mk;
      const u16x2_t mv0 = mv;
#pragma unroll
      for (int e = 0; e < 8; ++e) mk = fmaxf(mk, fmaxf(__builtin_fabsf(k[2 * e]), __builtin_fabsf(k[2 * e + 1])));
#pragma unroll
      for (int j = 0; j < 8; ++j) mv = __builtin_elementwise_max(mv, __builtin_bit_cast(u16x2_t, v[j] & 0x7FFF7FFFu));
      if (__builtin_amdgcn_ballot_w64(mk == INFINITY || mv[0] >= 0x7F80 || mv[1] >= 0x7F80)) {
        mk = mk0, mv = mv0;
#pragma unroll
        for (int e = 0; e < 16; ++e) mk = fmaxf(mk, __builtin_fabsf(k[e]) < INFINITY ? __builtin_fabsf(k[e]) : 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          u16x2_t w = __builtin_bit_cast(u16x2_t, v[j] & 0x7FFF7FFFu);
          w[0] = w[0] < 0x7F80 ? w[0] : 0, w[1] = w[1] < 0x7F80 ? w[1] : 0;
          mv = __builtin_elementwise_max(mv, w);
        }
      }
    };
    // Over the wave: K's for the lower lanes, V's for the upper ones.
    auto over_wave = [&] {
      float p = mk, q = __uint_as_float((uint32_t)(mv[0] > mv[1] ? mv[0] : mv[1]) << 16);
      asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(p), "+v"(q));
      p = q = fmaxf(p, q);
      asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(p), "+v"(q));
      return row16_all<MaxOp>(fmaxf(p, q));
    };
    // What a block's exponents become, and what was loaded, or what was there, to its codes.
    struct Block { uint8_t *kp, *vp; int old_k, old_v, ek, ev; };
    auto block_of = [&](uint32_t head, uint64_t &index) {
      index = (uint64_t)(uint32_t)id * a.kv_heads + head;
      Block w{a.k_pages + (index << shift) * DIM, a.v_pages + (index << shift) * DIM, 0, 0, 0, 0};
      if (from != 0) w.old_k = a.k_exps[index], w.old_v = a.v_exps[index];
      return w;
    };
    auto grow = [&](Block &w, uint64_t index, float top, bool write) {
      w.ek = block_exp(__builtin_amdgcn_readlane(__float_as_int(top), 0)), w.ev = block_exp(__builtin_amdgcn_readlane(__float_as_int(top), 32));
      if (from != 0) {
        w.ek = w.ek > w.old_k ? w.ek : w.old_k;
        w.ev = w.ev > w.old_v ? w.ev : w.old_v;
      }
      if (write && lane == 0) {
        a.k_exps[index] = (uint8_t)w.ek;
        a.v_exps[index] = (uint8_t)w.ev;
      }
    };
    auto store = [&](uint32_t u0, const Block &b, bool live) {
      const uint32_t t = u0 + tok;
      uint8_t *to_row = b.kp + t * DIM;
      if (live && t >= from && t < to) {
        const float by = power_of_two(127 - b.ek);
        const uint32_t p0 = codes4(k[0], k[1], k[2], k[3], by), p1 = codes4(k[4], k[5], k[6], k[7], by);
        const uint32_t q0 = codes4(k[8], k[9], k[10], k[11], by), q1 = codes4(k[12], k[13], k[14], k[15], by);
        const u32x2_nt u = {split ? p0 : __builtin_amdgcn_perm(q0, p0, 0x05010400u), split ? p1 : __builtin_amdgcn_perm(q0, p0, 0x07030602u)};
        const u32x2_nt w = {split ? q0 : __builtin_amdgcn_perm(q1, p1, 0x05010400u), split ? q1 : __builtin_amdgcn_perm(q1, p1, 0x07030602u)};
        *reinterpret_cast<u32x2_nt *>(to_row + one) = u;
        *reinterpret_cast<u32x2_nt *>(to_row + two) = w;
      } else if (t < from && b.ek != b.old_k) {
        const float by = power_of_two(b.old_k - b.ek);
        u32x2_nt u = *reinterpret_cast<u32x2_nt *>(to_row + one), w = *reinterpret_cast<u32x2_nt *>(to_row + two);
#pragma unroll
        for (int e = 0; e < 2; ++e) u[e] = shift_codes(u[e], by), w[e] = shift_codes(w[e], by);
        *reinterpret_cast<u32x2_nt *>(to_row + one) = u;
        *reinterpret_cast<u32x2_nt *>(to_row + two) = w;
      }
      // V: what is not all new is put together with what is there
      if (!live && b.ev == b.old_v) return;
      const uint32_t t0 = v_first(u0), dim = v_dim(u0);
      uint8_t *unit = b.vp + t0 / kUnit * (kUnit * DIM);
      uint32_t w[2][2];
      const float by = power_of_two(127 - b.ev);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        w[0][j] = live ? codes4(bf16_lo(v[4 * j]), bf16_lo(v[4 * j + 1]), bf16_lo(v[4 * j + 2]), bf16_lo(v[4 * j + 3]), by) : 0u;
        w[1][j] = live ? codes4(bf16_hi(v[4 * j]), bf16_hi(v[4 * j + 1]), bf16_hi(v[4 * j + 2]), bf16_hi(v[4 * j + 3]), by) : 0u;
      }
      const uint32_t begins = u0 / kUnit * kUnit;
      if (begins < from || begins + kUnit > to) {
        const float v_shift = power_of_two(b.old_v - b.ev);
        // bytes of the lane's eight tokens below a place
        auto below = [&](uint32_t place) { return place <= t0 ? 0ull : place >= t0 + 8 ? ~0ull : (1ull << 8 * (place - t0)) - 1; };
        const uint64_t before = below(from), fresh = live ? below(to) & ~before : 0ull;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const u32x2_nt old = *reinterpret_cast<const u32x2_nt *>(unit + (dim + d) * kUnit + t0 % kUnit);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t gone = (uint32_t)(before >> 32 * j), is_new = (uint32_t)(fresh >> 32 * j);
            uint32_t x = old[j];
            if (b.ev != b.old_v) x = (x & ~gone) | (shift_codes(x, v_shift) & gone);
            w[d][j] = (x & ~is_new) | (w[d][j] & is_new);
          }
        }
      }
      if constexpr (WHOLE) {
        // (the lower lanes take the first dim of the pair, the upper ones the second, all 16 tokens)
#pragma unroll
        for (int j = 0; j < 2; ++j) asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(w[0][j]), "+v"(w[1][j]));
        *reinterpret_cast<u32x4_nt *>(unit + (dim + lane / SIDE) * kUnit) = u32x4_nt{w[0][0], w[0][1], w[1][0], w[1][1]};
      } else {
#pragma unroll
        for (int d = 0; d < 2; ++d) *reinterpret_cast<u32x2_nt *>(unit + (dim + d) * kUnit + t0 % kUnit) = u32x2_nt{w[d][0], w[d][1]};
      }
    };

    __shared__ float s_top[2][2][WAVES];
    // The largest magnitudes over the page's waves.  (A row of 16 lanes has all of theirs, some more than once.)
    auto over_page = [&](float top, uint32_t turn) {
      if (per_page == 1) return top;
      if (lane % 32 == 0) s_top[turn][lane / 32][wave] = top;
      __syncthreads();
      return row16_all<MaxOp>(s_top[turn][lane / 32][wave - wave % per_page + lane % per_page]);
    };
    if constexpr (FEW) {
      uint64_t index;
      Block b = block_of(h0, index);
      const uint32_t mine = FEW == 1 ? 0 : wave * TOK, begins = from / TOK * TOK + mine;
      uint32_t have = ~0u;                                 // the piece that is loaded
      for (uint32_t u0 = begins; u0 < to; u0 += FEW * TOK) {
        ask(u0, h0);
        if (a.rot) make_turns(u0);
        take();
        tops();
        have = u0;
      }
      grow(b, index, over_page(over_wave(), 0), mine == 0);
      if (have != ~0u) store(have, b, true);
      for (uint32_t u0 = begins; u0 < to && u0 != have; u0 += FEW * TOK) {
        ask(u0, h0);
        if (a.rot) make_turns(u0);
        take();
        store(u0, b, true);
      }
      if (b.ek != b.old_k || b.ev != b.old_v)
        for (uint32_t u0 = mine; u0 < from / TOK * TOK; u0 += FEW * TOK) store(u0, b, false);
    } else {
      const uint32_t u0 = wave % per_page * TOK, begins = u0 / kUnit * kUnit;
      const bool live = there && begins < to && begins + kUnit > from, held = there && begins < from;   // new ones in the unit; old ones
      if (live) ask(u0, h0);
      if (live && a.rot) make_turns(u0);
      for (uint32_t i = 0; i < HN && h0 + i < a.kv_heads; ++i) {   // (the same for the whole workgroup)
        uint64_t index = 0;
        Block b{};
        float top = 0.f;
        if (live || held) b = block_of(h0 + i, index);
        if (live) {
          if (i) ask(u0, h0 + i);
          take();
          mk = 0.f, mv = u16x2_t{0, 0};
          tops();
          top = over_wave();
        }
        top = over_page(top, i & 1);
        if (!live && !held) continue;
        grow(b, index, top, u0 == 0);
        store(u0, b, live);
      }
    }
#endif
  }
};

// ---- single-token attention ----------------------------------------------------------------
// How a call is cut up.  How long sequences are is known on the device alone, and a batch's lengths may differ by any
// factor, so the parts are dealt out there: all sequences have T strips of 128 tokens together; a part is at most
// c = max(least, ceil(T / parts)) of one sequence, whose parts are then made equal.  So there are
// at most `parts` + batch of them however the tokens are spread, and each workgroup finds its own by counting
// through the lengths, 64 at a time.
//
// A workgroup has 16 query heads at most of one K/V head and a part's tokens, each wave a tile of 32 in turn, with a state
// of its own; the four are merged in LDS at the end.  128 registers and 17 KB of LDS: four of them on a compute unit, or one beside a
// paused 256 x 256 GEMM tile.
//
// 1024 workgroups are what is on the GPU at once (us with 512 / 768 / 1024 / 2048: 32 sequences of up to 4096, 8 K/V heads, 36.6 36.0 34.4 34.6; 8 of up to
// 131071 223 211 193 195; one of 32768 19.0 20.1 20.2 20.2).  A part has two strips at least (1 / 2 / 4: 16 of up to 3001, 4 K/V heads, 13.5 12.2 12.1; one of
// 4096, 8 heads, 9.2 9.3 10.4).  No more than 256 parts, for one K/V head 256 workgroups (128 / 256 / 512: one of 131071, 8 heads of 128 on one, 18.4 18.6
// 24.6, 16 of 64 on one, 14.3 13.7 17.4; 4 of up to 65536, 8 on one, 17.7 16.1 17.9): more of them find their part later than they read it sooner.
// The host knows the table's width and no lengths, so a wide table costs short sequences the second kernel (4 of up to 512 tokens 5.8 with a table for as many,
// 8.4 with one for 32768; 16 of up to 3001 12.3 and 13.5; 32 of up to 4096 32.1 and 32.1).
// One part a sequence saves the second kernel.  It pays up to 4 strips whatever the number of workgroups (4 sequences of 512, 12 heads of 64:
// 5.8, in two parts 8.2; one of 1024, 8 heads, 9.9 and 9.2), up to 8 from 256 workgroups on (8 of 600, 32 heads, 10.8 and 12.1; with 64 of them,
// 8 of 1024, 8 heads, 10.0 and 9.4), up to 16 from 512 on (64 of up to 2000, 8 heads, 32.8 and 34.9; with 128, 128 of 2000 on one head of 64,
// 14.3 and 12.2).  Eight waves a workgroup then: 6.2 for 5.8.
// A row of the second kernel is a wave's where sequences have few parts, else a workgroup's (a wave / a workgroup: 64 of up to 1000, 3 parts, 19.9
// 21.3; 64 of up to 8192, heads of 64, 3, 51.8 53.8; 32 of up to 4096, 5, 32.1 32.4; 16 of up to 3001, 17, 13.4 12.4; one of 32768 26.9 20.4).
// Caches above 256 MB, which is what the Infinity Cache holds, are read past it (non-temporal; three caches in turn, ordinary / so: capacity 192 MB
// 26.0 27.3, 224 29.7 28.3, 256 34.5 32.3, 320 40.3 37.2, 2.1 GB 192 173; one cache again and again 256 MB 28.8 31.4).
constexpr uint32_t kPagedStrip = 128, kPagedTile = 32, kPagedRows = 16;
struct PagedPlan {
  uint32_t group, row_tiles;                               // query heads of a K/V head; workgroups that share them
  uint32_t least, parts;                                   // strips of a part at least; parts over all sequences, beside one more for each
  uint32_t slots;                                          // parts that there may be
  uint32_t single;                                         // no sequence can have two: nothing to merge
  uint32_t past;                                           // the caches may be larger than what the GPU's caches hold
};
inline PagedPlan paged_plan(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t page, uint32_t seq_pages) {
  PagedPlan p;
  p.group = heads / kv_heads;
  p.row_tiles = (p.group + kPagedRows - 1) / kPagedRows;
  const uint64_t across = (uint64_t)kv_heads * p.row_tiles, strips = ((uint64_t)seq_pages * page + kPagedStrip - 1) / kPagedStrip;
  const uint64_t whole = batch * across / 32 < 4 ? 4 : batch * across / 32 > 16 ? 16 : batch * across / 32;
  p.least = (uint32_t)(strips <= whole ? strips : 2);
  p.parts = across >= 1024 ? 1 : (uint32_t)(1024 / across);
  if (p.parts > 256) p.parts = 256;
  const uint64_t most = (strips + p.least - 1) / p.least;  // of one sequence
  p.single = most <= 1;
  const uint64_t all = batch * (most ? most : 1);
  p.past = 2ull * batch * seq_pages * page * kv_heads * dim >= kInfinityCache;
  p.slots = (uint32_t)(all < (uint64_t)p.parts + batch ? all : (uint64_t)p.parts + batch);
  return p;
}
// Scratch: (max, sum) of each part's heads, and behind them each one's acc.
__host__ __device__ inline uint64_t paged_acc_at(uint64_t records) { return (records * 2 + 3) / 4 * 4; }   // in floats
inline size_t paged_scratch_bytes(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t page, uint32_t seq_pages) {
  const PagedPlan p = paged_plan(batch, heads, kv_heads, dim, page, seq_pages);
  const uint64_t n = p.single ? 0 : (uint64_t)p.slots * heads;
  return (size_t)(paged_acc_at(n) + n * dim) * sizeof(float);
}

#ifdef __HIP_DEVICE_COMPILE__
template <bool NT, class T>
__device__ __forceinline__ T past(const T *p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}
// A sequence's parts, and of them one.
struct PagedPart {
  uint32_t seq, len;                                       // len: tokens of the sequence
  uint32_t first, parts;                                   // its parts: first, first + 1, ...
  uint32_t strips;                                         // of each of them (the last may have fewer)
};
// Sums over the lanes up to each one.  (By DPP operands: within rows of 16, then a row's last lane to the rows behind.)
__device__ __forceinline__ uint32_t wave_scan_u32(uint32_t v) {
#define SCAN_STEP(ctrl, rows) v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false)
  SCAN_STEP(0x111, 0xf);
  SCAN_STEP(0x112, 0xf);
  SCAN_STEP(0x114, 0xf);
  SCAN_STEP(0x118, 0xf);
  SCAN_STEP(0x142, 0xa);
  SCAN_STEP(0x143, 0xc);
#undef SCAN_STEP
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
  const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)wave_scan_u32(sum), 63), even = (all + p.parts - 1) / p.parts, c = even > p.least ? even : p.least;
  uint32_t before = 0;
  for (uint32_t i0 = 0; i0 < a.batch; i0 += 64) {
    const uint32_t i = i0 + lane, len = i < a.batch ? paged_len(a, i) : 0u;
    const uint32_t strips = (len + kPagedStrip - 1) / kPagedStrip;
    const uint32_t mine = i < a.batch ? (strips ? (strips + c - 1) / c : 1u) : 0u;
    const uint32_t upto = wave_scan_u32(mine);             // with those of the lanes before
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

// SMALL: pages of 16 tokens, so that a tile's two units may lie in different ones.  Otherwise a tile has one page, whose
// address is the same for all lanes.  NT: caches that are larger than what the GPU's caches hold are read past them.
template <int DIM, bool SMALL, bool NT>
__global__ __launch_bounds__(256, 4) void attn_paged_partial(tally_attn_paged_args a, PagedPlan p, uint32_t urgent) {
#ifdef __HIP_DEVICE_COMPILE__
  if (urgent) __builtin_amdgcn_s_setprio(3);
  typedef OnePass<DIM, 16, 32, 3> F;
  constexpr int KH = DIM / 64, DT = DIM / 16;              // 64-byte pieces of a key; blocks of 16 dims
  constexpr int PAGES = SMALL ? 2 : 1;                     // of a tile
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
  const int32_t *table = a.table + (uint64_t)mine.seq * (a.ld_table ? a.ld_table : a.seq_pages);
  const uint32_t last_page = n ? (n - 1) / a.page : 0u, shift = (uint32_t)__builtin_ctz(a.page);

  // Where a tile lies: its pages (of one that does not exist, page 0), and in them the byte that it begins at.
  struct Place { uint32_t id[PAGES]; bool there[PAGES]; uint32_t in; };
  auto place_of = [&](uint32_t t0) {
    Place w;
#pragma unroll
    for (int u = 0; u < PAGES; ++u) {
      const uint32_t at = (t0 + u * kUnit) >> shift;
      const int32_t id = table[at < last_page ? at : last_page];
      w.there[u] = id >= 0 && (uint32_t)id < a.n_pages;
      w.id[u] = w.there[u] ? (uint32_t)id : 0u;
    }
    w.in = (t0 & (a.page - 1)) * DIM;
    return w;
  };
  // A lane's row of K in a tile is token 8 (r / 4) + 4 u + r % 4 for product u, so that it gets the scores of eight neighbours,
  // 8 quarter + 4 u + i, and of V eight neighbours of each dim.
  const uint32_t k_lane = ((SMALL ? 0 : r / 8 * kUnit) + r / 4 % 2 * 8 + r % 4) * DIM + quarter * 16;
  const uint32_t v_lane = (SMALL ? 0 : quarter / 2 * kUnit * DIM) + r * 16 + quarter % 2 * 8;
  auto block_of = [&](const Place &w, bool second) {       // of the lane
    const uint64_t one = (uint64_t)w.id[0] * a.kv_heads + kv;
    if constexpr (!SMALL) return one;
    const uint64_t two = (uint64_t)w.id[PAGES - 1] * a.kv_heads + kv;
    return second ? two : one;
  };
  uint4 k[2][KH];
  uint2 v[DT];
  uint32_t ke, ve;
  auto ask_keys = [&](const Place &w) {
    const uint8_t *at = a.k_pages + (block_of(w, r >= 8) << shift) * DIM + w.in + k_lane;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < KH; ++h) k[u][h] = __builtin_bit_cast(uint4, past<NT>(reinterpret_cast<const u32x4_nt *>(at + u * 4 * DIM + h * 64)));
  };
  auto ask_values = [&](const Place &w) {
    const uint8_t *at = a.v_pages + (block_of(w, quarter >= 2) << shift) * DIM + w.in + v_lane;
#pragma unroll
    for (int d = 0; d < DT; ++d) v[d] = __builtin_bit_cast(uint2, past<NT>(reinterpret_cast<const u32x2_nt *>(at + d * 256)));
  };
  auto ask_exps = [&](const Place &w) {
    const uint64_t block = block_of(w, quarter >= 2);
    ke = a.k_exps[block];
    ve = a.v_exps[block];
  };
  uint32_t t0 = s0 * kPagedStrip + wave * kPagedTile;
  Place now = place_of(t0), next = now;
  if (t0 < end) {
    ask_exps(now);
    ask_keys(now);
    ask_values(now);
    next = place_of(t0 + 4 * kPagedTile);
  }
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
  auto wide = [](uint32_t lo, uint32_t hi, float by) {     // eight codes as bf16, times a power of two
    uint4 w;
    w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false));
    w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true));
    w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false));
    w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true));
    return __builtin_bit_cast(bf16x8_t, w);
  };
  for (; t0 < end; t0 += 4 * kPagedTile) {
    const bool more = t0 + 4 * kPagedTile < end;
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
    const float by = c * __uint_as_float(ke << 23);
    float v_by = __uint_as_float(ve << 23);
    __builtin_amdgcn_sched_barrier(0);
    if (more) {                                            // (the registers of this tile's are free)
      ask_exps(next);
      ask_keys(next);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 2; ++u) s[u] *= by;
    if (t0 + kPagedTile > end || !now.there[0] || !now.there[PAGES - 1]) {
      // tokens of the lane's eight that count
      const uint32_t t = t0 + quarter * 8;
      const uint32_t count = !(quarter >= 2 ? now.there[PAGES - 1] : now.there[0]) || t >= end ? 0u : end - t < 8u ? end - t : 8u;
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j)
        if (j >= count) s[j / 4][j % 4] = -INFINITY;
      const uint32_t lo = count >= 4 ? ~0u : (1u << 8 * count) - 1, hi = count >= 8 ? ~0u : count > 4 ? (1u << 8 * (count - 4)) - 1 : 0u;
#pragma unroll
      for (int d = 0; d < DT; ++d) v[d].x &= lo, v[d].y &= hi;
      v_by = count ? v_by : 1.f;                           // (of a page that does not exist it is another's, which may be anything)
      some |= __builtin_amdgcn_ballot_w64(count != 0) != 0;
    } else {
      some = true;
    }
    float top = s[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j / 4][j % 4]);
    top = across_rows<MaxOp>(top);
    const float upto = fmaxf(m, top), fade = F::exp2(m - upto);
    m = upto;
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
    __builtin_amdgcn_sched_barrier(0);
    if (more) {
      ask_values(next);
      now = next;
      next = place_of(t0 + 8 * kPagedTile);
    }
    __builtin_amdgcn_sched_barrier(0);
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

// One row per workgroup of WAVES waves (a row: a query head of a sequence), or a row per wave: the parts' weights exp(m - max), 16
// bytes of a part's acc to a lane.
template <int DIM, int WAVES>
__global__ __launch_bounds__(256) void attn_paged_merge(tally_attn_paged_args a, PagedPlan p, uint32_t urgent) {
#ifdef __HIP_DEVICE_COMPILE__
  if (urgent) __builtin_amdgcn_s_setprio(3);
  constexpr uint32_t LANES = DIM / 4, SIDE = 64 / LANES;   // parts side by side in a wave
  __shared__ float s_acc[WAVES][DIM];
  __shared__ float s_sum[WAVES];
  const uint32_t lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : threadIdx.x >> 6;
  const uint32_t unit = WAVES == 1 ? same(blockIdx.x * 4 + (threadIdx.x >> 6)) : blockIdx.x;
  if (WAVES == 1 && unit >= a.heads * a.batch) return;
  const uint32_t head = unit % a.heads, seq = unit / a.heads;
  PagedPart mine;
  if (!paged_find(a, p, seq, true, mine) || mine.parts == 1) return;
  const uint64_t row = (uint64_t)mine.first * a.heads + head;
  const float2 *ml = reinterpret_cast<const float2 *>(a.scratch) + row;
  const float *rec = static_cast<const float *>(a.scratch) + paged_acc_at((uint64_t)p.slots * a.heads) + row * DIM + lane % LANES * 4;
  constexpr uint32_t ROUND = WAVES * SIDE, U = 4;          // parts at a time
  const uint32_t first = wave * SIDE + lane / LANES;
  // (the first round's loads do not wait for the weights)
  f32x4_t v[U];
  float2 own[U];
  auto ask = [&](uint32_t i) {
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      own[u] = make_float2(kNothing, kNoTokens);
      if (i + u * ROUND >= mine.parts) continue;
      v[u] = *reinterpret_cast<const f32x4_t *>(rec + (uint64_t)(i + u * ROUND) * a.heads * DIM);
      own[u] = ml[(uint64_t)(i + u * ROUND) * a.heads];
    }
  };
  ask(first);
  float top = kNothing;
  for (uint32_t i = lane; i < mine.parts; i += 64) top = fmaxf(top, ml[(uint64_t)i * a.heads].x);
  top = wave_max(top);
  float sum = 0.f;
  bool any = false;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t i = first;;) {
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      const bool none = own[u].y < 0.f;                    // (a part without tokens has an acc of zeros)
      const float w = none ? 0.f : __builtin_amdgcn_exp2f(own[u].x - top);
      any |= !none;
      sum += none ? 0.f : own[u].y * w;
      acc += v[u] * w;
    }
    i += ROUND * U;
    if (i - first >= mine.parts) break;                    // (the same for every lane)
    ask(i);
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
  any = __builtin_amdgcn_ballot_w64(any) != 0;
  const uint64_t at = (uint64_t)seq * (a.ld_out ? a.ld_out : a.heads * DIM) + head * DIM;
  if constexpr (WAVES == 1) {
    const float over = any ? 1.f / sum : 0.f;
    if (lane < LANES)
      *reinterpret_cast<uint2 *>(a.out + at + lane * 4) = make_uint2(OnePass<DIM, 16, 32, 3>::pack(acc[0] * over, acc[1] * over),
                                                                     OnePass<DIM, 16, 32, 3>::pack(acc[2] * over, acc[3] * over));
  } else {
    if (lane < LANES) *reinterpret_cast<f32x4_t *>(&s_acc[wave][lane * 4]) = acc;
    if (lane == 0) s_sum[wave] = any ? sum : kNoTokens;
    __syncthreads();
    if (threadIdx.x < DIM) {
      const uint32_t d = threadIdx.x;
      const float o = (s_acc[0][d] + s_acc[1][d]) + (s_acc[2][d] + s_acc[3][d]);
      float all = 0.f;
      bool some = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        some |= !(s_sum[i] < 0.f);
        all += s_sum[i] < 0.f ? 0.f : s_sum[i];
      }
      a.out[at + d] = f32_to_bf16(some ? o / all : 0.f);
    }
  }
#endif
}

inline PagedPlan paged_plan(const tally_attn_paged_args &a) { return paged_plan(a.batch, a.heads, a.kv_heads, a.dim, a.page, a.seq_pages); }

template <int DIM>
hipError_t launch_paged_dim(hipStream_t s, const tally_attn_paged_args &a, uint32_t urgent) {
  const PagedPlan p = paged_plan(a);
  auto kernel = a.page == 16 ? (p.past ? attn_paged_partial<DIM, true, true> : attn_paged_partial<DIM, true, false>)
                             : (p.past ? attn_paged_partial<DIM, false, true> : attn_paged_partial<DIM, false, false>);
  const hipError_t e = launch(kernel, dim3(p.slots * a.kv_heads * p.row_tiles), dim3(256), 0, s, a, p, urgent);
  if (e != hipSuccess || p.single) return e;
  if (p.slots <= 6 * a.batch) return launch(attn_paged_merge<DIM, 1>, dim3((a.heads * a.batch + 3) / 4), dim3(256), 0, s, a, p, urgent);
  return launch(attn_paged_merge<DIM, 4>, dim3(a.heads * a.batch), dim3(256), 0, s, a, p, urgent);
}
inline hipError_t launch_attn_paged(hipStream_t s, const void *args, uint32_t urgent) {
  tally_attn_paged_args a;
  memcpy(&a, args, sizeof(a));
  return a.dim == 64 ? launch_paged_dim<64>(s, a, urgent) : launch_paged_dim<128>(s, a, urgent);
}

}  // namespace tally
