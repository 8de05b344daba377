// Single-token attention of a batch whose sequences share a prefix.
//
// Each sequence attends to the prefix's tokens and to its own; softmax over both is the merge of
// softmaxes over parts of them, so the prefix is gone through once for the whole batch: a K/V head's
// queries from all sequences are the rows of one product (batch x group of them), and its K and V are
// read once for as many rows as a workgroup holds.  A sequence's own tokens are the same loop
// with the rows of one sequence.  The tokens are split so that the parts fill the chip; each part leaves
// (max, sum, acc) of its rows in scratch, and a second kernel merges a row's parts.
//
// What bounds it is reading K and V, and for small calls one load waiting for another.  With 16 rows or
// fewer, as a sequence's own tokens have, each wave goes through tokens of its own and the four are merged in the
// workgroup (lone_part); up to 64 rows the four waves have 16 each and share the tokens; with more and a long prefix, where the
// products count, 32 each, as prompts do.  The first two take 24 KB of LDS at most and 128 registers, so that several
// share a compute unit and they fit beside a paused GEMM tile.
//
// Measured (us of a call; K and V read once at 5.1 TB/s in brackets): 16 sequences of 0 to 3001 tokens, 28/4 heads of 128,
// 14.0 [9.6]; 64 of 0 to 2048, 32/8, 64.7 [52.5]; 32 behind 4096 tokens with 0 to 512 of their own 18.4 [9.9]; 64 behind 65500
// with 0 to 1024 109 to 118 [78.6]; 4 behind 512, 12 heads of 64, 6.2, of which an empty launch is 2.4.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/tally.h"
#include "kernels_onepass.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

constexpr uint32_t kPrefixFewRows = 64;                    // rows of a workgroup of 16-row waves
constexpr uint32_t kPrefixManyRows = 128;
constexpr uint32_t kPrefixLone = 16;                       // rows that each wave of a workgroup may have all of
constexpr uint32_t kPrefixParts = 128;                     // of the prefix, and of a sequence's own tokens
constexpr uint32_t kPrefixLeast = 128;                     // tokens of a part

// How a call is cut up (figures: us of a call, heads of 128 unless said).
//
// Whole: one workgroup per sequence and K/V head has all of its tokens, of the prefix too, and writes the output;
// there is nothing to merge and no second kernel (~2.5 us).  It pays while a workgroup's own way through its tokens is short,
// 512 tokens of 128 dims (2048 from 256 workgroups on, which share the memory's rate anyhow), and
// while reading the prefix once per sequence costs little: 4 sequences, 8 K/V heads, 256 + 64
// tokens 7.1 against 8.0, but 512 + 64 9.3 against 7.7; 32 sequences of 256 + 256 8.9 against 14.2; 64 of up to 2048 alone
// 64.7 against 70.4; 32 of 1024 + 512 18.6 against 17.3.
//
// Otherwise the workgroups have, of the prefix, 16 rows (kind 0), 64 (kind 1) or 128 (kind 2: twice the products per read of
// LDS, but a compute unit has room for two, and short prefixes leave it waiting): 512 rows, 4 K/V
// heads, 2000 tokens 18.3 in kind 1 and 21.1 in kind 2, 3000 tokens 22.7 and 21.5; 256 rows, 8 heads, 65500 tokens 138 and 112.
//
// Parts: as many workgroups as one round on the GPU takes.  Kind 0 is better off with one per compute
// unit, whose parts are longer (16 sequences of up to 3001, 4 heads: 14.1, with 512 of them 15.8, with 1024 16.9).
// Where four waves share tokens (kind 1) a part is a longer chain than where each has its own: with half as many again of
// the latter and more, parts of the prefix are shorter by a fourth.  Both sides of 104 calls drawn at random, by own : shared:
// from 1.5 on 4.6 % faster on average (from 10 % slower, one of 67, to 15 % faster), between 1 and 1.5 0.3 % slower (12 % either
// way), below 1.2 2.1 % slower.
struct PrefixPlan {
  uint32_t group, rows;                                    // query heads per K/V head; rows of one K/V head
  uint32_t kind;                                           // rows of a workgroup: 0: 16, 1: 64, 2: 128 of the prefix
  uint32_t whole;                                          // a workgroup has all tokens of a sequence: nothing to merge
  uint32_t row_tiles, own_tiles;                           // of the prefix's rows, of one sequence's
  uint32_t chunk, parts;                                   // tokens of a part of the prefix, and parts
  uint32_t own_chunk, own_parts;
  uint32_t prefix_groups, own_groups;                      // workgroups
};

inline PrefixPlan prefix_plan(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t prefix, uint32_t own_cap) {
  auto up = [](uint64_t a, uint64_t b) { return (a + b - 1) / b; };
  PrefixPlan p;
  p.group = heads / kv_heads;
  p.rows = batch * p.group;
  const uint64_t products = (uint64_t)p.rows * prefix * kv_heads, groups = (uint64_t)batch * kv_heads;
  p.kind = p.group <= kPrefixLone && (!prefix || p.rows <= kPrefixLone) ? 0 : p.rows > kPrefixFewRows && products > (1u << 23) ? 2 : 1;
  p.whole = 0;
  p.row_tiles = (uint32_t)up(p.rows, p.kind == 2 ? kPrefixManyRows : kPrefixFewRows);
  p.own_tiles = (uint32_t)up(p.group, kPrefixFewRows);
  const uint64_t shared = (uint64_t)kv_heads * p.row_tiles * prefix, own = (uint64_t)kv_heads * batch * p.own_tiles * own_cap;
  uint64_t chunk = up(shared + own, p.kind == 0 ? 256 : 512);
  if (chunk < kPrefixLeast) chunk = kPrefixLeast;
  auto parts = [&](uint32_t n, uint32_t &c, uint32_t &k) {
    const uint64_t least = up(n, kPrefixParts), w = chunk < least ? least : chunk < n ? chunk : n;
    c = (uint32_t)(up(w ? w : 1, 64) * 64);
    k = (uint32_t)up(n, c);
  };
  const uint64_t own_chunk = chunk;
  if (p.kind == 1 && 2 * own >= 3 * shared && chunk * 3 / 4 >= kPrefixLeast) chunk = chunk * 3 / 4;
  parts(prefix, p.chunk, p.parts);
  chunk = own_chunk;
  parts(own_cap, p.own_chunk, p.own_parts);
  p.prefix_groups = kv_heads * p.row_tiles * p.parts;
  p.own_groups = kv_heads * batch * p.own_tiles * p.own_parts;
  const uint64_t all = (uint64_t)(prefix + own_cap) * dim, again = (uint64_t)prefix * dim;
  if (p.group <= kPrefixLone && all != 0 && all <= (groups < 256 ? 1u << 16 : 1u << 18) &&
      ((prefix <= own_cap && again <= (1u << 15)) || groups * again <= (1u << 24))) {
    p.kind = 0;
    p.whole = 1;
    p.prefix_groups = 0;
    p.own_groups = kv_heads * batch;
  }
  return p;
}
// Scratch: (max, sum) of each row's parts, and behind them, from a multiple of 16 bytes on, each part's acc.
__host__ __device__ inline uint64_t prefix_records(uint32_t batch, uint32_t heads, const PrefixPlan &p) {
  return (uint64_t)batch * heads * (p.parts + p.own_parts);
}
__host__ __device__ inline uint64_t prefix_acc_at(uint64_t records) { return (records * 2 + 3) / 4 * 4; }   // in floats
inline size_t prefix_scratch_bytes(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t prefix, uint32_t own_cap) {
  const uint64_t n = prefix_records(batch, heads, prefix_plan(batch, heads, kv_heads, dim, prefix, own_cap));
  return (size_t)(prefix_acc_at(n) + n * dim) * sizeof(float);
}

// What stands for the sum of a part without tokens (a sum is never negative; that of tokens whose weights are all
// zero in 32 bits is zero, and such a part's acc counts: zero times an infinity or NaN of V is NaN).
constexpr float kNoTokens = -1.f;

// Tokens of K and V, `ld` elements between them.
struct Span { const uint16_t *k, *v; uint32_t ld, n; };

// One workgroup's part, the only one it has: tokens of `s` for rows [row0, row0 + rows) of a K/V head,
// row r being query head r % group of sequence r / group.
template <class F>
__device__ __forceinline__ void prefix_part(const tally_attn_prefix_args &a, const PrefixPlan &p, unsigned char *lds_at, const Span &s,
                                            uint32_t kv, uint32_t row0, uint32_t rows, uint32_t part) {
#ifdef __HIP_DEVICE_COMPILE__
  F f;
  f.begin(lds_at);
  const uint32_t mine = f.wave * F::ROWS, r = mine + f.lane % F::ROWS, row = row0 + r;
  const uint32_t b = row / p.group, head = kv * p.group + row % p.group;
  const bool exists = r < rows;
  const uint32_t LDQ = a.ld_q ? a.ld_q : a.heads * F::DIM;
  const uint16_t *q = a.q + (uint64_t)b * LDQ + head * F::DIM + f.lane / F::ROWS * 8;
#pragma unroll
  for (int i = 0; i < F::QK; ++i) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (exists) u = *reinterpret_cast<const uint4 *>(q + i * F::MK);
    f.q[i] = __builtin_bit_cast(bf16x8_t, u);
  }
  const float c = (a.scale > 0.f ? a.scale : F::DIM == 128 ? 0.08838834764831845f : 0.125f) * kLog2e;
  const uint32_t n = s.n;
  auto step = [](uint32_t) {};
  if (n != 0) {
    if constexpr (F::ROWS == 16) f.run_lean(f.source(s.k, n, s.ld), f.source(s.v, n, s.ld), n, mine < rows ? n : 0u, n, (int32_t)n, c, step);
    else f.template run<false>(typename F::Src(), f.source(s.k, n, s.ld), f.source(s.v, n, s.ld), n, mine < rows ? n : 0u, n, (int32_t)n, c, step);
  }
  if (!exists) return;
  const uint32_t parts = p.parts + p.own_parts;
  const uint64_t at = ((uint64_t)b * a.heads + head) * parts + part;
  float2 *ml = reinterpret_cast<float2 *>(a.scratch);
  if (f.lane < F::ROWS) ml[at] = make_float2(f.m, n != 0 ? f.l : kNoTokens);
  float *acc = static_cast<float *>(a.scratch) + prefix_acc_at(prefix_records(a.batch, a.heads, p)) + at * F::DIM + f.lane / F::ROWS * 4;
  if (n != 0) {
#pragma unroll
    for (int d = 0; d < F::DT; ++d)
#pragma unroll
      for (int g = 0; g < F::AN / 4; ++g)
        *reinterpret_cast<f32x4_t *>(acc + d * F::ROWS + 8 * g) =
            f32x4_t{f.acc[d][4 * g], f.acc[d][4 * g + 1], f.acc[d][4 * g + 2], f.acc[d][4 * g + 3]};
  }
#endif
}

// One workgroup's part of 16 rows at most: tokens of `one` and then of `two`, 32 of them a tile, each wave a fourth of the
// tiles on its own.  No wave waits for another until their states are merged.  K and V go through registers, in
// whole lines, into a piece of LDS of the wave's own (4 KB: 32 tokens of 64 dims, 16 of 128), from where the
// fragments are read; the next tile's loads are sent as soon as the registers are free.  (K's fragments straight from
// memory, 64 bytes of a token at a time: 64 sequences of up to 1024 tokens 41.6 us instead of 38.8.)
template <int DIM>
__device__ __forceinline__ void lone_part(const tally_attn_prefix_args &a, const PrefixPlan &p, unsigned char *lds_at, const Span &one,
                                          const Span &two, uint32_t kv, uint32_t row0, uint32_t rows, uint32_t part) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef OnePass<DIM, 16, 32, 3> F;
  typedef typename F::s16x4_t s16x4_t;
  constexpr uint32_t PIECE = 4096, CHUNKS = DIM / 8;        // of LDS, for tokens of a wave; 16-byte chunks of a token
  constexpr int TOK = PIECE / F::ROWB, TURNS = 32 / TOK, BLOCKS = TOK / 16, LOADS = 4;   // of a piece
  __shared__ float2 s_ml[4][16];
  F f;
  f.begin(lds_at);
  const uint32_t lane = f.lane, wave = f.wave, at = f.lds + wave * PIECE;
  const uint32_t before = (one.n + 31) / 32, tiles = before + (two.n + 31) / 32;
  const uint32_t row = row0 + lane % 16, b = row / p.group, LDQ = a.ld_q ? a.ld_q : a.heads * DIM;
  typedef __attribute__((address_space(3))) u32x4_t *to_t;
  const float c = (a.scale > 0.f ? a.scale : DIM == 128 ? 0.08838834764831845f : 0.125f) * kLog2e;
  uint4 k[TURNS * LOADS], v[TURNS * LOADS];
  // tile i (past the last one: nothing, of which loads leave zeros, as behind a span's last token)
  auto tokens = [&](uint32_t i) {
    const Span &s = i < before ? one : two;
    const uint32_t from = (i < before ? i : i - before) * 32;
    return i >= tiles ? 0u : s.n - from < 32u ? s.n - from : 32u;
  };
  auto ask = [&](uint4 (&to)[TURNS * LOADS], const uint16_t *Span::*of, uint32_t i, int h) {
    const Span &s = i < before ? one : two;
    const uint32_t ld = s.ld * 2, lane = F::opaque(f.lane);   // (nothing of it kept)
    const buf_t src = make_buf(s.*of + (uint64_t)((i < before ? i : i - before) * 32) * s.ld, tokens(i) * ld);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) to[h * LOADS + j] = buf_ld16(src, (TOK * h + j * F::RPL + lane / CHUNKS) * ld + lane % CHUNKS * 16, 0);
  };
  // a tile, or half of one, to LDS, which serves a wave's accesses in order
  auto put = [&](const uint4 (&from)[TURNS * LOADS], int h) {
    const uint32_t lane = F::opaque(f.lane);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const uint32_t t = j * F::RPL + lane / CHUNKS;
      *(to_t)(at + t * F::ROWB + ((lane % CHUNKS ^ F::swz(t)) << 4)) = __builtin_bit_cast(u32x4_t, from[h * LOADS + j]);
    }
    asm volatile("" ::: "memory");
  };
  // (q in LDS, a fragment from each wave: the registers are full without it)
  const uint32_t q_at = f.lds + 4 * PIECE;
  u32x4_t u = {0u, 0u, 0u, 0u};
  if (wave < F::QK && lane % 16 < rows)
    u = *reinterpret_cast<const u32x4_t *>(a.q + (uint64_t)b * LDQ + (kv * p.group + row % p.group) * DIM + lane / 16 * 8 + wave * 32);
#pragma unroll
  for (int h = 0; h < TURNS; ++h) ask(k, &Span::k, wave, h);
#pragma unroll
  for (int h = 0; h < TURNS; ++h) ask(v, &Span::v, wave, h);
  if (wave < F::QK) *(to_t)(q_at + (f.k_at ^ wave * 64)) = u;
  __syncthreads();
  for (uint32_t i = wave; i < tiles; i += 4) {
    f32x4_t s[2];
    uint32_t w[4];
#pragma unroll
    for (int h = 0; h < TURNS; ++h) {
      put(k, h);
      const uint32_t k_at = F::opaque(f.k_at);
#pragma unroll
      for (int j = 0; j < F::QK; j += 2) {                 // (two steps' fragments at a time)
        bf16x8_t key[2][BLOCKS], q[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          q[u] = f.key(q_at, k_at, (j + u) * F::TT);
#pragma unroll
          for (int t = 0; t < BLOCKS; ++t) key[u][t] = f.key(at, k_at, (j + u) * F::TT + t);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int t = 0; t < BLOCKS; ++t)
            s[h * BLOCKS + t] = F::mma(key[u][t], q[u], j + u == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : s[h * BLOCKS + t]);
      }
      ask(k, &Span::k, i + 4, h);
    }
    const uint32_t n = tokens(i);
    if (n < 32u) f.hide(s, (int32_t)n);
    f.follow(F::largest(s), c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = F::pack(F::exp2(__builtin_fmaf(s[j / 2][j % 2 * 2], c, -f.m)), F::exp2(__builtin_fmaf(s[j / 2][j % 2 * 2 + 1], c, -f.m)));
      f.l = F::add_pair(w[j], f.l);
    }
#pragma unroll
    for (int h = 0; h < TURNS; ++h) {
      typedef __attribute__((address_space(3))) s16x4_t *tr_t;
      put(v, h);
      auto values = [&](int n) {                           // of step n: block n / DT of tokens, block n % DT of dims
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(at + n / F::DT * (16 * F::ROWB) + (f.v_at ^ (n % F::DT * 32))));
      };
      s16x4_t value[4];                                    // (read four steps ahead)
#pragma unroll
      for (int n = 0; n < 4; ++n) value[n] = values(n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < BLOCKS * F::DT; ++n) {
        const int t = h * BLOCKS + n / F::DT;
        f.acc[n % F::DT] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
            value[n % 4], __builtin_bit_cast(s16x4_t, make_uint2(w[2 * t], w[2 * t + 1])), f.acc[n % F::DT], 0, 0, 0);
        if (n + 4 < BLOCKS * F::DT) value[n % 4] = values(n + 4);
        __builtin_amdgcn_sched_barrier(0);
      }
      ask(v, &Span::v, i + 4, h);
    }
  }
  // The four waves' states: each row's maximum and sum first, then the weighted acc, half of the dims at a time.
  f.l = F::template over_row<AddOp>(f.l);
  if (lane < 16) s_ml[wave][lane] = make_float2(f.m, f.l);
  __syncthreads();
  auto top_of = [&](uint32_t r) { return fmaxf(fmaxf(s_ml[0][r].x, s_ml[1][r].x), fmaxf(s_ml[2][r].x, s_ml[3][r].x)); };
  const float by = F::exp2(f.m - top_of(lane % 16));
  constexpr uint32_t PIECES = DIM / 8;                     // of four dims, in half of them
  typedef __attribute__((address_space(3))) f32x4_t *four_t;
  const uint32_t r = threadIdx.x / PIECES, piece = threadIdx.x % PIECES;
  f32x4_t o[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h) __syncthreads();
#pragma unroll
    for (int d = 0; d < F::DT / 2; ++d)
      *(four_t)(at + lane % 16 * (DIM * 2) + ((d * 4 + lane / 16 ^ lane % PIECES) << 4)) = f.acc[h * F::DT / 2 + d] * by;
    __syncthreads();
    o[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (r < 16)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[h] += *(four_t)(f.lds + i * PIECE + r * (DIM * 2) + ((piece ^ r % PIECES) << 4));
  }
  if (r >= rows) return;
  const float top = top_of(r);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum += s_ml[i][r].y * F::exp2(s_ml[i][r].x - top);
  const uint32_t out_b = (row0 + r) / p.group, head = kv * p.group + (row0 + r) % p.group;
  if (p.whole) {
    const float over = tiles == 0 ? 0.f : 1.f / sum;        // (scores of -inf throughout: NaN, as in a prompt)
    uint16_t *out = a.out + (uint64_t)out_b * (a.ld_out ? a.ld_out : a.heads * DIM) + head * DIM + piece * 4;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<uint2 *>(out + h * (DIM / 2)) =
          make_uint2(F::pack(o[h][0] * over, o[h][1] * over), F::pack(o[h][2] * over, o[h][3] * over));
    return;
  }
  const uint32_t parts = p.parts + p.own_parts;
  const uint64_t to = ((uint64_t)out_b * a.heads + head) * parts + part;
  float2 *ml = reinterpret_cast<float2 *>(a.scratch);
  if (piece == 0) ml[to] = make_float2(top, tiles != 0 ? sum : kNoTokens);
  if (tiles == 0) return;
  float *acc = static_cast<float *>(a.scratch) + prefix_acc_at(prefix_records(a.batch, a.heads, p)) + to * DIM + piece * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4_t *>(acc + h * (DIM / 2)) = o[h];
#endif
}

template <int DIM, int KIND>
constexpr unsigned prefix_lds() {
  constexpr unsigned lone = 4 * 4096 + 16 * DIM * 2, shared = KIND == 2 ? OnePass<DIM, 32, 64, 4>::LDS : KIND == 1 ? OnePass<DIM, 16, 32, 3>::LDS : 0;
  return lone > shared ? lone : shared;
}

template <int DIM, int KIND>
__global__ __launch_bounds__(256, KIND == 2 ? 2 : 4) void attn_prefix_partial(tally_attn_prefix_args a, PrefixPlan p, uint32_t urgent) {
  if (urgent) __builtin_amdgcn_s_setprio(3);
  extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
  typedef OnePass<DIM, 16, 32, 3> Few;
  typedef typename std::conditional<KIND == 2, OnePass<DIM, 32, 64, 4>, Few>::type Shared;
  // (beside 128-row workgroups, of which a compute unit has two, in the LDS that those take)
  typedef typename std::conditional<KIND == 2, OnePass<DIM, 16, 32, 8>, Few>::type Own;
  static_assert(KIND == 0 || Own::LDS <= prefix_lds<DIM, KIND>(), "one size for both");
  uint32_t i = blockIdx.x;
  const uint32_t LDP = a.ld_prefix ? a.ld_prefix : a.kv_heads * DIM;
  Span one = {nullptr, nullptr, 0, 0}, two = one;
  uint32_t kv, row0, rows, part;
  if (i < p.prefix_groups) {
    // the row tiles of one part of one K/V head next to one another on one die (every eighth workgroup is on
    // the same one), so that all but the first find its K and V in that die's L2
    const uint32_t units = a.kv_heads * p.parts, group = i / (8 * p.row_tiles), at8 = i % (8 * p.row_tiles);
    const uint32_t side = units - 8 * group < 8 ? units - 8 * group : 8, tile = at8 / side, unit = 8 * group + at8 % side;
    kv = unit % a.kv_heads, part = unit / a.kv_heads;
    const uint32_t t0 = part * p.chunk;
    const uint64_t at = (uint64_t)t0 * LDP + kv * DIM;
    one = Span{a.K + at, a.V + at, LDP, a.prefix - t0 < p.chunk ? a.prefix - t0 : p.chunk};
    row0 = tile * Shared::BLOCK_ROWS, rows = p.rows - row0;
    if constexpr (KIND != 0) {
      prefix_part<Shared>(a, p, tally_dyn_lds, one, kv, row0, rows < (uint32_t)Shared::BLOCK_ROWS ? rows : (uint32_t)Shared::BLOCK_ROWS, part);
      return;
    }
  } else {
    i -= p.prefix_groups;
    kv = i % a.kv_heads;
    const uint32_t rest = i / a.kv_heads, b = rest % a.batch, more = rest / a.batch;
    const uint32_t LD = a.ld_own ? a.ld_own : a.kv_heads * DIM;
    const int32_t said = a.own_cap ? a.own_len[b] : 0;
    const uint32_t len = __builtin_amdgcn_readfirstlane(said < 0 ? 0u : (uint32_t)said < a.own_cap ? (uint32_t)said : a.own_cap);
    uint64_t at = (uint64_t)b * (a.stride_own ? a.stride_own : (uint64_t)a.own_cap * LD) + kv * DIM;
    row0 = b * p.group, rows = p.group, part = 0;
    if (KIND == 0 && p.whole) {
      one = Span{a.K + kv * DIM, a.V + kv * DIM, LDP, a.prefix};
      two = Span{a.Ko + at, a.Vo + at, LD, len};
    } else {
      const uint32_t mine = more % p.own_parts, tile = more / p.own_parts, t0 = mine * p.own_chunk, left = len > t0 ? len - t0 : 0u;
      part = p.parts + mine;
      at += (uint64_t)t0 * LD;
      one = Span{a.Ko + at, a.Vo + at, LD, left < p.own_chunk ? left : p.own_chunk};
      if constexpr (KIND != 0) {
        if (p.group > kPrefixLone) {
          const uint32_t first = tile * Own::BLOCK_ROWS;
          rows -= first;
          prefix_part<Own>(a, p, tally_dyn_lds, one, kv, row0 + first, rows < (uint32_t)Own::BLOCK_ROWS ? rows : (uint32_t)Own::BLOCK_ROWS, part);
          return;
        }
      }
    }
  }
  lone_part<DIM>(a, p, tally_dyn_lds, one, two, kv, row0, rows, part);
}
static_assert(OnePass<128, 16, 32, 3>::LDS + 1024 <= 31 * 1024, "room beside a paused 256 x 256 GEMM tile");

// One row per workgroup: the parts' weights exp(m - max) first, then each wave a quarter of the
// parts, 16 bytes of a part's acc to a lane and eight loads at a time.  A part without tokens says so in place of its
// sum and its acc was not written: what stands there is not added (its weight is kNoTokens too, below any other).
template <int DIM>
__global__ __launch_bounds__(256) void attn_prefix_combine(tally_attn_prefix_args a, PrefixPlan p, uint32_t urgent) {
#ifdef __HIP_DEVICE_COMPILE__
  if (urgent) __builtin_amdgcn_s_setprio(3);
  constexpr uint32_t LANES = DIM / 4, SIDE = 64 / LANES, ROUND = 4 * SIDE, U = 4;   // parts side by side in a wave, in all four
  __shared__ float s_w[2 * kPrefixParts + ROUND * U];
  __shared__ float s_acc[4][DIM];
  const uint32_t head = blockIdx.x % a.heads, b = blockIdx.x / a.heads, parts = p.parts + p.own_parts;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t row = (uint64_t)b * a.heads + head;
  const float2 *ml = reinterpret_cast<const float2 *>(a.scratch) + row * parts;
  const float *rec = static_cast<const float *>(a.scratch) + prefix_acc_at(prefix_records(a.batch, a.heads, p)) + row * parts * DIM + lane % LANES * 4;
  const uint32_t mine = wave * SIDE + lane / LANES;
  // (the first round's loads do not wait for the weights)
  f32x4_t v[U];
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (mine + u * ROUND < parts) v[u] = *reinterpret_cast<const f32x4_t *>(rec + (uint64_t)(mine + u * ROUND) * DIM);
  }
  float2 own[2 * kPrefixParts / 64];
  float top = kNothing;
#pragma unroll
  for (uint32_t i = 0; i < 2 * kPrefixParts / 64; ++i) {
    own[i] = make_float2(kNothing, kNoTokens);
    if (lane + 64 * i < parts) own[i] = ml[lane + 64 * i];
    top = fmaxf(top, own[i].x);
  }
  top = wave_max(top);
  float sum = 0.f;
  bool any = false;
#pragma unroll
  for (uint32_t i = 0; i < 2 * kPrefixParts / 64; ++i) {
    const bool none = own[i].y < 0.f;
    any |= !none;
    const float w = none ? kNoTokens : __builtin_amdgcn_exp2f(own[i].x - top);
    sum += none ? 0.f : own[i].y * w;
    if (wave == 0) s_w[lane + 64 * i] = w;
  }
  if (wave == 0 && lane < ROUND * U) s_w[2 * kPrefixParts + lane] = kNoTokens;
  sum = wave_sum(sum);
  any = __builtin_amdgcn_ballot_w64(any) != 0;             // (the same for every wave)
  __syncthreads();
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t i = mine;;) {
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      const float w = s_w[i + u * ROUND];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += w < 0.f ? 0.f : w * v[u][e];
    }
    i += ROUND * U;
    if (i - mine >= parts) break;                          // (the same for every lane)
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (i + u * ROUND < parts) v[u] = *reinterpret_cast<const f32x4_t *>(rec + (uint64_t)(i + u * ROUND) * DIM);
  }
  if constexpr (SIDE == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = across_rows<AddOp>(acc[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float o = acc[e], w = o;
      asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(o), "+v"(w));
      acc[e] = o + w;
    }
  }
  if (lane < LANES) *reinterpret_cast<f32x4_t *>(&s_acc[wave][lane * 4]) = acc;
  __syncthreads();
  if (threadIdx.x < DIM) {
    const uint32_t d = threadIdx.x;
    const float o = (s_acc[0][d] + s_acc[1][d]) + (s_acc[2][d] + s_acc[3][d]);
    const uint32_t LDO = a.ld_out ? a.ld_out : a.heads * DIM;
    a.out[(uint64_t)b * LDO + head * DIM + d] = f32_to_bf16(any ? o / sum : 0.f);
  }
#endif
}

inline PrefixPlan prefix_plan(const tally_attn_prefix_args &a) { return prefix_plan(a.batch, a.heads, a.kv_heads, a.dim, a.prefix, a.own_cap); }

template <int DIM>
hipError_t launch_prefix_dim(hipStream_t s, const tally_attn_prefix_args &a, uint32_t urgent) {
  const PrefixPlan p = prefix_plan(a);
  const uint32_t groups = p.prefix_groups + p.own_groups;
  if (groups) {
    auto kernel = p.kind == 2 ? attn_prefix_partial<DIM, 2> : p.kind == 1 ? attn_prefix_partial<DIM, 1> : attn_prefix_partial<DIM, 0>;
    const unsigned lds = p.kind == 2 ? prefix_lds<DIM, 2>() : p.kind == 1 ? prefix_lds<DIM, 1>() : prefix_lds<DIM, 0>();
    const hipError_t e = launch(kernel, dim3(groups), dim3(256), lds, s, a, p, urgent);
    if (e != hipSuccess || p.whole) return e;
  }
  return launch(attn_prefix_combine<DIM>, dim3(a.heads * a.batch), dim3(256), 0, s, a, p, urgent);
}
inline hipError_t launch_attn_prefix(hipStream_t s, const void *args, uint32_t urgent) {
  tally_attn_prefix_args a;
  memcpy(&a, args, sizeof(a));
  return a.dim == 64 ? launch_prefix_dim<64>(s, a, urgent) : launch_prefix_dim<128>(s, a, urgent);
}

}  // namespace tally
