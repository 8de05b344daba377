// Single-token attention of a batch whose sequences share a prefix.
//
// Each sequence attends to the prefix's tokens and to its own; softmax over both is the merge of
// softmaxes over parts of them, so the prefix is gone through once for the whole batch: a K/V head's
// queries from all sequences are the rows of one product (batch x group of them), and its K and V are
// read once for as many rows as a workgroup holds.  A sequence's own tokens are the same loop
// with the rows of one sequence.  The tokens are split so that the parts fill the chip; each part leaves
// (max, sum, acc) of its rows in scratch, and a second kernel merges a row's parts.
//
// What bounds it is reading K and V: up to 64 rows the four waves of a workgroup have 16 each
// (24 KB of LDS and 128 registers, so that several share a compute unit and they fit beside a paused
// GEMM tile); with more rows, where the products count, 32 each, as prompts do.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/tally.h"
#include "kernels_flash.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

constexpr uint32_t kPrefixFewRows = 64;                    // rows of a workgroup of 16-row waves
constexpr uint32_t kPrefixManyRows = 128;
constexpr uint32_t kPrefixParts = 128;                     // of the prefix, and of a sequence's own tokens
constexpr uint32_t kPrefixLeast = 128;                     // tokens of a part

struct PrefixPlan {
  uint32_t group, rows;                                    // query heads per K/V head; rows of one K/V head
  uint32_t many;                                           // the prefix's workgroups have 128 rows
  uint32_t row_tiles, own_tiles;                           // of the prefix's rows, of one sequence's
  uint32_t chunk, parts;                                   // tokens of a part of the prefix, and parts
  uint32_t own_chunk, own_parts;
  uint32_t prefix_groups, own_groups;                      // workgroups
};

inline PrefixPlan prefix_plan(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t prefix, uint32_t own_cap) {
  auto up = [](uint64_t a, uint64_t b) { return (a + b - 1) / b; };
  PrefixPlan p;
  p.group = heads / kv_heads;
  p.rows = batch * p.group;
  p.many = prefix && p.rows > kPrefixFewRows;
  p.row_tiles = (uint32_t)up(p.rows, p.many ? kPrefixManyRows : kPrefixFewRows);
  p.own_tiles = (uint32_t)up(p.group, kPrefixFewRows);
  const uint64_t tokens = (uint64_t)kv_heads * p.row_tiles * prefix + (uint64_t)kv_heads * batch * p.own_tiles * own_cap;
  uint64_t chunk = up(tokens, p.many ? 512 : 1024);       // (workgroups that are on the GPU at once)
  if (chunk < kPrefixLeast) chunk = kPrefixLeast;
  auto parts = [&](uint32_t n, uint32_t &c, uint32_t &k) {
    const uint64_t least = up(n, kPrefixParts), w = chunk < least ? least : chunk < n ? chunk : n;
    c = (uint32_t)(up(w ? w : 1, 64) * 64);
    k = (uint32_t)up(n, c);
  };
  parts(prefix, p.chunk, p.parts);
  parts(own_cap, p.own_chunk, p.own_parts);
  p.prefix_groups = kv_heads * p.row_tiles * p.parts;
  p.own_groups = kv_heads * batch * p.own_tiles * p.own_parts;
  return p;
}
inline size_t prefix_scratch_bytes(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t prefix, uint32_t own_cap) {
  const PrefixPlan p = prefix_plan(batch, heads, kv_heads, prefix, own_cap);
  return (size_t)batch * heads * (p.parts + p.own_parts) * (dim + 2) * sizeof(float);
}

// One workgroup's part, the only one it has: tokens [0, n) of K and V at `k` and `v` for rows [row0, row0 + rows) of a K/V head,
// row r being query head r % group of sequence r / group.
template <class F>
__device__ __forceinline__ void prefix_part(const tally_attn_prefix_args &a, const PrefixPlan &p, unsigned char *lds_at, const uint16_t *k,
                                            const uint16_t *v, uint32_t ld, uint32_t n, uint32_t kv, uint32_t row0, uint32_t rows,
                                            uint32_t part) {
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
  auto step = [](uint32_t) {};
  if (n != 0) {
    if constexpr (F::ROWS == 16) f.run_lean(f.source(k, n, ld), f.source(v, n, ld), n, mine < rows ? n : 0u, n, (int32_t)n, c, step);
    else f.template run<false>(typename F::Src(), f.source(k, n, ld), f.source(v, n, ld), n, mine < rows ? n : 0u, n, (int32_t)n, c, step);
  }
  if (!exists) return;
  const uint32_t parts = p.parts + p.own_parts;
  const uint64_t at = ((uint64_t)b * a.heads + head) * parts + part;
  float2 *ml = reinterpret_cast<float2 *>(a.scratch);
  if (f.lane < F::ROWS) ml[at] = make_float2(f.m, f.l);
  float *acc = reinterpret_cast<float *>(ml + (uint64_t)a.batch * a.heads * parts) + at * F::DIM + f.lane / F::ROWS * 4;
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

template <int DIM, bool MANY>
constexpr unsigned prefix_lds() { return MANY ? Flash<DIM, 32, 64, 4>::LDS : Flash<DIM, 16, 32, 3>::LDS; }

template <int DIM, bool MANY>
__global__ __launch_bounds__(256, MANY ? 2 : 4) void attn_prefix_partial(tally_attn_prefix_args a, PrefixPlan p, uint32_t urgent) {
  if (urgent) __builtin_amdgcn_s_setprio(3);
  extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
  typedef Flash<DIM, 16, 32, 3> Few;
  typedef Flash<DIM, 32, 64, 4> Many;
  typedef typename std::conditional<MANY, Many, Few>::type Shared;
  // (beside 128-row workgroups, of which a compute unit has two, in the LDS that those take)
  typedef typename std::conditional<MANY, Flash<DIM, 16, 32, 8>, Few>::type Own;
  static_assert(Own::LDS <= prefix_lds<DIM, MANY>(), "one size for both");
  uint32_t i = blockIdx.x;
  if (i < p.prefix_groups) {
    // the row tiles of one part of one K/V head next to one another on one die (every eighth workgroup is on
    // the same one), so that all but the first find its K and V in that die's L2
    const uint32_t units = a.kv_heads * p.parts, group = i / (8 * p.row_tiles), at8 = i % (8 * p.row_tiles);
    const uint32_t side = units - 8 * group < 8 ? units - 8 * group : 8, tile = at8 / side, unit = 8 * group + at8 % side;
    const uint32_t kv = unit % a.kv_heads, part = unit / a.kv_heads;
    const uint32_t LD = a.ld_prefix ? a.ld_prefix : a.kv_heads * DIM, t0 = part * p.chunk;
    const uint32_t n = a.prefix - t0 < p.chunk ? a.prefix - t0 : p.chunk;
    const uint32_t row0 = tile * Shared::BLOCK_ROWS, left = p.rows - row0;
    const uint64_t at = (uint64_t)t0 * LD + kv * DIM;
    prefix_part<Shared>(a, p, tally_dyn_lds, a.K + at, a.V + at, LD, n, kv, row0,
                        left < (uint32_t)Shared::BLOCK_ROWS ? left : (uint32_t)Shared::BLOCK_ROWS, part);
  } else {
    i -= p.prefix_groups;
    const uint32_t kv = i % a.kv_heads, rest = i / a.kv_heads, b = rest % a.batch, more = rest / a.batch;
    const uint32_t part = more % p.own_parts, tile = more / p.own_parts;
    const uint32_t LD = a.ld_own ? a.ld_own : a.kv_heads * DIM, t0 = part * p.own_chunk;
    const int32_t said = a.own_len[b];
    const uint32_t len = said < 0 ? 0u : (uint32_t)said < a.own_cap ? (uint32_t)said : a.own_cap;
    const uint32_t left = len > t0 ? len - t0 : 0u, n = __builtin_amdgcn_readfirstlane(left < p.own_chunk ? left : p.own_chunk);
    const uint32_t row0 = tile * Own::BLOCK_ROWS, rows = p.group - row0;
    const uint64_t at = (uint64_t)b * (a.stride_own ? a.stride_own : (uint64_t)a.own_cap * LD) + (uint64_t)t0 * LD + kv * DIM;
    prefix_part<Own>(a, p, tally_dyn_lds, a.Ko + at, a.Vo + at, LD, n, kv, b * p.group + row0,
                     rows < (uint32_t)Own::BLOCK_ROWS ? rows : (uint32_t)Own::BLOCK_ROWS, p.parts + part);
  }
}
static_assert(Flash<128, 16, 32, 3>::LDS <= 31 * 1024, "room beside a paused 256 x 256 GEMM tile");

// One row per workgroup: the parts' weights exp(m - max) first, then each wave a quarter of the
// parts, 16 bytes of a part's acc to a lane and eight loads at a time.  A part without tokens has l = 0 and its
// acc was not written: what stands there is not added.
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
  const float *rec = reinterpret_cast<const float *>(reinterpret_cast<const float2 *>(a.scratch) + (uint64_t)a.batch * a.heads * parts) +
                     row * parts * DIM + lane % LANES * 4;
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
    own[i] = make_float2(kNothing, 0.f);
    if (lane + 64 * i < parts) own[i] = ml[lane + 64 * i];
    top = fmaxf(top, own[i].x);
  }
  top = wave_max(top);
  float sum = 0.f;
#pragma unroll
  for (uint32_t i = 0; i < 2 * kPrefixParts / 64; ++i) {
    const float w = own[i].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(own[i].x - top);
    sum += own[i].y == 0.f ? 0.f : own[i].y * w;
    if (wave == 0) s_w[lane + 64 * i] = w;
  }
  if (wave == 0 && lane < ROUND * U) s_w[2 * kPrefixParts + lane] = 0.f;
  sum = wave_sum(sum);
  __syncthreads();
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t i = mine;;) {
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) {
      const float w = s_w[i + u * ROUND];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += w == 0.f ? 0.f : w * v[u][e];
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
    a.out[(uint64_t)b * LDO + head * DIM + d] = f32_to_bf16(sum == 0.f ? 0.f : o / sum);
  }
#endif
}

inline PrefixPlan prefix_plan(const tally_attn_prefix_args &a) { return prefix_plan(a.batch, a.heads, a.kv_heads, a.prefix, a.own_cap); }

template <int DIM>
hipError_t launch_prefix_dim(hipStream_t s, const tally_attn_prefix_args &a, uint32_t urgent) {
  const PrefixPlan p = prefix_plan(a);
  const uint32_t groups = p.prefix_groups + p.own_groups;
  if (groups) {
    const hipError_t e = launch(p.many ? attn_prefix_partial<DIM, true> : attn_prefix_partial<DIM, false>, dim3(groups), dim3(256),
                                p.many ? prefix_lds<DIM, true>() : prefix_lds<DIM, false>(), s, a, p, urgent);
    if (e != hipSuccess) return e;
  }
  return launch(attn_prefix_combine<DIM>, dim3(a.heads * a.batch), dim3(256), 0, s, a, p, urgent);
}
inline hipError_t launch_attn_prefix(hipStream_t s, const void *args, uint32_t urgent) {
  tally_attn_prefix_args a;
  memcpy(&a, args, sizeof(a));
  return a.dim == 64 ? launch_prefix_dim<64>(s, a, urgent) : launch_prefix_dim<128>(s, a, urgent);
}

}  // namespace tally
