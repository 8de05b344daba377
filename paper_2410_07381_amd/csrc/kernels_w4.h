// Matrix-vector products with 4-bit weights and group scales for gfx950: up to 16 vectors at once.
//
// y[v][r] = sum over groups g of s[r][g] * sum over k of g of (code[r][k] - zero[r][g]) x[v][k].
//
// What bounds it is reading the codes, half a byte each.  A code becomes a bf16 with one AND-OR for
// two of them: 0x4300 | code is 128 + code.  The 128 and the zero point are taken out again by a second
// MFMA with the constant -(128 + zero), which is exact in bf16, so that a group's sum has the
// rounding of fp32 alone; then the scale is applied, in fp32.  The vectors are the 16 rows of an MFMA,
// weight rows its columns, so one vector costs what sixteen do and a lane needs the scale of one row.
//
// The codes lie in memory as the lanes want them: a tile is 16 rows by 128 weights, 1 KB that a wave
// reads with one 16-byte load a lane; word i of lane 16 q + r holds weights 32 i + 8 q to 32 i + 8 q + 7
// of row r, the even ones in its low half.  So MFMA i of a tile takes 32 neighbouring weights of each
// row, which always belong to one group.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tally.h"
#include "kernels_gemm.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

constexpr uint32_t kW4Rows = 16, kW4Block = 128, kW4Vectors = 16;

// SUB: MFMAs of a tile that share a scale (groups of 32, of 64, of 128 and more)
template <int SUB>
struct GemvW4BodyT {
  using Args = tally_gemv_w4_args;
  static constexpr int THREADS = 256;
  static constexpr int MIN_WAVES = 4;
  static constexpr unsigned DYN_LDS = 0;
  static constexpr bool YIELDS = false;
  static constexpr bool RANGE = false;
  static constexpr bool END_BARRIER = true;                // (the waves' sums are joined in LDS)
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) { run_t(a, bx); }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) { run_t(a, bx); }
  static __device__ __forceinline__ void run_t(const Args &a, uint32_t tile) {
#ifdef __HIP_DEVICE_COMPILE__
    __shared__ f32x4_t s_acc[4][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t col = lane & 15, quarter = lane >> 4;
    const uint32_t blocks = (a.k + kW4Block - 1) / kW4Block, groups = (a.k + a.group - 1) / a.group;
    const uint32_t LDX = a.ld_x ? a.ld_x : a.k;
    const uint4 *W = reinterpret_cast<const uint4 *>(a.W) + (uint64_t)tile * blocks * 64 + lane;
    const buf_t scales = make_buf(a.scales + (uint64_t)tile * groups * 16, groups * 32);
    const buf_t zeros = make_buf(a.zeros ? a.zeros + (uint64_t)tile * groups * 16 : nullptr, a.zeros ? groups * 16 : 0);
    const buf_t x = make_buf(a.x, 0x7fffffff);
    const uint32_t xrow = col < a.m ? (col * LDX + quarter * 8) * 2 : 0x80000000u;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t b = wave; b < blocks; b += 4) {
      const uint4 w = W[(uint64_t)b * 64];
      const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int g = 0; g < 4; g += SUB) {
        const uint32_t k0 = b * kW4Block + g * 32, at = k0 / a.group;
        const float s = bf16_lo(__builtin_amdgcn_raw_buffer_load_b16(scales, (at * 16 + col) * 2, 0, 0));
        const uint32_t z = a.zeros ? __builtin_amdgcn_raw_buffer_load_b8(zeros, at * 16 + col, 0, 0) : 8u;
        const uint32_t c = __float_as_uint(-(float)(128u + z)) >> 16, cc = c << 16 | c;
        f32x4_t part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = g; i < g + SUB; ++i) {
          // (8 elements of x at a time: k is a multiple of 8, and past it x counts as zero)
          const uint32_t k1 = b * kW4Block + i * 32;
          const uint32_t off = k1 + quarter * 8 < a.k ? xrow + k1 * 2 : 0x80000000u;
          const bf16x8_t xv = __builtin_bit_cast(bf16x8_t, buf_ld16(x, off, 0));
          uint32_t q[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) q[j] = (word[i] >> (4 * j) & 0x000F000Fu) | 0x43004300u;
          part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, __builtin_bit_cast(bf16x8_t, make_uint4(q[0], q[1], q[2], q[3])), part, 0, 0, 0);
          part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, __builtin_bit_cast(bf16x8_t, make_uint4(cc, cc, cc, cc)), part, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(s, part[e], acc[e]);
      }
    }
    s_acc[wave][lane] = acc;
    __syncthreads();
    // lane 16 q + r, element e: vector 4 q + e, row r
    const uint32_t v = threadIdx.x >> 4, r = threadIdx.x & 15, from = (v >> 2) * 16 + r, e = v & 3, row = tile * kW4Rows + r;
    if (v < a.m && row < a.n) {
      const float y = (s_acc[0][from][e] + s_acc[1][from][e]) + (s_acc[2][from][e] + s_acc[3][from][e]);
      a.y[(uint64_t)v * (a.ld_y ? a.ld_y : a.n) + row] = f32_to_bf16(y);
    }
#endif
  }
};

}  // namespace tally
