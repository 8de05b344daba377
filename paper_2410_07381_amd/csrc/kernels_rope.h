// Rotary positions for gfx950: pairs of a head's dims turned by position * frequency.
//
// With a the angle of a pair, (x1, x2) -> (x1 cos a - x2 sin a, x2 cos a + x1 sin a).  The angle of a far position
// needs more bits than fp32 has (position 2^20, one radian a position: 2^-4 of a radian is lost), so it
// is formed in fp64 and reduced there to an eighth of a turn either way, where the power series of sine and cosine, up to x^13
// and x^14, are off by 2e-14 at most.  An angle belongs to a token and a pair, not to a head: a workgroup makes a table of them
// in LDS for its tokens, a sine and a cosine per thread and turn, and all heads read it.
//
// What bounds it is reading and writing x once.  Measured (us of a call; the bytes at the 5.12 TB/s of a copy in brackets, an empty launch is
// 2.4): one token, 24 heads of 64, 3.3; 64 tokens, 40 heads of 128, 3.6; 4097 tokens, 32 heads, 11.6 [13.1, found in the Infinity Cache]; 13.5 thousand
// tokens, 40 heads, 52.9 [54.0].  A call that moves more than that cache holds goes past it (one buffer again and again / three in turn,
// ordinary: 192 MB 31.5 39.2, 256 MB 42.5 50.2, 320 MB 60.5 62.6; non-temporal 34.6 36.3, 45.1 46.7, 56.4 57.9).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tally.h"
#include "kernels_onepass.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

struct Turn { double c, s; };

// Cosine and sine of position * freq.  The product has 55 bits at most and is rounded from 2^29 positions on.  In quarter turns it
// is q = a 2 / pi; with n the nearest whole number, q - n is formed from the two halves of 2 / pi
// without losing what the first product rounds away.
__device__ __forceinline__ Turn turn_of(int32_t position, float freq) {
  constexpr double kHi = 0.63661977236758138, kLo = -3.935735335036497e-17, kQuarter = 1.5707963267948966;   // 2/pi = kHi + kLo
  const double a = (double)position * (double)freq, n = __builtin_rint(a * kHi);
  const double x = __builtin_fma(a, kLo, __builtin_fma(a, kHi, -n)) * kQuarter, z = x * x;
  double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  s = __builtin_fma(s * z, x, x);
  c = __builtin_fma(c, z, 1.0);
  const int quadrant = (int)__builtin_fma(-4.0, __builtin_floor(n * 0.25), n);
  const double u = quadrant & 1 ? s : c, v = quadrant & 1 ? c : s;
  return Turn{(quadrant + 1) & 2 ? -u : u, quadrant & 2 ? -v : v};
}

constexpr uint64_t kInfinityCache = 256ull << 20;          // bytes
constexpr uint32_t kRopeTable = 2048;                      // pairs of a workgroup's tokens
constexpr uint32_t kRopeItems = 1024;                      // pieces of 16 dims that a workgroup should have

// Tokens of a logical block: enough for four pieces per thread, while there are four workgroups per compute unit.  (us, a token a block / by
// this rule: 65536 tokens, one head of 64, 45.7 / 8.8; 32768, two of 64, 23.0 / 6.7; 32768, 8 of 128, 37.8 / 28.0; 4097, 8 of 64, 4.4 / 3.6; eight tokens at
// most / 32: 65536, one of 64, 12.0 / 8.8.  512 / 1024 / 2048 pieces: 32768, 8 of 128, 26.5 / 28.0 / 30.2; 13504, 40 of 128, 47.6 / 51.9 / 55.4, and 44.7 with a
// token a block: wide rows would gain from fewer; heads of 64 do not mind.  512 / 1024 / 2048 workgroups: 3000, 8 of 64, 3.4 / 3.5 / 4.2; 2048, 40 of 128,
// 8.5 / 7.9 / 7.9.)  As workers, 13504 tokens, 40 heads, 69, as one slice of the whole grid 67; 4097 35 and 32.
__host__ __device__ inline uint32_t rope_tokens(const tally_rope_args &a) {
  uint32_t g = 1;
  while (g < 32 && (uint64_t)g * a.heads * (a.dim / 16) < kRopeItems && a.total / (2 * g) >= 1024 && g * a.rot <= kRopeTable) g *= 2;
  return g;
}

struct RopeBody {
  using Args = tally_rope_args;
  static constexpr int THREADS = kThreads;
  static constexpr int MIN_WAVES = 4;
  static constexpr unsigned DYN_LDS = kRopeTable * sizeof(float2);
  static constexpr bool END_BARRIER = true;                // (the table)
  static constexpr bool YIELDS = false;
  static constexpr bool RANGE = false;
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) {
    if (4ull * a.total * a.heads * a.dim >= kInfinityCache) turn<true>(a, bx);
    else turn<false>(a, bx);
  }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) { turn<true>(a, bx); }

  template <bool NT>
  static __device__ __forceinline__ u32x4_nt load(const uint16_t *p) {
    if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt *>(p));
    else return *reinterpret_cast<const u32x4_nt *>(p);
  }
  template <bool NT>
  static __device__ __forceinline__ void store(uint16_t *p, u32x4_nt v) {
    if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_nt *>(p));
    else *reinterpret_cast<u32x4_nt *>(p) = v;
  }
  // A piece is 16 dims of a token and head: of the rotated part eight pairs, of the rest sixteen neighbours.
  template <bool NT>
  static __device__ __forceinline__ void turn(const Args &a, uint32_t block) {
#ifdef __HIP_DEVICE_COMPILE__
    extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
    float2 *table = reinterpret_cast<float2 *>(tally_dyn_lds);
    const uint32_t g = rope_tokens(a), t0 = block * g, n = a.total - t0 < g ? a.total - t0 : g, half = a.rot / 2;
    const double by = a.magnitude > 0.f ? (double)a.magnitude : 1.0, sign = a.flags & TALLY_ROPE_INVERSE ? -by : by;
    for (uint32_t i = threadIdx.x; i < n * half; i += kThreads) {
      const Turn w = turn_of(a.positions[t0 + i / half], a.freqs[i % half]);
      table[i] = make_float2((float)(w.c * by), (float)(w.s * sign));
    }
    __syncthreads();
    const uint32_t pieces = a.dim / 16, turned = a.rot / 16, LDX = a.ld_x ? a.ld_x : a.heads * a.dim, LDO = a.ld_out ? a.ld_out : a.heads * a.dim;
    const bool split = !(a.flags & TALLY_ROPE_INTERLEAVED);
    for (uint32_t i = threadIdx.x; i < n * a.heads * pieces; i += kThreads) {
      const uint32_t piece = i % pieces, head = i / pieces % a.heads, tok = i / pieces / a.heads;
      // (the two halves of a piece: eight dims each)
      const bool turns = piece < turned, apart = turns && split;
      const uint32_t one = head * a.dim + piece * (apart ? 8 : 16), two = one + (apart ? half : 8);
      const uint16_t *x = a.x + (uint64_t)(t0 + tok) * LDX;
      uint16_t *out = a.out + (uint64_t)(t0 + tok) * LDO;
      u32x4_nt u = load<NT>(x + one), v = load<NT>(x + two);
      if (turns) {
        const float2 *w = table + tok * half + piece * 8;
        if (split) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 w0 = w[2 * e], w1 = w[2 * e + 1];
            const float p0 = bf16_lo(u[e]), p1 = bf16_hi(u[e]), q0 = bf16_lo(v[e]), q1 = bf16_hi(v[e]);
            u[e] = pack(__builtin_fmaf(p0, w0.x, -(q0 * w0.y)), __builtin_fmaf(p1, w1.x, -(q1 * w1.y)));
            v[e] = pack(__builtin_fmaf(q0, w0.x, p0 * w0.y), __builtin_fmaf(q1, w1.x, p1 * w1.y));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 w0 = w[e], w1 = w[e + 4];
            const float p0 = bf16_lo(u[e]), q0 = bf16_hi(u[e]), p1 = bf16_lo(v[e]), q1 = bf16_hi(v[e]);
            u[e] = pack(__builtin_fmaf(p0, w0.x, -(q0 * w0.y)), __builtin_fmaf(q0, w0.x, p0 * w0.y));
            v[e] = pack(__builtin_fmaf(p1, w1.x, -(q1 * w1.y)), __builtin_fmaf(q1, w1.x, p1 * w1.y));
          }
        }
      }
      store<NT>(out + one, u);
      store<NT>(out + two, v);
    }
#endif
  }
#ifdef __HIP_DEVICE_COMPILE__
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return OnePass<128, 16, 32, 3>::pack(a, b); }
#endif
};

}  // namespace tally
