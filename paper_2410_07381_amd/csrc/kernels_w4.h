// Matrix-vector products with 4-bit weights and group scales for gfx950: up to 16 vectors at once.
//
// y[v][r] = sum over groups g of s[r][g] * sum over k of g of (code[r][k] - zero[r][g]) x[v][k].
//
// What bounds it is reading the codes, half a byte each.  A code becomes a bf16 with one AND-OR for two of
// them: 0x4300 | code is 128 + code, a small integer as the mantissa of a power of two.  The 128 and the zero
// point are taken out again by a second MFMA with the constant -(128 + zero), which is exact in bf16, so that a
// group's sum has the rounding of fp32 alone; then the scale is applied, in fp32.  The vectors are the 16 rows
// of an MFMA, weight rows its columns, so one vector costs what sixteen do and a lane needs the scale of one row.
//
// The codes lie in memory as the lanes want them: a tile is 16 rows by 128 weights, 1 KB that a wave
// reads with one 16-byte load a lane; word i of lane 16 q + r holds weights 32 i + 8 q to 32 i + 8 q + 7
// of row r, the even ones in its low half.  So MFMA i of a tile takes 32 neighbouring weights of each
// row, which always belong to one group.
//
// The eight waves of a workgroup share the tiles of a row of tiles and join their sums in LDS.  Which wave takes
// a tile and in what order sums are added depends on k alone, so a result's bits depend neither on the
// number of vectors nor on the variant.
//
// Measured (us; the codes, scales and zero points read once at 5.1 TB/s in brackets, and an empty launch is 2.4): 1 vector,
// 4096 x 4096 3.6 [1.7], 4096 x 11008 in groups of 64 with zero points 7.5 [4.8]; 16 vectors, 11008 x 4096 8.3 [4.6]; 5 vectors,
// 50257 x 4096 in groups of 32 with zero points 29.5 [23.9].  With many vectors a short product is bound by reading x
// from the L2s once per workgroup (16 vectors, 4096 x 16384: 19.7 [7.3]).  Beginning the rows of tiles at different columns, so that
// not all ask for the same x at once, gave 9.9 for 10.9 with 8 vectors, 16384 x 4096, and 33.1 for 31.5 with 5, 50257 x 4096.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tally.h"
#include "kernels_gemm.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

constexpr uint32_t kW4Rows = 16, kW4Block = 128, kW4Vectors = 16, kW4MaxGroup = 1u << 20;
constexpr int kW4Waves = 8;
constexpr uint32_t kW4Staged = 22 * 1024;                  // bytes of LDS for x, where it goes there
constexpr uint32_t kW4LongK = 8192;                        // ... from this k on
constexpr uint32_t kW4Piece = 1024;                        // bytes of x that one direct load brings

// Rows of tiles that a workgroup takes.  It reads x once for all of them (from the L2s, 24 bytes a clock and compute
// unit where all of them read the same): with many vectors that is more than the codes, so fewer workgroups
// with more rows each are faster, as long as each of the 256 compute units has the same number of them.  Cost of
// a workgroup: its rows, and a quarter of a row per vector; of equals the one with more rows.  Four rows are left out where
// that is one workgroup per compute unit at most, with nothing beside its long way (800 to 1024 tiles, 13 to 16 vectors, two
// rows and four: k = 2048, groups of 32, 6.5 to 7.2 and 7.2 to 9.1; 4096, of 64, 10.8 to 12.3 and 13.1 to 14.0; 1024 the
// same; 4096, of 128, 9.4 to 10.7 and 9.4 to 10.3).
// us by rows, groups of 128, k = 4096, 256 / 688 / 1024 / 2000 tiles:
//    1 vector   3.7 4.7 5.9 7.5 /  7.0  7.4 6.2  8.5 /  8.7  7.7  9.5  8.9 / 15.1 14.2 14.7 15.5
//    4 vectors  4.1 4.8 6.0 7.7 /  8.3  7.4 6.2  9.3 / 10.6  7.4  9.4  8.9 / 18.7 14.3 14.6 15.6
//    8 vectors  4.7 5.2 6.0 8.0 / 10.1  8.0 6.3  8.9 / 12.9  8.1  9.9  9.2 / 23.7 15.2 15.0 15.3
//   16 vectors  6.1 6.4 7.2 8.5 / 14.2 10.8 7.4 10.3 / 18.2 10.7 12.5 10.3 / 34.0 19.0 17.7 15.7
// k and the groups are not asked for.  Over 254 random calls (n to 65536, k to 11585, all groups) the choice is 2.4 % slower
// than the best of the four on average; worst with four rows, where two are faster with small groups or short k (17 of 20
// calls; 2889 tiles, k = 560, groups of 64, 16 vectors: 5.7 and 7.4).
inline uint32_t w4_rows(uint32_t m, uint32_t n) {
  const uint32_t tiles = (n + kW4Rows - 1) / kW4Rows, most = m <= 6 ? 2 : m <= 10 ? 3 : 4;
  if (m <= 2) return tiles > 1024 ? 2 : 1;
  uint32_t best = 1;
  uint64_t least = ~0ull;
  for (uint32_t r = 1; r <= most; ++r) {
    const uint64_t groups = (tiles + r - 1) / r, cost = (groups + 255) / 256 * (4 * r + m);
    if (r == 4 && groups <= 256) continue;
    if (cost <= least) { least = cost; best = r; }
  }
  return best;
}
// One vector goes to LDS where it fits (two from kW4LongK on do not) and a wave has many tiles to take one after the
// other, so that nothing but codes is on its way in the loop.  (us, straight from the L2s / so: 4096 x 11008, groups of
// 64 with zero points, 9.1 / 8.3; 11008 x 11008 13.9 / 12.8; 1024 x 11008, groups of 32, 8.4 / 7.6; but 11008 x 1024 3.4 / 3.8.)
static_assert(2 * kW4LongK * 2 > kW4Staged, "room for one vector alone");
inline bool w4_staged(const tally_gemv_w4_args &a) {
  return a.m == 1 && a.k >= kW4LongK && a.k * 2 <= kW4Staged && w4_rows(a.m, a.n) == 1;
}

// One tile of 16 rows by 128 weights, as loaded.  SUB: MFMAs of a tile that share a scale (groups of 32, of
// 64, of 128 and more).  Scales and zero points: a lane has those of row l % 16 and of the group that the
// quarter l / 16 of the tile lies in.
template <int SUB>
struct W4Tile {
  uint4 w;
  uint32_t scale, zero;
#ifdef __HIP_DEVICE_COMPILE__
  struct From {
    buf_t w, scales, zeros;
    uint32_t inverse;                                      // 2^31 over the tiles of a group, rounded up
    bool has_zeros;
    __device__ __forceinline__ From(const tally_gemv_w4_args &a, uint32_t rows, uint32_t blocks, uint32_t groups)
        : w(make_buf(reinterpret_cast<const unsigned char *>(a.W) + (uint64_t)rows * blocks * 1024, blocks * 1024)),
          scales(make_buf(a.scales + (uint64_t)rows * groups * 16, groups * 32)),
          zeros(make_buf(a.zeros ? a.zeros + (uint64_t)rows * groups * 16 : nullptr, a.zeros ? groups * 16 : 0)),
          inverse(SUB == 4 ? (0x7FFFFFFFu + a.group / kW4Block) / (a.group / kW4Block) : 0u), has_zeros(a.zeros != nullptr) {}
  };
  // (unless it is `there` nothing is read, and zeros come back: the lanes' offsets are past any buffer's end)
  __device__ __forceinline__ void load(const From &f, uint32_t b, uint32_t lane, bool there = true) {
    const uint32_t none = there ? 0u : 0x80000000u;
    b = there ? b : 0u;
    w = buf_ld16(f.w, lane * 16 | none, b * 1024);
    const uint32_t at = SUB == 4 ? __umulhi(2 * b, f.inverse) * 16 + (lane & 15)
                                 : b * (4 / SUB) * 16 + (SUB == 1 ? lane : (lane >> 5) * 16 + (lane & 15));
    scale = __builtin_amdgcn_raw_buffer_load_b16(f.scales, at * 2 | none, 0, 0);
    zero = f.has_zeros ? __builtin_amdgcn_raw_buffer_load_b8(f.zeros, at | none, 0, 0) : 8u;
  }
  // acc += this tile's rows times the vectors; x(i): the vectors' 32 elements for MFMA i
  template <class X>
  __device__ __forceinline__ void add(f32x4_t &acc, uint32_t lane, X x) const {
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
    // (in registers, or there would be an AND and an OR: an instruction has room for one constant)
    uint32_t mask = 0x000F000Fu, base = 0x43004300u;
    asm("" : "+s"(mask), "+v"(base));
    // scale in the upper half, -(128 + zero) in the lower
    const uint32_t both = scale << 16 | __float_as_uint(-(float)(128u + zero)) >> 16;
#pragma unroll
    for (int g = 0; g < 4; g += SUB) {
      const uint32_t u = SUB == 4 ? both : (uint32_t)__builtin_amdgcn_ds_bpermute((g * 16 + (lane & 15)) * 4, (int)both);
      const uint32_t cc = __builtin_amdgcn_perm(u, u, 0x01000100u);
      const bf16x8_t less = __builtin_bit_cast(bf16x8_t, make_uint4(cc, cc, cc, cc));
      f32x4_t part = {0.f, 0.f, 0.f, 0.f}, off = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = g; i < g + SUB; ++i) {
        const bf16x8_t xv = x(i);
        uint32_t q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = (word[i] >> (4 * j) & mask) | base;
        off = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, less, off, 0, 0, 0);
        // (of 64 and more two chains, as an MFMA waits for the one before: 16 vectors, 11008 x 4096, 8.6 us, in one 9.1;
        // of 32 one, which is short and saves additions: 5 vectors, 50257 x 4096, 30.3, in two 31.4)
        if (SUB == 1) part = off;
        part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, __builtin_bit_cast(bf16x8_t, make_uint4(q[0], q[1], q[2], q[3])), part, 0, 0, 0);
      }
      const float s = bf16_hi(u);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(s, SUB == 1 ? part[e] : part[e] + off[e], acc[e]);
    }
  }
#endif
};

// What the variants have in common.  ROWS: rows of tiles of a block.
template <int ROWS_>
struct W4Base {
  using Args = tally_gemv_w4_args;
  static constexpr int ROWS = ROWS_, THREADS = 64 * kW4Waves;
  static constexpr bool YIELDS = false;
  static constexpr bool RANGE = false;
  static constexpr bool END_BARRIER = true;                // (LDS holds the waves' sums, and x)
  // The waves' sums, joined in LDS, one row of tiles at a time; lane 16 q + r, element e: vector 4 q + e, row r
  static __device__ __forceinline__ void store(const Args &a, const f32x4_t (&acc)[ROWS], uint32_t block, uint32_t wave, uint32_t lane) {
    __shared__ f32x4_t s_acc[kW4Waves][64];
#pragma unroll
    for (int o = 0; o < ROWS; ++o) {
      if (o) __syncthreads();
      s_acc[wave][lane] = acc[o];
      __syncthreads();
      const uint32_t v = threadIdx.x >> 4, l = (v >> 2) * 16 + (threadIdx.x & 15), e = v & 3;
      const uint32_t row = (block * ROWS + o) * kW4Rows + (threadIdx.x & 15);
      if (v < a.m && row < a.n) {
        float y = 0.f;
#pragma unroll
        for (int w = 0; w < kW4Waves; ++w) y += s_acc[w][l][e];
        a.y[(uint64_t)v * (a.ld_y ? a.ld_y : a.n) + row] = f32_to_bf16(y);
      }
    }
  }
};

// One vector in LDS, straight from memory; behind its loads each wave keeps two tiles of codes on their way.
template <int SUB>
struct GemvW4StagedT : W4Base<1> {
  static constexpr int MIN_WAVES = 7;                      // 72 registers: two waves fit beside a paused GEMM tile
  static constexpr unsigned DYN_LDS = kW4Staged;
  static constexpr int DEEP = 2;
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) { run_t(a, bx); }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) { run_t(a, bx); }
  static __device__ __forceinline__ void run_t(const Args &a, uint32_t tile) {
#ifdef __HIP_DEVICE_COMPILE__
    extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
    uint32_t lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t blocks = (a.k + kW4Block - 1) / kW4Block, groups = (a.k + a.group - 1) / a.group;
    const uint32_t lds = (uint32_t)(uintptr_t)(lptr_t)tally_dyn_lds;
    const uint64_t p = (uint64_t)(uintptr_t)a.x;
    const u32x4_t x = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, a.k * 2, 0x00027000u};
    for (uint32_t at = wave * kW4Piece; at < a.k * 2; at += kW4Waves * kW4Piece) {
      // (as in OnePass::ask, the waits too: what is past the vector's end is left as zeros)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   ::"s"(lds + at), "v"(lane * 16 + at), "s"(x) : "memory");
    }
    const typename W4Tile<SUB>::From from(a, tile, blocks, groups);
    W4Tile<SUB> t[DEEP];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) t[j].load(from, wave + j * kW4Waves, lane);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * DEEP) : "memory");   // (at least so many loads are behind those of x)
    __syncthreads();
    const uint32_t at = lds + (lane >> 4) * 16;            // (the same for all 16 rows of an MFMA, of which one counts)
    f32x4_t acc[1] = {{0.f, 0.f, 0.f, 0.f}};
    for (uint32_t b = wave; b < blocks; b += DEEP * kW4Waves) {
#pragma unroll
      for (int j = 0; j < DEEP; ++j) {
        const uint32_t mine = b + j * kW4Waves;
        if (mine < blocks)
          t[j].add(acc[0], lane, [&](int i) {
            typedef const __attribute__((address_space(3))) bf16x8_t *frag_t;
            return *(frag_t)(at + mine * (kW4Block * 2) + i * 64);
          });
        t[j].load(from, mine + DEEP * kW4Waves, lane, mine + DEEP * kW4Waves < blocks);
      }
    }
    store(a, acc, tile, wave, lane);
#endif
  }
};

// x as each wave needs it, from the L2s, together with the codes of one tile of each row.  With one row there are
// often no more workgroups than compute units, and a wave's loads for its next tile are sent before it works on
// this one (4 vectors, 4096 x 11008, 9.3 us, without 12.3; 8 vectors, 2048 x 8192, 8.2 and 10.0; but one vector, 11008
// x 4096, where three workgroups share a compute unit, 7.3 and 7.1); more rows have no registers for that.
template <int SUB, int ROWS>
struct GemvW4T : W4Base<ROWS> {
  using Args = tally_gemv_w4_args;
  static constexpr int MIN_WAVES = ROWS <= 3 ? 7 : 4;   // (up to 72 registers: two waves fit beside a paused GEMM tile)
  static constexpr unsigned DYN_LDS = 0;
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) { run_t(a, bx); }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) { run_t(a, bx); }
  static __device__ __forceinline__ void run_t(const Args &a, uint32_t block) {
#ifdef __HIP_DEVICE_COMPILE__
    uint32_t lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t blocks = (a.k + kW4Block - 1) / kW4Block, groups = (a.k + a.group - 1) / a.group;
    const uint32_t tiles = (a.n + kW4Rows - 1) / kW4Rows;
    const uint32_t LDX = a.ld_x ? a.ld_x : a.k, col = lane & 15, k0 = (lane >> 4) * 8;
    // (a vector that does not exist lies past the buffer's end, and so does what is past the end of one)
    const buf_t x = make_buf(a.x, 0x7fffffff);
    const uint32_t xrow = col < a.m ? (col * LDX + k0) * 2 : 0x80000000u;
    f32x4_t acc[ROWS];
#pragma unroll
    for (int o = 0; o < ROWS; ++o) acc[o] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    struct Stage { W4Tile<SUB> t[ROWS]; uint4 xv[4]; };
    auto load = [&](Stage &s, uint32_t b) {
#pragma unroll
      for (int o = 0; o < ROWS; ++o) {
        const uint32_t tile = block * ROWS + o;
        const typename W4Tile<SUB>::From from(a, tile < tiles ? tile : tiles - 1, blocks, groups);
        s.t[o].load(from, b, lane, b < blocks);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t k1 = b * kW4Block + i * 32;
        s.xv[i] = buf_ld16(x, k1 + k0 < a.k ? xrow + k1 * 2 : 0x80000000u, 0);
      }
    };
    auto add = [&](const Stage &s) {
#pragma unroll
      for (int o = 0; o < ROWS; ++o) s.t[o].add(acc[o], lane, [&](int i) { return __builtin_bit_cast(bf16x8_t, s.xv[i]); });
    };
    if constexpr (ROWS == 1) {
      Stage s[2];
      uint32_t b = wave;
      load(s[0], b);
      while (b < blocks) {
        load(s[1], b + kW4Waves);
        __builtin_amdgcn_sched_barrier(0);
        add(s[0]);
        b += kW4Waves;
        if (b >= blocks) break;
        load(s[0], b + kW4Waves);
        __builtin_amdgcn_sched_barrier(0);
        add(s[1]);
        b += kW4Waves;
      }
    } else {
      for (uint32_t b = wave; b < blocks; b += kW4Waves) {
        Stage s;
        load(s, b);
        add(s);
      }
    }
    W4Base<ROWS>::store(a, acc, block, wave, lane);
#endif
  }
};

}  // namespace tally
