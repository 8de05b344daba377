// Attention in one pass over K and V for gfx950: a whole prompt (causal, grouped heads, sequences
// of different lengths packed one behind the other) and single-token queries of a batch that
// shares a prefix.
//
// Scores never leave the registers.  With m the running maximum of a row's scores and p = exp(s - m) (a softmax
// in one pass, Milakov and Gimelshein 2018), a row's state is (m, l = sum of p, acc = sum of p v); a new maximum rescales l and acc by
// exp(m_old - m_new), and the output is acc / l.  Everything is held in fp32; q, k, v and the p that
// enter the second product are bf16, so each p is off by at most 2^-8 of itself, which is
// what the output's own rounding costs.
//
// Both products are taken transposed, S^T = K Q^T and O^T = V^T P^T: a lane then holds scores of ONE
// row, so that maximum and sum need one or two lane swaps a tile, and the lanes that hold P^T after
// the exponential are the ones that the second product wants it from.  (The order of the tokens
// within one MFMA's k is free as long as V's fragments have it too, and the transposing LDS
// reads that make those take four consecutive tokens from anywhere.)
//
// Four waves share tiles of K and V in LDS; each has ROWS rows of its own (ROWS x ROWS MFMA blocks).
// A tile's K and V are items of one ring of NS places: item i is waited for and a barrier
// passed, which also says that everyone is done with item i - 1, whose place takes item i + NS - 1.
// A place holds its rows' 16-byte chunks xor-swizzled by the row, so that the 16 lanes that a
// 128-bit read serves at once, and the 16 tokens of a transposing read, fall into different banks.
//
// What bounds long prompts is the matrix pipe, and the clock that it is left with: 32768 tokens, 8 heads of 128 on one
// K/V head, take 1.87 to 1.94 ms, 1.13 to 1.18 PFLOP/s (8192^3 of the GEMM tile: 1.5), 3.06 million cycles in which the compute
// units have work, so 1.6 GHz, and in 69 % of them the pipe is busy.
// 8192 tokens, 32/8 heads, 487 us (1.13); 4097, 32 heads, 148 (0.93); 16384, 16 heads of 64, 567 (0.97).
// Short ones are a chain of latencies: 128 tokens, 12 heads of 64, 5.4 us, of which an empty launch is 2.4; 512
// tokens, 32/8 heads of 128, 13.6.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "../../include/tally.h"
#include "kernels_gemm.h"
#include "kernels_stream.h"
#include "launch_forms.h"
#include "turnaround.h"

namespace tally {

constexpr float kLog2e = 1.4426950408889634f;
// The maximum of a row that has seen nothing: below any score, but a number, so that exp(s - m) is zero for a score
// of -inf and exp(m - m_new) for any new maximum.
constexpr float kNothing = -3e38f;

template <int DIM_, int ROWS_, int TOK_, int NS_>
struct OnePass {
  static constexpr int DIM = DIM_, ROWS = ROWS_, TOK = TOK_, NS = NS_, WAVES = 4;
  static constexpr int BLOCK_ROWS = ROWS * WAVES;
  static constexpr uint32_t ROWB = DIM * 2;                // bytes of a token's row
  static constexpr uint32_t PLACE = TOK * ROWB;            // bytes of an item
  static constexpr int L = PLACE / 1024 / WAVES;           // direct loads per wave and item
  static constexpr uint32_t RPL = 1024 / ROWB;             // tokens per load
  static constexpr unsigned LDS = PLACE * NS;
  static constexpr uint32_t BEFORE = (L - 1) * 1024;       // (see ask)
  static constexpr int MK = ROWS == 32 ? 16 : 32;          // k of one MFMA
  static constexpr int QK = DIM / MK, PV = TOK / MK;
  static constexpr int TT = TOK / ROWS, DT = DIM / ROWS;   // blocks of tokens and of dims
  static constexpr int AN = ROWS == 32 ? 16 : 4;           // accumulators of a block
  static constexpr int PAIRS = TT * AN / 2;                // of a lane's scores in a tile
  static constexpr int AHEAD = 4;                          // fragments on their way from LDS
  static_assert((DIM == 64 || DIM == 128) && (ROWS == 32 || ROWS == 16), "shapes that the maps below know");
  static_assert((L == 1 || L == 2 || L == 4) && L * 1024 * WAVES == (int)PLACE && NS >= 3, "whole loads, two items on their way");
  static_assert(BEFORE < 4096, "an immediate has 12 bits");

#ifdef __HIP_DEVICE_COMPILE__
  typedef typename std::conditional<ROWS == 32, f32x16_t, f32x4_t>::type acc_t;
  typedef short s16x4_t __attribute__((ext_vector_type(4)));
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

  // tokens of K or of V that are still to be asked for
  struct Src {
    const unsigned char *at;
    uint32_t left, ld;                                     // tokens; bytes between them
    uint32_t voff[L];
  };

  uint32_t lane, wave, lds;
  uint32_t k_at, v_at;                                     // a lane's place in K's and V's fragment reads
  bf16x8_t q[QK];
  acc_t acc[DT];
  float m, l;

  // 16-byte chunk c of token t stands at chunk c xor swz(t): different for 16 neighbouring tokens (of
  // dim 64, whose rows are half as long, for every second one), and its high bits for four
  static __device__ __forceinline__ uint32_t swz(uint32_t t) {
    return DIM == 128 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3);
  }
  static __device__ __forceinline__ float exp2(float x) { return __builtin_amdgcn_exp2f(x); }
  // over the lanes that hold scores of one row
  template <class F>
  static __device__ __forceinline__ float over_row(float v) {
    if constexpr (ROWS == 16) return across_rows<F>(v);
    float w = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(v), "+v"(w));
    return F::of(v, w);
  }
  static __device__ __forceinline__ acc_t mma(bf16x8_t a, bf16x8_t b, acc_t c) {
    if constexpr (ROWS == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }

  __device__ __forceinline__ void begin(unsigned char *lds_at) {
    lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                         // (see the GEMM: nothing of it is kept across blocks)
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds = (uint32_t)(uintptr_t)(lptr_t)lds_at;
    const uint32_t row = lane % ROWS, part = lane / ROWS;
    k_at = row * ROWB + ((part ^ swz(row)) << 4);
    // a transposing read: 16 lanes take four tokens of 16 dims, lane i the i%4-th 8 bytes of token i/4
    const uint32_t i = lane & 15, tok = 4 * part + (i >> 2);
    const uint32_t chunk = (ROWS == 32 ? (lane >> 4 & 1) * 2 : 0) + (i >> 1 & 1);
    v_at = tok * ROWB + ((chunk ^ swz(tok)) << 4) + (i & 1) * 8;
    reset();
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = acc_t{};
    m = kNothing;
    l = 0.f;
  }
  __device__ __forceinline__ Src source(const uint16_t *at, uint32_t tokens, uint32_t ld) const {
    Src r;
    r.at = (const unsigned char *)at - BEFORE;
    r.left = tokens;
    r.ld = ld * 2;
#pragma unroll
    for (int n = 0; n < L; ++n) {
      const uint32_t row = (wave * L + n) * RPL + lane / (ROWB / 16), c = lane % (ROWB / 16);
      r.voff[n] = row * r.ld + ((c ^ swz(row)) << 4) + (BEFORE - n * 1024u);
    }
    return r;
  }
  // the next item of a source to a place of the ring; past its end nothing is moved and zeros are left
  __device__ __forceinline__ void ask(Src &r, uint32_t place) const {
    // (Assembly: knowing of the loads, the compiler waits for all of them before any transposing read.  They
    // have no destination in registers, sync() waits for them, and nothing else in these kernels uses m0.  The
    // immediate separates a wave's loads in LDS; it moves the global address too, which is taken out of
    // the lane's offset, and so that none is negative the buffer starts BEFORE bytes early.  An SGPR that a vector
    // instruction wrote (the buffer's words, where they had to be put away) may be read by a load five wait states
    // later, which the compiler sees to for its own instructions alone: the block opens with them.)
    const uint32_t n = r.left < (uint32_t)TOK ? r.left : (uint32_t)TOK, to = lds + place * PLACE + wave * (L * 1024u);
    const uint64_t p = (uint64_t)(uintptr_t)r.at;
    const u32x4_t b = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, n * r.ld + BEFORE, 0x00027000u};
#define LOAD_LDS(v, at) "buffer_load_dwordx4 " v ", %1, 0 offen offset:" at " lds"
#define OPEN_LDS "s_mov_b32 m0, %0\n\ts_nop 4\n\t"
    if constexpr (L == 1)
      asm volatile(OPEN_LDS LOAD_LDS("%2", "0") ::"s"(to), "s"(b), "v"(r.voff[0]) : "memory");
    else if constexpr (L == 2)
      asm volatile(OPEN_LDS LOAD_LDS("%2", "0") "\n\t" LOAD_LDS("%3", "0x400") ::"s"(to), "s"(b), "v"(r.voff[0]), "v"(r.voff[1]) : "memory");
    else
      asm volatile(OPEN_LDS LOAD_LDS("%2", "0") "\n\t" LOAD_LDS("%3", "0x400") "\n\t" LOAD_LDS("%4", "0x800") "\n\t" LOAD_LDS("%5", "0xC00")
                   ::"s"(to), "s"(b), "v"(r.voff[0]), "v"(r.voff[1]), "v"(r.voff[2]), "v"(r.voff[3])
                   : "memory");
#undef LOAD_LDS
#undef OPEN_LDS
    r.at += (uint64_t)TOK * r.ld;
    r.left -= n;
  }
  // all but the last LEFT loads of every wave are there, and every wave is done with what it has read
  template <int LEFT>
  static __device__ __forceinline__ void sync() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  }
  // (the compiler would wait for q in the loop, counting none of ask()'s loads)
  __device__ __forceinline__ void wait_q() {
#pragma unroll
    for (int k = 0; k < QK; ++k) asm volatile("" : "+v"(q[k]));
  }
  // (what is computed from it is not kept beside what another loop has computed)
  static __device__ __forceinline__ uint32_t opaque(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
  }

  // which token of a tile element e of block t stands for, without the lane's own part
  static constexpr uint32_t token(int t, int e) { return ROWS == 32 ? 32 * t + 8 * (e / 4) + e % 4 : 16 * t + e; }

  // fragment i of K, of the tile at `place`: block i % TT of tokens, MFMA step i / TT
  __device__ __forceinline__ bf16x8_t key(uint32_t place, uint32_t k_at, int i) const {
    typedef const __attribute__((address_space(3))) bf16x8_t *frag_t;
    return *(frag_t)(place + (k_at ^ (i / TT * (MK * 2))) + i % TT * (ROWS * ROWB));
  }
  // S^T of a tile; the fragments are read AHEAD MFMAs before they are needed
  __device__ __forceinline__ void products(acc_t (&s)[TT], uint32_t place, uint32_t k_at) const {
    constexpr int N = QK * TT;
    bf16x8_t f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = key(place, k_at, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[i % TT] = mma(f[i % AHEAD], q[i / TT], i < TT ? acc_t{} : s[i % TT]);
      if (i + AHEAD < N) f[i % AHEAD] = key(place, k_at, i + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // a lane's row attends to tokens of the tile below `lim` alone
  __device__ __forceinline__ void hide(acc_t (&s)[TT], int32_t lim) const {
    int32_t left = lim - 4 * (int32_t)(lane / ROWS);
    asm volatile("" : "+v"(left));                         // (computed here, where it is asked for)
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < AN; ++e) s[t][e] = (int32_t)token(t, e) < left ? s[t][e] : -INFINITY;
  }
  // a lane's largest score
  static __device__ __forceinline__ float largest(const acc_t (&s)[TT]) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < AN; ++e) top = fmaxf(top, s[t][e]);
    return top;
  }
  // The running maximum follows that of a tile (c: the scale times log2(e)).  One that has grown by less than 2^8 is
  // left as it is: p then stays below 2^8, which costs nothing in floating point, and acc is rarely rescaled (nor
  // do the lanes of a row have to exchange theirs).
  __device__ __forceinline__ void follow(float top, float c) {
    top *= c;
    if (__builtin_amdgcn_ballot_w64(top > m + 8.f) != 0) {
      const float now = fmaxf(m, over_row<MaxOp>(top)), a = exp2(m - now);
      m = now;
      l *= a;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < AN; ++e) acc[d][e] *= a;
    }
  }
  // to + times . p (two bf16 each)
  static __device__ __forceinline__ float add_pair(uint32_t p, float to, uint32_t times = 0x3F803F80u) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, p), __builtin_bit_cast(bf16x2_t, times), to, false);
  }

  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const f32x2_t p = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2_t));
  }
  // p of MFMA step k as the second operand: of 32 tokens' 16 pairs a lane has 8 (of 16 rows: 16 tokens' 4 in all)
  static __device__ __forceinline__ bf16x8_t weights(const uint32_t (&p)[PAIRS], int k) {
    return __builtin_bit_cast(bf16x8_t, make_uint4(p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]));
  }
  // V^T of dims [ROWS d, ROWS d + ROWS) for the tokens of MFMA step k, in the order of weights()
  static __device__ __forceinline__ uint4 values(uint32_t at, uint32_t v_at, int k, int d) {
    typedef __attribute__((address_space(3))) s16x4_t *tr_t;
    uint2 h[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // (the second four are 8 or 16 tokens further on; 8 tokens on the swizzle differs by 2)
      const uint32_t far = ROWS == 32 ? (uint32_t)j << 5 : 0u;
      const uint32_t off = at + (v_at ^ (d * (ROWS * 2)) ^ far) + (k * MK + j * (MK / 2)) * ROWB;
      h[j] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)off));
    }
    return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
  }
  // A tile's exponentials (p in pairs as bf16, whose sum, of what the product takes, goes to l) and its product with
  // V, each step's beside the product of the one before.
  __device__ __forceinline__ void finish(const acc_t (&s)[TT], uint32_t (&p)[PAIRS], uint32_t place, uint32_t v_at, float c) {
    constexpr int N = PV * DT, EACH = 2 * PAIRS / PV;      // scores of a lane in an MFMA step
    uint4 f[AHEAD];
    float sum[2] = {0.f, 0.f};
    auto exps = [&](int from, int to) {
#pragma unroll
      for (int i = from; i < to; i += 2) {
        p[i / 2] = pack(exp2(__builtin_fmaf(s[i / AN][i % AN], c, -m)), exp2(__builtin_fmaf(s[i / AN][i % AN + 1], c, -m)));
        sum[i / 2 & 1] = add_pair(p[i / 2], sum[i / 2 & 1]);
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD && i < N; ++i) f[i] = values(place, v_at, i / DT, i % DT);
    exps(0, EACH);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int k = i / DT, d = i % DT;
      acc[d] = mma(__builtin_bit_cast(bf16x8_t, f[i % AHEAD]), weights(p, k), acc[d]);
      if (i + AHEAD < N) f[i % AHEAD] = values(place, v_at, (i + AHEAD) / DT, (i + AHEAD) % DT);
      if (k + 1 < PV) exps((k + 1) * EACH + EACH * d / DT / 2 * 2, (k + 1) * EACH + EACH * (d + 1) / DT / 2 * 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sum[0] + sum[1];
  }
  // The same where V has tokens that are no numbers and that not every row sees.  Their p is zero, but zero times an
  // infinity or NaN is NaN: the product has zeros in their place, and the tile is then looked through
  // token by token, where a row takes what it sees.  (Rare: in few registers rather than fast.)
  __device__ __forceinline__ void finish_careful(const acc_t (&s)[TT], uint32_t (&p)[PAIRS], uint32_t at, uint32_t v_at, float c, int32_t lim) {
    const uint32_t lane = opaque(this->lane);
    asm volatile("" : "+v"(c));                            // (nothing in common with finish())
#pragma unroll
    for (int i = 0; i < 2 * PAIRS; i += 2) {
      p[i / 2] = pack(exp2(__builtin_fmaf(s[i / AN][i % AN], c, -m)), exp2(__builtin_fmaf(s[i / AN][i % AN + 1], c, -m)));
      l = add_pair(p[i / 2], l);
    }
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      const bf16x8_t w = weights(p, k);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint4 v = values(at, v_at, k, d);
        uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] &= (u[i] & 0x7F80u) == 0x7F80u ? 0xFFFF0000u : 0xFFFFFFFFu;
          u[i] &= (u[i] & 0x7F800000u) == 0x7F800000u ? 0xFFFFu : 0xFFFFFFFFu;
        }
        acc[d] = mma(__builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3])), w, acc[d]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    typedef const __attribute__((address_space(3))) uint2 *four_t;
#pragma unroll 1
    for (int32_t t = 0; t < TOK; ++t) {
      const bool sees = t < lim;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < AN / 4; ++g) {                 // four neighbouring dims
          const uint32_t dim = d * ROWS + 8 * g + 4 * (lane / ROWS);
          const uint2 v = *(four_t)(at + t * ROWB + ((dim >> 3 ^ swz(t)) << 4) + (dim & 4) * 2);
          const uint32_t w[2] = {v.x, v.y};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16;
            acc[d][4 * g + i] += sees && (x & 0x7F800000u) == 0x7F800000u ? __uint_as_float(x) : 0.f;
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  }

  // Tile j: its exponentials and its product with V beside the scores of tile j + 1, in an order that is pinned:
  // behind each MFMA one or two LDS reads (of what is needed AHEAD MFMAs later) and as many vector instructions
  // as run while the matrix pipe is busy with it.  s: tile j's scores; next: the next one's, whose largest is
  // returned (MASK: of those that a lane's row attends to, below `lim`); `ask` (the next loads) is called behind
  // the first MFMAs.
  template <bool MASK, class Ask>
  __device__ __forceinline__ float tile(acc_t (&next)[TT], const acc_t (&s)[TT], uint32_t k_place, uint32_t v_place, uint32_t k_at,
                                        uint32_t v_at, float c, int32_t lim, Ask ask) {
    static_assert(ROWS == 32 && TT == 2 && PV == 4, "32 scores of a lane, 16 for each half of the second product");
    constexpr int NQ = QK * TT, NV = PV * DT, EXPS = NQ + NV / 2;
    bf16x8_t kf[AHEAD];
    uint4 vf[AHEAD];
    uint32_t p[PAIRS];
    float even = 0.f, sum[2] = {0.f, 0.f}, top = -INFINITY;
    const int32_t left = lim - 4 * (int32_t)(lane / ROWS);
    auto read_v = [&](int i) { vf[i % AHEAD] = values(v_place, v_at, i / DT, i % DT); };
    auto exps = [&](int slot) {                            // 32 scores to p, over the first EXPS slots
#pragma unroll
      for (int i = slot * 32 / EXPS; i < (slot + 1) * 32 / EXPS; ++i) {
        const float x = exp2(__builtin_fmaf(s[i / AN][i % AN], c, -m));
        if (i & 1) p[i / 2] = pack(even, x);
        else even = x;
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = key(k_place, k_at, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      next[i % TT] = mma(kf[i % AHEAD], q[i / TT], i < TT ? acc_t{} : next[i % TT]);
      if (i + AHEAD < NQ) kf[i % AHEAD] = key(k_place, k_at, i + AHEAD);
      else read_v(i + AHEAD - NQ);
      exps(i);
      if (i == 1 || i == 3) ask(i / 2);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      acc[i % DT] = mma(__builtin_bit_cast(bf16x8_t, vf[i % AHEAD]), weights(p, i / DT), acc[i % DT]);
      if (i + AHEAD < NV) read_v(i + AHEAD);
      if (i < NV / 2) exps(NQ + i);
      else {
#pragma unroll
        for (int n = (i - NV / 2) * (64 / NV); n < (i - NV / 2 + 1) * (64 / NV); ++n) {
          if (MASK) next[n / AN][n % AN] = (int32_t)token(n / AN, n % AN) < left ? next[n / AN][n % AN] : -INFINITY;
          top = fmaxf(top, next[n / AN][n % AN]);
          if (n & 1) sum[n / 2 & 1] = add_pair(p[n / 2], sum[n / 2 & 1]);
        }
        asm volatile("" : "+v"(top), "+v"(sum[0]), "+v"(sum[1]));   // (here, not later)
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sum[0] + sum[1];
    return top;
  }

  // Tokens [0, n) of K and V, `n` the same for all four waves; `mine` of them are seen by rows of this
  // wave (none if 0).  A wave's rows attend to tokens below `lim`, or (CAUSAL) the first to those and each
  // further one to one more; full: below that every row does, and what is left of `mine` is one tile at
  // most.  `step(j)` is called behind the barrier of each tile.  What is behind a row's last token has a weight
  // of zero, and has to be numbers where it is not zeros, unless `careful`.
  //
  // LDS is nobody else's when they are called.  CAUSAL: the block's rows of q come from `qs`; otherwise q is there.
  //
  // Where reading K and V is what bounds it: one item of the ring after the other.
  template <class Step>
  __device__ __forceinline__ void run_lean(Src ks, Src vs, uint32_t n, uint32_t mine, uint32_t full, int32_t lim, float c, Step step) {
    const uint32_t tiles = (n + TOK - 1) / TOK, have = (mine + TOK - 1) / TOK, whole = full / TOK;
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) ask(i & 1 ? vs : ks, i);
    wait_q();
    acc_t s[TT];
    uint32_t p[PAIRS];
    uint32_t place = 0;                                    // of item i; item i + NS - 1 goes to the place before it
    auto next = [&]() { place = place + 1 == NS ? 0 : place + 1; };
    auto before = [&]() { return place == 0 ? NS - 1 : place - 1; };
    constexpr bool V_FIRST = (NS - 1) & 1;                 // what item i + NS - 1 is, behind a K
    for (uint32_t j = 0; j < tiles; ++j) {
      sync<(NS - 2) * L>();
      ask(V_FIRST ? vs : ks, before());
      step(j);
      if (j < have) {
        products(s, lds + place * PLACE, k_at);
        if (j >= whole) hide(s, lim - (int32_t)(j * TOK));
        follow(largest(s), c);
      }
      next();
      sync<(NS - 2) * L>();
      ask(V_FIRST ? ks : vs, before());
      if (j < have) finish(s, p, lds + place * PLACE, v_at, c);
      next();
    }
    // what is still on its way is the zeros of items past the last one
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    l = over_row<AddOp>(l);
  }

  // Where the products are: the scores of the next tile are computed beside the exponentials of this one,
  // which keeps the matrix pipe and the vector pipe busy at the same time, and there is one barrier a tile.  Behind
  // tile j's, K of tile j + 1 and V of tile j are in LDS, and tile j - 1's V and tile j's K are done with:
  // their places take those of tiles j + 1 and j + 2.
  template <bool CAUSAL, class Step>
  __device__ __forceinline__ void run(Src qs, Src ks, Src vs, uint32_t n, uint32_t mine, uint32_t full, int32_t lim, float c,
                                      Step step, bool careful = false) {
    static_assert(NS == 4 && BLOCK_ROWS == 2 * TOK, "two tiles, and q as one");
    const uint32_t tiles = (n + TOK - 1) / TOK, have = (mine + TOK - 1) / TOK;
    const uint32_t whole = full / TOK < have ? full / TOK : have;
    auto below = [&](uint32_t j) { return lim + (CAUSAL ? (int32_t)(opaque(lane) % ROWS) : 0) - (int32_t)(j * TOK); };   // in tile j
    if constexpr (CAUSAL) {                                // q's rows come as tokens of K do, and are read as those are
      ask(qs, 2);
      ask(qs, 3);
    }
    ask(ks, 0);
    ask(vs, 1);
    acc_t s[2][TT];
    if constexpr (CAUSAL) {
      sync<L>();
#pragma unroll
      for (int k = 0; k < QK; ++k) q[k] = key(lds + (2 + wave / TT) * PLACE, k_at + wave % TT * (ROWS * ROWB), k * TT);
      sync<L>();
    } else {
      wait_q();
      sync<L>();
    }
    ask(ks, 2);
    if (have) {
      products(s[0], lds, opaque(k_at));
      if (whole == 0) hide(s[0], below(0));
      follow(largest(s[0]), c);
    }
    uint32_t j = 0;
    auto both = [&](auto par) {                            // tile j, in the places of tiles with its parity
      constexpr int P = decltype(par)::value;
      sync<0>();
      step(j);
      follow(tile<false>(s[1 - P], s[P], lds + (2 - 2 * P) * PLACE, lds + (1 + 2 * P) * PLACE, k_at, v_at, c, 0,
                         [&](int i) { i ? ask(vs, 3 - 2 * P) : ask(ks, 2 * P); }), c);
      ++j;
    };
    auto keep = [&]() {
#pragma unroll
      for (int t = 0; t < TT; ++t) s[0][t] = s[1][t];
    };
    while (j + 2 < whole) {
      both(std::integral_constant<int, 0>());
      both(std::integral_constant<int, 1>());
    }
    if (j + 1 < whole) {
      both(std::integral_constant<int, 0>());
      keep();
    }
    auto asks = [&](int i) { i ? ask(vs, 3 - 2 * (j & 1)) : ask(ks, 2 * (j & 1)); };
    if (j < whole && whole < have) {                       // the last that every row sees whole
      sync<0>();
      step(j);
      follow(tile<true>(s[1], s[0], lds + (2 - 2 * (j & 1)) * PLACE, lds + (1 + 2 * (j & 1)) * PLACE, opaque(k_at), opaque(v_at), c,
                        below(j + 1), asks), c);
      keep();
      ++j;
    }
    if (j < have) {                                        // the last one
      sync<0>();
      step(j);
      uint32_t p[PAIRS];
      const uint32_t at = lds + (1 + 2 * (j & 1)) * PLACE;
      if (j + 1 < tiles) {
        asks(0);
        asks(1);
      }
      if (CAUSAL && careful) finish_careful(s[0], p, at, opaque(v_at), c, below(j));
      else finish(s[0], p, at, opaque(v_at), c);
      ++j;
    }
    for (; j < tiles; ++j) {                               // those of the other waves alone
      sync<0>();
      asks(0);
      asks(1);
      step(j);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (as above)
    l = over_row<AddOp>(l);
  }

  // four neighbouring dims of the lane's row, times `by`, as bf16: those from ROWS d + 8 g + 4 (l / ROWS) on
  __device__ __forceinline__ uint2 four(int d, int g, float by) const {
    const acc_t &a = acc[d];
    return make_uint2(pack(a[4 * g] * by, a[4 * g + 1] * by), pack(a[4 * g + 2] * by, a[4 * g + 3] * by));
  }
#endif
};

// ---- a whole prompt ---------------------------------------------------------------------
// Logical block heads x slot + nth: 128 rows of one sequence for one query head.  (With a multiple of eight heads those that
// share a K/V head are dealt to one die, every eighth block's, as far as they are neighbours: one sequence of 700
// tokens, 32/8 heads, 15.0 us, in the heads' own order 15.6; long ones the same.)  Where sequences begin is
// known on the device alone, so the slots are dealt out without counting: sequence s has those from
// start(s) = cu[s] / 128 + s on up to start(s + 1), which are enough for its rows wherever it
// begins, and at most one of them has none.  A sequence's last rows, which attend to most tokens, come first.
template <int DIM>
struct PromptBodyT {
  using Args = tally_attn_prompt_args;
  typedef OnePass<DIM, 32, 64, 4> F;
  static constexpr int THREADS = 256;
  static constexpr int MIN_WAVES = 2;
  static constexpr unsigned DYN_LDS = F::LDS;
  static constexpr bool END_BARRIER = false;               // (a block opens with a barrier)
  static constexpr bool YIELDS = true;
  static constexpr bool RANGE = false;
  static_assert(F::BLOCK_ROWS == (int)kPromptRows && F::TOK == (int)kPromptTile, "rows of a block, tokens of a tile");
  static double pause_fraction(const Args &a, uint32_t every) { return prompt_pause_share(a, every); }
  static __device__ __forceinline__ void run(const Args &a, uint32_t bx, uint32_t, uint32_t) {
    run_impl<false, false>(a, bx, YieldCtl{nullptr, 0, 0, 15, false});
  }
  static __device__ __forceinline__ void run_be(const Args &a, uint32_t bx, uint32_t, uint32_t) {
    run_impl<true, false>(a, bx, YieldCtl{nullptr, 0, 0, 15, false});
  }
  static __device__ __forceinline__ void run_yielding(const Args &a, uint32_t bx, uint32_t, uint32_t, const YieldCtl ctl) {
    run_impl<true, true>(a, bx, ctl);
  }
  template <bool NT, bool YIELD>
  static __device__ __forceinline__ void run_impl(const Args &a, uint32_t block, const YieldCtl ctl) {
#ifdef __HIP_DEVICE_COMPILE__
    const uint32_t slot = block / a.heads, nth = block % a.heads;
    const uint32_t head = a.heads % 8 ? nth : nth % 8 * (a.heads / 8) + nth / 8;
    extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
    // the sequence of this slot: the last one that starts at or before it, 63 candidates at a time; the lane behind
    // the last candidate has where that one ends
    const uint32_t ln = threadIdx.x & 63;
    uint32_t seq = 0, first, last;
    for (uint32_t n = a.n_seqs;;) {
      const uint32_t step = (n + 62) / 63, s = ln * step < n ? ln * step : n;
      const int32_t v = a.cu_seqlens[seq + s];
      const uint32_t edge = v < 0 ? 0u : (uint32_t)v < a.total ? (uint32_t)v : a.total;
      const bool ok = s < n && edge / kPromptRows + seq + s <= slot;
      const uint32_t c = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(ok)), i = c ? c - 1 : 0;
      seq += i * step;
      if (step == 1) {
        first = (uint32_t)__builtin_amdgcn_readlane((int)edge, (int)i);
        last = (uint32_t)__builtin_amdgcn_readlane((int)edge, (int)i + 1);
        break;
      }
      n = n - i * step < step ? n - i * step : step;
    }
    const uint32_t len = last > first ? last - first : 0u;
    const uint32_t at = slot - (first / kPromptRows + seq), blocks = (len + kPromptRows - 1) / kPromptRows;
    if (at >= blocks) return;                              // (the same for the whole workgroup; slots before the first sequence wrap)
    const uint32_t row0 = (blocks - 1 - at) * kPromptRows;
    const uint32_t LDQ = a.ld_q ? a.ld_q : a.heads * DIM, LDO = a.ld_out ? a.ld_out : a.heads * DIM;
    const uint32_t LDK = a.ld_k ? a.ld_k : a.kv_heads * DIM, LDV = a.ld_v ? a.ld_v : a.kv_heads * DIM;
    const uint32_t kv = head / (a.heads / a.kv_heads);
    F f;
    f.begin(tally_dyn_lds);
    const uint32_t wrow = row0 + f.wave * F::ROWS;         // this wave's first row
    const uint32_t rows = wrow < len ? (len - wrow < (uint32_t)F::ROWS ? len - wrow : (uint32_t)F::ROWS) : 0u;
    const uint64_t qrow = (uint64_t)first + wrow;
    const uint32_t n = len < row0 + kPromptRows ? len : row0 + kPromptRows;
    uint32_t left = ctl.ticks, look = 0;
    const bool looks = YIELD && ctl.ticks != 0 && f.wave == 0;
    const buf_t flag = make_buf(ctl.flag, 4);
    if (YIELD && ctl.look_first && looks) yield_while_preempted(ctl, left);
    const float c = (a.scale > 0.f ? a.scale : DIM == 128 ? 0.08838834764831845f : 0.125f) * kLog2e;
    constexpr int FOURS = F::DT * F::AN / 4;
    uint2 v[FOURS];
    __syncthreads();                                       // (LDS may still be read for the block before)
    __shared__ uint32_t s_none;
    if (threadIdx.x == 0) s_none = 0;
    // Once as if all of K and V were numbers; if an output of the block is none, again with care.
    for (bool careful = false;; careful = true) {
      // the pause word is asked for behind a tile's loads and the answer acted on a tile later (as in the GEMM)
      f.template run<true>(f.source(a.q + ((uint64_t)first + row0) * LDQ + head * DIM, n - row0, LDQ),
                           f.source(a.k + (uint64_t)first * LDK + kv * DIM, n, LDK),
                           f.source(a.v + (uint64_t)first * LDV + kv * DIM, n, LDV), n, rows ? wrow + rows : 0u,
                           rows ? wrow + 1 : 0u, (int32_t)wrow + 1, c, [&](uint32_t j) {
                             if constexpr (YIELD) {
                               if (!looks) return;
                               if (j != 0 && ((j - 1) & ctl.mask) == ctl.mask && __builtin_amdgcn_readfirstlane(look) == ctl.epoch)
                                 yield_while_preempted(ctl, left);
                               if ((j & ctl.mask) == ctl.mask) look = __builtin_amdgcn_raw_buffer_load_b32(flag, 0, 0, 16);
                             }
                           }, careful);
      const float by = 1.f / f.l;
      float none = 0.f;                                    // zero times the outputs: NaN if one is no number
#pragma unroll
      for (int i = 0; i < FOURS; ++i) {
        v[i] = f.four(i / (F::AN / 4), i % (F::AN / 4), by);
        none = F::add_pair(v[i].x, none, 0u);
        none = F::add_pair(v[i].y, none, 0u);
      }
      if (f.lane % F::ROWS < rows && none != none) s_none = 1;
      __syncthreads();
      if (careful || s_none == 0) break;
      f.reset();
    }
    // The wave's rows go through a piece of LDS of its own, so that whole rows are written.  (Straight from the
    // registers an instruction would write 16 bytes here and there, 32 rows of them: 128 tokens 8.2 us and so 7.7.)
    typedef __attribute__((address_space(3))) uint2 *four_t;
    typedef const __attribute__((address_space(3))) u32x4_nt *chunk_t;
    const uint32_t lane = F::opaque(f.lane), row = lane % F::ROWS, mine = f.lds + f.wave * (F::ROWS * F::ROWB);
    constexpr uint32_t CHUNKS = F::ROWB / 16, PER = 64 / CHUNKS;   // rows that an instruction writes
    // (a row's chunks are xor-swizzled as in the ring)
#pragma unroll
    for (int i = 0; i < FOURS; ++i)
      *(four_t)(mine + row * F::ROWB + ((i ^ F::swz(row)) << 4) + lane / F::ROWS * 8) = v[i];
    asm volatile("" ::: "memory");                         // (written in one type and read in another)
    uint16_t *o = a.out + (qrow + lane / CHUNKS) * LDO + head * DIM + lane % CHUNKS * 8;
#pragma unroll
    for (uint32_t i = 0; i < F::ROWS / PER; ++i) {
      const uint32_t r = i * PER + lane / CHUNKS;
      const u32x4_nt w = *(chunk_t)(mine + r * F::ROWB + ((lane % CHUNKS ^ F::swz(r)) << 4));
      if (r < rows) {
        if constexpr (NT) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_nt *>(o + (uint64_t)(i * PER) * LDO));
        else *reinterpret_cast<u32x4_nt *>(o + (uint64_t)(i * PER) * LDO) = w;
      }
    }
#endif
  }
};
using PromptBody = PromptBodyT<128>;
using PromptNarrowBody = PromptBodyT<64>;

}  // namespace tally
