// Attention in one pass over K and V for gfx950: a whole prompt (causal, grouped heads, sequences
// of different lengths packed one behind the other) and single-token queries of a batch that
// shares a prefix.
//
// Scores never leave the registers.  With m the running maximum of a row's scores and p = exp(s - m),
// a row's state is (m, l = sum of p, acc = sum of p v); a new maximum rescales l and acc by
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
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "../../include/tally.h"
#include "kernels_gemm.h"
#include "kernels_stream.h"
#include "launch_forms.h"

namespace tally {

constexpr float kLog2e = 1.4426950408889634f;

template <int DIM_, int ROWS_, int TOK_, int NS_>
struct Flash {
  static constexpr int DIM = DIM_, ROWS = ROWS_, TOK = TOK_, NS = NS_, WAVES = 4;
  static constexpr int BLOCK_ROWS = ROWS * WAVES;
  static constexpr uint32_t ROWB = DIM * 2;                // bytes of a token's row
  static constexpr uint32_t PLACE = TOK * ROWB;            // bytes of an item
  static constexpr int L = PLACE / 1024 / WAVES;           // direct loads per wave and item
  static constexpr uint32_t RPL = 1024 / ROWB;             // tokens per load
  static constexpr unsigned LDS = PLACE * NS;
  static constexpr int MK = ROWS == 32 ? 16 : 32;          // k of one MFMA
  static constexpr int QK = DIM / MK, PV = TOK / MK;
  static constexpr int TT = TOK / ROWS, DT = DIM / ROWS;   // blocks of tokens and of dims
  static constexpr int AN = ROWS == 32 ? 16 : 4;           // accumulators of a block
  static_assert((DIM == 64 || DIM == 128) && (ROWS == 32 || ROWS == 16), "shapes that the maps below know");
  static_assert(L >= 1 && L * 1024 * WAVES == (int)PLACE && NS >= 3, "whole loads, two items on their way");

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
  acc_t s[TT];                                             // scores, then p
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
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = acc_t{};
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ Src source(const uint16_t *at, uint32_t tokens, uint32_t ld) const {
    Src r;
    r.at = (const unsigned char *)at;
    r.left = tokens;
    r.ld = ld * 2;
#pragma unroll
    for (int n = 0; n < L; ++n) {
      const uint32_t row = (wave * L + n) * RPL + lane / (ROWB / 16), c = lane % (ROWB / 16);
      r.voff[n] = row * r.ld + ((c ^ swz(row)) << 4);
    }
    return r;
  }
  // rows of q: a lane's, of `rows` that exist (the others read as zeros)
  __device__ __forceinline__ void read_q(const uint16_t *at, uint32_t rows, uint32_t ld) {
    const buf_t b = make_buf(at, rows * ld * 2);
#pragma unroll
    for (int k = 0; k < QK; ++k)
      q[k] = __builtin_bit_cast(bf16x8_t, buf_ld16(b, (lane % ROWS) * ld * 2 + (lane / ROWS) * 16, k * MK * 2));
  }

  // the next item of a source to a place of the ring; past its end nothing is moved and zeros are left
  __device__ __forceinline__ void ask(Src &r, uint32_t place) const {
    // (Assembly: knowing of the loads, the compiler waits for all of them before any transposing read.  They
    // have no destination in registers, sync() waits for them, and nothing else in these kernels uses m0.)
    const uint32_t n = r.left < (uint32_t)TOK ? r.left : (uint32_t)TOK;
    const uint64_t p = (uint64_t)(uintptr_t)r.at;
    const u32x4_t b = {(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, n * r.ld, 0x00027000u};
    uint32_t to = lds + place * PLACE + wave * (L * 1024u);
#pragma unroll
    for (int j = 0; j < L; ++j)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   ::"s"(to + j * 1024u), "v"(r.voff[j]), "s"(b) : "memory");
    r.at += (uint64_t)TOK * r.ld;
    r.left -= n;
  }
  // item i is there for everyone, and everyone is done with item i - 1
  __device__ __forceinline__ void sync() const {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * L) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  }

  // which token of a tile element e of block t stands for, without the lane's own part
  static constexpr uint32_t token(int t, int e) { return ROWS == 32 ? 32 * t + 8 * (e / 4) + e % 4 : 16 * t + e; }

  // scores of a tile and the softmax's step.  c: the scale times log2(e); lim: the lane's row may
  // attend to tokens of the tile below it (MASK only).
  template <bool MASK>
  __device__ __forceinline__ void scores(uint32_t place, float c, int32_t lim) {
    typedef const __attribute__((address_space(3))) bf16x8_t *frag_t;
    const uint32_t at = lds + place * PLACE;
    uint32_t k_at = this->k_at;
    if constexpr (MASK) asm volatile("" : "+v"(k_at));     // (its eight variants are not kept beside the other loop's)
#pragma unroll
    for (int t = 0; t < TT; ++t) s[t] = acc_t{};
#pragma unroll
    for (int k = 0; k < QK; ++k)
#pragma unroll
      for (int t = 0; t < TT; ++t)
        s[t] = mma(*(frag_t)(at + (k_at ^ (k * (MK * 2))) + t * (ROWS * ROWB)), q[k], s[t]);
    if constexpr (MASK) {
      const int32_t left = lim - 4 * (int32_t)(lane / ROWS);
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int e = 0; e < AN; ++e) s[t][e] = (int32_t)token(t, e) < left ? s[t][e] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < AN; ++e) top = fmaxf(top, s[t][e]);
    top = over_row<MaxOp>(top) * c;
    // A maximum that has grown by less than 2^8 is left as it is: p then stays below 2^8, which
    // costs nothing in floating point, and acc is rarely rescaled.
    if (__builtin_amdgcn_ballot_w64(top > m + 8.f) != 0) {
      const float now = fmaxf(m, top);
      const float a = exp2(m - (now == -INFINITY ? 0.f : now));
      m = now;
      l *= a;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < AN; ++e) acc[d][e] *= a;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < AN; ++e) s[t][e] = exp2(__builtin_fmaf(s[t][e], c, -ref));
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < AN; ++e) sum[e & 3] += s[t][e];
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }

  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const f32x2_t p = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2_t));
  }
  // p of MFMA step k as the second operand
  __device__ __forceinline__ bf16x8_t weights(int k) const {
    uint4 w;
    if constexpr (ROWS == 32) {
      const acc_t &p = s[k / 2];
      const int o = 8 * (k & 1);
      w = make_uint4(pack(p[o], p[o + 1]), pack(p[o + 2], p[o + 3]), pack(p[o + 4], p[o + 5]), pack(p[o + 6], p[o + 7]));
    } else {
      const acc_t &a = s[2 * k], &b = s[2 * k + 1];
      w = make_uint4(pack(a[0], a[1]), pack(a[2], a[3]), pack(b[0], b[1]), pack(b[2], b[3]));
    }
    return __builtin_bit_cast(bf16x8_t, w);
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
  __device__ __forceinline__ void add_values(uint32_t place, uint32_t v_at) {
    const uint32_t at = lds + place * PLACE;
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      const bf16x8_t p = weights(k);
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] = mma(__builtin_bit_cast(bf16x8_t, values(at, v_at, k, d)), p, acc[d]);
    }
  }
  // The same where some rows must not see some of the tokens.  Their p is zero, but zero times an
  // infinity or NaN of V is NaN: a tile that holds any goes through the product with zeros in their
  // place, and is then looked through token by token, where a row takes what it sees.
  __device__ __forceinline__ void add_values_masked(uint32_t place, int32_t lim) {
    const uint32_t at = lds + place * PLACE;
    uint32_t v_at = this->v_at, lane = this->lane;
    asm volatile("" : "+v"(v_at), "+v"(lane));
    u16x2_t big = {0, 0};
#pragma unroll
    for (int k = 0; k < PV; ++k)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint4 v = values(at, v_at, k, d);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) big = __builtin_elementwise_max(big, __builtin_bit_cast(u16x2_t, w[i] & 0x7FFF7FFFu));
        __builtin_amdgcn_sched_barrier(0);
      }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(big.x >= 0x7F80 || big.y >= 0x7F80) == 0, 1)) {
      add_values(place, v_at);
      return;
    }
#pragma unroll
    for (int k = 0; k < PV; ++k) {
      const bf16x8_t p = weights(k);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint4 v = values(at, v_at, k, d);
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] &= (w[i] & 0x7F80u) == 0x7F80u ? 0xFFFF0000u : 0xFFFFFFFFu;
          w[i] &= (w[i] & 0x7F800000u) == 0x7F800000u ? 0xFFFFu : 0xFFFFFFFFu;
        }
        acc[d] = mma(__builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3])), p, acc[d]);
        __builtin_amdgcn_sched_barrier(0);                 // (rare: in few registers rather than fast)
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

  // Tokens [0, n) of K and V, `n` the same for all four waves; `mine` of them are seen by rows of this
  // wave (none if 0).  A row attends to tokens below its `lim`; full: below that every row does.
  // CAUSAL: there is data behind a row's last token (otherwise zeros).  `step(j)` is called behind
  // the barrier of each tile.
  template <bool CAUSAL, class Step>
  __device__ __forceinline__ void run(Src ks, Src vs, uint32_t n, uint32_t mine, uint32_t full, int32_t lim, float c, Step step) {
    __syncthreads();                                       // (LDS may still be read for the block before)
    const uint32_t tiles = (n + TOK - 1) / TOK, have = (mine + TOK - 1) / TOK, whole = full / TOK;
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) ask(i & 1 ? vs : ks, i);
    // (q is waited for here: the compiler would do so in the loop, counting none of the loads above)
#pragma unroll
    for (int k = 0; k < QK; ++k) asm volatile("" : "+v"(q[k]));
    uint32_t place = 0;                                    // of item i; item i + NS - 1 goes to the place before it
    auto next = [&]() { place = place + 1 == NS ? 0 : place + 1; };
    auto before = [&]() { return place == 0 ? NS - 1 : place - 1; };
    constexpr bool V_FIRST = (NS - 1) & 1;                 // what item i + NS - 1 is, behind a K
    uint32_t j = 0;
    for (; j < whole && j < have; ++j) {
      sync();
      ask(V_FIRST ? vs : ks, before());
      step(j);
      scores<false>(place, c, 0);
      next();
      sync();
      ask(V_FIRST ? ks : vs, before());
      add_values(place, v_at);
      next();
    }
    for (; j < have; ++j) {
      const int32_t below = lim - (int32_t)(j * TOK);
      sync();
      ask(V_FIRST ? vs : ks, before());
      step(j);
      scores<true>(place, c, below);
      next();
      sync();
      ask(V_FIRST ? ks : vs, before());
      if constexpr (CAUSAL) add_values_masked(place, below);
      else add_values(place, v_at);
      next();
    }
    for (; j < tiles; ++j) {
      sync();
      ask(V_FIRST ? vs : ks, before());
      step(j);
      next();
      sync();
      ask(V_FIRST ? ks : vs, before());
      next();
    }
    // what is still on its way is the zeros of items past the last one
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    l = over_row<AddOp>(l);
  }

  // eight neighbouring dims of the lane's row, as bf16: of dims 16 g .. 16 g + 16 of block d the lane holds
  // the first eight or the last (lanes of 32 x 32 blocks); returns where they start
  __device__ __forceinline__ uint32_t eight(int d, int g, float by, uint4 &out) const {
    static_assert(ROWS == 32, "the swap is made for these");
    const acc_t &a = acc[d];
    const int e = 8 * g;
    out.x = pack(a[e] * by, a[e + 1] * by);
    out.y = pack(a[e + 2] * by, a[e + 3] * by);
    out.z = pack(a[e + 4] * by, a[e + 5] * by);
    out.w = pack(a[e + 6] * by, a[e + 7] * by);
    // the upper half's first four against the lower half's last four
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(out.x), "+v"(out.z));
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(out.y), "+v"(out.w));
    return d * 32 + g * 16 + (lane >> 5) * 8;
  }
#endif
};

// ---- a whole prompt ---------------------------------------------------------------------
constexpr uint32_t kPromptRows = 128;                      // rows of a logical block

inline uint32_t prompt_slots(const tally_attn_prompt_args &a) { return a.total / kPromptRows + a.n_seqs; }

// Logical block heads x slot + head: 128 rows of one sequence for one query head.  Where sequences begin is
// known on the device alone, so the slots are dealt out without counting: sequence s has those from
// start(s) = cu[s] / 128 + s on up to start(s + 1), which are enough for its rows wherever it
// begins, and at most one of them has none.  A sequence's last rows, which attend to most tokens, come first.
template <int DIM>
struct PromptBodyT {
  using Args = tally_attn_prompt_args;
  typedef Flash<DIM, 32, 64, 4> F;
  static constexpr int THREADS = 256;
  static constexpr int MIN_WAVES = 2;
  static constexpr unsigned DYN_LDS = F::LDS;
  static constexpr bool END_BARRIER = false;               // (a block opens with a barrier)
  static constexpr bool YIELDS = true;
  static constexpr bool RANGE = false;
  static_assert(F::BLOCK_ROWS == (int)kPromptRows, "rows of a block");
  // share of the longest block between two looks at the pause word, `every` tiles apart, and the
  // tile after, in which the answer is acted on
  static double pause_fraction(const Args &a, uint32_t every) {
    const uint32_t tiles = (a.total + F::TOK - 1) / F::TOK;
    return tiles > every + 1 ? (double)(every + 1) / tiles : 1.0;
  }
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
    const uint32_t head = block % a.heads, slot = block / a.heads;
    extern __shared__ __align__(1024) unsigned char tally_dyn_lds[];
    // the sequence of this slot: the last one that starts at or before it, 64 candidates at a time
    const uint32_t ln = threadIdx.x & 63;
    auto edge = [&](uint32_t s) {
      const int32_t v = a.cu_seqlens[s];
      return v < 0 ? 0u : (uint32_t)v < a.total ? (uint32_t)v : a.total;
    };
    uint32_t seq = 0;
    for (uint32_t n = a.n_seqs;;) {
      const uint32_t step = (n + 63) / 64, s = ln * step;
      const bool ok = s < n && edge(seq + s) / kPromptRows + seq + s <= slot;
      const uint32_t c = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(ok)), i = c ? c - 1 : 0;
      seq += i * step;
      if (step == 1) break;
      n = n - i * step < step ? n - i * step : step;
    }
    const uint32_t first = __builtin_amdgcn_readfirstlane(edge(seq));
    const uint32_t last = __builtin_amdgcn_readfirstlane(edge(seq + 1));
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
    const uint64_t qrow = (uint64_t)first + (rows ? wrow : 0u);
    f.read_q(a.q + qrow * LDQ + head * DIM, rows, LDQ);
    const uint32_t n = len < row0 + kPromptRows ? len : row0 + kPromptRows;
    uint32_t left = ctl.ticks, look = 0;
    const bool looks = YIELD && ctl.ticks != 0 && f.wave == 0;
    const buf_t flag = make_buf(ctl.flag, 4);
    if (YIELD && ctl.look_first && looks) yield_while_preempted(ctl, left);
    // the pause word is asked for behind a tile's loads and the answer acted on a tile later (as in the GEMM)
    f.template run<true>(f.source(a.k + (uint64_t)first * LDK + kv * DIM, n, LDK), f.source(a.v + (uint64_t)first * LDV + kv * DIM, n, LDV),
                         n, rows ? wrow + rows : 0u, rows ? wrow + 1 : 0u, (int32_t)(wrow + f.lane % F::ROWS + 1),
                         (a.scale > 0.f ? a.scale : DIM == 128 ? 0.08838834764831845f : 0.125f) * kLog2e, [&](uint32_t j) {
                           if constexpr (YIELD) {
                             if (!looks) return;
                             if (j != 0 && ((j - 1) & ctl.mask) == ctl.mask && __builtin_amdgcn_readfirstlane(look) == ctl.epoch)
                               yield_while_preempted(ctl, left);
                             if ((j & ctl.mask) == ctl.mask) look = __builtin_amdgcn_raw_buffer_load_b32(flag, 0, 0, 16);
                           }
                         });
    const float by = 1.f / f.l;
    uint16_t *o = a.out + (qrow + f.lane % F::ROWS) * LDO + head * DIM;
#pragma unroll
    for (int d = 0; d < F::DT; ++d)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint4 v;
        const uint32_t dim = f.eight(d, g, by, v);
        const u32x4_nt w = {v.x, v.y, v.z, v.w};
        if (f.lane % F::ROWS < rows) {
          if constexpr (NT) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_nt *>(o + dim));
          else *reinterpret_cast<u32x4_nt *>(o + dim) = w;
        }
      }
#endif
  }
};
using PromptBody = PromptBodyT<128>;
using PromptNarrowBody = PromptBodyT<64>;

}  // namespace tally
