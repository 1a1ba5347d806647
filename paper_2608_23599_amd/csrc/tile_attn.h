// Attention of many query rows over tiles of keys and values in LDS: the part that the
// packed-prompt kernel (prompt.hip) and the chunk kernel (chunk.hip) share.
//
// Rows.  The G query heads of a KV head read the same keys, so the rows of one (sequence,
// KV head) are its (token, head) pairs in one order, row r = token r / G, head r % G: a
// tile of rows spans few tokens (little of a causal tile is masked away) and one token's
// heads fill a tile together.  A wavefront holds 32 rows.
//
// Arithmetic per 32-token group, on 32x32x16 MFMA (32 cycles each; the 16x16x32 form took
// 18.4 ns for the same products beside six vector instructions, this one 15.4):
//   S^T[token][row] = sum_d K[token][d] Q[row][d]          8 instructions
//   p = 2^(S sl2 - m)   (sl2 = log2(e) / sqrt(128), m per row)
//   O^T[d][row]    += sum_t V[t][d] p[t][row]              4 x 2 instructions
// With S transposed, a lane holds one row's scores in the accumulator layout (lane l: row
// l & 31, tokens 8 (i >> 2) + 4 (l >> 5) + (i & 3)), which is, two values a register, the
// layout of the second product's operand when its inner index runs over the tokens in that
// same order: the probabilities never leave their lane.  O^T has a row per lane too, so the
// rescale by a moved reference is one factor per lane.
//
// Weights are taken relative to a reference that is set kLead (log2 units) below the largest score so
// far and only moved when a score passes it by more than kRescale, 8 further: the sums are in fp32 and the
// common tile has no cross-lane step.  In fp16 (7 and 15) the largest weight of a row lies between 2^7 and
// 2^15, so that weights use the type's range on both sides: they stay below its 65504, are normal
// numbers down to 2^-21 of the largest one and vanish below 2^-32 of it.  (With the reference at
// the largest score itself they vanished below 2^-25: beside one token that took nearly all of a
// row's weight, 16384 others of together 5e-4 were lost.)  In bf16, which has fp32's range, the reference is
// the largest score (7 below, 16k tokens x 28/4 heads took 1844 us instead of 1820).  Weights enter the
// second product in the type of the values (one rounding of at most half a step each); the sum of a row
// adds the rounded ones, so the weights of a row sum to 1 as the product sees them.
//
// A masked score becomes -infinity by selection, never by arithmetic, so a NaN or infinity
// in a masked key has no effect; for masked values see find_odd.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#pragma clang diagnostic ignored "-Winline-asm"  // the LDS copies set M0 themselves (dma16)

namespace gkv {
namespace ta {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));

struct F16 {
  static constexpr float kRescale = 15.0f;  // an exponent above this moves the reference
  static constexpr float kLead = 7.0f;      // the largest one's exponent when it has moved
  static constexpr uint32_t kInf = 0x7C00u, kExp = 0x7C007C00u;  // infinity; the exponent bits of a pair
  __device__ static f16v mfma(u4 a, u4 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0,
                                                  0);
  }
  __device__ static uint32_t pack(float x, float y) {
    half2v h;
    h[0] = (_Float16)x;
    h[1] = (_Float16)y;
    return __builtin_bit_cast(uint32_t, h);
  }
  // acc + the two values of p
  __device__ static float add2(uint32_t p, float acc) {
    half2v one;
    one[0] = one[1] = (_Float16)1.0f;
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, p), one, acc, false);
  }
  // acc + 0 times each value of p: NaN if one is infinite or NaN
  __device__ static float times0(uint32_t p, float acc) {
    half2v none;
    none[0] = none[1] = (_Float16)0.0f;
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, p), none, acc, false);
  }
};
struct BF16 {
  static constexpr float kRescale = 8.0f, kLead = 0.0f;
  static constexpr uint32_t kInf = 0x7F80u, kExp = 0x7F807F80u;
  __device__ static f16v mfma(u4 a, u4 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  __device__ static uint32_t pack(float x, float y) {
    bf2 h;
    h[0] = (__bf16)x;
    h[1] = (__bf16)y;
    return __builtin_bit_cast(uint32_t, h);
  }
  __device__ static float add2(uint32_t p, float acc) {
    bf2 one;
    one[0] = one[1] = (__bf16)1.0f;
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, p), one, acc, false);
  }
  __device__ static float times0(uint32_t p, float acc) {
    bf2 none;
    none[0] = none[1] = (__bf16)0.0f;
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, p), none, acc, false);
  }
};

// ---------------------------------------------------------------- LDS tiles
// Keys: row-major rows of 256 B, 16-byte unit u of row r at place u ^ (r & 15): the 16 rows
// that a 16-byte read serves at once lie on distinct banks.
// Values, transposing form (kTr): row-major, unit u of row r at u ^ 4 (r & 3); read with
// ds_read_b64_tr_b16, which hands each of 16 lanes one column of four rows.
// Values, operand form: [16-token page][32-channel group][lane] units that hold what the
// lane feeds the MFMA (tokens 4 (l >> 5) .. + 3 and those + 8 of channel 32 ct + (l & 31)).
__device__ __forceinline__ uint32_t key_place(int row, int unit) { return row * 256 + ((unit ^ (row & 15)) << 4); }
__device__ __forceinline__ uint32_t value_place(int row, int unit) {
  return row * 256 + ((unit ^ ((row & 3) << 2)) << 4);
}

typedef __attribute__((address_space(3))) const u4 *LdsU4;
typedef __attribute__((address_space(3))) short4v *LdsTr;
__device__ __forceinline__ u4 lds_u4(uint32_t at) { return *(LdsU4)(uintptr_t)at; }
__device__ __forceinline__ u2 lds_tr(uint32_t at) {
  return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(uintptr_t)at));
}

// Lane addresses of the operand reads, relative to a tile's first byte.
struct Lane {
  int lane, col, hf;  // lane, row of the wavefront (l & 31), half (l >> 5)
  uint32_t k0;        // key operand of channels 0..15: the others are k0 ^ (s << 5)
  uint32_t v0;        // value operand of channel group 0: the others v0 ^ (ct << 6) (kTr), + 1024 ct (operand form)
  template <bool kTr>
  __device__ __forceinline__ void init() {
    lane = threadIdx.x & 63;
    col = lane & 31;
    hf = lane >> 5;
    k0 = key_place(col, hf);
    if (kTr) {
      const int r = (lane & 15) >> 2;
      v0 = value_place(4 * hf + r, 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
    } else {
      v0 = lane * 16;
    }
  }
};

// One wavefront's rows.
struct Rows {
  f16v o[4];  // O^T: register i of group ct is channel 32 ct + 8 (i >> 2) + 4 hf + (i & 3)
  float m;    // what exponents are taken relative to (log2 units, both halves alike)
  float raise;  // an exponent above this moves m: -infinity while the row has seen nothing
  float l;    // this half's sum
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    m = 0.f;
    raise = -__builtin_inff();
    l = 0.f;
  }
};

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// The value operand of 16-token page kk and channel group ct.
template <bool kTr>
__device__ __forceinline__ u4 value_operand(const Lane &ln, uint32_t vbase, int kk, int ct) {
  if constexpr (kTr) {
    const uint32_t at = vbase + (ln.v0 ^ (ct << 6)) + kk * 4096;
    const u2 a = lds_tr(at), b = lds_tr(at + 2048);
    return u4{a[0], a[1], b[0], b[1]};
  } else {
    return lds_u4(vbase + ln.v0 + (kk * 4 + ct) * 1024);
  }
}

// Pairs of v with infinity or NaN, as a mask of 16-bit halves.
template <class T>
__device__ __forceinline__ uint32_t bad_halves(uint32_t x) {
  const uint32_t lo = T::kExp & 0xFFFFu;
  return ((x & lo) == lo ? 0xFFFFu : 0u) | ((x & (lo << 16)) == (lo << 16) ? 0xFFFF0000u : 0u);
}

// What the scores of a 64-token tile start from: 0, or the tile's 64 floats at `bias`, in the
// accumulators' order.
template <bool kBias>
__device__ __forceinline__ void start_scores(f16v (&s)[2], const Lane &ln, uint32_t bias) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u4 x = {0, 0, 0, 0};
      if (kBias) x = lds_u4(bias + 128 * t + 32 * i + 16 * ln.hf);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t w = x[k];
        s[t][4 * i + k] = __builtin_bit_cast(float, w);
      }
    }
}

// Key operand of 32-token group t: channels 16 d .. + 15, or (d = 8) the second terms of the tile's
// hot channels, one unit a lane at `hot`.
__device__ __forceinline__ u4 key_operand(const Lane &ln, uint32_t kbase, uint32_t hot, int d, int t) {
  return d < 8 ? lds_u4(kbase + (ln.k0 ^ (d << 5)) + t * 8192) : lds_u4(hot + t * 1024 + ln.lane * 16);
}

// S^T of a 64-token tile.
template <class T, bool kBias, int NQ>
__device__ __forceinline__ void scores(f16v (&s)[2], const Lane &ln, const u4 (&q)[NQ], uint32_t kbase, uint32_t bias,
                                       uint32_t hot) {
  start_scores<kBias>(s, ln, bias);
#pragma unroll
  for (int d = 0; d < NQ; ++d)
#pragma unroll
    for (int t = 0; t < 2; ++t) s[t] = T::mfma(key_operand(ln, kbase, hot, d, t), q[d], s[t]);
}

// Scores of tokens whose bit in vis (of this lane's row) is clear become -infinity.
template <int NT>
__device__ __forceinline__ void mask_scores(f16v (&s)[NT], const Lane &ln, uint64_t vis) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint32_t w = (uint32_t)(vis >> (32 * t)) >> (4 * ln.hf);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      s[t][i] = (w >> (8 * (i >> 2) + (i & 3))) & 1u ? s[t][i] : -__builtin_inff();
  }
}

// Moves the references where a score passes one by more than kRescale, and turns scores into
// packed probabilities (two 16-token pages a group).
template <class T, int NT>
__device__ __forceinline__ void weights(u4 (&p)[2 * NT], Rows &r, const f16v (&s)[NT], float sl2) {
  // The maximum is taken of exponents (the compiler knows a product's result to be canonical;
  // of the MFMA's it would quiet every operand first), which are formed again after it: kept
  // across the rare branch, they and the outputs were copied on the common path (70 moves).
  float top = -__builtin_inff();
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, __builtin_fmaf(s[t][i], sl2, -r.m));
  if (__builtin_expect(__any(top > r.raise), 0)) {
    // only the rows that pass their own limit (one that has seen no score: at the first ones),
    // so that a row's rounding does not depend on its neighbours'
    const float high = fmaxf(top, other_half(top));
    const bool go = high > r.raise;
    const float up = go ? high - T::kLead : 0.f;
    const float f = r.raise < 0.f ? 0.f : __builtin_amdgcn_exp2f(-up);
    r.raise = go ? T::kRescale : r.raise;
    r.m += up;
    r.l *= f;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.o[c][i] *= f;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t w = T::pack(__builtin_amdgcn_exp2f(__builtin_fmaf(s[t][2 * j], sl2, -r.m)),
                                 __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][2 * j + 1], sl2, -r.m)));
      p[2 * t + (j >> 2)][j & 3] = w;
      r.l = T::add2(w, r.l);
    }
  // formed here, not past a barrier that follows
#pragma unroll
  for (int j = 0; j < 2 * NT; ++j) asm volatile("" : "+v"(p[j]));
  asm volatile("" : "+v"(r.l));
}

// Values (token t, channels 32 ct + 8 j + 4 hf .. + 3) of a tile.
template <bool kTr>
__device__ __forceinline__ u2 value_quad(int hf, uint32_t vbase, int t, int ct, int j) {
  if constexpr (kTr) {
    return *(__attribute__((address_space(3))) const u2 *)(uintptr_t)(vbase + value_place(t, 4 * ct + j) + 8 * hf);
  } else {
    const uint32_t at = vbase + ((t >> 4) * 4 + ct) * 1024 + 512 * ((t >> 2) & 1) + 8 * ((t >> 3) & 1) + 2 * (t & 3) +
                        16 * (8 * j + 4 * hf);
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = *(__attribute__((address_space(3))) const uint16_t *)(uintptr_t)(at + 16 * i);
    return u2{h[0] | h[1] << 16, h[2] | h[3] << 16};
  }
}

// A tile that is not whole for every row: a masked token has weight 0, and 0 times an
// infinity or NaN in its value would be NaN.  Finds whether a tile holds such values (a sum of
// all values times 0, a quarter of the product's time); if so they must not enter the
// product, and `odd` keeps, two bits for each of the lane's 64 outputs, which of them the
// row sees (1 infinity, 2 -infinity, 3 both or NaN), for add_odd to add in the end.
template <class T, int NT, bool kTr>
__device__ __forceinline__ bool find_odd(const Lane &ln, uint32_t vbase, uint64_t vis, u4 &odd) {
  float zero = 0.f;
#pragma unroll
  for (int kk = 0; kk < 2 * NT; ++kk)
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      const u4 v = value_operand<kTr>(ln, vbase, kk, ct);
#pragma unroll
      for (int j = 0; j < 4; ++j) zero = T::times0(v[j], zero);
    }
  const bool any = __any(zero != zero);
  if (__builtin_expect(any, 0)) {
    int hf = ln.hf;  // (opaque: no address of this path is kept in a register through the loop)
    asm volatile("" : "+s"(vbase), "+v"(hf));
#pragma unroll 1
    for (int t = 0; t < 32 * NT; ++t) {
      const uint32_t seen = (vis >> t) & 1 ? 3u : 0u;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u2 v = value_quad<kTr>(hf, vbase, t, i >> 2, i & 3);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t x = v[k >> 1] >> (16 * (k & 1)) & 0xFFFFu, e = x & 0x7FFFu;
          const uint32_t b = e < T::kInf ? 0u : e > T::kInf ? 3u : x == e ? 1u : 2u;
          odd[i >> 2] |= (b & seen) << (8 * (i & 3) + 2 * k);
        }
      }
    }
  }
  return any;
}

// The value product without infinities and NaN where `clean` (wave-uniform).
template <class T, int NT, bool kTr>
__device__ __forceinline__ void outputs_clean(Rows &r, const Lane &ln, const u4 (&p)[2 * NT], uint32_t vbase,
                                              bool clean) {
#pragma unroll
  for (int kk = 0; kk < 2 * NT; ++kk)
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
      u4 v = value_operand<kTr>(ln, vbase, kk, ct);
      if (__builtin_expect(clean, 0)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] &= ~bad_halves<T>(v[j]);
      }
      r.o[ct] = T::mfma(v, p[kk], r.o[ct]);
    }
}

__device__ __forceinline__ void add_odd(Rows &r, const u4 &odd) {
  if (__builtin_expect(!__any(odd[0] | odd[1] | odd[2] | odd[3]), 1)) return;
#pragma unroll
  for (int i = 0; i < 64; ++i) {
    const uint32_t b = odd[i >> 4] >> (2 * (i & 15)) & 3u;
    r.o[i >> 4][i & 15] += b == 0 ? 0.f : b == 3 ? __builtin_nanf("") : b == 1 ? __builtin_inff() : -__builtin_inff();
  }
}

// The value product of one 64-token tile and the key product of the next, one MFMA after the
// other with the operands read kAhead products before (the order is pinned: left alone, the
// compiler reads one ahead and every product waits for LDS).
template <class T, bool kTr, bool kBias, int NQ>
__device__ __forceinline__ void multiply(Rows &r, f16v (&s)[2], const Lane &ln, const u4 (&p)[4], const u4 (&q)[NQ],
                                         uint32_t vbase, uint32_t kbase, uint32_t bias, uint32_t hot) {
  constexpr int kAhead = 6, kAll = 16 + 2 * NQ;
  u4 x[kAhead];
  auto operand = [&](int i) {
    if (i < 16) return value_operand<kTr>(ln, vbase, i >> 2, i & 3);
    return key_operand(ln, kbase, hot, (i - 16) >> 1, i & 1);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) x[i] = operand(i);
  start_scores<kBias>(s, ln, bias);
#pragma unroll
  for (int i = 0; i < kAll; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    const u4 a = x[i % kAhead];
    if (i < 16) r.o[i & 3] = T::mfma(a, p[i >> 2], r.o[i & 3]);
    else s[i & 1] = T::mfma(a, q[(i - 16) >> 1], s[i & 1]);
    if (i + kAhead < kAll) x[i % kAhead] = operand(i + kAhead);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// A row's outputs, O / l, from its first element on.  The halves of a row's lanes exchange the
// quarters of two 8-channel groups, so that each stores 16 bytes.
template <class T>
__device__ __forceinline__ void store_row(uint16_t *row, const Rows &r, float inv, int hf) {
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      u4 w;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const u2 x = __builtin_bit_cast(
            u2, __builtin_amdgcn_permlane32_swap(
                    T::pack(r.o[c][4 * i + 2 * k] * inv, r.o[c][4 * i + 2 * k + 1] * inv),
                    T::pack(r.o[c][4 * i + 4 + 2 * k] * inv, r.o[c][4 * i + 5 + 2 * k] * inv), false, false));
        w[k] = x[0];
        w[2 + k] = x[1];
      }
      *(u4 *)(row + 32 * c + 8 * (i + hf)) = w;
    }
}

// ---------------------------------------------------------------- a workgroup's pass
constexpr int kTile = 64;                  // tokens of a tile
constexpr int kTileBytes = kTile * 128 * 2;  // of its keys, or of its values
constexpr int kBiasBytes = kTile * 4;
constexpr int kHot = 16;                     // hot channels: those whose keys have second terms
constexpr int kHotBytes = kTile * kHot * 2;
constexpr int kAttendLds = 4 * kTileBytes;   // two tiles; biases and second terms: 2 kBiasBytes, 2 kHotBytes more

// LDS copies of 16 bytes a lane, lane after lane from a wave-uniform LDS address.  The compiler puts
// no wait states in front of inline assembly: the base goes through a scalar move, as a vector
// memory instruction must not follow closely on a vector instruction that wrote its scalar operand
// (v_readlane), and that move stands between the write of M0 and its use.
__device__ __forceinline__ void dma16(uint32_t voff, const void *base, uint32_t lds) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds);
  uint64_t at;
  asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0"
               : "=&s"(at) : "v"(voff), "s"(base), "s"(m0v) : "memory", "m0");
}

// The rows of a workgroup over tiles t0 .. t1 - 1 (t0 < t1), those before `full` seen whole by
// every row; seen(t) gives a lane's row's visible tokens of any other.  src.keys(t, lds, bias, hot)
// and src.values(t, lds) issue the wavefront's part of a tile's copies.  load() gets the queries (a ninth operand
// for the hot channels, where there are any), after the first copies are on their way.
//
// The two wavefronts of a SIMD (w and w + WAVES / 2) work half a tile apart: while one
// multiplies (the last tile's values, this tile's keys) the other forms weights.  In the same
// phase they wait for one unit together: the MFMAs ran 43% of the time and the vector
// instructions 49% (16k tokens x 28 heads: 1975 us; half a tile apart 1744).
//
// Intervals, each ended by a barrier: the first wavefronts' key product of tile t is in interval
// 2 t, the second ones' in 2 t + 1.  Keys t + 1 and values t are copied from the start of
// interval 2 t on (whose buffers were last read in 2 t - 1; the first ones from the start on) and
// have arrived at the end of 2 t + 1.
template <class T, int WAVES, bool kTr, bool kBias, int NQ, class Src, class Seen, class Load>
__device__ __forceinline__ void attend(Rows &st, const Lane &ln, u4 (&q)[NQ], uint32_t lds, int wave, int t0, int t1,
                                       int full, float sl2, const Src &src, const Seen &seen, const Load &load) {
  const bool second = wave >= WAVES / 2;
  auto keys = [&](int t) { return lds + (t & 1) * kTileBytes; };
  auto values = [&](int t) { return lds + (2 + (t & 1)) * kTileBytes; };
  auto bias = [&](int t) { return lds + 4 * kTileBytes + (t & 1) * kBiasBytes; };
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
  auto meet = [] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto hot = [&](int t) { return lds + 4 * kTileBytes + 2 * kBiasBytes + (t & 1) * kHotBytes; };
  auto copy_keys = [&](int t) { src.keys(t, keys(t), bias(t), hot(t)); };
  auto copy = [&](int t) {
    if (t + 1 < t1) copy_keys(t + 1);
    if (t < t1) src.values(t, values(t));
  };
  auto before = [&](int t) {  // the value product of tile t
    if (!second) arrived();
    meet();
    if (!second) copy(t + 1);
  };
  auto after = [&](int t) {
    if (second) arrived();
    meet();
    if (second) copy(t + 2);
  };
  copy_keys(t0);
  copy(t0);
  load();
  // the queries have arrived (the loop's copies are in flight when they are used: a wait for
  // their loads there would wait for the copies)
#pragma unroll
  for (int d = 0; d < NQ; ++d) asm volatile("" : "+v"(q[d]));
  st.init();
  f16v s[2];
  u4 pr[4];
  if (full > t1 - 1) full = t1 - 1;
  arrived();
  meet();
  if (second) meet();
  scores<T, kBias>(s, ln, q, keys(t0), bias(t0), hot(t0));
  after(t0 - 1);
  int t = t0;
  for (; t < full; ++t) {
    weights<T, 2>(pr, st, s, sl2);
    before(t);
    multiply<T, kTr, kBias>(st, s, ln, pr, q, values(t), keys(t + 1), bias(t + 1), hot(t + 1));
    after(t);
  }
  u4 odd = {0, 0, 0, 0};  // infinities and NaN among the values from here on
  for (;; ++t) {
    const uint64_t vis = seen(t);
    mask_scores<2>(s, ln, vis);
    weights<T, 2>(pr, st, s, sl2);
    before(t);
    const bool clean = find_odd<T, 2, kTr>(ln, values(t), vis, odd);
    outputs_clean<T, 2, kTr>(st, ln, pr, values(t), clean);
    if (t == t1 - 1) break;
    scores<T, kBias>(s, ln, q, keys(t + 1), bias(t + 1), hot(t + 1));
    after(t);
  }
  if (!second) meet();
  add_odd(st, odd);
}

}  // namespace ta
}  // namespace gkv
