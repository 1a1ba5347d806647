// Attention of the newest tokens of every sequence (a prompt's chunk, a speculative step's
// drafts) over the graded cache (sections 3.1, 3.2, 3.4 and 3.7): the many-query form of the
// dense decode read.
//
// Two ways, chosen for each sequence by its rows (tokens times heads of a group):
//  * few rows: every wavefront holds 16 of a (sequence, KV head)'s rows, copies blocks of its own
//    to LDS and decodes them into operands;
//  * many rows: the cache is decoded once to fp16 tiles in the workspace, over which row tiles
//    go as a prompt's do (tile_attn.h).
// Either splits a long context over workgroups whose partials a merge kernel joins.
//
// A tile's entries are rounded to fp16 once, code * scale + zero in one step, but for the keys' outlier
// channels (see hot channels); of few rows only values with scales per token are, all other scales go into
// the queries and outputs.  Outputs are then off by 0.3e-3 to 0.4e-3 of their size with many rows, 2.4e-4 to
// 2.6e-4 with few, where the rounding of the outputs themselves takes 2.0e-4.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gkv_internal.h"
#include "tile_attn.h"

using namespace gkv;

namespace {

using ta::f16v;
using ta::half2v;
using ta::u2;
using ta::u4;
using T16 = ta::F16;

constexpr int kMaxSeqs = GKV_MAX_CHUNK_SEQS;
constexpr int kPart = D + 4;  // floats of a row's partial: O, m, l, none twice (16-byte rows)

struct ChunkParams {
  const uint16_t *q;
  uint16_t *out;
  float *part;
  int64_t qs, os;  // elements from a token's rows to the next one's
  const int8_t *level;
  const int64_t *koff, *voff;
  const uint8_t *arena;
  const uint64_t *res_mask;  // null without residual rows
  const int32_t *res_idx, *res_off;
  const uint8_t *res_rows;
  int32_t nblk_cap, Hkv, G, nseq, nres, nres_cap, nrb_cap, vtok;
  float sl2;
  int64_t part0;             // first partial row of this launch
  uint8_t *list;             // many rows: the decoded tiles
  int32_t *whole;            // and how many of each list every row sees whole
  uint8_t *hot;              // and each list's hot channels; bytes of a tile
  int32_t tile;
  int32_t list0[kMaxSeqs];   // first tile of a sequence's lists (one a KV head)
  int32_t T[kMaxSeqs], n[kMaxSeqs];  // its tokens, and the newest ones that attend
  int32_t row0[kMaxSeqs];    // their first packed row
  uint16_t split[kMaxSeqs];  // workgroups that share a row tile's context
  uint8_t seq[kMaxSeqs];     // sequence
  int32_t wg0[kMaxSeqs + 1]; // workgroups per KV head before each
};

// ---------------------------------------------------------------- records to tiles
// Table entries are the same for a whole wavefront and no kernel here writes them: scalar loads,
// which wait apart from the records' vector loads (as vector loads they would stand in line with
// those, and every block would wait for its table entries alone).
typedef const __attribute__((address_space(4))) uint64_t *ScalarU64;
typedef const __attribute__((address_space(4))) uint32_t *ScalarU32;
__device__ __forceinline__ uint64_t table64(const void *t, int64_t i) { return ((ScalarU64)(uintptr_t)t)[i]; }
__device__ __forceinline__ uint32_t table32(const void *t, int64_t i) { return ((ScalarU32)(uintptr_t)t)[i]; }
__device__ __forceinline__ int table8(const int8_t *t, int64_t i) {  // by the word it lies in
  const uintptr_t at = (uintptr_t)t + i;
  return *(ScalarU32)(at & ~(uintptr_t)3) >> (8 * (at & 3)) & 0xFFu;
}

// A block, or 64 residual rows, as it is read (wave-uniform).
struct Visit {
  const uint8_t *k, *v;  // records
  int level;
  uint64_t drop;  // tokens that are read elsewhere (residual rows) or are no rows
};

__device__ __forceinline__ Visit visit_at(const ChunkParams &p, int64_t u, int v, int nblk) {
  Visit x;
  if (v < nblk) {
    const int64_t ti = u * p.nblk_cap + v;
    x.level = table8(p.level, ti);
    x.k = p.arena + table64(p.koff, ti);
    x.v = p.arena + table64(p.voff, ti);
    x.drop = p.res_mask ? table64(p.res_mask, ti) : 0;
  } else {
    const int r = v - nblk;
    x.level = GKV_EXACT;
    x.k = p.res_rows + (u * p.nrb_cap + r) * (2 * kExactBytes);
    x.v = x.k + kExactBytes;
    const int left = p.nres - r * P;
    x.drop = left >= P ? 0 : ~0ull << left;
  }
  return x;
}

// What a lane reads of a record for its chunk of page pg (kg = lane >> 4, m = lane & 15): the
// codes of an integer level, the values of an exact one, a centroid block's four rows (keys:
// the one of the lane's token), a one-centroid block's row.
struct Raw {
  u4 w[4];
};
template <int TENSOR>
__device__ __forceinline__ void load_raw(Raw &x, const uint8_t *rec, int level, int pg, int lane) {
  const int kg = lane >> 4, m = lane & 15;
  if (level == GKV_EXACT) {
    const u4 *s = (const u4 *)(rec + (pg * 64 + lane) * 64);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.w[i] = s[i];
  } else if (level == GKV_INT8) {
    const u4 *s = (const u4 *)(rec + kSZBytes + (pg * 64 + lane) * 32);
    x.w[0] = s[0];
    x.w[1] = s[1];
  } else if (level == GKV_INT4) {
    x.w[0] = *(const u4 *)(rec + kSZBytes + (pg * 64 + lane) * 16);
  } else if (level == GKV_INT2) {
    const u2 s = *(const u2 *)(rec + kSZBytes + (pg * 64 + lane) * 8);
    x.w[0][0] = s[0];
    x.w[0][1] = s[1];
  } else if (TENSOR == GKV_KEYS) {
    const uint16_t *c = (const uint16_t *)rec + 8 * kg;
    if (level == GKV_CENTROID) c += (table32(rec + KC * D * 2, pg) >> (2 * m) & 3u) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.w[i] = *(const u4 *)(c + 32 * i);
  } else if (level == GKV_CENTROID) {
    const u4 *s = (const u4 *)(rec + m * 64);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.w[i] = s[i];
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c) x.w[c >> 2][c & 3] = ((const uint16_t *)rec)[16 * c + m] * 0x10001u;
  }
}

// Codes 2 q and 2 q + 1 of a chunk under a fixed exponent, 2^k + code in fp16 (exact), and that
// power of two; words 2 c and 2 c + 1 have the same one.  It is small (but for eight bits): where the
// codes are multiplied as they are, it is part of every product and taken off the sum.
template <int BITS>
__device__ __forceinline__ uint32_t raw_offset(int q) {
  if constexpr (BITS == 8) return 0x64006400u;
  if constexpr (BITS == 4) return (q & 2) ? 0x4C004C00u : 0x54005400u;
  const uint32_t e[4] = {0x44004400u, 0x4C004C00u, 0x54005400u, 0x44004400u};
  return e[(q & 7) >> 1];
}
// The exponents in vector registers, behind the compiler's back: an and-or takes one constant that
// is not in one, and as literals they make it two instructions.
struct Exponents {
  uint32_t e4, e16, e64, e1024;
  __device__ __forceinline__ Exponents() : e4(0x44004400u), e16(0x4C004C00u), e64(0x54005400u), e1024(0x64006400u) {
    asm("" : "+v"(e4), "+v"(e16), "+v"(e64), "+v"(e1024));
  }
};
template <int BITS>
__device__ __forceinline__ uint32_t raw_pair(const u4 (&w)[4], int q, const Exponents &x) {
  const bool odd = q & 1;
  if constexpr (BITS == 8) {
    return __builtin_amdgcn_perm(x.e1024, w[q >> 3][(q >> 1) & 3], odd ? 0x07030702u : 0x07010700u);
  } else if constexpr (BITS == 4) {
    const uint32_t y = w[0][q >> 2];
    if (q & 2) return ((odd ? y >> 2 : y << 6) & 0x03C003C0u) | x.e16;
    return ((odd ? y >> 8 : y) & 0x00F000F0u) | x.e64;
  } else {
    const uint32_t y = w[0][q >> 3];
    switch (q & 7) {
      case 0: case 1: return ((odd ? y >> 6 : y) & 0x03000300u) | x.e4;
      case 2: case 3: return ((odd ? y >> 6 : y) & 0x00C000C0u) | x.e16;
      case 4: case 5: return ((odd ? y >> 6 : y) & 0x00300030u) | x.e64;
      default: return ((odd ? y << 6 : y << 8) & 0x03000300u) | x.e4;
    }
  }
}
// The codes alone.
template <int BITS>
__device__ __forceinline__ half2v code_pair(const u4 (&w)[4], int q, const Exponents &e) {
  const uint32_t x = raw_pair<BITS>(w, q, e), off = raw_offset<BITS>(q);
  return __builtin_bit_cast(half2v, x) - __builtin_bit_cast(half2v, off);
}

typedef __attribute__((address_space(3))) u4 *LdsW4;
typedef __attribute__((address_space(3))) u2 *LdsW2;
typedef __attribute__((address_space(3))) uint32_t *LdsW1;

__device__ __forceinline__ uint32_t lds_u16(uint32_t at) {
  return *(__attribute__((address_space(3))) const uint16_t *)(uintptr_t)at;
}

// Scales and zeros in LDS: keys in the record's lane order (a lane's 32 are side by side);
// values per channel as [channel & 15][channel >> 4], so that a lane's 8 are; values per
// token in token order.  One wavefront loads both headers, 16 bytes a lane: keys in lanes
// 0..31, values in 32..63.
__device__ __forceinline__ u4 load_head(const Visit &x, int lane) {
  return *(const u4 *)((lane < 32 ? x.k : x.v) + (lane & 31) * 16);
}
__device__ __forceinline__ void store_head(uint32_t head, u4 x, int lane, bool vtok) {
  if (lane < 32 || vtok) {
    *(LdsW4)(uintptr_t)(head + lane * 16) = x;
    return;
  }
  const int l = lane - 32, e0 = (l & 15) * 8, a = e0 >> 5, c = (e0 >> 2) & 7;  // entries 32 a + 4 c + b
  const uint32_t at = head + 512 + (l >> 4) * 256 + (4 * a * 8 + c) * 2;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    *(__attribute__((address_space(3))) uint16_t *)(uintptr_t)(at + (i & 3) * 16 + (i >> 2) * 2) =
        (uint16_t)(x[i >> 1] >> (16 * (i & 1)));
}

// (taken by value: a bit cast of a vector's element itself reads the first one)
__device__ __forceinline__ half2v halves(uint32_t x) { return __builtin_bit_cast(half2v, x); }
__device__ __forceinline__ uint32_t decoded(half2v code, uint32_t scale, uint32_t zero) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code, halves(scale), halves(zero)));
}

// Entries past the largest fp16 number, which codes of values next to it can stand for (eight bits, values
// 0 .. 65504: 255 * 257), are that number: as infinities they would make whole outputs infinite or
// NaN.  What an infinite scale or zero, or a NaN, decodes to stays as it is.
template <int BITS, class Pairs>
__device__ __forceinline__ bool past_fp16(const Pairs &scales, const Pairs &zeros) {  // (or not a number, in some lane)
  half2v most;
  most[0] = most[1] = (_Float16)(float)((1 << BITS) - 1);
  float zero = 0.f;
#pragma unroll
  for (uint32_t i = 0; i < sizeof(Pairs) / 4; ++i) zero = T16::times0(decoded(most, scales[i], zeros[i]), zero);
  return __any(zero != zero);
}
__device__ __forceinline__ uint32_t bounded(uint32_t y, uint32_t scale, uint32_t zero) {
  const uint32_t off = ta::bad_halves<T16>(scale) | ta::bad_halves<T16>(zero);  // halves that stay
  const uint32_t lo = (y & 0xFFFFu) == T16::kInf ? 1u : 0u, hi = y >> 16 == T16::kInf ? 0x10000u : 0u;
  return y - ((lo | hi) & ~off);
}

template <int BITS>
__device__ __forceinline__ void stage_key_codes(uint32_t (&y)[16], const Raw &x, uint32_t head, int kg, const Exponents &e) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const u4 s = ta::lds_u4(head + kg * 64 + j * 16), z = ta::lds_u4(head + 256 + kg * 64 + j * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[4 * j + i] = decoded(code_pair<BITS>(x.w, 4 * j + i, e), s[i], z[i]);
    if (__builtin_expect(past_fp16<BITS>(s, z), 0))
#pragma unroll
      for (int i = 0; i < 4; ++i) y[4 * j + i] = bounded(y[4 * j + i], s[i], z[i]);
  }
}
__device__ __forceinline__ half2v twice(uint32_t pair, int i) {
  const half2v h = halves(pair);
  half2v r;
  r[0] = r[1] = h[i];
  return r;
}
template <int BITS>
__device__ __forceinline__ void stage_value_codes(uint32_t (&y)[16], const Raw &x, uint32_t head, int pg, int lane,
                                                  bool vtok, const Exponents &e) {
  const int kg = lane >> 4, m = lane & 15;
  if (vtok) {  // tokens 16 pg + 4 kg .. + 3
    const u2 s = *(LdsW2)(uintptr_t)(head + 512 + (16 * pg + 4 * kg) * 2);
    const u2 z = *(LdsW2)(uintptr_t)(head + 512 + 128 + (16 * pg + 4 * kg) * 2);
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] = decoded(code_pair<BITS>(x.w, q, e), s[q & 1], z[q & 1]);
    if (__builtin_expect(past_fp16<BITS>(s, z), 0))
#pragma unroll
      for (int q = 0; q < 16; ++q) y[q] = bounded(y[q], s[q & 1], z[q & 1]);
  } else {
    const u4 s = ta::lds_u4(head + 512 + m * 16), z = ta::lds_u4(head + 768 + m * 16);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int c = q >> 1;
      y[q] = __builtin_bit_cast(uint32_t,
                                __builtin_elementwise_fma(code_pair<BITS>(x.w, q, e), twice(s[c >> 1], c & 1),
                                                          twice(z[c >> 1], c & 1)));
    }
    if (__builtin_expect(past_fp16<BITS>(s, z), 0))
#pragma unroll
      for (int q = 0; q < 16; ++q)
        y[q] = bounded(y[q], __builtin_bit_cast(uint32_t, twice(s[q >> 2], q >> 1 & 1)),
                       __builtin_bit_cast(uint32_t, twice(z[q >> 2], q >> 1 & 1)));
  }
}

// A lane's key chunk of a page as fp16 pairs: words 4 j .. 4 j + 3 are channels 32 j + 8 kg .. + 7.
template <int LEVEL>
__device__ __forceinline__ void key_words(uint32_t (&y)[16], const Raw &x, uint32_t head, int kg, const Exponents &e) {
  if constexpr (LEVEL == GKV_INT8 || LEVEL == GKV_INT4 || LEVEL == GKV_INT2) {
    stage_key_codes<LEVEL>(y, x, head, kg, e);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x.w[i >> 2][i & 3];
  }
}

// The same of any level.
__device__ __forceinline__ void key_words_any(uint32_t (&y)[16], const Raw &x, int level, uint32_t head, int kg,
                                              const Exponents &e) {
  if (level == GKV_INT8) key_words<GKV_INT8>(y, x, head, kg, e);
  else if (level == GKV_INT4) key_words<GKV_INT4>(y, x, head, kg, e);
  else if (level == GKV_INT2) key_words<GKV_INT2>(y, x, head, kg, e);
  else key_words<GKV_EXACT>(y, x, head, kg, e);
}

// A lane's value chunk of a centroid block: its channels' centroids, four to a channel, by the two
// bits of each of its four tokens.
__device__ __forceinline__ void centroid_words(uint32_t (&y)[16], const u4 (&cent)[4], uint32_t ids) {
  uint32_t sel[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t a = ids >> (4 * i) & 3u, b = ids >> (4 * i + 2) & 3u;
    sel[i] = (2 * a) | (2 * a + 1) << 8 | (2 * b) << 16 | (2 * b + 1) << 24;
  }
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const int c = q >> 1;
    y[q] = __builtin_amdgcn_perm(cent[c >> 1][2 * (c & 1) + 1], cent[c >> 1][2 * (c & 1)], sel[q & 1]);
  }
}
// Zeros for the tokens of page pg in drop.
__device__ __forceinline__ void drop_words(uint32_t (&y)[16], uint64_t drop, int pg, int kg) {
  const uint32_t d = (uint32_t)(drop >> (16 * pg)) >> (4 * kg);
  const uint32_t keep[2] = {(d & 1 ? 0 : 0xFFFFu) | (d & 2 ? 0 : 0xFFFF0000u),
                            (d & 4 ? 0 : 0xFFFFu) | (d & 8 ? 0 : 0xFFFF0000u)};
#pragma unroll
  for (int q = 0; q < 16; ++q) y[q] &= keep[q & 1];
}

// A lane's value chunk of page pg as fp16 pairs: words 2 c and 2 c + 1 are tokens 4 kg .. + 3 of
// channel 16 c + m.  drop: the block's tokens that are not read, whose values become zero
// (their weight is zero, but 0 * infinity is NaN).
template <int LEVEL>
__device__ __forceinline__ void value_words(uint32_t (&y)[16], const Raw &x, const uint8_t *rec, uint64_t drop,
                                            uint32_t head, int pg, int lane, bool vtok, const Exponents &e) {
  const int kg = lane >> 4;
  if constexpr (LEVEL == GKV_INT8 || LEVEL == GKV_INT4 || LEVEL == GKV_INT2) {
    stage_value_codes<LEVEL>(y, x, head, pg, lane, vtok, e);
  } else if constexpr (LEVEL == GKV_CENTROID) {
    centroid_words(y, x.w, table32(rec + KC * D * 2, pg) >> (8 * kg));
  } else if constexpr (LEVEL == GKV_MEAN) {
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] = x.w[q >> 3][(q >> 1) & 3];
  } else {
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] = x.w[q >> 2][q & 3];
  }
  if (drop) drop_words(y, drop, pg, kg);
}

// The same of any level.
__device__ __forceinline__ void value_words_any(uint32_t (&y)[16], const Raw &x, const Visit &v, uint32_t head, int pg,
                                                int lane, bool vtok, const Exponents &e) {
#define GKV_WORDS(lv) value_words<lv>(y, x, v.v, v.drop, head, pg, lane, vtok, e)
  if (v.level == GKV_INT8) GKV_WORDS(GKV_INT8);
  else if (v.level == GKV_INT4) GKV_WORDS(GKV_INT4);
  else if (v.level == GKV_INT2) GKV_WORDS(GKV_INT2);
  else if (v.level == GKV_CENTROID) GKV_WORDS(GKV_CENTROID);
  else if (v.level == GKV_MEAN) GKV_WORDS(GKV_MEAN);
  else GKV_WORDS(GKV_EXACT);
#undef GKV_WORDS
}

// ---------------------------------------------------------------- rows
// The part of a call that one workgroup computes.
struct Job {
  int s, h, tile, part;  // place among the launch's sequences, KV head, row tile, share of the context
  int T, n, pos0;        // tokens, new ones, the first new one's position
  int rows, nblk;        // rows of the (sequence, KV head); blocks
  int64_t u, row0;
};

__device__ __forceinline__ Job job_of(const ChunkParams &p, int rows_tile, int h, int w) {
  Job j;
  j.h = h;
  int lo = 0, hi = p.nseq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.wg0[mid] <= w) lo = mid;
    else hi = mid;
  }
  w -= p.wg0[lo];
  j.s = lo;
  j.T = p.T[lo];
  j.n = p.n[lo];
  j.pos0 = j.T - j.n;
  j.rows = j.n * p.G;
  const int tiles = (j.rows + rows_tile - 1) / rows_tile;
  j.tile = w % tiles;
  j.part = w / tiles;
  j.nblk = (j.T + P - 1) / P;
  j.u = (int64_t)p.seq[lo] * p.Hkv + j.h;
  j.row0 = p.row0[lo];
  return j;
}

// The row of the launch's partials at which a workgroup's rows begin.
__device__ __forceinline__ int64_t part_row(const ChunkParams &p, const Job &j, int rows_tile) {
  // a KV head's partials lie tile after tile in the order of its workgroups
  const int tiles = (j.rows + rows_tile - 1) / rows_tile;
  return p.part0 + ((int64_t)j.h * p.wg0[p.nseq] + p.wg0[j.s] + j.part * tiles + j.tile) * rows_tile;
}

template <bool kRest, int NQ>
__device__ __forceinline__ void load_queries(u4 (&q)[NQ], const ChunkParams &p, const Job &j, int tok, int g, int hf) {
  const uint16_t *qp = p.q + (j.row0 + tok) * p.qs + (int64_t)(j.h * p.G + g) * D;
#pragma unroll
  for (int d = 0; d < 8; ++d) q[d] = *(const u4 *)(qp + 16 * d + 8 * hf);
  if constexpr (kRest) {  // the hot channels once more
    const int64_t at = ((int64_t)j.s * p.Hkv + j.h) * (ta::kHot / 4);
    const u4 ids = {table32(p.hot, at), table32(p.hot, at + 1), table32(p.hot, at + 2), table32(p.hot, at + 3)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = (hf ? ids[2 + (i >> 1)] : ids[i >> 1]) >> (16 * (i & 1));
      q[8][i] = qp[two & 0xFF] | (uint32_t)qp[two >> 8 & 0xFF] << 16;
    }
  }
}

__device__ __forceinline__ void store_part(float *part, const ta::Rows &st, float l, int hf) {
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(float4 *)(part + 32 * c + 8 * i + 4 * hf) =
          make_float4(st.o[c][4 * i], st.o[c][4 * i + 1], st.o[c][4 * i + 2], st.o[c][4 * i + 3]);
  if (!hf) *(float2 *)(part + D) = make_float2(st.m, l);
}

// Tokens of visit v that the token at position pos sees, of the ones not dropped.
__device__ __forceinline__ uint64_t seen_by(const ChunkParams &p, const Job &j, int v, uint64_t drop, int pos) {
  if (v < j.nblk) {
    const int n = pos + 1 - v * P;
    return (n >= P ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1) & ~drop;
  }
  const int32_t *idx = p.res_idx + j.u * p.nres_cap + (v - j.nblk) * P;  // ascending
  const int most = min(P, p.nres - (v - j.nblk) * P);
  int lo = 0, hi = most;  // rows whose token lies at or before pos
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (idx[mid] <= pos) lo = mid + 1;
    else hi = mid;
  }
  return lo >= P ? ~0ull : (1ull << lo) - 1;
}

// Whether every token of visit v lies at or before position pos.
__device__ __forceinline__ bool whole_at(const ChunkParams &p, const Job &j, int v, int pos) {
  if (v < j.nblk) return v * P + P - 1 <= pos;
  const int last = min(P, p.nres - (v - j.nblk) * P) - 1;
  return (int)table32(p.res_idx, j.u * p.nres_cap + (v - j.nblk) * P + last) <= pos;
}

// ---------------------------------------------------------------- many rows
// The cache of a (sequence, KV head) as a list of tiles (ta::attend's, 64 tokens each) in the
// workspace, decoded once for all row tiles:
//   the blocks before block c0 = pos0 / 64, which every row sees whole, but for one-centroid
//   ones | the residual rows of tokens before 64 c0 | the one-centroid blocks before c0, one
//   key each | the blocks from c0 on, each with its residual tokens in their places.
// A tile is 16 KB of keys, 16 KB of values and 64 floats that its scores start from: 0, minus
// infinity for a place that holds no token (a residual token's in its block, those behind
// the last row), log2(n) in a score's units for a one-centroid block, whose key counts for
// its n tokens that are no residual ones.  Where a sequence of the call has integer blocks, 2 KB more: what the
// rounding to fp16 took off the keys of the list's 16 hot channels, as operands of one more product.
//
// Hot channels are those of the largest keys (key channels are known to have outliers): a score's error is
// that of its largest products.  With four channels ten times larger than the others the keys' rounding put the
// outputs off by 0.7e-3 to 1.0e-3, over one level of codes, now by 2e-4.  (Rounding up or down at random,
// tokens apart, came to 1.1e-3: a long context's outputs are themselves sums in which the tokens' values
// cancel, so that errors that differ from token to token do not become less beside them.)  It costs a sixteenth
// of the products: 512 tokens over 64k 568 us against 531, mixed chunks 313 against 287.
constexpr int kListTile = 2 * ta::kTileBytes + ta::kBiasBytes;

// Room of a list: a tile for every block and for every 64 residual rows.
__host__ __device__ __forceinline__ int list_tiles(int T, int nres) { return (T + P - 1) / P + (nres + P - 1) / P; }
__device__ __forceinline__ int list_tiles(const ChunkParams &p, int T) { return list_tiles(T, p.nres); }

struct ListShape {  // of one (sequence, KV head)
  int plain, res, means;  // tiles of the first two parts, one-centroid blocks
  int whole;              // tiles before block c0's
};
__device__ __forceinline__ ListShape list_shape(const ChunkParams &p, int c0, int means) {
  ListShape l;
  l.means = means;
  l.plain = c0 - means;
  l.res = (p.nres + P - 1) / P;
  l.whole = l.plain + l.res + (means + P - 1) / P;
  return l;
}

// The hot channels of every list: the 16 with the largest keys in up to 16 integer blocks spread over the
// context, by the ends of their ranges.  A thread a channel.  Bound by latency (three dependent round trips).
__global__ void __launch_bounds__(D) hot_kernel(const ChunkParams p) {
  constexpr int kSamples = 16;
  __shared__ const _Float16 *heads[kSamples];
  __shared__ float most[kSamples];  // a sample's largest code (0: no integer block)
  __shared__ __align__(16) uint32_t size[D];
  const int s = blockIdx.y, h = blockIdx.x, e = threadIdx.x;  // (e: place in a record's header)
  const int nblk = (p.T[s] + P - 1) / P;
  const int64_t u = (int64_t)p.seq[s] * p.Hkv + h;
  int any = 0;
  if (e < kSamples) {
    const int64_t ti = u * p.nblk_cap + (int64_t)e * nblk / kSamples;
    const int level = p.level[ti];
    any = is_int_level(level);
    heads[e] = (const _Float16 *)(p.arena + p.koff[ti]);
    most[e] = any ? (float)((1 << level) - 1) : 0.f;
  }
  float sum = 0.f;
  if (__syncthreads_or(any)) {
    int last = 0;  // an integer block (the others' records may be shorter than a header)
#pragma unroll
    for (int i = 0; i < kSamples; ++i) last = most[i] != 0.f ? i : last;
    float scale[kSamples], zero[kSamples];
#pragma unroll
    for (int i = 0; i < kSamples; ++i) {
      const _Float16 *head = heads[most[i] != 0.f ? i : last];
      scale[i] = (float)head[e];
      zero[i] = (float)head[D + e];
    }
#pragma unroll
    for (int i = 0; i < kSamples; ++i) {
      const float end = __builtin_fmaf(most[i], scale[i], zero[i]);
      sum += most[i] != 0.f ? fmaxf(zero[i] * zero[i], end * end) : 0.f;
    }
    sum = fminf(sum, 3e38f);  // (a NaN, too, is only large)
  }
  // sums that are no less than 0 compare as their bits do; the last seven tell channels apart
  const int d = sz_channel(GKV_KEYS, e);
  const uint32_t mine = (__builtin_bit_cast(uint32_t, sum) & ~127u) | d;
  size[d] = mine;
  __syncthreads();
  int rank = 0;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) {
    const u4 x = *(const u4 *)(size + 4 * i);
    rank += (x[0] > mine) + (x[1] > mine) + (x[2] > mine) + (x[3] > mine);
  }
  if (rank < ta::kHot) p.hot[((int64_t)s * p.Hkv + h) * ta::kHot + rank] = (uint8_t)d;
}

// Token t's key in channel d of an integer record: the word its code is in, and (head: the record's header
// in LDS) what rounding to fp16 took off it.
__device__ __forceinline__ int key_entry(int d) { return (d >> 5) << 3 | (d & 7); }  // of a lane's chunk
__device__ __forceinline__ uint32_t key_code_word(const uint8_t *rec, int level, int t, int d) {
  const int lane = (t >> 4) * 64 + (d >> 3 & 3) * 16 + (t & 15);
  return *(const uint32_t *)(rec + kSZBytes + lane * 4 * level + 4 * (key_entry(d) * level >> 5));
}
__device__ __forceinline__ uint32_t key_rest(uint32_t w, int level, uint32_t head, int d) {
  const int kg = d >> 3 & 3, n = key_entry(d);
  const int pos = level == GKV_INT8   ? 8 * (n & 3)  // code_pos, without tables in memory
                  : level == GKV_INT4 ? 4 * (1 - (n >> 2 & 1)) + 8 * (n >> 1 & 1) + 16 * (n & 1)
                                      : (int)(0x20A4C6E8u >> 4 * (n >> 1 & 7) & 15) + 16 * (n & 1);
  const uint32_t code = w >> pos & ((1u << level) - 1);
  const uint32_t sc = lds_u16(head + (32 * kg + n) * 2), z = lds_u16(head + 2 * D + (32 * kg + n) * 2);
  half2v c;
  c[0] = c[1] = (_Float16)(float)code;
  const uint32_t y = bounded(decoded(c, sc, z), sc, z) & 0xFFFFu;
  if ((y & T16::kInf) == T16::kInf) return 0;
  const float rest = __builtin_fmaf((float)code, (float)halves(sc)[0], (float)halves(z)[0]) - (float)halves(y)[0];
  return T16::pack(rest, 0.f);
}

// One workgroup a block or 64 residual rows; a wavefront a page (kRest: tiles with second terms).  Bound by
// the bytes it writes: 55 us for six sequences of 1343 to 12311 tokens x 8 KV heads (209 MB, 3.8 TB/s).
template <bool kRest>
__global__ void __launch_bounds__(256) expand_kernel(const ChunkParams p) {
  __shared__ __align__(16) uint8_t sh[1024 + 64];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)sh;
  const int s = blockIdx.z, h = blockIdx.y, v = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, pg = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = lane >> 4, m = lane & 15;
  const int T = p.T[s], nblk = (T + P - 1) / P, c0 = (T - p.n[s]) / P;
  if (v >= nblk + (p.nres + P - 1) / P) return;
  const int64_t u = (int64_t)p.seq[s] * p.Hkv + h;
  // one-centroid blocks before this one, and before c0
  const int8_t *levels = p.level + u * p.nblk_cap;
  int here = 0, all = 0;
  for (int i = tid; i < c0; i += 256)
    if (levels[i] == GKV_MEAN) {
      ++all;
      here += i < v;
    }
  for (int k = 32; k; k >>= 1) {
    all += __shfl_xor(all, k);
    here += __shfl_xor(here, k);
  }
  int *sums = (int *)(sh + 1024);
  if (lane == 0) {
    sums[2 * pg] = all;
    sums[2 * pg + 1] = here;
  }
  __syncthreads();
  all = sums[0] + sums[2] + sums[4] + sums[6];
  here = sums[1] + sums[3] + sums[5] + sums[7];
  const ListShape l = list_shape(p, c0, all);
  uint8_t *list = p.list + (p.list0[s] + (int64_t)h * list_tiles(p, T)) * p.tile;
  if (v == 0 && tid == 0) p.whole[s * p.Hkv + h] = l.whole;
  const Visit x = visit_at(p, u, v, nblk);
  if (v < c0 && x.level == GKV_MEAN) {  // a row of the one-centroid tiles
    if (pg) return;
    uint8_t *tile = list + (int64_t)(l.plain + l.res + (here >> 6)) * p.tile;
    // the last one's workgroup also writes the places behind it
    const int end = here == l.means - 1 ? ((here >> 6) + 1) * P : here + 1;
    for (int r = here; r < end; ++r) {
      const int t = r & (P - 1), n = r == here ? P - __popcll(x.drop) : 0;
      const u4 none = {0, 0, 0, 0};
      if (lane < 16) *(u4 *)(tile + ta::key_place(t, lane)) = n ? ((const u4 *)x.k)[lane] : none;
      if (kRest && lane < 2) *(u4 *)(tile + kListTile + (t >> 5) * 1024 + ((t & 31) + 32 * lane) * 16) = none;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int d = lane + 64 * i;
        const int at = ((t >> 4) * 4 + (d >> 5)) * 1024 + 512 * ((t >> 2) & 1) + 16 * (d & 31) + 8 * ((t >> 3) & 1) + 2 * (t & 3);
        *(uint16_t *)(tile + ta::kTileBytes + at) = n ? ((const uint16_t *)x.v)[d] : 0;
      }
      if (lane == 0)
        ((float *)(tile + 2 * ta::kTileBytes))[t] = n ? __builtin_amdgcn_logf((float)n) / p.sl2 : -__builtin_inff();
    }
    return;
  }
  const int at = v < c0 ? v - here : v < nblk ? l.whole + v - c0 : l.plain + v - nblk;
  uint8_t *tile = list + (int64_t)at * p.tile;
  // places without a token: their keys and values are zero, their scores start from -infinity
  uint64_t drop = x.drop;
  if (v >= c0 && v < nblk) drop = 0;  // residual tokens are put in their places
  if (v >= nblk) {
    const int r = (v - nblk) * P + lane;
    const bool later = r < p.nres && p.res_idx[u * p.nres_cap + r] >= c0 * P;
    drop |= __ballot(later);
  }
  if (is_int_level(x.level)) {
    if (pg == 0) store_head(lds, load_head(x, lane), lane, p.vtok);
    __syncthreads();
  }
  Raw k, w;
  uint32_t y[16];
  load_raw<GKV_KEYS>(k, x.k, x.level, pg, lane);
  load_raw<GKV_VALUES>(w, x.v, x.level, pg, lane);
  // hot channels hc .. + 3 of token ht
  const int ht = tid >> 2, hc = 4 * (tid & 3);
  uint32_t ids = 0, hw[4] = {0, 0, 0, 0};
  if (kRest && is_int_level(x.level)) {
    const int64_t l4 = ((int64_t)s * p.Hkv + h) * (ta::kHot / 4);
    const uint32_t a = hc & 4 ? table32(p.hot, l4 + 1) : table32(p.hot, l4);
    ids = hc & 8 ? hc & 4 ? table32(p.hot, l4 + 3) : table32(p.hot, l4 + 2) : a;
#pragma unroll
    for (int i = 0; i < 4; ++i) hw[i] = key_code_word(x.k, x.level, ht, ids >> (8 * i) & 0xFF);
  }
  const Exponents e;
  key_words_any(y, k, x.level, lds, kg, e);
  if (drop >> (16 * pg + m) & 1)
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *(u4 *)(tile + ta::key_place(16 * pg + m, 4 * j + kg)) = u4{y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]};
  if constexpr (kRest) {
    u2 rest = {0, 0};
    if (is_int_level(x.level) && !(x.drop >> ht & 1))
#pragma unroll
      for (int i = 0; i < 4; ++i) rest[i >> 1] |= key_rest(hw[i], x.level, lds, ids >> (8 * i) & 0xFF) << (16 * (i & 1));
    *(u2 *)(tile + kListTile + (ht >> 5) * 1024 + ((ht & 31) + 4 * (hc & 8)) * 16 + 2 * (hc & 7)) = rest;
  }
  Visit xd = x;
  xd.drop = drop;
  value_words_any(y, w, xd, lds, pg, lane, p.vtok, e);
  // operand form; two lanes' halves of a unit are exchanged, so that each stores 16 bytes: a lane
  // of the lower groups the units of even channel groups, its partner those of odd ones
  uint8_t *to = tile + ta::kTileBytes + pg * 4096 + (kg & 1) * 512 + m * 16;
#pragma unroll
  for (int c = 0; c < 8; c += 2) {
    const bool low = kg < 2;
    uint32_t mine[2], other[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t give = low ? y[2 * (c + 1) + i] : y[2 * c + i];
      mine[i] = low ? y[2 * c + i] : y[2 * (c + 1) + i];
      other[i] = __shfl_xor(give, 32);
    }
    const int cc = low ? c : c + 1;
    *(u4 *)(to + (cc >> 1) * 1024 + (cc & 1) * 256) =
        low ? u4{mine[0], mine[1], other[0], other[1]} : u4{other[0], other[1], mine[0], mine[1]};
  }
  if (pg == 0) ((float *)(tile + 2 * ta::kTileBytes))[lane] = drop >> lane & 1 ? -__builtin_inff() : 0.f;
  if (v >= c0 && v < nblk && x.drop) {  // the residual tokens' exact rows
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the graded ones are written
    __syncthreads();
    const int32_t *off = p.res_off + u * (p.nblk_cap + 1) + v;
    for (int t = tid >> 4; t < P; t += 16) {
      if (!(x.drop >> t & 1)) continue;
      const int r = off[0] + __popcll(x.drop & ((1ull << t) - 1));
      const uint8_t *rec = p.res_rows + (u * p.nrb_cap + (r >> 6)) * (2 * kExactBytes);
      const int rt = r & 63, un = tid & 15;
      *(u4 *)(tile + ta::key_place(t, un)) =
          *(const u4 *)(rec + (((rt >> 4) * 64 + (un & 3) * 16 + (rt & 15)) * 4 + (un >> 2)) * 16);
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // channels 8 un + i
        const int d = 8 * un + i;
        const int src = ((rt >> 4) * 64 + ((rt >> 2) & 3) * 16 + (d & 15)) * 32 + (d >> 4) * 4 + (rt & 3);
        const int dst = ((t >> 4) * 4 + (d >> 5)) * 1024 + 512 * ((t >> 2) & 1) + 16 * (d & 31) + 8 * ((t >> 3) & 1) + 2 * (t & 3);
        *(uint16_t *)(tile + ta::kTileBytes + dst) = ((const uint16_t *)(rec + kExactBytes))[src];
      }
    }
  }
}

constexpr int kTileWaves = 8, kTileRows = 32 * kTileWaves;

// A list's tiles: 1 KB a copy.
template <bool kRest>
struct ListTiles {
  const uint8_t *list;
  int bytes, wave, lane;
  __device__ __forceinline__ void copy(const uint8_t *src, uint32_t lds) const {
#pragma unroll
    for (int i = 0; i < 16 / kTileWaves; ++i) {
      const uint32_t at = (wave + kTileWaves * i) * 1024;
      ta::dma16(lane * 16, src + at, lds + at);
    }
  }
  __device__ __forceinline__ void keys(int t, uint32_t lds, uint32_t bias, uint32_t hot) const {
    const uint8_t *tile = list + (int64_t)t * bytes;
    copy(tile, lds);
    if (wave == 0 && lane < 16) ta::dma16(lane * 16, tile + 2 * ta::kTileBytes, bias);
    if (kRest && (wave == 1 || wave == 2)) {
      const uint32_t at = (wave - 1) * 1024;
      ta::dma16(lane * 16 + at, tile + kListTile, hot + at);
    }
  }
  __device__ __forceinline__ void values(int t, uint32_t lds) const {
    copy(list + (int64_t)t * bytes + ta::kTileBytes, lds);
  }
};

// 256 rows over a share of a list, as a prompt's row tile (and as it bound by matrix and vector
// issue): 512 tokens x 28/4 heads over 64k 515 us with second terms (0.93 PFLOP/s without counting them) and
// 476 without.
template <bool kRest>
__global__ void __launch_bounds__(64 * kTileWaves, 2) tiles_kernel(const ChunkParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
  const Job j = job_of(p, kTileRows, blockIdx.x % p.Hkv, blockIdx.x / p.Hkv);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  ta::Lane ln;
  ln.init<false>();
  const int row = j.tile * kTileRows + 32 * wave + ln.col;
  const int rc = row < j.rows ? row : j.rows - 1;  // rows past the last are copies, not stored
  const int tok = rc / p.G, g = rc - tok * p.G;
  const int first = j.pos0 + (j.tile * kTileRows) / p.G;  // seen by every row up to here
  const int last = j.pos0 + min(j.tile * kTileRows + kTileRows - 1, j.rows - 1) / p.G;
  const int c0 = j.pos0 / P, whole = (int)table32(p.whole, j.s * p.Hkv + j.h);
  const int ntile = whole + last / P - c0 + 1;
  const int split = p.split[j.s];
  const int t0 = (int)((int64_t)ntile * j.part / split), t1 = (int)((int64_t)ntile * (j.part + 1) / split);
  const ListTiles<kRest> src = {p.list + (p.list0[j.s] + (int64_t)j.h * list_tiles(p, j.T)) * p.tile, p.tile, wave, ln.lane};
  ta::Rows st;
  u4 q[kRest ? 9 : 8];
  st.init();
  if (t0 < t1)  // (a row tile with fewer tiles than shares leaves some of them none)
    ta::attend<T16, kTileWaves, false, true>(
        st, ln, q, lds, wave, t0, t1, whole + (first + 1) / P - c0, p.sl2, src,
        [&](int t) {  // this row's visible tokens of tile t
          const int n = t < whole ? P : j.pos0 + tok + 1 - (c0 + t - whole) * P;
          return n >= P ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
        },
        [&] { load_queries<kRest>(q, p, j, tok, g, ln.hf); });
  const float l = st.l + ta::other_half(st.l);
  if (row >= j.rows) return;
  if (split == 1)
    ta::store_row<T16>(p.out + (j.row0 + tok) * p.os + (int64_t)(j.h * p.G + g) * D, st, l > 0.f ? 1.f / l : l, ln.hf);
  else store_part(p.part + (part_row(p, j, kTileRows) + 32 * wave + ln.col) * kPart, st, l, ln.hf);
}

// ---------------------------------------------------------------- few rows
// Row tiles of 16: every wavefront holds one and reads blocks of its own.  The records are laid out
// for 16x16x32 MFMA (a lane's key chunk is the four operands of its page, its value chunk of two
// pages the eight operands of 32 tokens), and the scores' layout (lane l: row l & 15, token 16
// page + 4 (l >> 4) + i) is the second product's operand layout again.
//
// The records are copied to LDS as they are (asynchronous copies, 16 bytes a lane, with an exact or
// int8 chunk's pieces one behind the other so that a read finds each bank once) and decoded
// from there: the copies hold no registers, so that two wavefronts fit a SIMD.  A step is a
// block, or half an exact one; its values are copied from the start of its key product on,
// the next step's keys from the end of that.  No other vector memory instruction runs in the
// loop (but every 64 blocks), so the wait for a copy is a constant count.
//
// The scales and zeros of an integer block stay out of its codes' operands, which are 2^k + code as
// they come from the bits:
//   q . k = sum (2^k + code) (q s) + sum z q - sum 2^k (q s), with q s as two fp16 terms and the
//   constant part from the matrix units too, for any token the same;
//   sum p v = s (sum p (2^k + code) - 2^k sum p) + z sum p, once a step.
// Both sums are held in 32 bits, of which 2^k takes some: it is 1024 for eight bits, 16 and 64 for four, 4 to
// 64 for two (with the 1024 that costs a shift less, 2 tokens over 128k were off by 7e-4 of their
// outputs' size, which a long context leaves small, and now by 2.5e-4, as fp16 outputs are).  The rows of
// q are brought below 1 (a channel that is 2^-14 of its row's largest or less loses bits then, at most 2^-25 of
// that largest) and s is at most 65504 2 / 3 (two bits), 8734 or 514, so that no q s
// overflows; those of eight bits are raised by 2^6, so that the second term of one is lost only
// where 2^-12 of the code's span is less than a step of fp16's smallest numbers.
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) f4 *LdsF4;
typedef __attribute__((address_space(3))) f2 *LdsF2;

constexpr int kFewWaves = 4, kFewRows = 16;
constexpr int kFewBuf = kSZBytes + P * D;  // an int8 record, the largest that is copied at once
constexpr float kRaise = 64.f;

// The visits of a wavefront, 64 at a time: lane i holds the i-th.  Their table entries are read together
// and handed out from registers; read one at a time each block waited for its own.
struct Visits {
  int level;
  uint64_t k, v, drop;
  __device__ __forceinline__ void read(const ChunkParams &p, const Job &j, int first, int stride, int v1, int lane) {
    const int64_t at = first + (int64_t)lane * stride;
    if (at >= v1) return;
    if (at < j.nblk) {
      const int64_t ti = j.u * p.nblk_cap + at;
      level = p.level[ti];
      k = (uint64_t)p.arena + p.koff[ti];
      v = (uint64_t)p.arena + p.voff[ti];
      drop = p.res_mask ? p.res_mask[ti] : 0;
    } else {
      const int r = (int)at - j.nblk, left = p.nres - r * P;
      level = GKV_EXACT;
      k = (uint64_t)(p.res_rows + (j.u * p.nrb_cap + r) * (2 * kExactBytes));
      v = k + kExactBytes;
      drop = left >= P ? 0 : ~0ull << left;
    }
  }
  static __device__ __forceinline__ uint64_t lane64(uint64_t x, int i) {
    return (uint32_t)__builtin_amdgcn_readlane((int)x, i) |
           (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32;
  }
  __device__ __forceinline__ Visit at(int i) const {
    Visit x;
    x.level = __builtin_amdgcn_readlane(level, i);
    x.k = (const uint8_t *)lane64(k, i);
    x.v = (const uint8_t *)lane64(v, i);
    x.drop = lane64(drop, i);
    return x;
  }
};

struct FewRows {
  f4 o[8];  // O^T: register i of group c is channel 16 c + 4 kg + i
  float m, raise, l;
};

__device__ __forceinline__ f4 mfma16(u4 a, u4 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ta::half8, a), __builtin_bit_cast(ta::half8, b), c,
                                                0, 0, 0);
}

__device__ __forceinline__ float over_groups(float x) {  // the maximum over a row's four lanes
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// Scores to packed probabilities (two words a page), moving the references as tile_attn.h does.
__device__ __forceinline__ void few_weights(uint32_t (&p)[8], FewRows &r, const f4 (&s)[4], float sl2) {
  float top = -__builtin_inff();
  f4 x[4];
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[g][i] = __builtin_fmaf(s[g][i], sl2, -r.m);
      top = fmaxf(top, x[g][i]);
    }
  if (__builtin_expect(__any(top > r.raise), 0)) {
    const float high = over_groups(top);
    const bool mine = high > r.raise;
    const float up = mine ? high - T16::kLead : 0.f;
    const float f = r.raise < 0.f ? 0.f : __builtin_amdgcn_exp2f(-up);
    r.raise = mine ? T16::kRescale : r.raise;
    r.m += up;
    r.l *= f;
#pragma unroll
    for (int c = 0; c < 8; ++c) r.o[c] *= f;
    // formed from the scores again: with the move taken off the exponents above they would keep the
    // rounding of large ones (in a wavefront's first block those of the whole score)
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[g][i] = __builtin_fmaf(s[g][i], sl2, -r.m);
  }
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      p[2 * g + i] = T16::pack(__builtin_amdgcn_exp2f(x[g][2 * i]), __builtin_amdgcn_exp2f(x[g][2 * i + 1]));
}

// Copies of a record (exact: of its pages 2 half, 2 half + 1) to LDS.
__device__ __forceinline__ void few_copy(const uint8_t *record, int level, int half, uint32_t buf, int lane) {
  const uint8_t *rec = (const uint8_t *)(  // (the copies take their base from scalar registers)
      (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint64_t)record) |
      (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)record >> 32)) << 32);
  if (level == GKV_EXACT) {
    const uint8_t *src = rec + half * (kExactBytes / 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) ta::dma16(lane * 64, src + (i >> 2) * 4096 + (i & 3) * 16, buf + i * 1024);
    return;
  }
  if (level == GKV_MEAN) {
    if (lane < kMeanBytes / 16) ta::dma16(lane * 16, rec, buf);
    return;
  }
  if (level == GKV_CENTROID) {
    ta::dma16(lane * 16, rec, buf);
    if (lane < 1) ta::dma16(0, rec + 1024, buf + 1024);
    return;
  }
  if (lane < kSZBytes / 16) ta::dma16(lane * 16, rec, buf);
  rec += kSZBytes;
  buf += kSZBytes;
  if (level == GKV_INT8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) ta::dma16(lane * 32, rec + (i >> 1) * 2048 + (i & 1) * 16, buf + i * 1024);
  } else {
    for (int i = 0; i < level; ++i) ta::dma16(lane * 16, rec + i * 1024, buf + i * 1024);
  }
}
// Waits until at most the copies of a record of this level (none: -1) are on their way.
__device__ __forceinline__ void few_wait(int level) {
  if (level == GKV_INT4) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
  else if (level == GKV_INT2) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
  else if (level == GKV_INT8) asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
  else if (level == GKV_EXACT) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if (level == GKV_CENTROID) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
  else if (level == GKV_MEAN) asm volatile("s_waitcnt vmcnt(1)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}
// LDS reads of what is copied over next have returned.
__device__ __forceinline__ void few_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// The codes of a lane's chunk of page g.
template <int BITS>
__device__ __forceinline__ void few_codes(Raw &x, uint32_t buf, int g, int lane) {
  const uint32_t at = buf + kSZBytes;
  if constexpr (BITS == 8) {
    x.w[0] = ta::lds_u4(at + 2 * g * 1024 + lane * 16);
    x.w[1] = ta::lds_u4(at + (2 * g + 1) * 1024 + lane * 16);
  } else if constexpr (BITS == 4) {
    x.w[0] = ta::lds_u4(at + g * 1024 + lane * 16);
  } else {
    const u2 y = *(LdsW2)(uintptr_t)(at + g * 512 + lane * 8);
    x.w[0][0] = y[0];
    x.w[0][1] = y[1];
  }
}

constexpr bool is_codes(int level) { return level == GKV_INT8 || level == GKV_INT4 || level == GKV_INT2; }

// The operands of pages 2 pp and 2 pp + 1 (exact: of the half's two): keys, four a page; values, one for each 16
// channels.  Only these depend on the level, so that the products' accumulators stand in no
// branch (in one for each level they were copied from one to the next: 1100 moves).
template <int LEVEL>
__device__ __forceinline__ void few_keys(u4 (&a)[8], uint32_t buf, int pp, int lane, const Exponents &e) {
  const int kg = lane >> 4, m = lane & 15;
#pragma unroll
  for (int g = 0; g < (LEVEL == GKV_MEAN ? 1 : 2); ++g) {
    if constexpr (is_codes(LEVEL)) {
      Raw x;
      few_codes<LEVEL>(x, buf, 2 * pp + g, lane);
#pragma unroll
      for (int q = 0; q < 16; ++q) a[4 * g + (q >> 2)][q & 3] = raw_pair<LEVEL>(x.w, q, e);
    } else {
      uint32_t at = buf + (LEVEL == GKV_EXACT ? g * 4096 + lane * 16 : kg * 16);
      if constexpr (LEVEL == GKV_CENTROID)
        at += (*(LdsW1)(uintptr_t)(buf + KC * D * 2 + 4 * (2 * pp + g)) >> (2 * m) & 3u) * (D * 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) a[4 * g + j] = ta::lds_u4(at + j * (LEVEL == GKV_EXACT ? 1024 : 64));
    }
  }
}
template <int LEVEL>
__device__ __forceinline__ void few_values(u4 (&a)[8], const Visit &x, int half, uint32_t buf, int pp, bool vtok,
                                           int lane, const Exponents &e) {
  const int kg = lane >> 4, m = lane & 15;
  // word q of page g's chunk (tokens 4 kg + 2 (q & 1) and the next, channel 16 (q >> 1) + m) is
  // a[q >> 1][2 g + (q & 1)]
  // A token that is read elsewhere has weight 0, but 0 * infinity is NaN: its values become zeros
  // (but where scales are of channels: what those decode to is infinite or NaN for every token).
  if constexpr (LEVEL == GKV_MEAN) {  // the one key's place alone, if it stands for any token
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t v = lds_u16(buf + 2 * (16 * c + m));
      a[c] = u4{lane < 16 && x.drop != ~0ull ? v : 0, 0, 0, 0};
    }
  } else if constexpr (is_codes(LEVEL)) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      Raw w;
      few_codes<LEVEL>(w, buf, 2 * pp + g, lane);
#pragma unroll
      for (int q = 0; q < 16; ++q) a[q >> 1][2 * g + (q & 1)] = raw_pair<LEVEL>(w.w, q, e);
    }
    if (vtok) {  // scales of tokens: into the values here
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const uint32_t at = buf + (16 * (2 * pp + g) + 4 * kg) * 2;
        const u2 s = *(LdsW2)(uintptr_t)at, z = *(LdsW2)(uintptr_t)(at + 128);
        uint32_t y[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const uint32_t w = a[q >> 1][2 * g + (q & 1)];
          y[q] = decoded(halves(w) - halves(raw_offset<LEVEL>(q)), s[q & 1], z[q & 1]);
        }
        if (__builtin_expect(past_fp16<LEVEL>(s, z), 0))
#pragma unroll
          for (int q = 0; q < 16; ++q) y[q] = bounded(y[q], s[q & 1], z[q & 1]);
        if (x.drop) drop_words(y, x.drop, 2 * pp + g, kg);
#pragma unroll
        for (int q = 0; q < 16; ++q) a[q >> 1][2 * g + (q & 1)] = y[q];
      }
    }
  } else {
    u4 cent[4];
    if constexpr (LEVEL == GKV_CENTROID)
#pragma unroll
      for (int i = 0; i < 4; ++i) cent[i] = ta::lds_u4(buf + m * 64 + 16 * i);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t y[16];
      if constexpr (LEVEL == GKV_CENTROID) {
        centroid_words(y, cent, *(LdsW1)(uintptr_t)(buf + KC * D * 2 + 4 * (2 * pp + g)) >> (8 * kg));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u4 b = ta::lds_u4(buf + g * 4096 + j * 1024 + lane * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[4 * j + i] = b[i];
        }
      }
      if (x.drop) drop_words(y, x.drop, 2 * (half + pp) + g, kg);
#pragma unroll
      for (int q = 0; q < 16; ++q) a[q >> 1][2 * g + (q & 1)] = y[q];
    }
  }
}

// q s of a block in two terms, and what its scores start from (eight bits: that times 2^6, and what
// they end with).
template <int LEVEL>
__device__ __forceinline__ void few_fold(u4 (&hi)[4], u4 (&lo)[4], f4 &start, f4 &zero, uint32_t buf, uint32_t lds,
                                         int lane) {
  const int kg = lane >> 4;
  start = zero = f4{0.f, 0.f, 0.f, 0.f};
  half2v raise;
  raise[0] = raise[1] = (_Float16)kRaise;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const u4 q = ta::lds_u4(lds + d * 1024 + lane * 16), sc = ta::lds_u4(buf + kg * 64 + d * 16);
    u4 off;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      half2v s = halves(sc[i]);
      if (LEVEL == GKV_INT8) s *= raise;
      const half2v x = halves(q[i]) * s;
      hi[d][i] = __builtin_bit_cast(uint32_t, x);
      lo[d][i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(halves(q[i]), s, -x));
      off[i] = raw_offset<LEVEL>(4 * d + i) | 0x80008000u;
    }
    f4 &z = LEVEL == GKV_INT8 ? zero : start;
    z = mfma16(ta::lds_u4(buf + 256 + kg * 64 + d * 16), q, z);
    start = mfma16(off, hi[d], start);
    start = mfma16(off, lo[d], start);
  }
}

// Infinities and NaN among an exact half block's values where some row does not see all of it:
// out of the product, and noted for the rows that see them (two bits an output, as in
// ta::find_odd).  The copied values are made clean in place.
// vis: the row's visible tokens of the half.
__device__ __forceinline__ void few_odd(u4 &odd, uint32_t vis, uint32_t buf, int lane) {
  const int kg = lane >> 4;
  float zero = 0.f;
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    const u4 a = ta::lds_u4(buf + i * 1024 + lane * 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) zero = T16::times0(a[k], zero);
  }
  if (__builtin_expect(!__any(zero != zero), 1)) return;
  // token 16 g + 4 a + b, channel 16 c + 4 kg + i: lane 16 a + 4 kg + i's word 2 c + (b >> 1)
#pragma unroll 1
  for (int tok = 0; tok < 32; ++tok) {
    const uint32_t at = buf + (tok >> 4) * 4096 + (16 * (tok >> 2 & 3) + 4 * kg) * 16 + 2 * (tok & 3);
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t h = lds_u16(at + (c >> 1) * 1024 + (c & 1) * 8 + i * 16);
        const uint32_t e = h & 0x7FFFu, b = e < T16::kInf ? 0u : e > T16::kInf ? 3u : h == e ? 1u : 2u;
        odd[c >> 1] |= (vis >> tok & 1 ? b : 0u) << (8 * (c & 1) + 2 * i);
      }
  }
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    u4 a = ta::lds_u4(buf + i * 1024 + lane * 16);
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] &= ~ta::bad_halves<T16>(a[k]);
    *(LdsW4)(uintptr_t)(buf + i * 1024 + lane * 16) = a;
  }
}

#define GKV_LEVELS(level, f, ...)                                \
  do {                                                           \
    if (level == GKV_INT4) f<GKV_INT4>(__VA_ARGS__);             \
    else if (level == GKV_INT2) f<GKV_INT2>(__VA_ARGS__);        \
    else if (level == GKV_INT8) f<GKV_INT8>(__VA_ARGS__);        \
    else if (level == GKV_EXACT) f<GKV_EXACT>(__VA_ARGS__);      \
    else if (level == GKV_CENTROID) f<GKV_CENTROID>(__VA_ARGS__); \
    else f<GKV_MEAN>(__VA_ARGS__);                               \
  } while (0)

// Bound by vector issue (560 instructions a block, half of the cycles) and what it waits for in
// between with two wavefronts a SIMD: 2 tokens x 28/4 heads over 8 x 128k 157 us (4.2 TB/s; with the copies
// left out 118, the copies alone 112), five over 8 x up to 32k in three row tiles 66.
__global__ void __launch_bounds__(64 * kFewWaves, 2) few_kernel(const ChunkParams p) {
  // the queries' operands, then each wavefront's keys and values, the rows' largest; in the end
  // two wavefronts' states
  constexpr int kQ = 4096, kTops = kQ + kFewWaves * 2 * kFewBuf, kState = 8 * 1024 + 512;
  __shared__ __align__(16) uint8_t sh[kTops + kFewWaves * 64];
  static_assert(2 * kState <= sizeof(sh), "two wavefronts' states");
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)sh;
  // the row tiles of a share of the context read the same blocks: side by side on one XCD (workgroups
  // go round the eight of them), from whose L2 all but the first take them
  const int x8 = blockIdx.x & 7, each = gridDim.x >> 3, wgs = p.wg0[p.nseq];
  const int place = x8 * each + min(x8, (int)(gridDim.x & 7)) + (int)(blockIdx.x >> 3);
  const Job j = job_of(p, kFewRows, place / wgs, place % wgs);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int kg = lane >> 4, m = lane & 15;
  const int row = j.tile * kFewRows + m, rc = min(row, j.rows - 1);  // rows past the last are copies
  const int tok = rc / p.G, g = rc - tok * p.G;
  const int nvis = j.nblk + (p.nres + P - 1) / P;
  const int split = p.split[j.s];
  // every workgroup takes blocks from the whole context in turn, so that each gets as many of
  // each level (in runs of blocks the ones with the exact blocks took a third longer)
  const int stride = split * kFewWaves;
  const uint32_t kbuf = lds + kQ + wave * 2 * kFewBuf, vbuf = kbuf + kFewBuf;
  int at = j.part * kFewWaves + wave, half = 0, nth = 0;
  Visits batch = {};
  Visit x, next;
  if (at < nvis) {
    batch.read(p, j, at, stride, nvis, lane);
    x = batch.at(0);
    few_copy(x.k, x.level, 0, kbuf, lane);
  }
  float sl2 = p.sl2;
  {  // a wavefront copies channels 32 wave .. + 31 of the queries, times the power of two that brings
     // the row's largest below 1
    u4 q = *(const u4 *)(p.q + (j.row0 + tok) * p.qs + (int64_t)(j.h * p.G + g) * D + 8 * kg + 32 * wave);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(q[i] & 0x7FFFu, q[i] >> 16 & 0x7FFFu));
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (lane < 16) *(LdsW1)(uintptr_t)(lds + kTops + (wave * 16 + m) * 4) = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) top = max(top, *(LdsW1)(uintptr_t)(lds + kTops + (i * 16 + m) * 4));
    const int k = top == 0 || top >= T16::kInf ? 0 : 14 - (int)(top >> 10);
    const uint32_t f = (k >= -14 ? (15 + k) << 10 : 0x400 >> (-14 - k)) * 0x10001u;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = __builtin_bit_cast(uint32_t, halves(q[i]) * halves(f));
    sl2 = ldexpf(sl2, -k);
    *(LdsW4)(uintptr_t)(lds + wave * 1024 + lane * 16) = q;
  }
  const Exponents e;
  FewRows r;
  u4 odd = {0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < 8; ++c) r.o[c] = f4{0.f, 0.f, 0.f, 0.f};
  r.m = r.l = 0.f;
  r.raise = -__builtin_inff();
  __syncthreads();
  while (at < nvis) {
    const bool again = x.level == GKV_EXACT && half == 0;  // the block's other half is next
    const int after = again ? at : at + stride;
    const bool more = after < nvis;
    next = x;
    if (!again && more) {
      nth = (nth + 1) & 63;
      if (nth == 0) batch.read(p, j, after, stride, nvis, lane);
      next = batch.at(nth);
    }
    const bool whole = whole_at(p, j, at, j.pos0);
    few_copy(x.v, x.level, half, vbuf, lane);
    few_wait(x.level);
    const bool codes = is_codes(x.level);
    const bool two = x.level != GKV_EXACT && x.level != GKV_MEAN;  // pairs of pages
    f4 s[4], start = {0.f, 0.f, 0.f, 0.f}, zero;
    {
      u4 hi[4], lo[4];
      if (x.level == GKV_INT4) few_fold<GKV_INT4>(hi, lo, start, zero, kbuf, lds, lane);
      else if (x.level == GKV_INT2) few_fold<GKV_INT2>(hi, lo, start, zero, kbuf, lds, lane);
      else if (x.level == GKV_INT8) few_fold<GKV_INT8>(hi, lo, start, zero, kbuf, lds, lane);
      else
#pragma unroll
        for (int d = 0; d < 4; ++d) hi[d] = ta::lds_u4(lds + d * 1024 + lane * 16);
#pragma unroll
      for (int pp = 0; pp < 2; ++pp)
        if (pp == 0 || two) {
          u4 a[8];
          GKV_LEVELS(x.level, few_keys, a, kbuf, pp, lane, e);
          s[2 * pp] = s[2 * pp + 1] = start;
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[2 * pp + h] = mfma16(a[4 * h + d], hi[d], s[2 * pp + h]);
          if (codes)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
              for (int h = 0; h < 2; ++h) s[2 * pp + h] = mfma16(a[4 * h + d], lo[d], s[2 * pp + h]);
        }
    }
    few_read();
    if (more) few_copy(next.k, next.level, again ? 1 : 0, kbuf, lane);
    if (x.level == GKV_INT8) {
#pragma unroll
      for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = __builtin_fmaf(s[h][i], 1.f / kRaise, zero[i]);
    }
    const float no = -__builtin_inff();
    if (!two) s[2] = s[3] = f4{no, no, no, no};
    if (x.level == GKV_MEAN) {
      // one key stands for all the block's tokens: its weight times their number, in the first
      // group's first place alone
      const int n = P - __popcll(x.drop);
      const float plus = __builtin_amdgcn_logf((float)n) / sl2;
      s[0] = f4{lane < 16 && n ? s[0][0] + plus : no, no, no, no};
      s[1] = f4{no, no, no, no};
    }
    uint32_t seen = 0;
    if (!whole || (x.drop && x.level != GKV_MEAN)) {
      const uint64_t vis = (whole ? ~x.drop : seen_by(p, j, at, x.drop, j.pos0 + tok)) >> (32 * half);
      seen = (uint32_t)vis;
      const uint64_t w = vis >> (4 * kg);
#pragma unroll
      for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = w >> (16 * h + i) & 1 ? s[h][i] : no;
    }
    uint32_t w[8];
    few_weights(w, r, s, sl2);
    float sum = 0.f;  // of the step's weights
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = T16::add2(w[i], sum);
    r.l += sum;
    const bool scaled = codes && !p.vtok;
    f4 acc[8];
    if (scaled) {
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {  // (repeats after four)
      const uint32_t off = x.level == GKV_INT8   ? raw_offset<8>(2 * (c & 3))
                           : x.level == GKV_INT4 ? raw_offset<4>(2 * (c & 3))
                                                 : raw_offset<2>(2 * (c & 3));
      const float z = scaled ? -(float)halves(off)[0] * sum : 0.f;
      acc[c] = c < 4 ? f4{z, z, z, z} : acc[c & 3];
    }
    few_wait(more ? next.level : -1);
    if (!whole) few_odd(odd, seen, vbuf, lane);  // an exact block (the host sees to it)
#pragma unroll
    for (int pp = 0; pp < 2; ++pp)
      if (pp == 0 || two) {
        u4 a[8];
        GKV_LEVELS(x.level, few_values, a, x, half, vbuf, pp, p.vtok, lane, e);
#pragma unroll
        for (int c = 0; c < 8; ++c)
          acc[c] = mfma16(a[c], u4{w[4 * pp], w[4 * pp + 1], w[4 * pp + 2], w[4 * pp + 3]}, acc[c]);
      }
    if (scaled && x.drop == ~0ull) {
      // no token of it is read here: sums of zeros, which an infinite scale would make NaN
    } else if (scaled) {  // channels 16 c + 4 kg .. + 3 lie side by side in the header's lane order
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const u4 sc = ta::lds_u4(vbuf + kg * 64 + h * 16), z = ta::lds_u4(vbuf + 256 + kg * 64 + h * 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f4 &o = r.o[2 * h + (i >> 2)];
          const float y = __builtin_fmaf((float)halves(sc[i >> 1])[i & 1], acc[2 * h + (i >> 2)][i & 3], o[i & 3]);
          o[i & 3] = __builtin_fmaf((float)halves(z[i >> 1])[i & 1], sum, y);
        }
      }
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) r.o[c] += acc[c];
    }
    few_read();
    x = next;
    half = again;
    at = after;
  }
  r.l += __shfl_xor(r.l, 16);
  r.l += __shfl_xor(r.l, 32);
  if (__any(odd[0] | odd[1] | odd[2] | odd[3]))  // the values that stayed out of the products
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const uint32_t b = odd[i >> 3] >> (8 * (i >> 2 & 1) + 2 * (i & 3)) & 3u;  // 0, infinity, -infinity, NaN
      const uint32_t v = (b & 1u ? 0x7F800000u : b ? 0xFF800000u : 0u) | (b == 3 ? 0x400000u : 0u);
      r.o[i >> 2][i & 3] += __builtin_bit_cast(float, v);
    }
  // the wavefronts' states, joined two and two in LDS, each value in the lane that holds its like
#pragma unroll
  for (int n = kFewWaves / 2; n >= 1; n >>= 1) {
    __syncthreads();
    const uint32_t mine = lds + (wave & (n - 1)) * kState + lane * 16, ends = mine - lane * 8 + 8192;
    if (wave >= n && wave < 2 * n) {
#pragma unroll
      for (int c = 0; c < 8; ++c) *(LdsF4)(uintptr_t)(mine + c * 1024) = r.o[c];
      *(LdsF2)(uintptr_t)ends = f2{r.m, r.l};
    }
    __syncthreads();
    if (wave < n) {
      const f2 ml = *(LdsF2)(uintptr_t)ends;
      // a state that has seen nothing has no maximum
      const float top = r.l == 0.f ? ml[0] : ml[1] == 0.f ? r.m : fmaxf(r.m, ml[0]);
      const float a = r.l == 0.f ? 0.f : __builtin_amdgcn_exp2f(r.m - top);
      const float b = ml[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[0] - top);
      r.m = top;
      r.l = r.l * a + ml[1] * b;
#pragma unroll
      for (int c = 0; c < 8; ++c) r.o[c] = r.o[c] * a + *(LdsF4)(uintptr_t)(mine + c * 1024) * b;
    }
  }
  if (wave || row >= j.rows) return;
  if (split == 1) {
    const float inv = r.l > 0.f ? 1.f / r.l : r.l;
    uint16_t *op = p.out + (j.row0 + tok) * p.os + (int64_t)(j.h * p.G + g) * D + 4 * kg;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      *(u2 *)(op + 16 * c) = u2{T16::pack(r.o[c][0] * inv, r.o[c][1] * inv),
                                T16::pack(r.o[c][2] * inv, r.o[c][3] * inv)};
  } else {
    float *part = p.part + (part_row(p, j, kFewRows) + m) * kPart;
#pragma unroll
    for (int c = 0; c < 8; ++c) *(f4 *)(part + 16 * c + 4 * kg) = r.o[c];
    if (kg == 0) *(float2 *)(part + D) = make_float2(r.m, r.l);
  }
}
#undef GKV_LEVELS

// Joins the partials of a row: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.  Sixteen lanes a
// row, eight channels a lane.  Bound by latency (7 us for 16 partials of 448 rows), then by the partials'
// bytes (14 us for 3584 rows x 4 KV heads).  A wavefront a row took 5.5 and 15 (and 22 us where
// 14 are now).
__global__ void __launch_bounds__(256) chunk_merge_kernel(const ChunkParams p, int rows_tile) {
  const int lane = threadIdx.x & 15, h = blockIdx.y;
  int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  int s = 0;
  for (; s < p.nseq; ++s) {  // the row's sequence
    const int rows = p.split[s] > 1 ? p.n[s] * p.G : 0;
    if (r < rows) break;
    r -= rows;
  }
  if (s == p.nseq) return;
  const int tiles = (p.n[s] * p.G + rows_tile - 1) / rows_tile;
  const int tile = (int)r / rows_tile, in = (int)r - tile * rows_tile;
  const int tok = (int)r / p.G, g = (int)r - tok * p.G;
  const float *part = p.part + (p.part0 + ((int64_t)h * p.wg0[p.nseq] + p.wg0[s] + tile) * rows_tile + in) * kPart;
  const int64_t step = (int64_t)tiles * rows_tile * kPart;
  const int n = p.split[s];
  float m = -__builtin_inff();
  for (int i = lane; i < n; i += 16) {
    const float2 ml = *(const float2 *)(part + i * step + D);
    if (ml.y != 0.f) m = fmaxf(m, ml.x);  // (one that saw nothing has no maximum)
  }
#pragma unroll
  for (int k = 8; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
  float o[8], l = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) o[k] = 0.f;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const float *x = part + i * step;
    const float2 ml = *(const float2 *)(x + D);
    const f4 y0 = *(const f4 *)(x + 8 * lane), y1 = *(const f4 *)(x + 8 * lane + 4);
    const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
    l += f * ml.y;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      o[k] += f * y0[k];
      o[4 + k] += f * y1[k];
    }
  }
  const float inv = l > 0.f ? 1.f / l : l;
  *(u4 *)(p.out + (p.row0[s] + tok) * p.os + (int64_t)(h * p.G + g) * D + 8 * lane) =
      u4{T16::pack(o[0] * inv, o[1] * inv), T16::pack(o[2] * inv, o[3] * inv), T16::pack(o[4] * inv, o[5] * inv),
         T16::pack(o[6] * inv, o[7] * inv)};
}

// ---------------------------------------------------------------- host
// Rows of a (sequence, KV head) up to which its blocks are read by few_kernel, decoded for every 16 rows
// anew; beyond, the cache is decoded to tiles first, which costs its bytes written and read
// again, and row tiles are of 256.  4 KV heads, few and many rows' form in us: 8 x 32k tokens 14
// rows 52 and 307, 63 rows 148 and 297, 126 rows 275 and 305; 1 x 64k 39 and 84, 49 and 86, 80 and
// 89; 16 x 2000 25 and 51, 35 and 53, 45 and 57.
constexpr int kFewMost = 128;
constexpr int kLeastVisits = 4;  // blocks that a workgroup takes at least

// One launch's part of a call.
struct Part {
  ChunkParams p;
  int rows_tile;
  int64_t wgs, merged, part_rows, tiles;  // workgroups per KV head, rows to merge per KV head, partial
                                          // rows and list tiles over all KV heads
};

// Shares of the contexts: every row tile of a sequence is cut into ceil(blocks / per) workgroups,
// with the least `per` for which all workgroups are resident at once (fill of them), or in two
// or three rounds where the row tiles alone are more.  What a workgroup takes beside its blocks
// counts as kAlone blocks, and as kShared where it leaves a partial: 256 rows' partial is
// 133 KB to write and to read again, 13 us at a compute unit's part of the memory rate,
// where a block takes 2 us.
gkv_status plan_part(Part &t, const gkv_cache *c, int64_t fill) {
  constexpr int64_t kAlone = 2, kShared = 8, kRounds = 3;
  ChunkParams &p = t.p;
  const int G = c->Hq / c->Hkv;
  auto tiles = [&](int i) { return ((int64_t)p.n[i] * G + t.rows_tile - 1) / t.rows_tile; };
  auto blocks = [&](int i) { return (int64_t)list_tiles(p.T[i], c->nres); };
  int64_t total = 0, plain = 0, longest = 0;
  t.wgs = t.merged = t.part_rows = t.tiles = 0;
  for (int i = 0; i < p.nseq; ++i) {
    total += tiles(i) * blocks(i) * c->Hkv;
    plain += tiles(i) * c->Hkv;
    longest = std::max(longest, blocks(i));
  }
  auto count = [&](int64_t per) {
    int64_t n = 0;
    for (int i = 0; i < p.nseq; ++i) n += (blocks(i) + per - 1) / per * tiles(i);
    return n * c->Hkv;
  };
  int64_t best = longest, cost = (longest + kAlone) * ((plain + fill - 1) / fill);
  for (int64_t r = 1; r <= kRounds && p.nseq; ++r) {
    if (plain > r * fill) continue;
    int64_t lo = std::max<int64_t>(kLeastVisits, (total + r * fill - 1) / (r * fill)), hi = std::max(longest, lo);
    while (lo < hi) {  // the least that fits
      const int64_t mid = (lo + hi) / 2;
      if (count(mid) <= r * fill) hi = mid;
      else lo = mid + 1;
    }
    if (r * (lo + kShared) < cost) {
      best = lo;
      cost = r * (lo + kShared);
    }
  }
  for (int i = 0; i < p.nseq; ++i) {
    const int64_t s = std::min<int64_t>((blocks(i) + best - 1) / best, 0xffff);
    p.split[i] = (uint16_t)s;
    p.wg0[i] = (int32_t)t.wgs;
    p.list0[i] = (int32_t)t.tiles;
    if (s > 1) t.merged += (int64_t)p.n[i] * G;
    t.wgs += s * tiles(i);
    t.tiles += blocks(i) * c->Hkv;
    if (t.wgs * c->Hkv > GKV_MAX_LAUNCH / 512 || t.tiles > 0x7fffffff) return GKV_E_UNSUPPORTED;
  }
  p.wg0[p.nseq] = (int32_t)t.wgs;
  t.part_rows = t.merged ? t.wgs * c->Hkv * t.rows_tile : 0;
  return GKV_OK;
}

struct Plan {
  Part few, many;
  bool rest;                               // tiles with second terms
  int64_t part, whole, hot, list, bytes;  // workspace: partials | whole counts | hot channels | lists
};

gkv_status chunk_plan(const gkv_cache *c, const int32_t *n_new, Plan &pl) {
  const int G = c->Hq / c->Hkv;
  pl.few.p.nseq = pl.many.p.nseq = 0;
  pl.rest = false;
  int64_t rows = 0;
  for (int b = 0; b < c->B; ++b) {
    const int64_t T = seq_tokens(c, b), n = n_new[b];
    if (n < 0) return GKV_E_SHAPE;
    if (!n) continue;
    if (T < 0) return GKV_E_ARG;
    if (n > T) return GKV_E_SHAPE;
    if (T > 0x7fffff00 || n * G > 0x7fffff00 || rows + n > 0x7fffffff ||
        list_tiles((int)T, c->nres) > GKV_MAX_LAUNCH / 256)
      return GKV_E_UNSUPPORTED;
    bool few = n * G <= kFewMost;  // and the blocks that some row sees in part are exact
    for (int h = 0; h < c->Hkv && few; ++h)
      for (int64_t i = (T - n) / P; i < (T + P - 1) / P; ++i)
        few &= c->level_host[((int64_t)b * c->Hkv + h) * c->nblk_cap + i] == GKV_EXACT;
    if (!few && !pl.rest) {
      const int8_t *lv = c->level_host + (int64_t)b * c->Hkv * c->nblk_cap;
      for (int h = 0; h < c->Hkv && !pl.rest; ++h, lv += c->nblk_cap) {
        int8_t bits = 0;  // (a level is its own bit: no exit, so that the loop takes many at once)
        for (int64_t i = 0; i < (T + P - 1) / P; ++i) bits |= lv[i];
        pl.rest = bits & (GKV_INT8 | GKV_INT4 | GKV_INT2);
      }
    }
    ChunkParams &p = few ? pl.few.p : pl.many.p;
    const int i = p.nseq++;
    p.seq[i] = (uint8_t)b;
    p.T[i] = (int32_t)T;
    p.n[i] = (int32_t)n;
    p.row0[i] = (int32_t)rows;
    rows += n;
  }
  pl.few.rows_tile = kFewRows;
  pl.many.rows_tile = kTileRows;
  const int64_t cus = gkv_device_cus();
  gkv_status st = plan_part(pl.few, c, 2 * cus);
  if (!st) st = plan_part(pl.many, c, cus);
  if (st) return st;
  auto align = [](int64_t x) { return (x + 255) & ~(int64_t)255; };
  pl.part = 0;
  pl.whole = align((pl.few.part_rows + pl.many.part_rows) * kPart * 4);
  const int64_t lists = (int64_t)pl.many.p.nseq * c->Hkv;
  pl.hot = align(pl.whole + lists * 4);
  pl.list = align(pl.hot + (pl.rest ? lists * ta::kHot : 0));
  pl.many.p.tile = kListTile + (pl.rest ? ta::kHotBytes : 0);
  pl.bytes = pl.list + pl.many.tiles * pl.many.p.tile;
  return GKV_OK;
}

}  // namespace

extern "C" int64_t gkv_chunk_ws_bytes(const gkv_cache *c, const int32_t *n_new) {
  if (gkv_validate_cache(c) || !n_new || c->B > kMaxSeqs) return -1;
  Plan pl;
  if (chunk_plan(c, n_new, pl)) return -1;
  return pl.bytes;
}

extern "C" gkv_status gkv_chunk_attn(const uint16_t *q, int64_t q_stride, const gkv_cache *c, const int32_t *n_new,
                                     uint16_t *out, int64_t out_stride, void *ws, int64_t ws_bytes, void *stream) {
  gkv_status st = gkv_validate_cache(c);
  if (st) return st;
  if (!n_new) return GKV_E_ARG;
  if (c->B > kMaxSeqs || c->Hkv > 65535) return GKV_E_UNSUPPORTED;
  Plan pl;
  st = chunk_plan(c, n_new, pl);
  if (st) return st;
  if (!pl.few.p.nseq && !pl.many.p.nseq) return GKV_OK;
  if (!q || !out || (uintptr_t)q % 16 || (uintptr_t)out % 16) return GKV_E_ARG;
  for (const int64_t s : {q_stride, out_stride}) {
    if (s < (int64_t)c->Hq * D) return GKV_E_SHAPE;
    if (s % 8) return GKV_E_ARG;
    if (s > GKV_MAX_ROW_STRIDE) return GKV_E_UNSUPPORTED;
  }
  if (pl.bytes && (!ws || (uintptr_t)ws % 16)) return GKV_E_ARG;
  if (ws_bytes < pl.bytes) return GKV_E_WORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  for (Part *t : {&pl.few, &pl.many}) {
    ChunkParams &p = t->p;
    if (!p.nseq) continue;
    p.q = q;
    p.out = out;
    p.part = (float *)ws;
    p.qs = q_stride;
    p.os = out_stride;
    p.level = c->level;
    p.koff = c->koff;
    p.voff = c->voff;
    p.arena = c->arena;
    p.res_mask = c->nres ? c->res_mask : nullptr;
    p.res_idx = c->res_idx;
    p.res_off = c->res_off;
    p.res_rows = c->res_rows;
    p.nblk_cap = c->nblk_cap;
    p.Hkv = c->Hkv;
    p.G = c->Hq / c->Hkv;
    p.nres = c->nres;
    p.nres_cap = c->nres_cap;
    p.nrb_cap = (c->nres_cap + P - 1) / P;
    p.vtok = c->v_per_token;
    p.sl2 = 1.4426950408889634f / sqrtf((float)D);
    p.part0 = t == &pl.few ? 0 : pl.few.part_rows;
    p.whole = (int32_t *)((uint8_t *)ws + pl.whole);
    p.hot = (uint8_t *)ws + pl.hot;
    p.list = (uint8_t *)ws + pl.list;
    const dim3 grid((unsigned)(t->wgs * c->Hkv));
    if (t == &pl.few) {
      hipLaunchKernelGGL(few_kernel, grid, dim3(64 * kFewWaves), 0, s, p);
    } else {
      int most = 0;
      for (int i = 0; i < p.nseq; ++i) most = std::max(most, list_tiles(p.T[i], c->nres));
      const dim3 blocks(most, c->Hkv, p.nseq);
      const dim3 blk(64 * kTileWaves);
      const int lds = ta::kAttendLds + 2 * ta::kBiasBytes;
      if (pl.rest) {
        hipLaunchKernelGGL(hot_kernel, dim3(c->Hkv, p.nseq), dim3(D), 0, s, p);
        hipLaunchKernelGGL(expand_kernel<true>, blocks, dim3(256), 0, s, p);
        hipLaunchKernelGGL(tiles_kernel<true>, grid, blk, lds + 2 * ta::kHotBytes, s, p);
      } else {
        hipLaunchKernelGGL(expand_kernel<false>, blocks, dim3(256), 0, s, p);
        hipLaunchKernelGGL(tiles_kernel<false>, grid, blk, lds, s, p);
      }
    }
    if (hipGetLastError() != hipSuccess) return GKV_E_HIP;
    if (t->merged) {
      hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)((t->merged + 15) / 16), c->Hkv), dim3(256), 0, s, p,
                         t->rows_tile);
      if (hipGetLastError() != hipSuccess) return GKV_E_HIP;
    }
  }
  return GKV_OK;
}
