// Attention of the newest tokens of every sequence (a prompt's chunk, a speculative step's
// drafts) over the graded cache (sections 3.1, 3.2, 3.4 and 3.7): the many-query form of the
// dense decode read.
//
// The records are decoded to fp16 tiles in LDS (one rounding of code * scale + zero), the form
// that the row tiles of tile_attn.h read.  Two shapes of workgroup:
//  * shared (kWaves row groups): the wavefronts hold 32 rows each and share every tile, so
//    a record is decoded once for all of a workgroup's rows;
//  * private (at most 32 rows of a (sequence, KV head)): every wavefront holds all the rows
//    and takes half blocks of its own, without barriers, and the wavefronts' states are
//    merged at the end.
// Either splits a long context over workgroups whose partials a merge kernel joins.
#include <hip/hip_runtime.h>

#include <new>

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
constexpr int kRecTile = P * D * 2;  // bytes of a tile's keys, or of its values
constexpr int kPart = D + 2;         // floats of a row's partial: O, m, l

struct ChunkParams {
  const uint16_t *q;
  uint16_t *out;
  float *part;
  int64_t qs, os;  // elements from a token's rows to the next one's
  const int8_t *level;
  const int64_t *koff, *voff;
  const uint8_t *arena;
  const uint64_t *res_mask;  // null without residual rows
  const int32_t *res_idx;
  const uint8_t *res_rows;
  int32_t nblk_cap, Hkv, G, nseq, nres, nres_cap, nrb_cap, vtok;
  float sl2;
  int64_t part0;             // first partial row of this launch
  int32_t seq[kMaxSeqs];     // sequence
  int32_t T[kMaxSeqs], n[kMaxSeqs];  // its tokens, and the newest ones that attend
  int32_t row0[kMaxSeqs];    // their first packed row
  int32_t split[kMaxSeqs];   // workgroups that share a row tile's context
  int32_t wg0[kMaxSeqs + 1]; // workgroups per KV head before each
};

// ---------------------------------------------------------------- records to tiles
__device__ __forceinline__ int64_t uni64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
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
    x.level = __builtin_amdgcn_readfirstlane((int)p.level[ti]);
    x.k = p.arena + uni64(p.koff[ti]);
    x.v = p.arena + uni64(p.voff[ti]);
    x.drop = p.res_mask ? (uint64_t)uni64((int64_t)p.res_mask[ti]) : 0;
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
    if (level == GKV_CENTROID) c += (*(const uint32_t *)(rec + KC * D * 2 + 4 * pg) >> (2 * m) & 3u) * D;
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

// Codes 2 q and 2 q + 1 of a chunk, as fp16 (exact): their bits under a fixed exponent, less
// the power of two that makes.
template <int BITS>
__device__ __forceinline__ half2v code_pair(const u4 (&w)[4], int q) {
  uint32_t x, off;
  if constexpr (BITS == 8) {
    x = __builtin_amdgcn_perm(0x64646464u, w[q >> 3][(q >> 1) & 3], (q & 1) ? 0x04030402u : 0x04010400u);
    off = 0x64006400u;
  } else if constexpr (BITS == 4) {
    const uint32_t s = w[0][q >> 2] >> ((q & 1) ? 8 : 0);
    x = (q & 2) ? (s & 0x000F000Fu) | 0x64006400u : (s & 0x00F000F0u) | 0x54005400u;
    off = (q & 2) ? 0x64006400u : 0x54005400u;
  } else {
    const uint32_t y = w[0][q >> 3];
    switch (q & 7) {
      case 0: case 1: x = ((q & 1 ? y >> 6 : y) & 0x03000300u) | (off = 0x44004400u); break;
      case 2: case 3: x = ((q & 1 ? y >> 6 : y) & 0x00C000C0u) | (off = 0x4C004C00u); break;
      case 4: case 5: x = ((q & 1 ? y >> 6 : y) & 0x00300030u) | (off = 0x54005400u); break;
      case 6: x = (y & 0x00030003u) | (off = 0x64006400u); break;
      default: x = (y & 0x000C000Cu) | (off = 0x5C005C00u); break;
    }
  }
  return __builtin_bit_cast(half2v, x) - __builtin_bit_cast(half2v, off);
}

typedef __attribute__((address_space(3))) u4 *LdsW4;
typedef __attribute__((address_space(3))) u2 *LdsW2;

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

template <int BITS>
__device__ __forceinline__ void stage_key_codes(uint32_t (&y)[16], const Raw &x, uint32_t head, int kg) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const u4 s = ta::lds_u4(head + kg * 64 + j * 16), z = ta::lds_u4(head + 256 + kg * 64 + j * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[4 * j + i] = decoded(code_pair<BITS>(x.w, 4 * j + i), s[i], z[i]);
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
                                                  bool vtok) {
  const int kg = lane >> 4, m = lane & 15;
  if (vtok) {  // tokens 16 pg + 4 kg .. + 3
    const u2 s = *(LdsW2)(uintptr_t)(head + 512 + (16 * pg + 4 * kg) * 2);
    const u2 z = *(LdsW2)(uintptr_t)(head + 512 + 128 + (16 * pg + 4 * kg) * 2);
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] = decoded(code_pair<BITS>(x.w, q), s[q & 1], z[q & 1]);
  } else {
    const u4 s = ta::lds_u4(head + 512 + m * 16), z = ta::lds_u4(head + 768 + m * 16);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int c = q >> 1;
      y[q] = __builtin_bit_cast(uint32_t,
                                __builtin_elementwise_fma(code_pair<BITS>(x.w, q), twice(s[c >> 1], c & 1),
                                                          twice(z[c >> 1], c & 1)));
    }
  }
}

// A lane's chunk of page pg into the key tile (row pg_at * 16 + m of the tile).
__device__ __forceinline__ void stage_keys(const Raw &x, int level, uint32_t head, uint32_t tile, int pg_at, int lane) {
  const int kg = lane >> 4, m = lane & 15;
  uint32_t y[16];
  if (level == GKV_INT8) stage_key_codes<8>(y, x, head, kg);
  else if (level == GKV_INT4) stage_key_codes<4>(y, x, head, kg);
  else if (level == GKV_INT2) stage_key_codes<2>(y, x, head, kg);
  else
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x.w[i >> 2][i & 3];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *(LdsW4)(uintptr_t)(tile + ta::key_place(16 * pg_at + m, 4 * j + kg)) =
        u4{y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]};
}

// The same for the value tile (operand form); drop: the block's tokens that are not read,
// whose values become zero (their weight is zero, but 0 * infinity is NaN).
__device__ __forceinline__ void stage_values(const Raw &x, int level, const uint8_t *rec, uint64_t drop, uint32_t head,
                                             uint32_t tile, int pg, int pg_at, int lane, bool vtok) {
  const int kg = lane >> 4, m = lane & 15;
  uint32_t y[16];
  if (level == GKV_INT8) stage_value_codes<8>(y, x, head, pg, lane, vtok);
  else if (level == GKV_INT4) stage_value_codes<4>(y, x, head, pg, lane, vtok);
  else if (level == GKV_INT2) stage_value_codes<2>(y, x, head, pg, lane, vtok);
  else if (level == GKV_CENTROID) {
    const uint32_t ids = *(const uint32_t *)(rec + KC * D * 2 + 4 * pg) >> (8 * kg);  // of the lane's four tokens
    uint32_t sel[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = ids >> (4 * i) & 3u, b = ids >> (4 * i + 2) & 3u;
      sel[i] = (2 * a) | (2 * a + 1) << 8 | (2 * b) << 16 | (2 * b + 1) << 24;
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int c = q >> 1;
      y[q] = __builtin_amdgcn_perm(x.w[c >> 1][2 * (c & 1) + 1], x.w[c >> 1][2 * (c & 1)], sel[q & 1]);
    }
  } else if (level == GKV_MEAN) {
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] = x.w[q >> 3][(q >> 1) & 3];
  } else {
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] = x.w[q >> 2][q & 3];
  }
  if (drop) {
    const uint32_t d = (uint32_t)(drop >> (16 * pg)) >> (4 * kg);
    const uint32_t keep[2] = {(d & 1 ? 0 : 0xFFFFu) | (d & 2 ? 0 : 0xFFFF0000u),
                              (d & 4 ? 0 : 0xFFFFu) | (d & 8 ? 0 : 0xFFFF0000u)};
#pragma unroll
    for (int q = 0; q < 16; ++q) y[q] &= keep[q & 1];
  }
  const uint32_t at = tile + pg_at * 4096 + (kg & 1) * 512 + m * 16 + (kg >> 1) * 8;
#pragma unroll
  for (int c = 0; c < 8; ++c) *(LdsW2)(uintptr_t)(at + (c >> 1) * 1024 + (c & 1) * 256) = u2{y[2 * c], y[2 * c + 1]};
}

// ---------------------------------------------------------------- rows
// The part of a call that one workgroup computes.
struct Job {
  int s, h, tile, part;  // place among the launch's sequences, KV head, row tile, share of the context
  int T, n, pos0;        // tokens, new ones, the first new one's position
  int rows, nblk;        // rows of the (sequence, KV head); blocks
  int64_t u, row0;
};

__device__ __forceinline__ Job job_of(const ChunkParams &p, int rows_tile) {
  Job j;
  j.h = blockIdx.x % p.Hkv;
  int w = blockIdx.x / p.Hkv, lo = 0, hi = p.nseq;
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

__device__ __forceinline__ void load_queries(u4 (&q)[8], const ChunkParams &p, const Job &j, int tok, int g, int hf) {
  const uint16_t *qp = p.q + (j.row0 + tok) * p.qs + (int64_t)(j.h * p.G + g) * D + 8 * hf;
#pragma unroll
  for (int d = 0; d < 8; ++d) q[d] = *(const u4 *)(qp + 16 * d);
}

__device__ __forceinline__ void store_row(const ChunkParams &p, const Job &j, int tok, int g, const ta::Rows &st,
                                          float inv, int hf) {
  uint16_t *op = p.out + (j.row0 + tok) * p.os + (int64_t)(j.h * p.G + g) * D + 4 * hf;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u2 w;
      w[0] = T16::pack(st.o[c][4 * i] * inv, st.o[c][4 * i + 1] * inv);
      w[1] = T16::pack(st.o[c][4 * i + 2] * inv, st.o[c][4 * i + 3] * inv);
      *(u2 *)(op + 32 * c + 8 * i) = w;
    }
}

__device__ __forceinline__ void store_part(float *part, const ta::Rows &st, float l, int hf) {
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float4 w = make_float4(st.o[c][4 * i], st.o[c][4 * i + 1], st.o[c][4 * i + 2], st.o[c][4 * i + 3]);
      float2 *d = (float2 *)(part + 32 * c + 8 * i + 4 * hf);
      d[0] = make_float2(w.x, w.y);
      d[1] = make_float2(w.z, w.w);
    }
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
  return __builtin_amdgcn_readfirstlane(p.res_idx[j.u * p.nres_cap + (v - j.nblk) * P + last]) <= pos;
}

// ---------------------------------------------------------------- shared tiles
template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) chunk_kernel(const ChunkParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
  constexpr int kTileRows = 32 * WAVES;
  const Job j = job_of(p, kTileRows);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  ta::Lane ln;
  ln.init<false>();
  const int row = j.tile * kTileRows + 32 * wave + ln.col;
  const int rc = row < j.rows ? row : j.rows - 1;  // rows past the last are copies, not stored
  const int tok = rc / p.G, g = rc - tok * p.G;
  u4 q[8];
  load_queries(q, p, j, tok, g, ln.hf);
#pragma unroll
  for (int d = 0; d < 8; ++d) asm volatile("" : "+v"(q[d]));

  const int first = j.pos0 + (j.tile * kTileRows) / p.G;  // seen by every row up to here
  const int last = j.pos0 + min(j.tile * kTileRows + kTileRows - 1, j.rows - 1) / p.G;
  const int nblk = last / P + 1;  // blocks that some row sees
  const int nvis = nblk + (p.nres + P - 1) / P;
  const int split = p.split[j.s];
  const int v0 = (int)((int64_t)nvis * j.part / split), v1 = (int)((int64_t)nvis * (j.part + 1) / split);
  auto visit = [&](int v) { return visit_at(p, j.u, v < nblk ? v : j.nblk + v - nblk, j.nblk); };

  const uint32_t head = lds + 4 * kRecTile;
  auto tiles = [&](int v) { return lds + (v & 1) * 2 * kRecTile; };
  constexpr bool kBoth = WAVES == 4;  // a wavefront stages a page of both tensors, or of one
  const int pg = wave & 3;
  const bool key_wave = wave < 4;
  Raw raw[kBoth ? 2 : 1];
  u4 hd;
  auto load = [&](const Visit &x) {
    if (kBoth) {
      load_raw<GKV_KEYS>(raw[0], x.k, x.level, pg, ln.lane);
      load_raw<GKV_VALUES>(raw[kBoth], x.v, x.level, pg, ln.lane);
    } else if (key_wave) {
      load_raw<GKV_KEYS>(raw[0], x.k, x.level, pg, ln.lane);
    } else {
      load_raw<GKV_VALUES>(raw[0], x.v, x.level, pg, ln.lane);
    }
  };
  auto stage = [&](const Visit &x, int v) {
    const uint32_t to = tiles(v), hv = head + (v & 1) * 1024;
    if (kBoth || key_wave) stage_keys(raw[0], x.level, hv, to, pg, ln.lane);
    if (kBoth || !key_wave)
      stage_values(raw[kBoth], x.level, x.v, x.drop, hv, to + kRecTile, pg, pg, ln.lane, p.vtok);
  };
  auto meet = [] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Tile v is staged, and the header of v + 1 lies in LDS, when its turn comes; the codes of
  // v + 1 and the header of v + 2 are in registers, the tables of v + 2 read.
  ta::Rows st;
  st.init();
  u4 odd = {0, 0, 0, 0};
  if (v0 < v1) {  // (a tile that sees few blocks may leave some of its workgroups nothing)
    auto fetch_head = [&](const Visit &x) {
      if (wave == 0 && is_int_level(x.level)) hd = load_head(x, ln.lane);
    };
    auto put_head = [&](const Visit &x, int v) {
      if (wave == 0 && is_int_level(x.level)) store_head(head + (v & 1) * 1024, hd, ln.lane, p.vtok);
    };
    Visit x0 = visit(v0), x1 = v0 + 1 < v1 ? visit(v0 + 1) : x0, x2 = v0 + 2 < v1 ? visit(v0 + 2) : x1;
    load(x0);
    fetch_head(x0);
    put_head(x0, v0);
    meet();
    stage(x0, v0);
    load(x1);
    fetch_head(x1);
    put_head(x1, v0 + 1);
    fetch_head(x2);
    for (int v = v0; v < v1; ++v) {
      meet();
      if (v + 1 < v1) {
        stage(x1, v + 1);
        put_head(x2, v);
        load(x2);
      }
      __builtin_amdgcn_sched_barrier(0);
      f16v s[2];
      u4 pr[4];
      ta::scores<T16, 2>(s, ln, q, tiles(v));
      const int vv = v < nblk ? v : j.nblk + v - nblk;
      const bool whole = whole_at(p, j, vv, first);
      uint64_t vis = ~0ull;
      if (!whole || x0.drop) {
        vis = seen_by(p, j, vv, x0.drop, j.pos0 + tok);
        ta::mask_scores<2>(s, ln, vis);
      }
      x0 = x1;
      x1 = x2;
      if (v + 3 < v1) x2 = visit(v + 3);
      fetch_head(x2);
      ta::weights<T16, 2>(pr, st, s, p.sl2);
      const uint32_t values = tiles(v) + kRecTile;
      if (!whole && ta::find_odd<T16, 2, false>(ln, values, vis, odd)) {  // alike for all wavefronts
        meet();  // each has found them
        for (int i = threadIdx.x; i < kRecTile / 16; i += 64 * WAVES) {
          u4 y = ta::lds_u4(values + 16 * i);
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] &= ~ta::bad_halves<T16>(y[k]);
          *(LdsW4)(uintptr_t)(values + 16 * i) = y;
        }
        meet();
      }
      ta::outputs<T16, 2, false>(st, ln, pr, values);
    }
    ta::add_odd(st, odd);
  }
  const float l = st.l + ta::other_half(st.l);
  if (split == 1) {
    if (row < j.rows) store_row(p, j, tok, g, st, l > 0.f ? 1.f / l : l, ln.hf);
  } else if (row < j.rows) {
    store_part(p.part + (part_row(p, j, kTileRows) + 32 * wave + ln.col) * kPart, st, l, ln.hf);
  }
}

// Joins the partials of a row: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.  A wavefront
// per row, two channels a lane.
__global__ void __launch_bounds__(256) chunk_merge_kernel(const ChunkParams p, int rows_tile) {
  const int lane = threadIdx.x & 63, h = blockIdx.y;
  int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
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
  float m = -__builtin_inff();
  for (int i = 0; i < p.split[s]; ++i) {
    const float2 ml = *(const float2 *)(part + i * step + D);
    if (ml.y != 0.f) m = fmaxf(m, ml.x);  // (one that saw nothing has no maximum)
  }
  float a = 0.f, b = 0.f, l = 0.f;
  for (int i = 0; i < p.split[s]; ++i) {
    const float2 ml = *(const float2 *)(part + i * step + D);
    if (ml.y == 0.f) continue;
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    const float2 o = *(const float2 *)(part + i * step + 2 * lane);
    a += f * o.x;
    b += f * o.y;
    l += f * ml.y;
  }
  const float inv = l > 0.f ? 1.f / l : l;
  *(uint32_t *)(p.out + (p.row0[s] + tok) * p.os + (int64_t)(h * p.G + g) * D + 2 * lane) = T16::pack(a * inv, b * inv);
}

// ---------------------------------------------------------------- host
struct Plan {
  int rows_tile;
  int64_t wgs, part_rows;  // workgroups per KV head; partial rows over all KV heads
};

}  // namespace

// Visits a workgroup takes at least, and the workgroups that fill the chip.
constexpr int kLeastVisits = 4;
constexpr int64_t kFill = 256;

static gkv_status chunk_plan(const gkv_cache *c, const int32_t *n_new, ChunkParams &p, Plan &pl) {
  p.nseq = 0;
  const int G = c->Hq / c->Hkv;
  int64_t rows = 0, visits = 0, most = 0;
  for (int b = 0; b < c->B; ++b) {
    const int64_t T = seq_tokens(c, b), n = n_new[b];
    if (n < 0) return GKV_E_SHAPE;
    if (!n) continue;
    if (T < 0) return GKV_E_ARG;
    if (n > T) return GKV_E_SHAPE;
    if (T > 0x7fffff00 || n * G > 0x7fffff00 || rows + n > 0x7fffffff) return GKV_E_UNSUPPORTED;
    const int i = p.nseq++;
    p.seq[i] = b;
    p.T[i] = (int32_t)T;
    p.n[i] = (int32_t)n;
    p.row0[i] = (int32_t)rows;
    rows += n;
    most = n * G > most ? n * G : most;
  }
  pl.rows_tile = most <= 128 ? 128 : 256;
  auto vis = [&](int i) { return (p.T[i] + P - 1) / P + (c->nres + P - 1) / P; };
  auto tiles = [&](int i) { return ((int64_t)p.n[i] * G + pl.rows_tile - 1) / pl.rows_tile; };
  int64_t total = 0, plain = 0;
  for (int i = 0; i < p.nseq; ++i) {
    total += tiles(i) * vis(i) * c->Hkv;
    plain += tiles(i) * c->Hkv;
  }
  const int64_t fill = pl.rows_tile == 128 ? 2 * kFill : kFill;
  int64_t per = plain >= fill ? 0x7fffffff : (total + fill - 1) / fill;  // visits a workgroup
  if (per < kLeastVisits) per = kLeastVisits;
  pl.wgs = 0;
  bool any = false;
  for (int i = 0; i < p.nseq; ++i) {
    int64_t s = vis(i) / per;
    s = s < 1 ? 1 : s;
    p.split[i] = (int32_t)s;
    p.wg0[i] = (int32_t)pl.wgs;
    any |= s > 1;
    pl.wgs += s * tiles(i);
    if (pl.wgs * c->Hkv > 0x7fffffff) return GKV_E_UNSUPPORTED;
  }
  p.wg0[p.nseq] = (int32_t)pl.wgs;
  pl.part_rows = any ? pl.wgs * c->Hkv * pl.rows_tile : 0;
  return GKV_OK;
}

extern "C" int64_t gkv_chunk_ws_bytes(const gkv_cache *c, const int32_t *n_new) {
  if (gkv_validate_cache(c) || !n_new || c->B > kMaxSeqs) return -1;
  ChunkParams p;
  Plan pl;
  if (chunk_plan(c, n_new, p, pl)) return -1;
  return pl.part_rows * kPart * 4;
}

extern "C" gkv_status gkv_chunk_attn(const uint16_t *q, int64_t q_stride, const gkv_cache *c, const int32_t *n_new,
                                     uint16_t *out, int64_t out_stride, void *ws, int64_t ws_bytes, void *stream) {
  gkv_status st = gkv_validate_cache(c);
  if (st) return st;
  if (!n_new) return GKV_E_ARG;
  if (c->B > kMaxSeqs) return GKV_E_UNSUPPORTED;
  ChunkParams p;
  Plan pl;
  st = chunk_plan(c, n_new, p, pl);
  if (st) return st;
  if (!p.nseq) return GKV_OK;
  if (!q || !out || (uintptr_t)q % 16 || (uintptr_t)out % 16) return GKV_E_ARG;
  for (const int64_t s : {q_stride, out_stride}) {
    if (s < (int64_t)c->Hq * D) return GKV_E_SHAPE;
    if (s % 8) return GKV_E_ARG;
    if (s > GKV_MAX_ROW_STRIDE) return GKV_E_UNSUPPORTED;
  }
  if (pl.part_rows && (!ws || (uintptr_t)ws % 16)) return GKV_E_ARG;
  if (ws_bytes < pl.part_rows * kPart * 4) return GKV_E_WORKSPACE;
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
  p.res_rows = c->res_rows;
  p.nblk_cap = c->nblk_cap;
  p.Hkv = c->Hkv;
  p.G = c->Hq / c->Hkv;
  p.nres = c->nres;
  p.nres_cap = c->nres_cap;
  p.nrb_cap = (c->nres_cap + P - 1) / P;
  p.vtok = c->v_per_token;
  p.sl2 = 1.4426950408889634f / sqrtf((float)D);
  p.part0 = 0;
  const hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(pl.wgs * c->Hkv));
  constexpr size_t lds = 4 * kRecTile + 2 * 1024;
  if (pl.rows_tile == 128)
    hipLaunchKernelGGL((chunk_kernel<4>), grid, dim3(256), lds, s, p);
  else
    hipLaunchKernelGGL((chunk_kernel<8>), grid, dim3(512), lds, s, p);
  if (hipGetLastError() != hipSuccess) return GKV_E_HIP;
  if (pl.part_rows) {
    int64_t rows = 0;
    for (int i = 0; i < p.nseq; ++i) rows += p.split[i] > 1 ? (int64_t)p.n[i] * p.G : 0;
    hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)((rows + 3) / 4), c->Hkv), dim3(256), 0, s, p, pl.rows_tile);
    if (hipGetLastError() != hipSuccess) return GKV_E_HIP;
  }
  return GKV_OK;
}
