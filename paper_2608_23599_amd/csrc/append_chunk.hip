// Many tokens of every sequence appended at once (section 3.2's incremental append for a
// prompt's chunk or a speculative step's drafts), and the newest ones dropped again.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>
#include <vector>

#include "encode_block.h"
#include "gkv_internal.h"

#pragma clang fp contract(off)

using namespace gkv;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxSeqs = GKV_MAX_CHUNK_SEQS;
constexpr int kMaxRuns = 48;
constexpr int kRowPad = D + 8;  // halves: the rows of a 16-byte access lie on distinct banks

typedef uint32_t w4 __attribute__((ext_vector_type(4)));

// The opened blocks' slots, in the order of (sequence, KV head, block): runs of slots that lie
// evenly apart (the pool hands them out side by side while it is not fragmented), so that
// a chunk of any size needs few arguments and the tables are written on the GPU.
struct SlotRun {
  int32_t first, count;  // among the call's opened blocks
  int64_t k, v, step;
};

struct ChunkAppend {
  const uint16_t *k_new, *v_new;
  int64_t ks, vs;  // elements from a token's rows to the next one's
  int8_t *level;
  int64_t *koff, *voff;
  uint8_t *arena;
  uint16_t *boxes;  // or null
  int64_t npage_cap;
  float *cert;       // or null
  int64_t *seq_len;  // or null
  int32_t page, Hkv, nblk_cap;
  int32_t first_launch, nrun;
  SlotRun run[kMaxRuns];
  int64_t T[kMaxSeqs];  // tokens before the call (-1: retired)
  int32_t n[kMaxSeqs];  // new ones
};

__device__ __forceinline__ int key_half(int tok, int d) {  // half index of an exact key record's element
  return ((tok >> 4) * 64 + ((d >> 3) & 3) * 16 + (tok & 15)) * 32 + (((d >> 5) << 3) | (d & 7));
}

// One workgroup per (touched block, KV head).  Rows pass through LDS once, 16 bytes a lane
// from the tokens' rows and 16 bytes a lane into the records.  Bound by the latency of its three
// passes over a block (rows, records, norms and boxes), with four workgroups on a compute unit: 8192
// tokens x 8 KV heads 24 us (2.8 TB/s of rows and records), drafts 5 to 9 us.
__global__ void __launch_bounds__(kThreads) append_chunk_kernel(const ChunkAppend p) {
  __shared__ __align__(16) uint16_t kt[P * kRowPad], vt[P * kRowPad];
  const int h = blockIdx.y, tid = threadIdx.x;
  // the sequence and block of this workgroup, the sequence's first packed row and first slot
  int64_t row0 = 0;
  int item = blockIdx.x, slot = 0, b = 0;
  for (;; ++b) {  // ends inside: the grid is the touched blocks of all sequences
    const int64_t T = p.T[b];
    const int n = p.n[b];
    const int touched = n ? (int)((T + n - 1) / P - T / P) + 1 : 0;
    if (item < touched) break;
    item -= touched;
    row0 += n;
    if (n) slot += ((int)((T + n + P - 1) / P) - (int)((T + P - 1) / P)) * p.Hkv;
  }
  const int64_t T = p.T[b];
  const int n = p.n[b];
  const int blk = (int)(T / P) + item;
  const int64_t t0 = (int64_t)blk * P;
  const int lo = t0 >= T ? 0 : (int)(T - t0);  // rows lo .. hi - 1 of the block are new
  const int hi = (int)(T + n - t0 < P ? T + n - t0 : P);
  const bool open = t0 >= T;
  const int64_t u = (int64_t)b * p.Hkv + h;
  const int64_t ti = u * p.nblk_cap + blk;
  if (p.first_launch && p.seq_len && item == 0 && h == 0 && tid == 0) p.seq_len[b] = T + n;
  int64_t ko, vo;
  if (open) {
    const int nopen = (int)((T + n + P - 1) / P) - (int)((T + P - 1) / P);
    slot += h * nopen + (blk - (int)((T + P - 1) / P));
    int r = 0;
    while (r < p.nrun && !(slot >= p.run[r].first && slot < p.run[r].first + p.run[r].count)) ++r;
    if (r == p.nrun) return;  // another launch's
    ko = p.run[r].k + (slot - p.run[r].first) * p.run[r].step;
    vo = p.run[r].v + (slot - p.run[r].first) * p.run[r].step;
    if (tid == 0) {
      p.level[ti] = GKV_EXACT;
      p.koff[ti] = ko;
      p.voff[ti] = vo;
    }
  } else {
    if (!p.first_launch) return;
    ko = p.koff[ti];
    vo = p.voff[ti];
  }
  uint16_t *kr = (uint16_t *)(p.arena + ko), *vr = (uint16_t *)(p.arena + vo);

  // the block's rows in LDS: new ones from their tokens, the older ones' keys from the record
  // (the page boxes need them), zeros behind the last
  const uint16_t *ks = p.k_new + (row0 + t0 - T) * p.ks + (int64_t)h * D;
  const uint16_t *vs = p.v_new + (row0 + t0 - T) * p.vs + (int64_t)h * D;
  for (int i = tid; i < P * 16; i += kThreads) {
    const int t = i >> 4, d = (i & 15) * 8;
    w4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (t >= lo && t < hi) {
      k = *(const w4 *)(ks + t * p.ks + d);
      v = *(const w4 *)(vs + t * p.vs + d);
    } else if (t < lo && p.boxes) {
      k = *(const w4 *)(kr + key_half(t, d));
    }
    *(w4 *)(kt + t * kRowPad + d) = k;
    *(w4 *)(vt + t * kRowPad + d) = v;
  }
  __syncthreads();

  // keys: a unit of 8 channels of one token; values: a lane's chunk, 4 tokens of 8 channels
  for (int i = tid; i < P * 16; i += kThreads) {
    const int t = i >> 4, d = (i & 15) * 8;
    if (open || (t >= lo && t < hi)) *(w4 *)(kr + key_half(t, d)) = *(const w4 *)(kt + t * kRowPad + d);
  }
  {
    const int pg = tid >> 6, kg = (tid >> 4) & 3, m = tid & 15, t4 = 16 * pg + 4 * kg;
    if (open || (t4 + 4 > lo && t4 < hi)) {
      uint16_t x[32];
      if (!open && (t4 < lo || t4 + 4 > hi))  // some of the four are older, or not there yet
#pragma unroll
        for (int i = 0; i < 4; ++i) *(w4 *)(x + 8 * i) = *(const w4 *)(vr + tid * 32 + 8 * i);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int t = t4 + (i & 3);
        if (open || (t >= lo && t < hi)) x[i] = vt[t * kRowPad + 16 * (i >> 2) + m];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) *(w4 *)(vr + tid * 32 + 8 * i) = *(const w4 *)(x + 8 * i);
    }
  }

  if (p.cert) {  // an exact block: no error; the value norms, each a channel-ascending sum
    if (tid < P) {  // (one wavefront)
      double s = 0.0;
      if (tid >= lo && tid < hi)
#pragma unroll 4
        for (int d = 0; d < D; d += 8) {
          const w4 w = *(const w4 *)(vt + tid * kRowPad + d);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double x = (double)__builtin_bit_cast(_Float16, (uint16_t)(w[i >> 1] >> (16 * (i & 1))));
            s += x * x;
          }
        }
      for (int k = 1; k < P; k <<= 1) {
        const double y = __shfl_xor(s, k);
        s = y > s ? y : s;
      }
      if (tid == 0) {
        const float vn = enc::round_up_f32(__builtin_sqrt(s));
        float *cb = p.cert + ti * 4;
        if (open) {
          cb[0] = 0.f;
          cb[1] = 0.f;
          cb[2] = vn;
          cb[3] = 0.f;
        } else {
          cb[2] = vn > cb[2] ? vn : cb[2];
        }
      }
    }
  }
  if (p.boxes) {  // the pages that the new rows complete
    const int d = tid & (D - 1);
    for (int pg = lo / p.page + (tid >> 7); (pg + 1) * p.page <= hi; pg += 2) {
      const uint16_t *row = kt + pg * p.page * kRowPad + d;
      _Float16 mn = __builtin_bit_cast(_Float16, row[0]), mx = mn;
      for (int t = 1; t < p.page; ++t) {
        const _Float16 x = __builtin_bit_cast(_Float16, row[t * kRowPad]);
        mn = x < mn ? x : mn;
        mx = x > mx ? x : mx;
      }
      uint16_t *bx = p.boxes + u * p.npage_cap * 2 * D + box_index(t0 / p.page + pg, d);
      bx[0] = canon_zero(__builtin_bit_cast(uint16_t, mn));
      bx[1] = canon_zero(__builtin_bit_cast(uint16_t, mx));
    }
  }
}

struct ChunkDrop {
  const int64_t *koff, *voff;
  uint8_t *arena;
  int64_t *seq_len;
  int32_t nblk_cap;
  int64_t from[kMaxSeqs], to[kMaxSeqs];  // tokens before and after (-1: retired)
};

// The dropped rows of the block that stays partial become zero again: reads mask them, but
// 0 * NaN is NaN.  Grid (Hkv, B).  Bound by its two dependent round trips: 3 to 5 us.
__global__ void __launch_bounds__(kThreads) truncate_kernel(const ChunkDrop p) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int64_t T = p.from[b], L = p.to[b];
  if (L >= T) return;  // nothing dropped (or retired)
  if (p.seq_len && h == 0 && tid == 0) p.seq_len[b] = L;
  const int lo = (int)(L % P);
  if (!lo) return;
  const int64_t ti = ((int64_t)b * gridDim.x + h) * p.nblk_cap + L / P;
  uint16_t *kr = (uint16_t *)(p.arena + p.koff[ti]), *vr = (uint16_t *)(p.arena + p.voff[ti]);
  const w4 zero = {0, 0, 0, 0};
  for (int i = tid; i < P * 16; i += kThreads)
    if ((i >> 4) >= lo) *(w4 *)(kr + key_half(i >> 4, (i & 15) * 8)) = zero;
  const int pg = tid >> 6, kg = (tid >> 4) & 3, t4 = 16 * pg + 4 * kg;
  if (t4 + 4 <= lo) return;
  for (int i = 0; i < 32; ++i)
    if (t4 + (i & 3) >= lo) vr[tid * 32 + i] = 0;
}

}  // namespace

// ---------------------------------------------------------------- C ABI
static gkv_status append_chunk(gkv_cache *c, const uint16_t *k_new, const uint16_t *v_new, int64_t k_stride,
                               int64_t v_stride, const int32_t *n_new, const int64_t *koff, const int64_t *voff,
                               int32_t n_open, hipStream_t stream) {
  gkv_status st = gkv_validate_cache(c);
  if (st) return st;
  if (!n_new || n_open < 0 || (n_open && (!koff || !voff))) return GKV_E_ARG;
  if (c->B > kMaxSeqs) return GKV_E_UNSUPPORTED;
  ChunkAppend p;
  int64_t rows = 0, items = 0, opened = 0, longest = c->seq_len_host ? 0 : c->T;
  for (int b = 0; b < c->B; ++b) {
    const int64_t T = seq_tokens(c, b), n = n_new[b];
    if (n < 0) return GKV_E_SHAPE;
    if (T < 0 && n) return GKV_E_ARG;  // retired
    if (!c->seq_len_host && n != n_new[0]) return GKV_E_SHAPE;
    p.T[b] = T;
    p.n[b] = (int32_t)n;
    if (T >= 0 && T + n > longest) longest = T + n;
    if (!n) continue;
    if ((T + n + P - 1) / P > c->nblk_cap) return GKV_E_SHAPE;
    if (c->page && (T + n) / c->page > c->npage_cap) return GKV_E_SHAPE;
    if (T % P)
      for (int h = 0; h < c->Hkv; ++h)
        if (c->level_host[((int64_t)b * c->Hkv + h) * c->nblk_cap + T / P] != GKV_EXACT) return GKV_E_ARG;
    rows += n;
    items += (T + n - 1) / P - T / P + 1;
    opened += ((T + n + P - 1) / P - (T + P - 1) / P) * c->Hkv;
  }
  if (opened != n_open) return GKV_E_ARG;
  if (!rows) return GKV_OK;
  if (items > GKV_MAX_LAUNCH / kThreads || c->Hkv > 65535) return GKV_E_UNSUPPORTED;
  if (!k_new || !v_new || (uintptr_t)k_new % 16 || (uintptr_t)v_new % 16) return GKV_E_ARG;
  for (const int64_t s : {k_stride, v_stride}) {
    if (s < (int64_t)c->Hkv * D) return GKV_E_SHAPE;
    if (s % 8) return GKV_E_ARG;
    if (s > GKV_MAX_ROW_STRIDE) return GKV_E_UNSUPPORTED;
  }
  // every slot in the arena, no two in one place: seen at once where they stand in order, as an
  // unfragmented pool hands them out
  bool up = true, down = true;
  int64_t last = 0;
  for (int i = 0; i < 2 * n_open; ++i) {
    const int64_t off = i & 1 ? voff[i >> 1] : koff[i >> 1];
    if (off < 0 || off % 16 || off + kExactBytes > c->arena_bytes) return GKV_E_ARG;
    up &= !i || off - last >= kExactBytes;
    down &= !i || last - off >= kExactBytes;
    last = off;
  }
  if (!up && !down) {
    std::vector<int64_t> slots(koff, koff + n_open);
    slots.insert(slots.end(), voff, voff + n_open);
    std::sort(slots.begin(), slots.end());
    for (size_t i = 1; i < slots.size(); ++i)
      if (slots[i] - slots[i - 1] < kExactBytes) return GKV_E_ARG;
  }
  p.k_new = k_new;
  p.v_new = v_new;
  p.ks = k_stride;
  p.vs = v_stride;
  p.level = c->level;
  p.koff = c->koff;
  p.voff = c->voff;
  p.arena = c->arena;
  p.boxes = c->page ? c->boxes : nullptr;
  p.npage_cap = c->npage_cap;
  p.cert = c->cert;
  p.seq_len = c->seq_len;
  p.page = c->page ? c->page : P;
  p.Hkv = c->Hkv;
  p.nblk_cap = c->nblk_cap;
  p.first_launch = 1;
  int i = 0;
  do {  // one launch, more if the slots make more runs than one takes
    p.nrun = 0;
    while (i < n_open && p.nrun < kMaxRuns) {
      SlotRun r = {i, 1, koff[i], voff[i], 0};
      if (i + 1 < n_open && koff[i + 1] - koff[i] == voff[i + 1] - voff[i]) {
        r.step = koff[i + 1] - koff[i];
        while (i + r.count < n_open && koff[i + r.count] == r.k + r.count * r.step &&
               voff[i + r.count] == r.v + r.count * r.step)
          ++r.count;
      }
      i += r.count;
      p.run[p.nrun++] = r;
    }
    hipLaunchKernelGGL(append_chunk_kernel, dim3((unsigned)items, c->Hkv), dim3(kThreads), 0, stream, p);
    if (hipGetLastError() != hipSuccess) return GKV_E_HIP;
    p.first_launch = 0;
  } while (i < n_open);
  for (int b = 0; b < c->B; ++b) {
    const int64_t T = p.T[b], n = p.n[b];
    if (T < 0) continue;
    for (int64_t blk = (T + P - 1) / P; blk < (T + n + P - 1) / P; ++blk)
      for (int h = 0; h < c->Hkv; ++h) c->level_host[((int64_t)b * c->Hkv + h) * c->nblk_cap + blk] = GKV_EXACT;
    if (c->seq_len_host) c->seq_len_host[b] = T + n;
  }
  c->T = longest;
  if (n_open) gkv_stamp(c);
  return GKV_OK;
}

extern "C" gkv_status gkv_append_chunk(gkv_cache *c, const uint16_t *k_new, const uint16_t *v_new, int64_t k_stride,
                                       int64_t v_stride, const int32_t *n_new, const int64_t *new_koff,
                                       const int64_t *new_voff, int32_t n_open, void *stream) {
  try {
    return append_chunk(c, k_new, v_new, k_stride, v_stride, n_new, new_koff, new_voff, n_open, (hipStream_t)stream);
  } catch (const std::bad_alloc &) {  // the host's slot list, before anything is enqueued
    return GKV_E_HIP;
  }
}

extern "C" gkv_status gkv_truncate(gkv_cache *c, gkv_pool *pool, const int64_t *koff, const int64_t *voff,
                                   const int64_t *len, void *stream) {
  gkv_status st = gkv_validate_cache(c);
  if (st) return st;
  if (!pool || !koff || !voff || !len) return GKV_E_ARG;
  if (c->B > kMaxSeqs || c->Hkv > 65535) return GKV_E_UNSUPPORTED;
  if (c->nres) return GKV_E_UNSUPPORTED;
  ChunkDrop p;
  bool any = false, any_block = false;
  int64_t longest = 0;
  for (int b = 0; b < c->B; ++b) {
    const int64_t T = seq_tokens(c, b), L = T < 0 ? -1 : len[b];
    if (T >= 0 && (L < 0 || L > T)) return GKV_E_SHAPE;
    if (!c->seq_len_host && L != len[0]) return GKV_E_SHAPE;
    p.from[b] = T;
    p.to[b] = L;
    longest = L > longest ? L : longest;
    any |= L < T;
    any_block |= L < T && (L + P - 1) / P < (T + P - 1) / P;
    if (L < T && L % P)
      for (int h = 0; h < c->Hkv; ++h)  // a block its sequence does not fill is exact
        if (c->level_host[((int64_t)b * c->Hkv + h) * c->nblk_cap + L / P] != GKV_EXACT) return GKV_E_SHAPE;
  }
  if (!any) return GKV_OK;
  // The slots go back in the reverse of the order in which an append of the same tokens takes
  // them: the next one takes them again.  A slot that is not a used one of its level, or is
  // listed twice, fails the call with every slot as it was.
  int64_t freed[GKV_EXACT + 1] = {0};
  gkv_status bad = GKV_OK;
  auto give = [&](int level, int64_t off) {
    bad = gkv_pool_free(pool, level, off);
    freed[bad ? 0 : level] += !bad;
    return !bad;
  };
  for (int b = c->B - 1; b >= 0 && !bad; --b)
    for (int h = c->Hkv - 1; h >= 0 && !bad; --h)
      for (int64_t blk = (p.from[b] + P - 1) / P - 1; blk >= (p.to[b] + P - 1) / P && blk >= 0; --blk) {
        const int64_t e = ((int64_t)b * c->Hkv + h) * c->nblk_cap + blk;
        if (!give(c->level_host[e], voff[e]) || !give(c->level_host[e], koff[e])) break;
      }
  if (!bad) {
    p.koff = c->koff;
    p.voff = c->voff;
    p.arena = c->arena;
    p.seq_len = c->seq_len;
    p.nblk_cap = c->nblk_cap;
    hipLaunchKernelGGL(truncate_kernel, dim3(c->Hkv, c->B), dim3(kThreads), 0, (hipStream_t)stream, p);
    if (hipGetLastError() != hipSuccess) bad = GKV_E_HIP;
  }
  if (bad) {  // a pool gives out the slots last freed first: as many again, and it is as it was
    for (int level = 0; level <= GKV_EXACT; ++level)
      for (; freed[level] > 0; --freed[level]) gkv_pool_alloc(pool, level);
    return bad;
  }
  for (int b = 0; b < c->B; ++b)
    if (c->seq_len_host) c->seq_len_host[b] = p.to[b];
  c->T = longest;
  if (any_block) {
    c->truncated = 1;
    gkv_stamp(c);
  }
  return GKV_OK;
}
