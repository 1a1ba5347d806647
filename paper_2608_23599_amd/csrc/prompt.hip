// Causal attention over packed prompts of different lengths (section 3.1's dense attention,
// before anything is graded): the step that makes a prompt's outputs while its keys and
// values are still exact.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "gkv_internal.h"
#include "tile_attn.h"

using namespace gkv;

namespace {

constexpr int kMaxSeqs = GKV_MAX_PROMPTS;

struct PromptParams {
  const uint16_t *q, *k, *v;
  uint16_t *out;
  int64_t qs, ks, vs, os;  // elements from a token's rows to the next one's
  int32_t Hkv, G, nseq;
  float sl2;
  int32_t start[kMaxSeqs], len[kMaxSeqs];  // sequences, the longest first
  int32_t tiles[kMaxSeqs + 1];             // row tiles before each
};

// A prompt's tiles: 4 rows of 256 B a copy, each row's 16-byte units in the places the reads
// want them in; rows past the end are the last token's again (masked).
template <int WAVES>
struct PromptTiles {
  const uint8_t *k, *v;
  uint32_t ks, vs;  // bytes from token to token
  int L, wave, lane;
  __device__ __forceinline__ void copy(int t, uint32_t lds, const uint8_t *base, uint32_t stride, bool keys) const {
    const int left = L - 1 - t * ta::kTile;
    const uint8_t *src = base + (int64_t)t * ta::kTile * stride;
#pragma unroll
    for (int i = 0; i < 16 / WAVES; ++i) {
      const int r4 = 4 * (wave + WAVES * i), r = r4 + (lane >> 4);
      const int u = (lane & 15) ^ (keys ? r & 15 : (r & 3) << 2);
      ta::dma16((uint32_t)min(r, left) * stride + (u << 4), src, lds + r4 * 256);
    }
  }
  __device__ __forceinline__ void keys(int t, uint32_t lds, uint32_t, uint32_t) const { copy(t, lds, k, ks, true); }
  __device__ __forceinline__ void values(int t, uint32_t lds) const { copy(t, lds, v, vs, false); }
};

// One workgroup for 32 WAVES rows of a (prompt, KV head), up to 220 registers and 64 KB of LDS: two
// wavefronts a SIMD, in one workgroup or two (see launch).  Bound by matrix and vector issue beside one another (1.87 us
// for 256 rows x 64 tokens), and in short prompts by the first copies, masked tiles and stores, about
// 6 us a workgroup of eight wavefronts with nothing else on its unit.  28/4 heads in bf16: one prompt of 16k tokens
// 1770 to 1840 us from card to card (1.05 to 1.09 PFLOP/s; a large library product reaches 1.27), sixteen of 107 to 2000 210 to 226;
// 32/8 heads in fp16, 4k tokens: 146 us.
template <class T, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) prompt_kernel(const PromptParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
  const int h = blockIdx.x % p.Hkv, j = blockIdx.x / p.Hkv;
  int lo = 0, hi = p.nseq;  // the sequence of row tile j
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.tiles[mid] <= j) lo = mid;
    else hi = mid;
  }
  const int L = p.len[lo], G = p.G;
  const int64_t start = p.start[lo];
  const int rows = L * G;
  const int tile = p.tiles[lo + 1] - 1 - j;  // the last rows, which see most, first
  const int r0 = tile * (32 * WAVES);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  ta::Lane ln;
  ln.init<true>();

  // this lane's row; rows past the last are copies of it and not stored
  const int row = r0 + 32 * wave + ln.col;
  const int rc = row < rows ? row : rows - 1;
  const int tok = rc / G, g = rc - tok * G;
  const int first = r0 / G;  // tokens up to this one are seen by every row
  const int ntile = min(r0 + 32 * WAVES - 1, rows - 1) / G / ta::kTile + 1;
  const PromptTiles<WAVES> src = {(const uint8_t *)(p.k + start * p.ks + (int64_t)h * D),
                                  (const uint8_t *)(p.v + start * p.vs + (int64_t)h * D),
                                  (uint32_t)p.ks * 2, (uint32_t)p.vs * 2, L, wave, ln.lane};
  ta::Rows st;
  ta::u4 q[8];
  ta::attend<T, WAVES, true, false>(
      st, ln, q, lds, wave, 0, ntile, first / ta::kTile, p.sl2, src,
      [&](int t) {  // this row's visible tokens of tile t
        const int n = tok - t * ta::kTile + 1;
        return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
      },
      [&] {
        const uint16_t *qp = p.q + (start + tok) * p.qs + (int64_t)(h * G + g) * D + 8 * ln.hf;
#pragma unroll
        for (int d = 0; d < 8; ++d) q[d] = *(const ta::u4 *)(qp + 16 * d);
      });
  const float l = st.l + ta::other_half(st.l);
  const float inv = l > 0.f ? 1.f / l : l;  // (a NaN stays)
  if (row < rows) ta::store_row<T>(p.out + (start + tok) * p.os + (int64_t)(h * G + g) * D, st, inv, ln.hf);
}

// Row tiles of every sequence at so many rows each; returns their number.
int64_t row_tiles(PromptParams &p, int rows) {
  int64_t tiles = 0;
  for (int i = 0; i < p.nseq; ++i) {
    p.tiles[i] = (int32_t)tiles;
    tiles += ((int64_t)p.len[i] * p.G + rows - 1) / rows;
  }
  p.tiles[p.nseq] = (int32_t)tiles;
  return tiles;
}

// Eight wavefronts a workgroup, or four, of which a compute unit holds two: those share no tiles, so that
// a step takes 5% longer, but one works through the other's first copies and stores, and half as
// many rows leave fewer units idle.  Four, in us against eight:
//  * up to half a workgroup of eight a unit: 28/4 heads, one prompt of 512 tokens 19.6 and 23.7;
//  * up to one a unit, where row tiles are of many lengths: one of 1200 to 2300 tokens 31.7 to 59.9 and
//    40.1 to 69.2, but four of 512 26.3 and 26.1, with 32/8 heads 27.6 and 25.0;
//  * beyond, where row tiles are short, up to 12 steps of 64 tokens on the mean.  Four over eight at 8
//    steps 0.90 to 1.01, at 10 and 11 0.92 to 1.03 (sixteen prompts of 107 to 2000 tokens in bf16 209.7 and
//    225.6), at 12 1.00 to 1.03, at 13 1.00 to 1.02, at 14 0.98 to 1.07, at 16 0.98 to 1.08, at 18
//    1.02 to 1.09 (28/4 and 32/8 heads; one of 4096 at 32 steps 1.06 and 1.08).
template <class T>
gkv_status launch(PromptParams &p, hipStream_t s) {
  const int64_t wide = row_tiles(p, 256) * p.Hkv;
  int64_t steps = 0;  // of 64 tokens, over all row tiles (twice)
  for (int i = 0; i < p.nseq; ++i) steps += (int64_t)(p.tiles[i + 1] - p.tiles[i]) * (p.len[i] / ta::kTile + 1);
  steps = steps * p.Hkv / (2 * wide);
  const int64_t cus = gkv_device_cus();
  const bool narrow = wide <= cus / 2 || (wide <= cus ? steps >= 8 : steps <= 12);
  const int64_t wgs = narrow ? row_tiles(p, 128) * p.Hkv : wide;
  const int threads = narrow ? 256 : 512;
  if (wgs > GKV_MAX_LAUNCH / threads) return GKV_E_UNSUPPORTED;
  const dim3 grid((unsigned)wgs), blk(threads);
  if (narrow) hipLaunchKernelGGL((prompt_kernel<T, 4>), grid, blk, ta::kAttendLds, s, p);
  else hipLaunchKernelGGL((prompt_kernel<T, 8>), grid, blk, ta::kAttendLds, s, p);
  return hipGetLastError() == hipSuccess ? GKV_OK : GKV_E_HIP;
}

}  // namespace

extern "C" gkv_status gkv_prompt_attn(const void *q, const void *k, const void *v, void *out, int32_t dtype,
                                      int32_t Hkv, int32_t Hq, int32_t nseq, const int64_t *len_host,
                                      int64_t q_stride, int64_t k_stride, int64_t v_stride, int64_t out_stride,
                                      void *stream) {
  if (dtype != GKV_F16 && dtype != GKV_BF16) return GKV_E_ARG;
  if (nseq < 0 || (nseq && !len_host)) return GKV_E_ARG;
  if (Hkv <= 0 || Hq <= 0 || Hq % Hkv || Hq / Hkv > 16) return GKV_E_SHAPE;
  if (nseq > kMaxSeqs) return GKV_E_UNSUPPORTED;
  const int G = Hq / Hkv;
  PromptParams p;
  int64_t total = 0;
  std::pair<int64_t, int64_t> seqs[kMaxSeqs];  // (length, start)
  int n = 0;
  for (int b = 0; b < nseq; ++b) {
    if (len_host[b] < 0) return GKV_E_SHAPE;
    if (len_host[b] > GKV_MAX_PROMPT_TOKENS - total) return GKV_E_UNSUPPORTED;
    if (len_host[b]) seqs[n++] = {len_host[b], total};
    total += len_host[b];
  }
  if (!total) return GKV_OK;
  if (!q || !k || !v || !out) return GKV_E_ARG;
  for (const void *x : {q, k, v, (const void *)out})
    if ((uintptr_t)x % 16) return GKV_E_ARG;
  const int64_t least[4] = {(int64_t)Hq * D, (int64_t)Hkv * D, (int64_t)Hkv * D, (int64_t)Hq * D};
  const int64_t strides[4] = {q_stride, k_stride, v_stride, out_stride};
  for (int i = 0; i < 4; ++i) {
    if (strides[i] < least[i]) return GKV_E_SHAPE;
    if (strides[i] % 8) return GKV_E_ARG;
    if (strides[i] > GKV_MAX_ROW_STRIDE) return GKV_E_UNSUPPORTED;
  }
  std::stable_sort(seqs, seqs + n, [](const auto &a, const auto &b) { return a.first > b.first; });
  p.q = (const uint16_t *)q;
  p.k = (const uint16_t *)k;
  p.v = (const uint16_t *)v;
  p.out = (uint16_t *)out;
  p.qs = q_stride;
  p.ks = k_stride;
  p.vs = v_stride;
  p.os = out_stride;
  p.Hkv = Hkv;
  p.G = G;
  p.nseq = n;
  p.sl2 = 1.4426950408889634f / sqrtf((float)D);
  for (int i = 0; i < n; ++i) {
    p.len[i] = (int32_t)seqs[i].first;
    p.start[i] = (int32_t)seqs[i].second;
  }
  return dtype == GKV_F16 ? launch<ta::F16>(p, (hipStream_t)stream) : launch<ta::BF16>(p, (hipStream_t)stream);
}
