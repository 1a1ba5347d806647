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
  __device__ __forceinline__ void keys(int t, uint32_t lds, uint32_t) const { copy(t, lds, k, ks, true); }
  __device__ __forceinline__ void values(int t, uint32_t lds) const { copy(t, lds, v, vs, false); }
};

// One workgroup for 32 WAVES rows of a (prompt, KV head), 215 registers and 64 KB of LDS: one on a
// compute unit, two wavefronts a SIMD.  Bound by matrix and vector issue beside one another (1.87 us
// for 256 rows x 64 tokens), and in short prompts by the first copies, masked tiles and stores, about
// 6 us a workgroup with nothing else on its unit.  28/4 heads in bf16: one prompt of 16k tokens
// 1790 us (1.08 PFLOP/s; a large library product reaches 1.27), sixteen of 107 to 2000 220 us;
// 32/8 heads in fp16, 4k tokens: 148 us.
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
  constexpr int kWaves = 8;
  int64_t tiles = 0;
  for (int i = 0; i < n; ++i) {
    p.len[i] = (int32_t)seqs[i].first;
    p.start[i] = (int32_t)seqs[i].second;
    p.tiles[i] = (int32_t)tiles;
    tiles += (seqs[i].first * G + 32 * kWaves - 1) / (32 * kWaves);
  }
  p.tiles[n] = (int32_t)tiles;
  if (tiles * Hkv > GKV_MAX_LAUNCH / (64 * kWaves)) return GKV_E_UNSUPPORTED;
  const dim3 grid((unsigned)(tiles * Hkv)), blk(64 * kWaves);
  const size_t lds = ta::kAttendLds;
  if (dtype == GKV_F16)
    hipLaunchKernelGGL((prompt_kernel<ta::F16, kWaves>), grid, blk, lds, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL((prompt_kernel<ta::BF16, kWaves>), grid, blk, lds, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? GKV_OK : GKV_E_HIP;
}
