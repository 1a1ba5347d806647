// Causal attention over packed prompts of different lengths (section 3.1's dense attention,
// before anything is graded): the step that makes a prompt's outputs while its keys and
// values are still exact.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "gkv_internal.h"
#include "tile_attn.h"

#pragma clang diagnostic ignored "-Winline-asm"

using namespace gkv;

namespace {

constexpr int kTile = 64;                   // tokens of a key/value tile
constexpr int kTileBytes = kTile * D * 2;   // of keys, or of values
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

__device__ __forceinline__ void dma_row(uint32_t voff, const void *base, uint32_t lds) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(m0v) : "memory", "m0");
}

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
  const int ntile = min(r0 + 32 * WAVES - 1, rows - 1) / G / kTile + 1;

  const uint8_t *kb = (const uint8_t *)(p.k + start * p.ks + (int64_t)h * D);
  const uint8_t *vb = (const uint8_t *)(p.v + start * p.vs + (int64_t)h * D);
  // copies: instruction i of this wavefront moves rows 4 (wave + WAVES i) .. + 3 of a tile
  constexpr int kCopies = 16 / WAVES;
  const int cr = ln.lane >> 4, cu = ln.lane & 15;
  auto copy_keys = [&](int t) {
    const int left = L - 1 - t * kTile;
    const uint8_t *src = kb + (int64_t)t * kTile * p.ks * 2;
    const uint32_t buf = lds + (t & 1) * kTileBytes;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r4 = 4 * (wave + WAVES * i), r = r4 + cr;  // past the end: the last token's row again, masked
      dma_row((uint32_t)(min(r, left) * (int)p.ks * 2) + ((cu ^ (r & 15)) << 4), src, buf + r4 * 256);
    }
  };
  auto copy_values = [&](int t) {
    const int left = L - 1 - t * kTile;
    const uint8_t *src = vb + (int64_t)t * kTile * p.vs * 2;
    const uint32_t buf = lds + (2 + (t & 1)) * kTileBytes;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r4 = 4 * (wave + WAVES * i), r = r4 + cr;
      dma_row((uint32_t)(min(r, left) * (int)p.vs * 2) + ((cu ^ ((r & 3) << 2)) << 4), src, buf + r4 * 256);
    }
  };
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
  auto meet = [] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  copy_keys(0);
  ta::u4 q[8];
  {
    const uint16_t *qp = p.q + (start + tok) * p.qs + (int64_t)(h * G + g) * D + 8 * ln.hf;
#pragma unroll
    for (int d = 0; d < 8; ++d) q[d] = *(const ta::u4 *)(qp + 16 * d);
  }
  ta::Rows st;
  st.init();
  ta::f16v s[2];
  ta::u4 pr[4];
  // The two wavefronts of a SIMD work half a tile apart: while one multiplies (the last
  // tile's values, this tile's keys) the other forms weights.  In the same phase they wait
  // for one unit together: 43% of the time the MFMAs ran and 49% the vector instructions.
  const bool second = wave >= WAVES / 2;
  auto keys = [&](int t) { return lds + (t & 1) * kTileBytes; };
  auto values = [&](int t) { return lds + (2 + (t & 1)) * kTileBytes; };
  auto copy = [&](int t) {  // in the interval of the first wavefronts' key product of tile t
    if (t + 1 < ntile) copy_keys(t + 1);
    if (t < ntile) copy_values(t);
  };
  auto seen = [&](int t) {  // this row's visible tokens of tile t
    const int n = tok - t * kTile + 1;
    return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
  };
  // Intervals, each ended by a barrier: the first wavefronts' key product of tile t is in
  // interval 2 t, the second ones' in 2 t + 1.  Keys t + 1 and values t are copied from the
  // start of interval 2 t on (whose buffers were last read in 2 t - 1) and have arrived at
  // the end of 2 t + 1.
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
  const int full = min(first / kTile, ntile - 1);  // tiles before this one are seen whole by every row
  arrived();
  meet();
  copy(0);
  if (second) {
    arrived();
    meet();
  }
  ta::scores<T, 2>(s, ln, q, keys(0));
  after(-1);
  int t = 0;
  for (; t < full; ++t) {
    ta::weights<T, 2>(pr, st, s, p.sl2);
    before(t);
    ta::multiply<T, true>(st, s, ln, pr, q, values(t), keys(t + 1));
    after(t);
  }
  ta::u4 odd = {0, 0, 0, 0};  // infinities and NaN there
  for (;; ++t) {
    const uint64_t vis = seen(t);
    ta::mask_scores<2>(s, ln, vis);
    ta::weights<T, 2>(pr, st, s, p.sl2);
    before(t);
    const bool clean = ta::find_odd<T, 2, true>(ln, values(t), vis, odd);
    ta::outputs_clean<T, 2, true>(st, ln, pr, values(t), clean);
    if (t == ntile - 1) break;
    ta::scores<T, 2>(s, ln, q, keys(t + 1));
    after(t);
  }
  if (!second) meet();
  ta::add_odd(st, odd);
  if (row < rows) {
    const float l = st.l + ta::other_half(st.l);
    const float inv = l > 0.f ? 1.f / l : l;  // (a NaN stays)
    uint16_t *op = p.out + (start + tok) * p.os + (int64_t)(h * G + g) * D + 4 * ln.hf;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ta::u2 w;
        w[0] = T::pack(st.o[c][4 * i] * inv, st.o[c][4 * i + 1] * inv);
        w[1] = T::pack(st.o[c][4 * i + 2] * inv, st.o[c][4 * i + 3] * inv);
        *(ta::u2 *)(op + 32 * c + 8 * i) = w;
      }
  }
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
  if (tiles * Hkv > 0x7fffffff) return GKV_E_UNSUPPORTED;
  const dim3 grid((unsigned)(tiles * Hkv)), blk(64 * kWaves);
  const size_t lds = 4 * kTileBytes;
  if (dtype == GKV_F16)
    hipLaunchKernelGGL((prompt_kernel<ta::F16, kWaves>), grid, blk, lds, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL((prompt_kernel<ta::BF16, kWaves>), grid, blk, lds, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? GKV_OK : GKV_E_HIP;
}
