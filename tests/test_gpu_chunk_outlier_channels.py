"""Chunks of many rows over integer blocks whose keys have outlier channels.

Scores are sums of products of which the outliers' are the largest, and a rounding of their keys to fp16 would be
the largest error of a row: it is held to 22 bits in the 16 channels with the largest keys.  The rest rounds
independently, each with a root mean square of at most u / sqrt(3), u = 2^-11: the outputs, the weights,
the decoded values and, by way of the scores, the other channels' keys.  Their squares add as in the
rows' bound; over all rows and channels of a test the sum is within a quarter of its expectation."""
import numpy as np
import pytest

from oracle import cache as ocache, fp16 as ofp16
from tests.test_gpu_chunk_accuracy import U, causal, rows_and_bounds, softmax_rows

T, N = 64 * 80 + 3, 150


def data(seed, heads, outliers):
    r = np.random.default_rng(seed)
    gain = np.ones((1, heads, 1, 128))
    for h in range(heads):
        gain[0, h, 0, r.permutation(128)[:outliers]] = 10.0
    k, v = (r.standard_normal((1, heads, T, 128)) for _ in range(2))
    q = r.standard_normal((N, heads, 128)).astype(np.float16)
    return ofp16.from_f64(k * gain), ofp16.from_f64(v), q


def expected(q, kh, vh, codes):
    """Outputs and the expected square of all their errors together at most."""
    hot = np.argsort(-(kh * kh).sum(0))[:16]
    rest = kh.copy()
    rest[:, hot] = 0.0
    o = softmax_rows(q, kh, causal(T, N)) @ vh
    w = softmax_rows(q, kh, causal(T, N))
    w2, v2 = w * w, (vh * vh).sum(1)
    off = v2[None, :] - 2 * o @ vh.T + (o * o).sum(1)[:, None]
    s2 = (q * q) @ (rest * rest).T / 128
    return o, U * U / 3 * ((o * o).sum() + (w2 * (off * (1 + s2 * codes) + v2 * codes)).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("outliers", [0, 4, 16])
@pytest.mark.parametrize("level", [2, 4, 8])
def test_error_with_outlier_channels(gpu, level, outliers):
    ks, vs, q = data(level + outliers, 2, outliers)
    levels = np.array([level] * 77 + [16] * 4, np.int8)
    cache = gpu.GradedCache.build(ks, vs, Hq=2, levels=levels)
    out = cache.chunk_attn(q.view(np.uint16), [N]).double().cpu().numpy()
    codes = np.repeat(levels == level, 64)[:T]
    for h in range(2):
        kh, vh = ocache.UnitCache(ks[0, h], vs[0, h], levels).khat_vhat()
        o, square = expected(q[:, h].astype(np.float64), kh, vh, codes)
        assert np.linalg.norm(out[:, h] - o) <= 1.25 * square ** 0.5, (np.linalg.norm(out[:, h] - o) / square ** 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [0x7C00, 0x7E00, 0xFC00])
def test_infinite_key_scales(gpu, bits):
    """An infinite or NaN scale of one block's keys shows in its own KV head alone."""
    import torch
    ks, vs, q = data(1, 2, 4)
    cache = gpu.GradedCache.build(ks, vs, Hq=2, levels=np.array([4] * 77 + [16] * 4, np.int8))
    want = cache.chunk_attn(q.view(np.uint16), [N])
    at = int(cache.koff_host[0, 0, 30]) + 2 * 17
    cache.arena[at:at + 2].view(torch.int16).fill_(bits - (bits >> 15 << 16))
    got = cache.chunk_attn(q.view(np.uint16), [N])
    assert torch.equal(got[:, 1], want[:, 1]) and not bool(torch.isfinite(got[:, 0]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("places", [(3,), (0,), (76,), (3, 4, 50)])
def test_few_integer_blocks(gpu, places):
    """Blocks of codes between exact and centroid ones, some of them in no sample."""
    ks, vs, q = data(7, 1, 4)
    levels = np.array([0, 1, 16] * 27, np.int8)
    levels[list(places)] = 8
    levels[-4:] = 16
    cache = gpu.GradedCache.build(ks, vs, Hq=1, levels=levels)
    out = cache.chunk_attn(q.view(np.uint16), [N]).double().cpu().numpy()
    kh, vh = ocache.UnitCache(ks[0, 0], vs[0, 0], levels).khat_vhat()
    codes = np.repeat(levels == 8, 64)[:T]
    o, bound = rows_and_bounds(q[:, 0].astype(np.float64), kh, vh, codes, codes)
    assert (np.linalg.norm(out[:, 0] - o, axis=1) / bound).max() <= 1.0


@pytest.mark.gpu
def test_captured_calls(gpu):
    """Two captured calls of many rows, replayed with new queries between eager calls of the same cache."""
    import torch
    ks, vs, q = data(11, 2, 4)
    cache = gpu.GradedCache.build(ks, vs, Hq=2, levels=np.array([2] * 20 + [4] * 30 + [8] * 27 + [16] * 4, np.int8))
    q = torch.from_numpy(q).cuda()
    outs, graphs = [torch.empty_like(q) for _ in range(2)], []
    cache.chunk_attn(q, [N])
    for out in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            cache.chunk_attn(q, [N], out=out)
    for _ in range(4):
        q.copy_(torch.roll(q, 1, 0))
        for g, out in zip(graphs, outs):
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        want = cache.chunk_attn(q, [N])
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
