"""Tokens that residual rows override: what their graded entries hold has no effect, in the form for
few rows and in the one for many."""
import numpy as np
import pytest

from oracle import cache as ocache, fp16 as ofp16
from tests._util import kv_all
from tests.test_gpu_chunk import rows_reference

T, EXACT_BLOCKS = 64 * 12, 3


def build(gpu, ks, vs, levels, kept, vtok):
    """A cache of one sequence with the tokens of `kept` (ascending) as residual rows."""
    H = ks.shape[1]
    cache = gpu.GradedCache.build(ks, vs, Hq=2 * H, levels=np.array(levels, np.int8), nres_cap=len(kept), v_per_token=vtok)
    mass = np.zeros((1, H, T), np.float32)
    mass[..., kept] = 1.0
    cache.rd_residual_select(ks, vs, mass, len(kept))
    assert cache.res_idx[0, 0].cpu().tolist() == list(kept)
    return cache


def queries(n, heads):
    return np.random.default_rng(3).standard_normal((n, heads, 128)).astype(np.float16).view(np.uint16)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 150])
@pytest.mark.parametrize("bits", [8, 4, 2])
def test_entries_past_fp16(gpu, n, bits):
    """An overridden token whose scale per token takes its entries past the largest fp16 number (8 bits:
    255 * 257 = 65535; 4 bits: 15 * 4368 = 65520; 2 bits: 3 * 21840 = 65520)."""
    ks, vs = kv_all(91, 1, 2, T)
    kept = [64 * 4 + 9, 64 * 4 + 40]
    for t in kept:
        vs[0, :, t] = ofp16.from_f64(np.linspace(0.0, 65504.0, 128))
    levels = [bits] * 9 + [16] * EXACT_BLOCKS
    q = queries(n, 4)
    out = build(gpu, ks, vs, levels, kept, True).chunk_attn(q, [n]).double().cpu().numpy()
    for h in range(2):
        u = ocache.UnitCache(ks[0, h], vs[0, h], levels, v_per_token=True)
        kh, vh = u.khat_vhat()
        assert (vh[kept].max(1) >= 65520).all()
        kh[kept], vh[kept] = ofp16.to_f64(ks[0, h, kept]), ofp16.to_f64(vs[0, h, kept])
        exact = np.repeat(np.array(levels) == 16, 64)
        exact[kept] = True
        for g in (2 * h, 2 * h + 1):
            ref, tol = rows_reference(q[:, g], kh, vh, range(T - n, T), exact)
            worst = np.abs(out[:, g] - ref) / tol
            assert worst.max() <= 1.0, (g, worst.max())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 150])
@pytest.mark.parametrize("bits", [0x7C00, 0xFC00, 0x7E00])
@pytest.mark.parametrize("level,vtok", [(0, False), (1, False), (8, True), (4, True), (2, True),
                                        (8, False), (4, False), (2, False)])
def test_infinite_and_nan_entries(gpu, level, vtok, bits, n):
    """A block or (with scales per token) a token whose record is infinite or NaN, all of
    whose tokens are residual rows: the outputs are those of the record as it was."""
    import torch
    ks, vs = kv_all(93, 1, 1, T)
    # four clusters of 16 values, so that no token is a centroid itself (one without error is not kept)
    x = ofp16.to_f64(vs[0, 0, 64 * 4:64 * 5])
    vs[0, 0, 64 * 4:64 * 5] = ofp16.from_f64(np.repeat(x[::16], 16, 0) + 0.1 * x)
    kept = [64 * 4 + 9] if vtok else list(range(64 * 4, 64 * 5))
    cache = build(gpu, ks, vs, [level] * 9 + [16] * EXACT_BLOCKS, kept, vtok)
    q = queries(n, 2)
    want = cache.chunk_attn(q, [n])
    # the mean's channel 9; the four centroids' channel 9; the token's scale; channel 9's scale
    first, count = (9, 1) if level == 0 or vtok else (9 * 8 * 4, 4) if level == 1 else (65, 1)
    at = int(cache.voff_host[0, 0, 4]) + 2 * first
    cache.arena[at:at + 2 * count].view(torch.int16).fill_(bits - (bits >> 15 << 16))
    assert bool(torch.isfinite(want).all()) and torch.equal(cache.chunk_attn(q, [n]), want)
