"""Graded keys and values next to the largest fp16 number, whose codes stand for up to 65535: the outputs
are finite and as the definition's, in both forms.  (A form that rounds such an entry to fp16 takes 65504:
31 of 65535 away, less than the half step that the tolerance has for every graded entry.)"""
import numpy as np
import pytest

from oracle import cache as ocache, fp16 as ofp16
from tests._util import kv_all
from tests.test_gpu_chunk import rows_reference

T = 64 * 12


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 150])
@pytest.mark.parametrize("bits", [8, 4, 2])
@pytest.mark.parametrize("what", ["keys", "values", "values per token"])
def test_entries_at_the_top(gpu, what, bits, n):
    ks, vs = kv_all(95, 1, 1, T)
    r = np.random.default_rng(bits)
    block = slice(64 * 4, 64 * 5)
    q = r.standard_normal((n, 2, 128)).astype(np.float16)
    if what == "values per token":
        vs[0, 0, block] = ofp16.from_f64(r.permuted(np.tile(np.linspace(0.0, 65504.0, 128), (64, 1)), axis=1))
    else:
        x = ks if what == "keys" else vs
        x[0, 0, block, 9] = ofp16.from_f64(r.permuted(np.linspace(0.0, 65504.0, 64)))
        if what == "keys":  # scores within some units of the others'
            q[:, :, 9] = 2.0 ** -13
    levels = [bits] * 9 + [16] * 3
    vtok = what == "values per token"
    u = ocache.UnitCache(ks[0, 0], vs[0, 0], levels, v_per_token=vtok)
    kh, vh = u.khat_vhat()
    assert 65520 <= (kh if what == "keys" else vh)[block].max() <= 65535
    cache = gpu.GradedCache.build(ks, vs, Hq=2, levels=np.array(levels, np.int8), v_per_token=vtok)
    out = cache.chunk_attn(q.view(np.uint16), [n]).double().cpu().numpy()
    exact = np.repeat(np.array(levels) == 16, 64)
    for g in range(2):
        ref, tol = rows_reference(q[:, g].view(np.uint16), kh, vh, range(T - n, T), exact)
        worst = np.abs(out[:, g] - ref) / tol
        assert worst.max() <= 1.0, (g, worst.max())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 150])
@pytest.mark.parametrize("vtok", [False, True])
@pytest.mark.parametrize("bits", [0x7C00, 0xFC00, 0x7E00])
def test_infinite_scales_stay(gpu, bits, vtok, n):
    """An infinite or NaN scale is not hidden: the channel (or token) it scales shows in every row."""
    import torch
    ks, vs = kv_all(97, 1, 1, T)
    cache = gpu.GradedCache.build(ks, vs, Hq=2, levels=np.array([8] * 9 + [16] * 3, np.int8), v_per_token=vtok)
    q = np.random.default_rng(1).standard_normal((n, 2, 128)).astype(np.float16).view(np.uint16)
    want = cache.chunk_attn(q, [n])
    at = int(cache.voff_host[0, 0, 4]) + 2 * (9 if vtok else 65)  # token 9's scale, or channel 9's
    cache.arena[at:at + 2].view(torch.int16).fill_(bits - (bits >> 15 << 16))
    got = cache.chunk_attn(q, [n])
    other = torch.arange(128) != 9
    if vtok:
        assert not bool(torch.isfinite(got).any())
    else:
        assert not bool(torch.isfinite(got[..., 9]).any()) and torch.equal(got[..., other], want[..., other])
