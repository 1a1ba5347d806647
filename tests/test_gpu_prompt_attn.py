"""Causal attention over packed prompts against the definition in fp64.

Tolerance of an output element, with u half a rounding step of the type and A the row's
sum of weight x |value|: each weight is rounded once (u A), their sum adds the rounded ones
(u |out| more), the output is rounded once (u |out|); a logit is an fp32 sum of 128
products, off by at most 129 x 2^-24 of the sum of their magnitudes, and its exponent is
rounded twice more, which changes every weight by that much (2 E A, numerator and sum); fp16
weights below 2^-14 of the row's reference are off by up to 2^-25 each instead.  The hardware
exponential's error (under 2^-22) is counted with E."""
import numpy as np
import pytest

HALF_STEP = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def reference(q, k, v, lens):
    """fp64 outputs and tolerances of packed q [n][Hq][128], k, v [n][Hkv][128] tensors."""
    import torch
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    u = HALF_STEP[str(q.dtype).split(".")[1]]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    at = 0
    for t in lens:
        if not t:
            continue
        hidden = torch.ones(t, t, dtype=torch.bool).triu(1)
        for g in range(Hq):
            qs, ks, vs = q[at:at + t, g], k[at:at + t, g // G], v[at:at + t, g // G]
            x = (qs @ ks.T / D ** 0.5).masked_fill(hidden, -float("inf"))
            # a masked token has no effect, whatever it holds: rows are formed one weight at a time
            w = torch.softmax(x, -1)
            bad = ~torch.isfinite(vs).all(-1)
            good = torch.where(bad[:, None], 0.0, vs)
            o = w @ good
            a = w @ good.abs()
            for j in torch.nonzero(bad)[:, 0].tolist():
                o[j:] += w[j:, j:j + 1] * vs[j]
            mag = (qs.abs() @ torch.where(torch.isfinite(ks), ks, 0.0).abs().T).masked_fill(hidden, 0.0).amax(-1)
            top = torch.where(torch.isfinite(x), x, 0.0).abs().amax(-1)
            e = 129 * 2.0 ** -24 * mag / D ** 0.5 + 4 * top * 2.0 ** -24 + 2.0 ** -22
            small = 2.0 ** -25 * t * good.abs().amax() if u == 2.0 ** -11 else 0.0
            out[at:at + t, g] = o
            sums = 2 * t * 2.0 ** -24  # fp32 sums over the tokens, of the products and of the weights
            tol[at:at + t, g] = (u + sums + 2 * e[:, None]) * a + 2 * u * o.abs() + small + 1e-6
        at += t
    return out, tol


def make(seed, lens, Hq, Hkv, dtype):
    import torch
    g = torch.Generator().manual_seed(seed)
    n = int(sum(lens))
    t = getattr(torch, dtype)
    q, k, v = (torch.randn(n, h, 128, generator=g) for h in (Hq, Hkv, Hkv))
    k[..., torch.randperm(128, generator=g)[:4]] *= 10.0
    return [x.to(t) for x in (q, k, v)]


def check(out, q, k, v, lens):
    import torch
    want, tol = reference(q, k, v, lens)
    got = out.double().cpu()
    assert out.dtype == q.dtype and got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    fine = torch.isfinite(want)
    worst = ((got - want).abs() / tol)[fine]
    assert not worst.numel() or float(worst.max()) <= 1.0, float(worst.max())


LENS = [[1], [2], [63], [64], [65], [255, 1, 0, 130], [0, 0, 7], [300], [1] * 40, [129, 511, 64, 3]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (7, 1), (6, 6), (16, 1), (20, 4)])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_prompts_match_the_definition(gpu, lens, Hq, Hkv, dtype):
    q, k, v = make(len(lens) + lens[0], lens, Hq, Hkv, dtype)
    out = gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), lens)
    check(out, q, k, v, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 2049), (3, 3, 1500), (16, 1, 1100)])
def test_long_prompts(gpu, Hq, Hkv, T):
    q, k, v = make(5, [T, 17], Hq, Hkv, "float16")
    check(gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), [T, 17]), q, k, v, [T, 17])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_slices_of_one_projection_are_read_in_place(gpu, dtype):
    import torch
    lens, Hq, Hkv = [70, 33], 8, 2
    q, k, v = make(9, lens, Hq, Hkv, dtype)
    fused = torch.cat([q.view(103, -1), k.view(103, -1), v.view(103, -1)], 1).cuda()
    parts = [x.unflatten(1, (-1, 128)) for x in fused.split([Hq * 128, Hkv * 128, Hkv * 128], 1)]
    wide = torch.full((103, Hq + 1, 128), 7.0, dtype=q.dtype, device="cuda")
    out = gpu.prompt_attn(*parts, lens, out=wide[:, :Hq])
    assert out.data_ptr() == wide.data_ptr() and bool((wide[:, Hq] == 7.0).all())
    check(out, q, k, v, lens)
    assert torch.equal(out, gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), lens))
    # other orders and alignments are copied
    odd = torch.zeros(103 * Hkv * 128 + 3, dtype=q.dtype, device="cuda")
    odd[3:] = k.cuda().reshape(-1)
    assert torch.equal(out, gpu.prompt_attn(parts[0].transpose(0, 1).contiguous().transpose(0, 1),
                                            odd[3:].view(103, Hkv, 128), parts[2], lens))


@pytest.mark.gpu
def test_bit_patterns_are_fp16(gpu):
    import torch
    q, k, v = make(3, [50], 4, 2, "float16")
    want = gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), [50])
    assert torch.equal(want, gpu.prompt_attn(*(x.cuda().view(torch.int16) for x in (q, k, v)), [50]))
    assert torch.equal(want, gpu.prompt_attn(*(x.numpy().view(np.uint16) for x in (q, k, v)), [50]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_masked_tokens_have_no_effect(gpu, what, value, dtype):
    """Rows before an infinite or NaN token, and every other prompt, are as without it."""
    import torch
    lens, Hq, Hkv = [90, 40, 200], 8, 2
    q, k, v = make(11, lens, Hq, Hkv, dtype)
    clean = gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), lens)
    bad = 90 + 23
    x = k if what == "k" else v
    x[bad, 0, 5] = value
    x[90 + 40 + 199, 1, 77] = value  # the last token of the last prompt
    out = gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), lens)
    same = torch.ones(330, Hq, dtype=torch.bool)
    same[bad:130, :4] = False
    same[329, 4:] = False
    assert torch.equal(out.cpu()[same], clean.cpu()[same])
    if what == "v":
        check(out, q, k, v, lens)
    elif value != value:
        assert bool(torch.isnan(out.cpu()[~same]).all())


@pytest.mark.gpu
def test_large_logits_and_rising_maxima(gpu):
    """Scores that rise by more than the rescale step from tile to tile, and rows whose
    scores are all far below zero."""
    import torch
    T = 400
    q, k, v = make(13, [T], 4, 1, "float16")
    q[:, 0] = 1.0
    k[:, 0] = (torch.arange(T)[:, None] * 0.02 - 4.0).half()
    q[:, 1] = -1.0
    q[:, 2] = 4.0
    k[:, 0, 7] = -100.0
    check(gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), [T]), q, k, v, [T])


@pytest.mark.gpu
def test_offsets_past_32_bits(gpu):
    """Rows 2^20 elements apart: the last ones lie past 4 GiB."""
    import torch
    T, S = 2200, 1 << 20
    q, k, v = make(17, [T], 2, 1, "float16")
    big = torch.empty((T - 1) * S + 4 * 128, dtype=torch.float16, device="cuda")
    views = [big[lo:lo + (T - 1) * S + h * 128].as_strided((T, h, 128), (S, 128, 1)) for lo, h in ((0, 2), (256, 1), (384, 1))]
    for x, y in zip(views, (q, k, v)):
        x.copy_(y.cuda())
    want = gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), [T])
    assert torch.equal(want, gpu.prompt_attn(*views, [T]))
    check(want, q, k, v, [T])


@pytest.mark.gpu
def test_streams_and_graphs(gpu):
    import torch
    lens = [77, 300]
    q, k, v = (x.cuda() for x in make(19, lens, 8, 2, "float16"))
    want = gpu.prompt_attn(q, k, v, lens)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = gpu.prompt_attn(q, k, v, lens)
    s.synchronize()
    assert torch.equal(want, other)
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gpu.prompt_attn(q, k, v, lens, out=out)
    for i in range(3):
        q.copy_(torch.roll(q, 1, 0))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, gpu.prompt_attn(q, k, v, lens))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("odd", [False, True])
def test_both_widths_of_a_workgroup(gpu, dtype, odd):
    """Long prompts together (row tiles of 256) and one by one (of 128): the same outputs, also where
    tokens hold infinities and NaN."""
    import torch
    lens = [2000, 1777, 1, 64, 1999]
    q, k, v = (x.cuda() for x in make(29, lens, 32, 8, dtype))
    if odd:
        for i, (at, x) in enumerate(((1900, float("inf")), (1950, float("nan")), (2000 + 1700, -float("inf")),
                                     (2000 + 1776, float("nan")))):
            (v if i % 2 == 0 else k)[at, i, 5 * i] = x
    got, at = gpu.prompt_attn(q, k, v, lens), 0
    for n in lens:
        one = gpu.prompt_attn(q[at:at + n], k[at:at + n], v[at:at + n], [n])
        same = (got[at:at + n] == one) | (got[at:at + n].isnan() & one.isnan())
        assert bool(same.all())
        assert odd or not bool(one.isnan().any())
        at += n


def _call(B, dtype=0, Hkv=2, Hq=4, lens=(5, 3), strides=None, ptr=4096, null=None):
    import ctypes
    lens = np.array(lens, dtype=np.int64)
    strides = strides or (Hq * 128, Hkv * 128, Hkv * 128, Hq * 128)
    p = [ptr if i != null else None for i in range(4)]
    return B._prompt_attn(*p, dtype, Hkv, Hq, len(lens), ctypes.c_void_p(lens.ctypes.data), *strides, None)


def test_refusals():
    """Checked on the host before anything is enqueued (no GPU here)."""
    from paper_2608_23599_amd import binding as B
    assert _call(B, lens=()) == 0 and _call(B, lens=(0, 0), ptr=None) == 0  # nothing to do
    assert _call(B, dtype=2) == -1
    assert _call(B, Hq=5) == -2 and _call(B, Hkv=0) == -2 and _call(B, Hkv=1, Hq=17) == -2
    assert _call(B, lens=(5, -1)) == -2
    for i in range(4):
        assert _call(B, null=i) == -1
        s = [512, 256, 256, 512]
        s[i] -= 8
        assert _call(B, strides=s) == -2
        s[i] += 12
        assert _call(B, strides=s) == -1
        s[i] = (1 << 20) + 8
        assert _call(B, strides=s) == -6
    assert _call(B, ptr=4104) == -1
    assert _call(B, lens=(1,) * 257) == -6
    assert _call(B, lens=(100000000, 1)) == -6
    assert _call(B, Hkv=64, Hq=64, lens=(100000000,)) == -6  # more threads than a launch takes


def test_binding_refusals():
    """Shapes and types that do not fit, before anything reaches a device."""
    import torch
    from paper_2608_23599_amd import binding as B
    with pytest.raises(B.GkvError):
        B._rows_dev(torch.zeros(3, 4, 64, dtype=torch.float16), "prompt_attn")
    with pytest.raises(B.GkvError):
        B._rows_dev(torch.zeros(3, 4, 128), "prompt_attn")


@pytest.mark.gpu
def test_binding_refuses_what_does_not_fit(gpu):
    import torch
    q, k, v = (x.cuda() for x in make(23, [9], 4, 2, "float16"))
    for bad in ((q, k, v, [8]), (q, k, v[:8], [9]), (q, k, v.bfloat16(), [9]), (q, k[:, :1], v, [9])):
        with pytest.raises(gpu.GkvError):
            gpu.prompt_attn(*bad)
    with pytest.raises(gpu.GkvError):
        gpu.prompt_attn(q, k, v, [9], out=torch.empty_like(q, dtype=torch.float32))
    assert gpu.prompt_attn(q[:0], k[:0], v[:0], []).shape == (0, 4, 128)
