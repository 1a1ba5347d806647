"""chunk_attn and prompt_attn row by row: the whole of a row's error against the definition, where the elementwise bounds
of worst cases are wide.

Of a row, the 128 channels' errors together (2-norm) are at most R = 2 u S, u = 2^-11 (half a step of
fp16, 2^-8 for bf16 prompts), with S^2 the sum of what independent roundings of one u each would make:
  |o|^2                     the output's,
  sum_t w_t^2 |v_t - o|^2   the weights' (their sum adds the rounded ones),
  sum_t w_t^2 |v_t|^2       the decoded values', and
  sum_t w_t^2 |v_t - o|^2 s_t^2, s_t^2 = sum_d (q_d k_td)^2 / 128, the decoded keys' by way of the scores,
the last two where the form rounds them (graded blocks: where many rows attend; values with scales
per token in both).  A rounding's root mean square is u / sqrt(3) at most, so that R
is 3.5 times what independent ones make: that is for codes of one channel that round alike, and for rows
of which one token has most of the weight.  A score is an fp32 sum of
129 terms; with independent roundings it is off by sqrt(129) x 2^-24 of their sizes' sum, which counts as a
rounding of the key does."""
import numpy as np
import pytest

from oracle import cache as ocache, fp16 as ofp16, ladder as olad
from tests._util import kv_all
from tests.test_gpu_chunk import Case, mixed_levels

U = 2.0 ** -11


def softmax_rows(q, kh, seen):
    """Weights [n][T] of fp64 rows; seen [n][T] truth values."""
    x = np.where(seen, q @ kh.T / np.sqrt(128.0), -np.inf)
    w = np.exp(x - x.max(1, keepdims=True))
    return w / w.sum(1, keepdims=True)


def causal(T, n):
    return np.arange(T)[None, :] <= np.arange(T - n, T)[:, None]


def rows_and_bounds(q, kh, vh, keys_rounded, values_rounded, u=U):
    """Outputs [n][128] of the newest n rows and the bound R of each; *_rounded: [T] truth values, u: half
    a step of the weights and outputs."""
    T, n = kh.shape[0], q.shape[0]
    w = softmax_rows(q, kh, causal(T, n))
    o = w @ vh
    w2, v2 = w * w, (vh * vh).sum(1)
    off = v2[None, :] - 2 * o @ vh.T + (o * o).sum(1)[:, None]  # |v_t - o|^2
    s2 = (q * q) @ (kh * kh).T / 128
    var = (o * o).sum(1) + (w2 * (off * (1 + s2 * keys_rounded) + v2 * values_rounded)).sum(1)
    size = np.abs(q) @ np.abs(kh).T / np.sqrt(128.0)
    var += (w2 * off * (129 ** 0.5 * 2.0 ** -24 / u * size) ** 2).sum(1)
    return o, 2 * u * np.sqrt(var) + 2.0 ** -25 * np.sqrt(128)


def ratio(got, o, bound):
    return np.linalg.norm(got - o, axis=1) / bound


def check(case, out, pick=None):
    """out against the definition over the oracle's records; pick: the newest rows that attend."""
    got = out.double().cpu().numpy()
    at, worst = 0, 0.0
    for b, (t, n) in enumerate(zip(case.lens, case.news)):
        m = n if pick is None else pick[b]
        for h in range(case.Hkv if m else 0):
            e = case.end[b]
            kh, vh = ofp16.to_f64(case.ks[b, h, :e]), ofp16.to_f64(case.vs[b, h, :e])
            graded = np.zeros(e, bool)
            codes = np.zeros(e, bool)
            if t > 0:
                u = case.units[b, h]
                kh[:t], vh[:t] = u.khat_vhat()
                lv = np.repeat(np.asarray(u.levels), 64)[:t]
                codes[:t] = (lv == 8) | (lv == 4) | (lv == 2)
                codes[u.res_idx] = False
            if m * case.G > 128:
                graded = codes
            vtok = t > 0 and case.units[b, h].v_per_token
            for g in range(h * case.G, (h + 1) * case.G):
                q = ofp16.to_f64(case.queries(b, m)[:, g])
                r = ratio(got[at:at + m, g], *rows_and_bounds(q, kh, vh, graded, codes if vtok else graded))
                assert r.max() <= 1.0, (b, g, r.max())
                worst = max(worst, r.max())
        at += m
    assert at == got.shape[0]
    return worst


@pytest.mark.gpu
@pytest.mark.parametrize("vtok", [False, True])
@pytest.mark.parametrize("prof,T,n", [("graded", 64 * 70 + 9, 90), ("graded", 64 * 120, 1), ("graded", 64 * 120, 40),
                                      ("rdv2", 64 * 60 + 1, 20), ("tiny", 64 * 40, 33), (mixed_levels, 64 * 90 + 63, 5),
                                      ("exact", 64 * 100 + 1, 3), ("exact", 64 * 100 + 1, 200)])
def test_long_contexts(gpu, prof, T, n, vtok):
    c = Case(gpu, 53, (T, 200), (n, 1), 8, 2, prof, vtok=vtok)
    check(c, c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,n", [(1, 1), (1, 17), (7, 3), (5, 13), (16, 8), (16, 9), (4, 100)])
@pytest.mark.parametrize("nres", [0, 70])
def test_mixed_levels(gpu, Hq, n, nres):
    T = 64 * 40 + 5
    c = Case(gpu, 73, (T,), (n,), Hq, 1, mixed_levels, nres=nres, ragged=False)
    check(c, c.run())


@pytest.mark.gpu
def test_many_sequences(gpu):
    r = np.random.default_rng(87)
    lens, news = r.integers(0, 1500, 40), r.choice([0, 1, 2, 7, 150], 40, p=[0.2, 0.3, 0.2, 0.2, 0.1])
    lens[:3], news[:3] = (0, 64 * 70, -1), (0, 150, 0)
    c = Case(gpu, 87, lens, news, 4, 2, "tiny")
    check(c, c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("lens,Hq,Hkv", [([2049, 17, 300], 8, 2), ([1], 3, 3), ([64, 65, 1100], 7, 1)])
def test_prompts(gpu, lens, Hq, Hkv, dtype):
    import torch
    g = torch.Generator().manual_seed(sum(lens))
    q, k, v = (torch.randn(sum(lens), h, 128, generator=g).to(getattr(torch, dtype)) for h in (Hq, Hkv, Hkv))
    out = gpu.prompt_attn(q.cuda(), k.cuda(), v.cuda(), lens).double().cpu().numpy()
    q, k, v = (x.double().numpy() for x in (q, k, v))
    at = 0
    for t in lens:
        own = slice(at, at + t)
        none = np.zeros(t, bool)
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            r = ratio(out[own, h], *rows_and_bounds(q[own, h], k[own, kv], v[own, kv], none, none,
                                                    U if dtype == "float16" else 2.0 ** -8))
            assert r.max() <= 1.0, (t, h, r.max())
        at += t


# ---------------------------------------------------------------- what the check sees (host only)
def emulate(q, kh, vh, seen, keys_rounded, values_rounded):
    """The outputs with every rounding the kernels make, of one pass over the context."""
    f16 = lambda x: np.asarray(x, np.float16).astype(np.float64)
    kh = np.where(keys_rounded[:, None], f16(kh), kh)
    vh = np.where(values_rounded[:, None], f16(vh), vh)
    x = np.where(seen, q @ kh.T / np.sqrt(128.0), -np.inf)
    w = f16(np.exp(x - x.max(1, keepdims=True)) * 2.0 ** 7)
    return f16(w @ vh / w.sum(1, keepdims=True))


@pytest.mark.parametrize("prof,T,n,many", [("graded", 64 * 120, 1, False), ("graded", 64 * 70 + 9, 90, False),
                                           ("graded", 64 * 70 + 9, 90, True), (mixed_levels, 64 * 40 + 5, 5, False),
                                           (mixed_levels, 64 * 40 + 5, 150, True), ("rdv2", 64 * 60 + 1, 20, False)])
def test_the_check_sees_lost_and_extra_tokens(prof, T, n, many):
    """The kernels' roundings pass; a block left out, a share of 16 left out of the join, a row's own
    token missing and the next one's visible do not."""
    ks, vs = kv_all(53, 1, 1, T + 1)
    lv = prof(T) if callable(prof) else olad.ladder(prof, T)
    u = ocache.UnitCache(ks[0, 0, :T], vs[0, 0, :T], lv)
    kh, vh = u.khat_vhat()
    codes = np.isin(np.repeat(lv, 64)[:T], (8, 4, 2))
    graded = codes if many else np.zeros(T, bool)
    seen, tokens = causal(T, n), np.arange(T)
    blocks = -(-T // 64)
    lost = [seen & (tokens // 64 != i) for i in (0, blocks // 2, blocks - 3)]
    lost.append(seen & (tokens // 64 * 16 // blocks != 5))
    lost.append(seen & (tokens[None, :] != np.arange(T - n, T)[:, None]))
    k1, v1 = np.concatenate([kh, ofp16.to_f64(ks[0, 0, T:])]), np.concatenate([vh, ofp16.to_f64(vs[0, 0, T:])])
    later = np.arange(T + 1)[None, :] <= np.arange(T - n, T)[:, None] + 1
    worst = np.zeros(len(lost) + 1)
    for head in range(8):  # (one head's weight of a token may be next to nothing)
        q = np.random.default_rng(head).standard_normal((n, 128)).astype(np.float16).astype(np.float64)
        o, bound = rows_and_bounds(q, kh, vh, graded, graded)
        assert ratio(emulate(q, kh, vh, seen, graded, graded), o, bound).max() <= 1.0
        wrong = [softmax_rows(q, kh, s) @ vh for s in lost] + [softmax_rows(q, k1, later) @ v1]
        worst = np.maximum(worst, [ratio(x, o, bound).max() for x in wrong])
    assert worst.min() > 1.0, worst
