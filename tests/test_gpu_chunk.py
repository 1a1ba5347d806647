"""Chunks of new tokens: append_chunk against as many single appends (bit for bit), truncate,
and chunk_attn against the definition in fp64 over the oracle's decoded records.

Tolerance of an output element of chunk_attn, with u = 2^-11 (half a step of fp16) and A the row's
sum of weight x |value|: a graded key is rounded to fp16 once, which moves a logit by at
most u sum |q_d k_d| / sqrt(128), and its fp32 sum is off by 129 x 2^-24 of the same sum;
both change every weight by that much (2 E A, numerator and sum); a graded value and a
weight are rounded once each (2 u A), the sum adds rounded weights and the output is rounded
(2 u |out|); weights below 2^-14 are off by up to 2^-25 each."""
import numpy as np
import pytest

from oracle import cache as ocache, fp16 as ofp16, ladder as olad
from paper_2608_23599_amd import synth
from tests._util import kv_all

U = 2.0 ** -11


def rows_reference(q, kh, vh, pos, exact_rows):
    """q [n][128], kh, vh [T][128] fp64, row i sees tokens 0..pos[i]: (outputs, tolerances).
    exact_rows: tokens that are read without rounding."""
    q = ofp16.to_f64(q)
    T = kh.shape[0]
    x = q @ kh.T / np.sqrt(128.0)
    x[np.arange(T)[None, :] > np.asarray(pos)[:, None]] = -np.inf
    w = np.exp(x - x.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    mag = np.abs(q) @ np.abs(kh).T / np.sqrt(128.0)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(1)
    unit = np.where(exact_rows, 0.0, U) + 129 * 2.0 ** -24
    e = (mag * unit * (x > -np.inf)).max(1) + 4 * top * 2.0 ** -24 + 2.0 ** -22
    out, a = w @ vh, w @ np.abs(vh)
    tol = (2 * U + 2 * T * 2.0 ** -24 + 2 * e[:, None]) * a + 2 * U * np.abs(out) + 2.0 ** -25 * T * np.abs(vh).max() + 1e-6
    return out, tol


def level_table(lens, Hkv, prof):
    lv = np.full((len(lens), Hkv, max(1, -(-max(lens) // 64))), 16, np.int8)
    for b, t in enumerate(lens):
        if t > 0:
            own = prof(t) if callable(prof) else olad.ladder(prof, t)
            lv[b, :, :len(own)] = own
    return lv


def mixed_levels(T):
    """All six levels in turn, the last three blocks exact."""
    n = -(-T // 64)
    lv = np.array([[0, 1, 2, 4, 8, 16][i % 6] for i in range(n)], np.int8)
    lv[-3:] = 16
    return lv


class Case:
    """A cache of lens tokens and the rows that are appended to it."""

    def __init__(self, gpu, seed, lens, news, Hq, Hkv, prof="tiny", page=0, vtok=False, nres=0, ragged=True, slack=0,
                 scale=1.0):
        self.lens, self.news, self.Hq, self.Hkv, self.G = list(lens), list(news), Hq, Hkv, Hq // Hkv
        B, T = len(lens), max(1, max(lens))
        self.end = [max(t, 0) + n for t, n in zip(lens, news)]
        self.ks, self.vs = kv_all(seed, B, Hkv, max(self.end))
        if scale != 1.0:
            self.ks, self.vs = (ofp16.from_f64(ofp16.to_f64(x) * scale) for x in (self.ks, self.vs))
        lv = level_table(lens, Hkv, prof)
        opened = sum(-(-e // 64) - -(-max(t, 0) // 64) for e, t in zip(self.end, lens)) * Hkv
        self.cache = gpu.GradedCache.build(
            np.ascontiguousarray(self.ks[:, :, :T]), np.ascontiguousarray(self.vs[:, :, :T]), Hq=Hq, levels=lv,
            page=page, nres_cap=nres, extra_blocks=-(-max(self.end) // 64) - -(-T // 64), slack={16: opened + slack},
            v_per_token=vtok, seq_lens=list(lens) if ragged else None)
        self.units = {}
        for b, t in enumerate(lens):
            for h in range(Hkv):
                if t > 0:
                    self.units[b, h] = ocache.UnitCache(self.ks[b, h, :t], self.vs[b, h, :t],
                                                        lv[b, h, :-(-t // 64)], v_per_token=vtok)
        if nres:
            mass = np.stack([[synth.mass_unit(seed, b, h, T) for h in range(Hkv)] for b in range(B)]).astype(np.float32)
            self.cache.rd_residual_select(self.ks[:, :, :T].copy(), self.vs[:, :, :T].copy(), mass, nres)
            for (b, h), u in self.units.items():
                u.select_residual(self.ks[b, h, :T], self.vs[b, h, :T], mass[b, h], nres)
        self.q = synth.rng(seed, 2, 9).standard_normal((sum(news), Hq, 128), dtype=np.float32).astype(np.float16)

    def new_rows(self):
        """Packed new keys and values [n][Hkv][128] (fp16 bits)."""
        pick = lambda x: np.concatenate([x[b, :, max(t, 0):max(t, 0) + n].transpose(1, 0, 2)
                                         for b, (t, n) in enumerate(zip(self.lens, self.news))])
        return np.ascontiguousarray(pick(self.ks)), np.ascontiguousarray(pick(self.vs))

    def append(self):
        self.cache.append_chunk(*self.new_rows(), self.news)

    def check(self, out, pick=None):
        """out against the definition; pick: the newest rows of each sequence that attend."""
        got = out.float().cpu().numpy().astype(np.float64)
        at = 0
        for b, (t, n) in enumerate(zip(self.lens, self.news)):
            m = n if pick is None else pick[b]
            for h in range(self.Hkv if m else 0):
                e = self.end[b]
                kh, vh = ofp16.to_f64(self.ks[b, h, :e]), ofp16.to_f64(self.vs[b, h, :e])
                exact = np.ones(e, bool)
                if t > 0:
                    kh[:t], vh[:t] = self.units[b, h].khat_vhat()
                    exact[:t] = np.repeat(np.asarray(self.units[b, h].levels) == 16, 64)[:t]
                    exact[self.units[b, h].res_idx] = True
                for g in range(h * self.G, (h + 1) * self.G):
                    ref, tol = rows_reference(self.queries(b, m)[:, g], kh, vh, range(e - m, e), exact)
                    worst = np.abs(got[at:at + m, g] - ref) / tol
                    assert worst.max() <= 1.0, (b, g, worst.max())
            at += m
        assert at == got.shape[0]

    def queries(self, b, m):
        lo = sum(self.news[:b + 1])
        return self.q[lo - m:lo].view(np.uint16)

    def run(self):
        self.append()
        return self.cache.chunk_attn(self.q.view(np.uint16), self.news)


# ---------------------------------------------------------------- append_chunk
@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 16, 32, 64])
@pytest.mark.parametrize("lens,news", [((1, 63, 64, 100), (3, 1, 1, 200)), ((0, -1, 130, 17), (70, 0, 0, 46)),
                                       ((61, 5), (2, 190)), ((64,), (53,))])
def test_append_chunk_equals_single_appends(gpu, lens, news, page):
    """The same records, tables, boxes, certificate numbers and lengths as one append per token
    (the sequences that still have tokens to append at a step, one at a time)."""
    import torch
    Hkv = 2
    a = Case(gpu, 31, lens, news, 4, Hkv, "exact", page=page)
    a.append()
    # single appends advance every active sequence: a cache of its own for each
    for s, (t, n) in enumerate(zip(lens, news)):
        assert int(a.cache.lengths()[s]) == int(a.cache.seq_len[s]) == (t + n if t >= 0 else -1)
        if t < 0:
            continue
        one = gpu.GradedCache(1, Hkv, 4, 0, 8, {16: 2 * Hkv * 8}, page=page, npage_cap=64 if page else 0, seq_lens=[0])
        for i in range(t + n):
            one.append(a.ks[s, :, i].copy(), a.vs[s, :, i].copy())
        for h in range(Hkv):
            for i in range(-(-(t + n) // 64)):
                assert int(a.cache.level[s, h, i]) == 16 == a.cache.level_host[s, h, i]
                assert int(a.cache.koff[s, h, i]) == a.cache.koff_host[s, h, i]
                assert int(a.cache.voff[s, h, i]) == a.cache.voff_host[s, h, i]
                for tensor in (0, 1):
                    assert a.cache.record_bytes(s, h, i, tensor) == one.record_bytes(0, h, i, tensor)
                if i * 64 >= t:
                    assert torch.equal(a.cache.cert[s, h, i], one.cert[0, h, i])
                else:  # the build's block encoder sums a row's squares in another order
                    assert torch.allclose(a.cache.cert[s, h, i], one.cert[0, h, i], rtol=2.0 ** -22, atol=0.0)
            if page:
                m = (t + n) // page
                for x, y in zip(a.cache.boxes_host(s, h, m), one.boxes_host(0, h, m)):
                    assert np.array_equal(x, y)


@pytest.mark.gpu
def test_append_chunk_from_a_strided_projection(gpu):
    import torch
    c, d = (Case(gpu, 33, (5, 60), (90, 7), 4, 2, "exact") for _ in range(2))
    k, v = (torch.from_numpy(x.view(np.int16)).view(torch.float16) for x in c.new_rows())
    fused = torch.cat([torch.zeros(97, 512, dtype=torch.float16), k.flatten(1), v.flatten(1)], 1).cuda()
    c.cache.append_chunk(fused[:, 512:768].unflatten(1, (2, 128)), fused[:, 768:].unflatten(1, (2, 128)), c.news)
    d.append()
    assert torch.equal(c.cache.arena, d.cache.arena)


@pytest.mark.gpu
def test_fragmented_slots_take_several_launches(gpu):
    """Slots in shuffled order make a run each: the tables and records are the same."""
    import ctypes
    import torch
    c = Case(gpu, 35, (10,), (64 * 70,), 2, 2, "exact")
    n = 70 * 2
    kv = c.cache.pool.alloc_many(16, 2 * n)
    order = np.random.default_rng(1).permutation(2 * n)
    nk, nv = kv[order[:n]].copy(), kv[order[n:]].copy()
    k, v = (torch.from_numpy(x.view(np.int16)).cuda() for x in c.new_rows())
    lens = np.array(c.news, np.int32)
    p = lambda a: ctypes.c_void_p(a.ctypes.data)
    assert gpu._append_chunk(ctypes.byref(c.cache.c), k.data_ptr(), v.data_ptr(), 256, 256, p(lens), p(nk), p(nv), n,
                             gpu._stream()) == 0
    c.cache.koff_host[0, :, 1:] = nk.reshape(2, 70)
    c.cache.voff_host[0, :, 1:] = nv.reshape(2, 70)
    assert np.array_equal(c.cache.koff.cpu().numpy(), c.cache.koff_host)
    assert np.array_equal(c.cache.voff.cpu().numpy(), c.cache.voff_host)
    for h in range(2):
        for i in (0, 1, 23, 24, 25, 48, 69):
            got = c.cache.record(0, h, i, 0)["values"]
            assert np.array_equal(got, ofp16.to_f64(c.ks[0, h, 64 * i:64 * i + 64])), i
            assert np.array_equal(c.cache.record(0, h, i, 1)["values"], ofp16.to_f64(c.vs[0, h, 64 * i:64 * i + 64]))


@pytest.mark.gpu
def test_append_chunk_with_a_ladder_demotes(gpu):
    c = Case(gpu, 37, (100,), (64 * 9,), 2, 1, "tiny")
    d = Case(gpu, 37, (100,), (64 * 9,), 2, 1, "tiny")
    c.cache.pool = c.cache.pool  # the pool of the build has slots for exact blocks only
    with pytest.raises(gpu.GkvError):
        c.cache.append_chunk(*c.new_rows(), c.news, profile="tiny")
    T = 676
    big = gpu.GradedCache(1, 1, 2, 0, 16, {16: 40, 8: 40, 4: 40, 2: 40}, seq_lens=[0])
    big.append_chunk(d.ks[0, :, :T].transpose(1, 0, 2).copy(), d.vs[0, :, :T].transpose(1, 0, 2).copy(), [T],
                     profile="tiny")
    assert np.array_equal(big.level_host[0, 0, :11], olad.ladder("tiny", T))


# ---------------------------------------------------------------- truncate
@pytest.mark.gpu
@pytest.mark.parametrize("lens,news,keep", [((70, 5, 130), (10, 70, 200), (70, 5, 130)),
                                            ((70, -1, 130), (60, 0, 1), (3, -1, 131)),
                                            ((64, 129), (1, 63), (64, 128)), ((5,), (300,), (0,))])
def test_truncate_gives_back_what_was_appended(gpu, lens, news, keep):
    import torch
    c = Case(gpu, 41, lens, news, 4, 2, "exact", page=16)
    used = c.cache.pool.used(16)
    c.append()
    first = c.cache.koff_host.copy(), c.cache.voff_host.copy()
    c.cache.truncate(keep)
    assert c.cache.lengths().tolist() == [k if t >= 0 else -1 for k, t in zip(keep, lens)]
    assert c.cache.seq_len.tolist() == c.cache.lengths().tolist()
    assert c.cache.T == max(max(keep), 0)
    assert c.cache.pool.used(16) == used + sum(
        4 * (-(-k // 64) - -(-t // 64)) for k, t in zip(keep, lens) if t >= 0)
    for b, k in enumerate(keep):
        if k > 0 and k % 64:
            for h in range(2):
                rec = c.cache.record(b, h, k // 64, 0)["values"], c.cache.record(b, h, k // 64, 1)["values"]
                for x, src in zip(rec, (c.ks, c.vs)):
                    assert np.array_equal(x[:k % 64], ofp16.to_f64(src[b, h, k - k % 64:k]))
                    assert not x[k % 64:].any()
    if list(keep) == list(lens):  # the same tokens again take the same slots
        before = c.cache.arena.clone()
        c.append()
        assert np.array_equal(first[0], c.cache.koff_host) and np.array_equal(first[1], c.cache.voff_host)
        c.cache.truncate(keep)
        c.append()
        assert not torch.equal(before, c.cache.arena)
        c.check(c.cache.chunk_attn(c.q.view(np.uint16), c.news))


@pytest.mark.gpu
def test_truncate_refusals_leave_everything_as_it_was(gpu):
    c = Case(gpu, 43, (64 * 20,), (5,), 2, 1, "tiny")
    c.append()
    used = {L: c.cache.pool.used(L) for L in gpu.LEVELS}
    for keep in ((64 * 20 + 6,), (-1,), (64 * 3 + 5,)):  # longer, negative, inside a demoted block
        with pytest.raises(gpu.GkvError):
            c.cache.truncate(keep)
    bad = c.cache.koff_host.copy()
    c.cache.koff_host[0, 0, 20] = c.cache.koff_host[0, 0, 19]  # a slot listed twice
    with pytest.raises(gpu.GkvError):
        c.cache.truncate((64,))
    c.cache.koff_host[:] = bad
    assert used == {L: c.cache.pool.used(L) for L in gpu.LEVELS}
    assert c.cache.T == 64 * 20 + 5
    c.check(c.cache.chunk_attn(c.q.view(np.uint16), c.news))


# ---------------------------------------------------------------- chunk_attn
@pytest.mark.gpu
@pytest.mark.parametrize("vtok", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (7, 1), (3, 3), (16, 1)])
@pytest.mark.parametrize("lens,news", [((0, 64), (1, 1)), ((130, 1), (3, 130)), ((700,), (1,)), ((385, 70), (40, 5)),
                                       ((64 * 7, 65, -1, 900), (0, 64, 0, 2))])
def test_chunks_match_the_definition(gpu, lens, news, Hq, Hkv, vtok):
    c = Case(gpu, 51, lens, news, Hq, Hkv, mixed_levels, vtok=vtok)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("prof,T,n", [("graded", 64 * 70 + 9, 90), ("graded", 64 * 120, 1), ("rdv2", 64 * 60 + 1, 20),
                                      ("tiny", 64 * 40, 33), (mixed_levels, 64 * 90 + 63, 5)])
def test_long_contexts_are_split(gpu, prof, T, n):
    """More workgroups than row tiles: partials over the context, joined."""
    c = Case(gpu, 53, (T, 200), (n, 1), 8, 2, prof)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,n", [(1, 15), (1, 16), (1, 17), (1, 31), (1, 32), (1, 33), (1, 48), (1, 49), (1, 64), (1, 65),
                                  (4, 4), (4, 5), (7, 2), (7, 3), (5, 9), (5, 13), (16, 4), (16, 5), (16, 8), (16, 9)])
@pytest.mark.parametrize("vtok,nres", [(False, 0), (True, 70)])
def test_row_counts(gpu, Hq, n, vtok, nres):
    """Rows about every bound of a row tile and of the two forms, over all six levels."""
    T = 64 * 40 + 5
    c = Case(gpu, 73, (T,), (n,), Hq, 1, mixed_levels, vtok=vtok, nres=nres, ragged=False)
    c.check(c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 3, 40, 100])
@pytest.mark.parametrize("prof", [mixed_levels, "exact"])
def test_queries_of_all_sizes(gpu, n, prof):
    """Rows scaled by 2^-14 .. 2^12, rows of zeros, and keys and values near the ends of fp16."""
    c = Case(gpu, 75, (64 * 25,), (n,), 4, 1, prof)
    size = np.exp2(np.resize([-14, 12, 0, -7, 5, -20, 9], n * 4)).reshape(n, 4, 1)
    size[n // 2, 1] = 0.0
    c.q = (c.q.astype(np.float64) * size).astype(np.float16)
    c.check(c.run())
    for scale in (2.0 ** 10, 2.0 ** -10):
        d = Case(gpu, 75, (64 * 25,), (n,), 4, 1, prof, scale=scale)
        d.q = (d.q.astype(np.float64) / scale).astype(np.float16)
        d.check(d.run())


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,nres", [(500, 7, 60), (64 * 30 + 5, 100, 200), (64 * 12, 1, 64), (130, 2, 130)])
def test_residual_rows_override_their_tokens(gpu, T, n, nres):
    c = Case(gpu, 55, (T, T), (n, n), 4, 2, mixed_levels, nres=nres, ragged=False)
    c.check(c.run())


@pytest.mark.gpu
def test_chunk_inside_the_selected_tokens(gpu):
    """Rows older than the newest residual rows: a residual row later than the row's own token
    is not seen."""
    T = 64 * 6 + 20
    c = Case(gpu, 57, (T,), (0,), 4, 2, "exact", nres=150, ragged=False)
    n = 100
    q = synth.rng(57, 2, 3).standard_normal((n, 4, 128), dtype=np.float32).astype(np.float16)
    out = c.cache.chunk_attn(q.view(np.uint16), [n]).float().cpu().numpy()
    for g in range(4):
        kh, vh = c.units[0, g // 2].khat_vhat()
        ref, tol = rows_reference(q.view(np.uint16)[:, g], kh, vh, range(T - n, T), np.ones(T, bool))
        assert (np.abs(out[:, g] - ref) / tol).max() <= 1.0


@pytest.mark.gpu
def test_rows_in_demoted_blocks(gpu):
    """A chunk whose own tokens the ladder has demoted since."""
    T, n = 64 * 20, 64 * 9 + 3
    c = Case(gpu, 59, (T,), (0,), 4, 2, mixed_levels)
    q = synth.rng(59, 2, 3).standard_normal((n, 4, 128), dtype=np.float32).astype(np.float16)
    out = c.cache.chunk_attn(q.view(np.uint16), [n]).float().cpu().numpy()
    for g in range(4):
        kh, vh = c.units[0, g // 2].khat_vhat()
        ref, tol = rows_reference(q.view(np.uint16)[:, g], kh, vh, range(T - n, T), np.zeros(T, bool))
        assert (np.abs(out[:, g] - ref) / tol).max() <= 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("tensor", [0, 1])
@pytest.mark.parametrize("bits", [0x7E00, 0x7C00, 0xFC00])
@pytest.mark.parametrize("n", [3, 70])
def test_unseen_tokens_have_no_effect(gpu, n, bits, tensor):
    """Rows before an infinite or NaN token are as without it; rows behind it see it."""
    import torch
    clean = Case(gpu, 61, (200, 64), (n, 2), 4, 2, mixed_levels)
    want = clean.run()
    c = Case(gpu, 61, (200, 64), (n, 2), 4, 2, mixed_levels)
    (c.ks if tensor == 0 else c.vs)[0, 1, 200 + n // 2, 9] = bits
    got = c.run()
    at = n // 2
    same = torch.ones(n + 2, 4, dtype=torch.bool)
    same[at:n, 2:] = False
    assert torch.equal(got.cpu()[same], want.cpu()[same])
    if tensor:
        hit = got[at:n, 2:, 9].float()
        assert bool(torch.isnan(hit).all()) if bits == 0x7E00 else bool((hit == (1 if bits == 0x7C00 else -1) * float("inf")).all())
        other = torch.arange(128) != 9
        assert torch.equal(got[at:n, 2:, other].cpu(), want[at:n, 2:, other].cpu())


@pytest.mark.gpu
def test_recycled_slots_with_nan_patterns(gpu):
    """Slots of retired sequences hold old bytes: a partial block's unused rows do not leak."""
    c = Case(gpu, 63, (70, 5), (1, 1), 4, 2, "exact", slack=8)
    free = c.cache.pool.alloc_many(16, c.cache.pool._caps[0] - c.cache.pool.used(16))
    for off in free:
        c.cache.arena[int(off):int(off) + 16384] = 0xFF
    for off in free[::-1]:
        c.cache.pool.free(16, int(off))
    c.check(c.run())


@pytest.mark.gpu
def test_single_tokens_agree_with_decode(gpu):
    """One new token: the chunk read and the decode read of the same cache."""
    c = Case(gpu, 65, (64 * 30 + 1, 77), (1, 1), 8, 2, "graded")
    out = c.run()
    c.check(out)
    dec = c.cache.decode(c.q.view(np.uint16))
    assert float((out.float() - dec).abs().max()) <= 2e-3 + 2.0 ** -11 * float(dec.abs().max())


@pytest.mark.gpu
def test_a_speculative_loop(gpu):
    """Append drafts, attend, drop some, again; then single appends and decode go on."""
    import torch
    Hq, Hkv, B = 4, 2, 3
    r = np.random.default_rng(5)
    ks, vs = kv_all(67, B, Hkv, 400)
    cache = gpu.GradedCache(B, Hkv, Hq, 0, 8, {16: 2 * B * Hkv * 8}, seq_lens=[0, 0, 0])
    have = np.zeros(B, np.int64)
    for step in range(12):
        n = r.integers(0, 60 if step == 0 else 9, B)
        pick = lambda x: np.concatenate([x[b, :, have[b]:have[b] + n[b]].transpose(1, 0, 2) for b in range(B)])
        cache.append_chunk(pick(ks), pick(vs), n)
        q = r.standard_normal((int(n.sum()), Hq, 128)).astype(np.float16)
        out = cache.chunk_attn(q.view(np.uint16), n).float().cpu().numpy()
        at = 0
        for b in range(B):
            e = have[b] + n[b]
            for g in range(Hq if n[b] else 0):
                ref, tol = rows_reference(q[at:at + n[b], g].view(np.uint16), ofp16.to_f64(ks[b, g // 2, :e]),
                                          ofp16.to_f64(vs[b, g // 2, :e]), range(have[b], e), np.ones(e, bool))
                assert (np.abs(out[at:at + n[b], g] - ref) / tol).max() <= 1.0
            at += n[b]
        have = have + n - np.array([r.integers(0, x + 1) for x in n])
        cache.truncate(have)
    cache.append(np.stack([ks[b, :, have[b]] for b in range(B)]), np.stack([vs[b, :, have[b]] for b in range(B)]))
    q = r.standard_normal((B, Hq, 128)).astype(np.float16)
    a = cache.decode(q.view(np.uint16))
    b = cache.chunk_attn(q.view(np.uint16), 1)
    assert float((a - b.float()).abs().max()) <= 4e-3


@pytest.mark.gpu
def test_prefill_by_chunks_equals_the_prompt(gpu):
    """A prompt attended whole, and appended and attended chunk by chunk to an exact cache."""
    T, Hq, Hkv = 333, 4, 2
    ks, vs = kv_all(69, 1, Hkv, T)
    q = np.random.default_rng(7).standard_normal((T, Hq, 128)).astype(np.float16).view(np.uint16)
    k, v = (np.ascontiguousarray(x[0].transpose(1, 0, 2)) for x in (ks, vs))
    whole = gpu.prompt_attn(q, k, v, [T])
    cache = gpu.GradedCache(1, Hkv, Hq, 0, 6, {16: 2 * Hkv * 6}, seq_lens=[0])
    at = 0
    for n in (1, 63, 100, 5, 164):
        cache.append_chunk(k[at:at + n], v[at:at + n], [n])
        out = cache.chunk_attn(q[at:at + n], [n])
        assert float((out.float() - whole[at:at + n].float()).abs().max()) <= 4e-3
        at += n


@pytest.mark.gpu
def test_workspaces_streams_and_graphs(gpu):
    import torch
    c = Case(gpu, 71, (64 * 60, 300), (9, 4), 8, 2, "graded")
    c.append()
    q = torch.from_numpy(c.q).cuda()
    want = c.cache.chunk_attn(q, c.news)
    c.check(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = c.cache.chunk_attn(q, c.news)
    s.synchronize()
    assert torch.equal(want, other)
    outs = [torch.empty_like(q) for _ in range(2)]
    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.cache.chunk_attn(q, c.news, out=out)
        graphs.append(g)
    for i in range(3):
        q.copy_(torch.roll(q, 1, 0))
        for g, out in zip(graphs, outs):
            out.zero_()
            g.replay()
        torch.cuda.synchronize()
        want = c.cache.chunk_attn(q, c.news)
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.gpu
@pytest.mark.parametrize("newest", [16, 8])
def test_contexts_past_every_count(gpu, newest):
    """A million tokens a head, blocks that repeat a few records (as many of each, so that the
    output is that of one of each): lists of more blocks than a wavefront reads table entries
    of at once, tiles past 4 GB."""
    import torch
    Hq, Hkv, order = 16, 8, [0, 1, 2, 4, 8, 16]
    order = [x for x in order if x != newest] + [newest]
    small = Case(gpu, 81, (64 * 6,), (0,), Hq, Hkv, lambda T: np.array(order, np.int8), ragged=False)
    times = 2834
    c = small.cache
    big = gpu.GradedCache(1, Hkv, Hq, 64 * 6 * times, 6 * times, {16: 1})
    big.arena = c.arena
    for name in ("level_host", "koff_host", "voff_host"):
        getattr(big, name)[:] = np.tile(getattr(c, name)[:, :, :6], (1, 1, times))
    big._bind(64 * 6 * times, 0)
    big._upload_tables()
    q = synth.rng(81, 2, 3).standard_normal((1, Hq, 128), dtype=np.float32).astype(np.float16)
    out = big.chunk_attn(q.view(np.uint16), [1]).float().cpu().numpy()
    del big
    torch.cuda.empty_cache()
    for g in range(Hq):
        kh, vh = small.units[0, g // 2].khat_vhat()
        ref, tol = rows_reference(q.view(np.uint16)[:, g], kh, vh, [383], np.zeros(384, bool))
        # (fp32 sums of a million weights, of which a wavefront's are some 4000 one after the other)
        tol = tol + 4096 * 2.0 ** -24 * (np.abs(vh).max() + np.abs(ref))
        assert (np.abs(out[:, g] - ref) / tol).max() <= 1.0, g


@pytest.mark.gpu
def test_rows_and_records_past_32_bits(gpu):
    """Tokens' rows 2 MB apart and slots behind 4 GB."""
    import torch
    T, Hq, Hkv = 2200, 4, 2
    ks, vs = kv_all(83, 1, Hkv, T)
    q, k, v = (torch.randn(T, Hq, 128).half().cuda(),
               *(torch.from_numpy(np.ascontiguousarray(x[0].transpose(1, 0, 2)).view(np.int16)).view(torch.float16).cuda()
                 for x in (ks, vs)))
    want = gpu.prompt_attn(q, k, v, [T])
    wide = torch.zeros(T, 1 << 20, dtype=torch.float16, device="cuda")
    assert wide.numel() > 1 << 31
    parts, at = [], 0
    for x in (q, k, v, torch.zeros_like(q)):
        view = wide[:, at:at + x.shape[1] * 128].unflatten(1, (x.shape[1], 128))
        view.copy_(x)
        parts.append(view)
        at += x.shape[1] * 128
    qw, kw, vw, out = parts
    gpu.prompt_attn(qw, kw, vw, [T], out=out)
    assert torch.equal(out, want)
    cache = gpu.GradedCache(1, Hkv, Hq, 0, 40, {16: 300000}, seq_lens=[0])
    cache.pool.alloc_many(16, 300000 - 2 * Hkv * 40)
    cache.append_chunk(kw, vw, [T])
    assert int(cache.koff_host[0, 0, 0]) > 1 << 32
    out.zero_()
    cache.chunk_attn(qw, [T], out=out)
    assert float((out.float() - want.float()).abs().max()) <= 4e-3
    near = cache.chunk_attn(q, [T])
    assert torch.equal(out, near)
    few = cache.chunk_attn(qw[-3:], [3])
    assert float((few.float() - want[-3:].float()).abs().max()) <= 4e-3
    assert torch.equal(few, cache.chunk_attn(q[-3:], [3]))
    cache.truncate([64 * 34])
    assert int((cache.record(0, 1, 33, 0)["values"] != ofp16.to_f64(ks[0, 1, 64 * 33:64 * 34])).sum()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,nres", [(64 * 130, 100, 0), (64 * 81, 65, 0), (64 * 96 + 7, 130, 900), (64 * 20, 70, 1100)])
def test_one_centroid_tiles(gpu, T, n, nres):
    """One-centroid blocks by the tile: more than 64, 64 and fewer, and blocks of which residual
    rows leave nothing."""
    c = Case(gpu, 85, (T,), (n,), 4, 2, "rdv2", nres=nres, ragged=False)
    c.check(c.run())
    m = min(n, 9)  # and the few-row form over the same cache
    q = c.q[n - m:]
    c.check(c.cache.chunk_attn(np.ascontiguousarray(q).view(np.uint16), [m]), [m])


@pytest.mark.gpu
def test_many_sequences(gpu):
    """128 sequences, idle, short, of single tokens and of chunks, both forms in one call."""
    r = np.random.default_rng(87)
    lens, news = r.integers(0, 260, 128), r.choice([0, 1, 2, 7, 150], 128, p=[0.2, 0.3, 0.2, 0.2, 0.1])
    lens[:3], news[:3] = (0, 64 * 70, -1), (0, 150, 0)
    c = Case(gpu, 87, lens, news, 2, 1, "tiny")
    c.check(c.run())


@pytest.mark.gpu
def test_calls_at_once(gpu):
    """Two streams, each with a cache of its own and one shared, the default workspaces."""
    import torch
    cs = [Case(gpu, 89 + i, (64 * 50 + 3, 400), (40, 3), 8, 2, "graded") for i in range(3)]
    qs = [torch.from_numpy(c.q).cuda() for c in cs]
    for c in cs:
        c.append()
    want = [c.cache.chunk_attn(q, c.news) for c, q in zip(cs, qs)]
    cs[0].check(want[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got += [(j, cs[j].cache.chunk_attn(qs[j], torch.tensor(cs[j].news))) for j in (i, 2)]
        torch.cuda.synchronize()
        for j, out in got:
            assert torch.equal(out, want[j])


@pytest.mark.gpu
def test_binding_refusals(gpu):
    """Arguments that the binding or the library turns away; the cache is as it was."""
    import torch
    c = Case(gpu, 91, (64 * 40, 70), (3, 2), 4, 2, "graded")
    k, v = (torch.from_numpy(x.view(np.int16)).view(torch.float16).cuda() for x in c.new_rows())
    q, cache = torch.from_numpy(c.q).cuda(), c.cache
    for a in ((k[:-1], v, c.news), (k, v[:, :1], c.news), (k.bfloat16(), v, c.news), (k, v, [3]), (k, v, [3.0, 2.0]),
              (k, v, [6, -1]), (k, v, [1 << 40, 2]), (k, v, [5])):
        with pytest.raises(gpu.GkvError):
            cache.append_chunk(*a)
    assert cache.lengths().tolist() == c.lens
    c.append()
    need = int(gpu._chunk_ws(gpu.ctypes.byref(cache.c), np.array(c.news, np.int32).ctypes.data))
    assert need > 0
    empty = lambda n, t=torch.uint8: torch.empty(n, dtype=t, device="cuda")
    for a, kw in (((q, [3, 3]), {}), ((q[:, :3], c.news), {}), ((q.bfloat16(), c.news), {}), ((q, [5, 0, 0]), {}),
                  ((q, c.news), {"ws": empty(need - 1)}), ((q, c.news), {"ws": empty(need, torch.float32)}),
                  ((q, c.news), {"ws": empty(2 * need)[::2]}), ((q, c.news), {"out": q.float()}),
                  ((q, c.news), {"out": torch.empty_like(q).transpose(0, 1)}),
                  ((q, c.news), {"out": empty(5 * 512, torch.float16).as_strided((5, 4, 128), (256, 128, 1))})):
        with pytest.raises(gpu.GkvError):
            cache.chunk_attn(*a, **kw)
    with pytest.raises(gpu.GkvError):
        cache.truncate([64 * 40])
    want = cache.chunk_attn(q, c.news)
    c.check(want)
    assert torch.equal(want, cache.chunk_attn(q, np.array(c.news), ws=empty(need)))


# ---------------------------------------------------------------- refusals (host only)


@pytest.fixture()
def host():
    """A cache descriptor whose device pointers are never followed: every call here is refused."""
    from paper_2608_23599_amd import binding as B
    Bn, Hkv, cap = 2, 2, 4
    lv = np.full((Bn, Hkv, cap), 16, np.int8)
    lens = np.array([70, 5], np.int64)
    c = B.CacheStruct()
    c.B, c.Hkv, c.Hq, c.D, c.T, c.nblk_cap = Bn, Hkv, 4, 128, 70, cap
    c.level = c.koff = c.voff = c.arena = c.seq_len = 4096
    c.arena_bytes = 64 * 16384
    c.level_host, c.seq_len_host = lv.ctypes.data, lens.ctypes.data
    return B, c, lv, lens


def _append(B, c, n, k=4096, stride=256, koff=None, voff=None, n_open=0):
    import ctypes
    n = np.array(n, np.int32)
    p = lambda a: None if a is None else ctypes.c_void_p(np.ascontiguousarray(a, np.int64).ctypes.data)
    keep = [None if x is None else np.ascontiguousarray(x, np.int64) for x in (koff, voff)]
    return B._append_chunk(ctypes.byref(c), k, k, stride, stride, ctypes.c_void_p(n.ctypes.data),
                           *[None if x is None else ctypes.c_void_p(x.ctypes.data) for x in keep], n_open, None)


def test_append_chunk_refusals(host):
    B, c, lv, lens = host
    assert _append(B, c, (0, 0)) == 0
    assert _append(B, c, (-1, 0)) == -2
    assert _append(B, c, (1, 0), k=None) == -1 and _append(B, c, (1, 0), k=4104) == -1
    assert _append(B, c, (1, 0), stride=248) == -2 and _append(B, c, (1, 0), stride=260) == -1
    assert _append(B, c, (1, 0), stride=(1 << 20) + 8) == -6
    assert _append(B, c, (200, 0)) == -2  # past the block capacity
    assert _append(B, c, (60, 0)) == -1  # opens a block, no slots
    ok = [0, 16384], [32768, 49152]
    assert _append(B, c, (60, 0), koff=ok[0], voff=ok[1], n_open=1) == -1
    for k, v in (([0, 0], ok[1]), ([0, 8], ok[1]), ([0, 32768 + 16], ok[1]), ([0, -16], ok[1]),
                 ([0, 64 * 16384 - 16], ok[1])):
        assert _append(B, c, (60, 0), koff=k, voff=v, n_open=2) == -1
    lv[0, 1, 1] = 8
    assert _append(B, c, (1, 0)) == -1  # its last block is not exact
    lv[0, 1, 1] = 16
    lens[1] = -1
    assert _append(B, c, (0, 1)) == -1  # retired
    lens[1] = 5
    c.seq_len = c.seq_len_host = None
    assert _append(B, c, (1, 2)) == -2  # one length, two counts


def test_chunk_attn_refusals(host):
    import ctypes
    B, c, lv, lens = host

    def call(n, q=4096, out=8192, stride=512, ws=None, ws_bytes=0):
        n = np.array(n, np.int32)
        p = ctypes.c_void_p(n.ctypes.data)
        return (B._chunk_attn(q, stride, ctypes.byref(c), p, out, stride, ws, ws_bytes, None),
                B._chunk_ws(ctypes.byref(c), p))

    assert call((0, 0)) == (0, 0)
    assert call((71, 0)) == (-2, -1) and call((-1, 0)) == (-2, -1)
    assert call((1, 0), q=None)[0] == -1 and call((1, 0), out=None)[0] == -1
    assert call((1, 0), q=4104)[0] == -1 and call((1, 0), stride=504)[0] == -2
    assert call((1, 0), stride=516)[0] == -1 and call((1, 0), stride=(1 << 20) + 8)[0] == -6
    lens[1] = -1
    assert call((0, 1)) == (-1, -1)
    lens[1] = 5
    big = np.full((2, 2, 4096), 16, np.int8)
    c.level_host = big.ctypes.data
    c.nblk_cap, c.T = 4096, 64 * 4096
    lens[0] = 64 * 4096
    nb = call((1, 1))[1]
    assert nb > 0 and call((1, 1))[0] == -1 and call((1, 1), ws=4096, ws_bytes=nb - 1)[0] == -4
    huge = np.full((1, 1, 1 << 25), 16, np.int8)  # more threads than a launch takes
    c.B = c.Hkv = c.Hq = 1
    c.level_host, c.nblk_cap = huge.ctypes.data, 1 << 25
    c.T = lens[0] = 1 << 31 - 1
    assert call((1, 0), ws=4096, ws_bytes=1 << 50) == (-6, -1)


def test_truncate_refusals(host):
    import ctypes
    B, c, lv, lens = host
    pool = B.Pool({16: 64})
    off = np.array([pool.alloc(16) for _ in range(32)], np.int64).reshape(2, 2, 2, 4)
    p = lambda a: ctypes.c_void_p(a.ctypes.data)
    ko, vo = off[0].copy(), off[1].copy()

    def call(n, pool_h=pool.h):
        n = np.array(n, np.int64)
        return B._truncate(ctypes.byref(c), pool_h, p(ko), p(vo), p(n), None)

    assert call((70, 5)) == 0  # nothing dropped
    assert call((71, 5)) == -2 and call((70, -1)) == -2 and call((70, 5), None) == -1
    lv[0, 0, 0] = 8
    assert call((63, 5)) == -2  # inside a demoted block
    lv[0, 0, 0] = 16
    vo[0, 1, 1] = vo[0, 0, 1]
    used = pool.used(16)
    assert call((64, 5)) == -1 and pool.used(16) == used
    c.nres = c.nres_cap = 1
    c.res_idx = c.res_rows = c.res_mask = c.res_off = 4096
    assert call((64, 5)) == -6


def test_pool_alloc_many():
    from paper_2608_23599_amd import binding as B
    a, b = B.Pool({16: 9, 8: 2}), B.Pool({16: 9, 8: 2})
    assert a.alloc_many(16, 7).tolist() == [b.alloc(16) for _ in range(7)]
    with pytest.raises(B.GkvError):
        a.alloc_many(16, 3)
    assert a.used(16) == 7 and a.alloc_many(16, 0).size == 0 and a.alloc_many(16, 2).size == 2
    with pytest.raises(B.GkvError):
        a.alloc_many(3, 1)
