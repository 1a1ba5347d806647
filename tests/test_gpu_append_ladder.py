"""append_chunk with a ladder: the device's tables, the demoted records and the attention over them, and a
refused ladder step leaves the cache as it was."""
import numpy as np
import pytest

from oracle import cache as ocache, fp16 as ofp16, ladder as olad
from tests._util import compare_record, kv_all
from tests.test_gpu_chunk import rows_reference


@pytest.mark.gpu
@pytest.mark.parametrize("news", [(64 * 26 + 5, 700), (64 * 5, 64 * 30)])
def test_tables_records_and_attention(gpu, news):
    Hkv, B = 2, 2
    ks, vs = kv_all(101, B, Hkv, max(news))
    cache = gpu.GradedCache(B, Hkv, 2 * Hkv, 0, -(-max(news) // 64), {16: 400, 8: 64, 4: 96, 2: 96}, seq_lens=[0, 0])
    pick = lambda x: np.concatenate([x[b, :, :n].transpose(1, 0, 2) for b, n in enumerate(news)])
    moves = cache.append_chunk(pick(ks), pick(vs), news, profile="tiny")
    want = [olad.ladder("tiny", n) for n in news]
    assert sorted((b, h, i, new) for b, h, i, old, new in moves if old == 16) == \
        [(b, h, i, int(lv)) for b in range(B) for h in range(Hkv) for i, lv in enumerate(want[b]) if lv != 16]
    n = 40
    q = np.random.default_rng(3).standard_normal((B * n, 2 * Hkv, 128)).astype(np.float16).view(np.uint16)
    out = cache.chunk_attn(q, [n] * B).double().cpu().numpy()
    for b in range(B):
        for h in range(Hkv):
            assert np.array_equal(cache.level[b, h, :len(want[b])].cpu().numpy(), want[b])
            assert np.array_equal(cache.level_host[b, h, :len(want[b])], want[b])
            u = ocache.UnitCache(ks[b, h, :news[b]], vs[b, h, :news[b]], want[b])
            for i in range(len(want[b])):
                for t in (0, 1):
                    compare_record(cache, u, b, h, i, t)
            kh, vh = u.khat_vhat()
            exact = np.repeat(np.asarray(want[b]) == 16, 64)[:news[b]]
            for g in (2 * h, 2 * h + 1):
                ref, tol = rows_reference(q[b * n:b * n + n, g], kh, vh, range(news[b] - n, news[b]), exact)
                assert (np.abs(out[b * n:b * n + n, g] - ref) / tol).max() <= 1.0


@pytest.mark.gpu
def test_a_refused_ladder_step_leaves_the_cache_as_it_was(gpu):
    import torch
    T, n = 300, 64 * 9
    ks, vs = kv_all(103, 1, 1, T + n)
    rows = lambda at, m: [np.ascontiguousarray(x[0, :, at:at + m].transpose(1, 0, 2)) for x in (ks, vs)]
    cache = gpu.GradedCache(1, 1, 2, 0, 16, {16: 32, 8: 10}, seq_lens=[0])
    cache.append_chunk(*rows(0, T), [T])
    before = cache.arena[:10 * 16384].clone()
    for _ in range(2):
        with pytest.raises(gpu.GkvError):
            cache.append_chunk(*rows(T, n), [n], profile="tiny")
        assert cache.T == T and cache.seq_len.tolist() == [T]
        assert cache.pool.used(16) == 10 and cache.pool.used(8) == 0
    assert torch.equal(before, cache.arena[:10 * 16384])
    cache.append_chunk(*rows(T, n), [n])
    for t, x in enumerate((ks, vs)):
        got = np.concatenate([cache.record(0, 0, i, t)["values"] for i in range(-(-(T + n) // 64))])[:T + n]
        assert np.array_equal(got, ofp16.to_f64(x[0, 0]))
