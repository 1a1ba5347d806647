"""A ladder on a cache whose newest tokens were dropped: blocks that it demoted at the greater length stay
as they are, and the cache goes on."""
import ctypes

import numpy as np
import pytest

from oracle import fp16 as ofp16
from tests._util import kv_all
from tests.test_gpu_chunk import rows_reference


def host_cache(B, levels, T):
    c = B.CacheStruct()
    c.B, c.Hkv, c.Hq, c.D, c.T, c.nblk_cap = 1, 1, 1, 128, T, levels.shape[2]
    c.level = c.koff = c.voff = c.arena = 4096
    c.arena_bytes = 64 * 16384
    c.level_host = levels.ctypes.data
    return c


def test_crossings_of_a_truncated_cache():
    """"tiny" at five blocks wants blocks 1 .. 4 exact; block 1 was demoted at six."""
    from paper_2608_23599_amd import binding as B
    levels = np.array([[[16, 8, 16, 16, 16, 16, 0, 0]]], np.int8)
    c = host_cache(B, levels, 64 * 4 + 10)
    jobs, to = np.zeros(12, np.int32), np.zeros(4, np.int8)
    call = lambda: B._ladder_crossings(ctypes.byref(c), 0, int(c.T), B._np_ptr(jobs), B._np_ptr(to), 4)
    assert call() == -3
    c.truncated = 1
    assert call() == 1 and jobs[:3].tolist() == [0, 0, 0] and to[0] == 8


class Grown:
    """A cache that grows by chunks under the ladder, beside the rows it holds."""

    def __init__(self, gpu):
        self.cache = gpu.GradedCache(1, 1, 2, 0, 16, {16: 32, 8: 32, 4: 32, 2: 32}, seq_lens=[0])
        self.ks, self.vs = kv_all(99, 1, 1, 1024)

    def rows(self, at, n):
        return [np.ascontiguousarray(x[0, :, at:at + n].transpose(1, 0, 2)) for x in (self.ks, self.vs)]

    def append(self, n):
        return self.cache.append_chunk(*self.rows(self.cache.T, n), [n], profile="tiny")

    def levels(self):
        n = -(-self.cache.T // 64)
        assert np.array_equal(self.cache.level[0, 0, :n].cpu().numpy(), self.cache.level_host[0, 0, :n])
        return self.cache.level_host[0, 0, :n].tolist()

    def check(self):
        """The newest rows' attention over the records the cache holds."""
        T, n = self.cache.T, 5
        q = np.random.default_rng(T).standard_normal((n, 2, 128)).astype(np.float16).view(np.uint16)
        out = self.cache.chunk_attn(q, [n]).double().cpu().numpy()
        kh, vh = (np.concatenate([self.cache.record(0, 0, i, t)["values"] for i in range(-(-T // 64))])[:T]
                  for t in (0, 1))
        for g in range(2):
            ref, tol = rows_reference(q[:, g], kh, vh, range(T - n, T), np.zeros(T, bool))
            assert (np.abs(out[:, g] - ref) / tol).max() <= 1.0


@pytest.mark.gpu
def test_appends_after_a_truncation(gpu):
    g = Grown(gpu)
    g.append(64 * 6)
    assert g.levels() == [8, 8, 16, 16, 16, 16]
    g.cache.truncate([64 * 4 + 10])
    assert g.append(1) == [] and g.levels() == [8, 8, 16, 16, 16]
    g.check()
    g.append(100)
    assert g.levels() == [8, 8, 16, 16, 16, 16]
    g.cache.truncate([64 * 5])
    assert g.cache.append(g.ks[:, :, 320].copy(), g.vs[:, :, 320].copy(), profile="tiny") == []
    g.append(64 * 3)
    assert g.levels() == [8, 8, 8, 8, 8, 16, 16, 16, 16]
    g.check()


@pytest.mark.gpu
def test_layers_step_after_a_truncation(gpu):
    g = [Grown(gpu) for _ in range(2)]
    for x in g:
        x.append(64 * 6)
        x.cache.truncate([64 * 4 + 10])
    layers = gpu.LayerCaches([x.cache for x in g], "tiny")
    for _ in range(130):
        T = g[0].cache.T
        layers.step(np.stack([x.ks[:, :, T] for x in g]), np.stack([x.vs[:, :, T] for x in g]))
    for x in g:
        assert x.levels() == [8, 8, 8, 16, 16, 16, 16]
        x.check()
