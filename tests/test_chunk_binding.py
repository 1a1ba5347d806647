"""The binding's part of appending and dropping chunks, on the host: the library's device calls are stand-ins."""
import numpy as np
import pytest

from paper_2608_23599_amd import binding as B


@pytest.fixture()
def calls(monkeypatch):
    """Device calls are noted as (device, function) and succeed; none finds a current stream."""
    done = []

    def no_stream():
        raise AssertionError("a call on the current device's stream")

    monkeypatch.setattr(B, "_call_on", lambda device, f, *args: done.append((device, f)) or 0)
    monkeypatch.setattr(B, "_stream", no_stream)
    return done


def cache(T=0, caps=None, blocks=16):
    c = B.GradedCache(1, 1, 1, 0, blocks, caps or {16: 2 * blocks, 8: 2 * blocks}, seq_lens=[T], device="cpu")
    for i in range(-(-T // 64)):
        c.level_host[0, 0, i] = 16
        c.koff_host[0, 0, i], c.voff_host[0, 0, i] = c.pool.alloc(16), c.pool.alloc(16)
    return c


def test_demotions_run_on_the_caches_device(calls):
    c = cache(64 * 6)
    c.demote([(0, 0, 0), (0, 0, 1)], [8, 8])
    assert calls == [(c._dev, B._demote)]
    assert c.pool.used(8) == 4 and c.pool.used(16) == 8


@pytest.mark.parametrize("dtype", [np.float32, np.float64, np.int32, np.int64, np.uint8])
def test_arrays_of_other_types_are_no_bit_patterns(dtype):
    """Whose bytes would make rows of 128 halves."""
    width = 256 // np.dtype(dtype).itemsize
    with pytest.raises(B.GkvError):
        B._rows_dev(np.zeros((3, 2, width), dtype), "prompt_attn")
    with pytest.raises(B.GkvError):
        B._rows_dev(np.zeros((3, 2, 128), dtype), "prompt_attn")
