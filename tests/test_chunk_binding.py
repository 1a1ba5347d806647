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


def rows(n):
    return np.zeros((n, 1, 128), np.float16), np.zeros((n, 1, 128), np.float16)


@pytest.mark.parametrize("caps,levels,status", [
    ({16: 32, 8: 2}, None, -7),  # "tiny" at 15 blocks: 8 int8 and 3 int4
    ({16: 32, 8: 16, 4: 5}, None, -7),
    ({16: 32, 8: 32, 4: 32, 2: 32}, [16, 16, 4, 16, 16, 16], -3),  # block 2 of 15 is an int4 one, of 10 int8
])
def test_a_ladder_that_cannot_be_applied_appends_nothing(calls, caps, levels, status):
    c = cache(64 * 6, caps)
    if levels:
        c.level_host[0, 0, :6] = levels
    used = {level: c.pool.used(level) for level in B.LEVELS}
    n = 64 * (4 if levels else 9)
    with pytest.raises(B.GkvError) as e:
        c.append_chunk(*rows(n), [n], profile="tiny")
    assert e.value.status == status
    assert calls == [] and used == {level: c.pool.used(level) for level in B.LEVELS}
    c.c.truncated = 1
    if levels:  # demoted at a greater length: stays
        c.append_chunk(*rows(n), [n], profile="tiny")
        assert calls[0] == (c._dev, B._append_chunk)


def test_a_ladder_with_just_enough_slots(calls):
    c = cache(64 * 6, {16: 30, 8: 16, 4: 6})
    c.append_chunk(*rows(64 * 9), [64 * 9], profile="tiny")
    assert calls[0] == (c._dev, B._append_chunk)


@pytest.mark.parametrize("lens", [[-1], [64 * 11]])
def test_lengths_that_the_append_refuses_reach_it(calls, monkeypatch, lens):
    """(with slots for them)"""
    c = cache(64 * 6, {16: 100, 8: 32, 4: 32})
    monkeypatch.setattr(B, "_call_on", lambda device, f, *args: calls.append((device, f)) or -2)
    k = np.zeros((max(lens[0], 0), 1, 128), np.float16)
    with pytest.raises(B.GkvError) as e:
        c.append_chunk(k, k, lens, profile="tiny")
    assert e.value.status == -2 and c.pool.used(16) == 12
