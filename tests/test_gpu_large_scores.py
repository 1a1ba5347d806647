"""Scores of millions that differ by a few units: what the softmax takes of them is their difference, which
fp32 holds exactly.

Queries and keys are 2048 in channel 0 and integers in channel 1, so that every product and sum
is exact; the keys' channel 1 is a multiple of 8, up to 56.  An exponent is then one rounding
(2^-24 of at most 30) and the constant's (2^-25 of the difference) away from its value, the
exponential 2^-22; weights and output are rounded to fp16 (2^-11 each, the sum adds rounded ones), and
fp32 sums are off by 2^-24 for each token."""
import numpy as np
import pytest


def rows(T, seed):
    r = np.random.default_rng(seed)
    q, k = np.zeros((2, T, 1, 128), np.float16)
    q[:, :, 0] = k[:, :, 0] = 2048.0
    q[:, :, 1] = 1.0
    k[:, 0, 1] = 8.0 * r.integers(0, 8, T)
    v = r.standard_normal((T, 1, 128)).astype(np.float16)
    return q, k, v


def check(out, q, k, v, n):
    """out: the newest n rows of a causal read of all T tokens."""
    T = k.shape[0]
    x = np.asarray(k[:, 0, 1], np.float64)[None, :] / np.sqrt(128.0)
    x = np.where(np.arange(T)[None, :] > np.arange(T - n, T)[:, None], -np.inf, x)
    w = np.exp(x - x.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    vs = v[:, 0].astype(np.float64)
    ref, size = w @ vs, w @ np.abs(vs)
    u, e = 2.0 ** -11, 30 * 2.0 ** -24 + 10 * 2.0 ** -25 + 2.0 ** -22
    tol = (u + 2 * e + 2 * T * 2.0 ** -24) * size + 2 * u * np.abs(ref) + 1e-6
    worst = np.abs(out.double().cpu().numpy()[:, 0] - ref) / tol
    assert worst.max() <= 1.0, worst.max()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 64, 1000, 3000])
def test_prompt(gpu, T):
    import torch
    q, k, v = rows(T, T)
    check(gpu.prompt_attn(*(torch.from_numpy(x).cuda() for x in (q, k, v)), [T]), q, k, v, T)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5, 130])
@pytest.mark.parametrize("T", [200, 3000])
def test_chunk(gpu, T, n):
    import torch
    q, k, v = rows(T, T + n)
    cache = gpu.GradedCache(1, 1, 1, 0, -(-T // 64), {16: 2 * -(-T // 64)}, seq_lens=[0])
    cache.append_chunk(*(torch.from_numpy(x).cuda() for x in (k, v)), [T])
    check(cache.chunk_attn(torch.from_numpy(q[T - n:]).cuda(), [n]), q, k, v, n)
