"""Rows of which one token takes nearly all of the weight, and many others the rest together.

Keys are zero but for one token's, whose score lies `above` nats over the others'; so a row that
sees n tokens beside it has the output sum_j w v_j / (1 + n w), w = exp(-above), of values v_j that
are zero for the one token.  Weights enter the value product rounded to the type, taken
relative to a reference from which the largest one lies at least 2^7 up: in fp16 (half a step 2^-11,
at the least 2^-25) each is off by at most max(2^-11 w, 2^-32) of the one token's, in bf16 by
2^-8 w; the output is rounded once.  An exponent of up to 30 in fp32 and the hardware's
exponential are off by 2^-19 of a weight together, and fp32 sums by 2^-24 for each of their tokens."""
import numpy as np
import pytest

ABOVE = [8.0, 14.0, 16.7, 17.4, 20.0]


def expect(above, n, total, half_step, least):
    """Output and tolerance of rows that see n tokens, whose values add to total [rows][channels]."""
    w = np.exp(-above)
    out = w * total / (1 + n * w)
    each = max(half_step * w, least)
    tol = each * total + out * (half_step + n * each + 2.0 ** -18 + 2 * n * 2.0 ** -24) + 2.0 ** -25
    return out, tol


def sink_key(above):
    """The value of the one key's channels under queries of ones, and the score it makes."""
    c = np.float16(above * np.sqrt(128.0) / 128)
    return c, float(c) * 128 / np.sqrt(128.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("above", ABOVE)
def test_prompt(gpu, above, dtype):
    import torch
    T, t = 16384, getattr(torch, dtype)
    c = float(torch.tensor(above * 128 ** 0.5 / 128).to(t))
    q = torch.ones(T, 2, 128, dtype=t, device="cuda")
    k = torch.zeros(T, 1, 128, dtype=t, device="cuda")
    v = (1 + torch.arange(128, device="cuda") / 128).to(t).repeat(T, 1, 1).contiguous()
    k[0], v[0] = c, 0.0
    out = gpu.prompt_attn(q, k, v, [T]).double().cpu().numpy()
    n = np.arange(T, dtype=np.float64)[:, None]
    u, least = (2.0 ** -11, 2.0 ** -32) if dtype == "float16" else (2.0 ** -8, 0.0)
    ref, tol = expect(c * 128 / 128 ** 0.5, n, n * v[1, 0].double().cpu().numpy(), u, least)
    worst = np.abs(out - ref[:, None]) / tol[:, None]
    assert worst.max() <= 1.0, worst.max()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 150])
@pytest.mark.parametrize("at", [5, 64 * 60 + 1])
@pytest.mark.parametrize("above", ABOVE)
def test_chunk(gpu, above, at, n):
    """The values of one share of the context count (the one token's block), in both forms."""
    import torch
    T = 8192
    c, score = sink_key(above)
    k = torch.zeros(T, 1, 128, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    v[at // 64 * 64:at // 64 * 64 + 64] = 1000.0
    k[at], v[at] = float(c), 0.0
    cache = gpu.GradedCache(1, 1, 1, 0, T // 64, {16: 2 * T // 64}, seq_lens=[0])
    cache.append_chunk(k, v, [T])
    out = cache.chunk_attn(torch.ones(n, 1, 128, dtype=torch.float16, device="cuda"), [n]).double().cpu().numpy()
    seen = np.arange(T - n, T, dtype=np.float64)[:, None]
    ref, tol = expect(score, seen, 63 * 1000.0, 2.0 ** -11, 2.0 ** -32)
    worst = np.abs(out[:, 0] - ref) / tol
    assert worst.max() <= 1.0, worst.max()
