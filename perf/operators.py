"""The performance cases of the many-query operators around the graded KV cache.

Four kinds of work, each through the calls a serving program makes:

* ``prompt``: causal attention over a batch of packed prompts (``prompt_attn``);
* ``append``: the drafts or prompt chunks of a batch written into its cache, what the last
  step left behind them dropped first (``GradedCache.truncate``, ``append_chunk``);
* ``chunk``: attention of a chunk of new tokens over the graded cache (``chunk_attn``);
* ``verify``: a speculative step's three calls together: drop the rejected drafts, append
  the new ones, attend with them.

Keys and values are normal rows, four key channels of each (sequence, KV head) ten times
larger (outlier channels); queries are normal; the attention mass that chooses the residual
rows is heavy-tailed.
"""
import math

import numpy as np
import torch

own = False  # set from outside: the framework's calls instead of the plain forms

P, D = 64, 128
EXACT, INT8, INT4, INT2, CENTROID, MEAN = 16, 8, 4, 2, 1, 0
HEADS = ((8, 2), (32, 8), (28, 4), (40, 8), (16, 1), (6, 6))  # (query heads, KV heads)
MOST_PAIRS = 28 * 16384 * 16384  # (query row, key) pairs of the largest case


# ---------------------------------------------------------------- the cases
def _prompt(batch, heads, kv_heads, tokens, dtype="float16", **more):
    return dict(kind="prompt", batch=batch, heads=heads, kv_heads=kv_heads, tokens=tokens, dtype=dtype, **more)


def _append(batch, heads, kv_heads, tokens, new, page=16, mixed=False, **more):
    return dict(kind="append", batch=batch, heads=heads, kv_heads=kv_heads, tokens=tokens, new=new, page=page,
                ladder="exact", residual=0, per_token=False, ragged=True, mixed=mixed, **more)


def _chunk(batch, heads, kv_heads, tokens, new, ladder="graded", residual=0, per_token=False, ragged=False,
           mixed=False, kind="chunk", **more):
    return dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, tokens=tokens, new=new, page=0,
                ladder=ladder, residual=residual, per_token=per_token, ragged=ragged, mixed=mixed, **more)


def listed():
    return [
        # the smallest call: one short question to a small model, where the launch counts
        _prompt(1, 8, 2, 37, name="prompt 37"),
        # an admission batch: sixteen prompts of all lengths up to 2000 tokens
        _prompt(16, 28, 4, 2000, "bfloat16", name="prompts ragged"),
        # one document of an 8B-shaped model
        _prompt(1, 32, 8, 4096, name="prompt 4k"),
        # a long document of a 7B-shaped model, and the largest case
        _prompt(1, 28, 4, 16384, "bfloat16", name="prompt 16k"),
        # a speculative step's drafts of eight conversations
        _append(8, 28, 4, 1900, 4, name="append drafts"),
        # a prompt's chunk of 8192 tokens, page boxes with it
        _append(1, 32, 8, 1000, 8192, name="append 8k"),
        # verification of a small model's three drafts: launches and latency
        _chunk(1, 8, 2, 2045, 3, "tiny", ragged=True, kind="verify", name="verify 2k"),
        # verification of five drafts in each of eight 32k conversations: bound by the cache's bytes
        _chunk(8, 28, 4, 32768, 5, ragged=True, kind="verify", name="verify 32k batch"),
        # the headline cache, 128k tokens a sequence with 2% residual rows, two new tokens each
        _chunk(8, 28, 4, 131072, 2, residual=20, name="chunk 2 over 128k"),
        # chunked prefill: 512 tokens over 64k of graded context
        _chunk(1, 28, 4, 65536, 512, name="chunk 512 over 64k"),
        # a mixed step: prompt chunks beside single tokens, lengths of all kinds, values grouped per token
        _chunk(9, 32, 8, 12011, 300, per_token=True, ragged=True, mixed=True, name="chunk mixed"),
        # the low-rate configuration: one-centroid base, 10.2% exact residual rows
        _chunk(2, 32, 8, 20000, 1000, "rdv2", residual=102, name="chunk low rate"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(("prompt", "prompt", "prompt", "append", "chunk", "chunk", "chunk", "verify"))
    heads, kv = rng.choice(HEADS)
    batch = rng.choice((1, 1, 2, 3, 4, 6, 8, 16))
    if kind == "prompt":
        tokens = _log(rng, 1, min(16384, math.isqrt(MOST_PAIRS // (batch * heads))))
        return _prompt(batch, heads, kv, tokens, rng.choice(("float16", "bfloat16")))
    if kind == "append":
        new = _log(rng, 1, 8192 // batch)
        return _append(batch, heads, kv, _log(rng, 1, 4000), new, rng.choice((0, 16, 32, 64)), rng.random() < 0.4)
    batch = min(batch, 8)
    tokens = _log(rng, 100, min(131072, 8 * 4 * 131072 // (batch * kv)))
    most = min(2048, tokens, max(1, MOST_PAIRS // (2 * batch * heads * (tokens + 2048))))
    new = _log(rng, 1, most if kind == "chunk" else min(8, most))
    ladder = rng.choice(("graded", "graded", "tiny", "rdv2"))
    ragged = batch > 1 and rng.random() < 0.5
    residual = 0 if ragged or kind == "verify" else 102 if ladder == "rdv2" else rng.choice((0, 20))
    return _chunk(batch, heads, kv, tokens, new, ladder, residual, rng.random() < 0.3, ragged or kind == "verify",
                  ragged and kind == "chunk" and rng.random() < 0.6, kind)


# ---------------------------------------------------------------- lengths
def _lengths(case):
    """Tokens of each sequence before the new ones (a prompt's whole length); the first is the longest."""
    B, T = case["batch"], case["tokens"]
    if case["kind"] != "prompt" and not case["ragged"]:
        return [T] * B
    return [T] + [max(1, int(T * (0.02 + 0.98 * (b * 0.6180339887 % 1.0)))) for b in range(1, B)]


def _news(case):
    """New tokens of each sequence: all alike, or chunks beside single tokens and idle sequences."""
    n = case["new"]
    return [(n, 1, n // 7)[b % 3] if case["mixed"] else n for b in range(case["batch"])]


def _kept(case):
    return case["tokens"] * case["residual"] // 1000


def _levels(ladder, tokens):
    """Levels of the age ladders by block, oldest first."""
    n = -(-tokens // P)
    age = np.arange(n)[::-1]
    if ladder == "exact":
        lv = np.full(n, EXACT)
    elif ladder == "tiny":
        lv = np.select([age < 4, age < 12, age < 24], [EXACT, INT8, INT4], INT2)
    elif ladder == "rdv2":
        lv = np.where(age < 16, EXACT, MEAN)
    else:
        rest = max(0, n - 16)
        lv = np.select([age < 16 + 25 * rest // 100, age < 16 + 60 * rest // 100], [INT8, INT4], INT2)
        lv = np.where(np.arange(n) < 10 * n // 100, CENTROID, lv)
        lv = np.where(age < 16, EXACT, lv)
    return lv.astype(np.int8)


def _level_table(case):
    """[batch][kv_heads][blocks] levels of the cached tokens, each sequence by the ladder at its own length."""
    lv = np.full((case["batch"], case["kv_heads"], -(-case["tokens"] // P)), EXACT, np.int8)
    for b, t in enumerate(_lengths(case)):
        lv[b, :, :-(-t // P)] = _levels(case["ladder"], t)
    return lv


# ---------------------------------------------------------------- inputs
def _generator(seed, *more):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash((int(seed),) + tuple(int(m) for m in more)) % (1 << 62))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(g, gain, *shape):
    """Normal rows in fp16; negative zeros become zeros."""
    return (_normal(g, *shape) * gain).half() + 0.0


def _gains(case, seed):
    """[batch][kv_heads][1][128]: the four outlier channels of each (sequence, KV head)."""
    B, H = case["batch"], case["kv_heads"]
    top = torch.rand((B, H, D), generator=_generator(seed, 1), device="cuda").topk(4, -1).indices
    return torch.ones((B, H, D), device="cuda").scatter_(-1, top, 10.0)[:, :, None]


def _cached(case, seed):
    """Exact keys and values of the cached tokens, [batch][kv_heads][tokens][128] fp16."""
    B, H, T = case["batch"], case["kv_heads"], case["tokens"]
    gain = _gains(case, seed)
    k = torch.empty((B, H, T, D), dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    for b in range(B):
        g = _generator(seed, 2, b)
        k[b] = _rows(g, gain[b], H, T, D)
        v[b] = _rows(g, 1.0, H, T, D)
    return k, v


def _new_rows(case, seed):
    """The new tokens' queries [n][heads][128] and keys and values [n][kv_heads][128], packed."""
    n = sum(_news(case))
    g = _generator(seed, 3)
    gain = _gains(case, seed)[:, :, 0].repeat_interleave(torch.tensor(_news(case), device="cuda"), 0)
    return (_normal(g, n, case["heads"], D).half(), _rows(g, gain, n, case["kv_heads"], D),
            _rows(g, 1.0, n, case["kv_heads"], D))


def _prompt_rows(case, seed):
    """Queries [n][heads][128], keys and values [n][kv_heads][128] of the packed prompts."""
    lens = _lengths(case)
    n, t = sum(lens), getattr(torch, case["dtype"])
    g = _generator(seed, 4)
    gain = _gains(case, seed)[:, :, 0].repeat_interleave(torch.tensor(lens, device="cuda"), 0)
    return (_normal(g, n, case["heads"], D).to(t), (_normal(g, n, case["kv_heads"], D) * gain).to(t),
            _normal(g, n, case["kv_heads"], D).to(t))


def _mass(case, seed):
    m = torch.exp(3.0 * _normal(_generator(seed, 5), case["batch"], case["kv_heads"], case["tokens"]))
    return m / m.sum(-1, keepdim=True)


def _places(lens):
    """Sequence and place within it of every packed row."""
    b = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))
    first = torch.tensor([0] + list(np.cumsum(lens)))[:-1]
    return b.cuda(), (torch.arange(int(sum(lens))) - first[b]).cuda()


def prepare(case, seed):
    s = {"case": case}
    if case["kind"] == "prompt":
        s["q"], s["k"], s["v"] = _prompt_rows(case, seed)
        s["lens"] = _lengths(case)
        if not own:
            s["places"] = _places(s["lens"])
        return s
    lens, news = _lengths(case), _news(case)
    s["lens"], s["news"] = lens, news
    s["q"], s["k"], s["v"] = _new_rows(case, seed)
    k, v = _cached(case, seed)
    if own:
        s["cache"] = _own_cache(case, seed, k, v)
        if case["kind"] == "chunk":
            s["cache"].append_chunk(s["k"], s["v"], news)
        return s
    s["places"] = _places(news)
    s["start"] = torch.tensor(lens, device="cuda")
    if case["kind"] == "append":
        _plain_append_state(s, k, v)
        return s
    s["store"] = _store(case, seed, k, v)
    return s


def _own_cache(case, seed, k, v):
    """The cache of the tokens so far, with slots for the new ones."""
    from paper_2608_23599_amd import binding as gkv
    lens, news = _lengths(case), _news(case)
    opened = [-(-(t + n) // P) - -(-t // P) for t, n in zip(lens, news)]
    extra = max(-(-(t + n) // P) for t, n in zip(lens, news)) - -(-case["tokens"] // P)
    # (a cache whose capacity holds no whole page has no boxes)
    page = case["page"] if case["page"] and (case["tokens"] + extra * P) // case["page"] else 0
    cache = gkv.GradedCache.build(k.view(torch.int16), v.view(torch.int16), Hq=case["heads"],
                                  levels=_level_table(case), page=page, nres_cap=_kept(case),
                                  extra_blocks=extra, slack={EXACT: sum(opened) * case["kv_heads"]},
                                  v_per_token=case["per_token"], seq_lens=lens if case["ragged"] else None)
    if _kept(case):
        cache.rd_residual_select(k.view(torch.int16), v.view(torch.int16), _mass(case, seed), _kept(case))
    return cache


# ---------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        if kind == "prompt":
            from paper_2608_23599_amd import binding as gkv
            return {"out": gkv.prompt_attn(s["q"], s["k"], s["v"], s["lens"])}
        cache = s["cache"]
        if kind != "chunk":
            cache.truncate(s["lens"])
            cache.append_chunk(s["k"], s["v"], s["news"])
        if kind == "append":
            out = {"records": cache.arena, "certificate": cache.cert}
            if s["case"]["page"]:
                none = torch.empty((cache.B, cache.Hkv, 0), dtype=torch.int16, device="cuda")
                out["boxes"] = cache.boxes if cache.page else none
            return out
        return {"out": cache.chunk_attn(s["q"], s["news"])}
    if kind == "prompt":
        return {"out": _plain_prompt(s)}
    if kind == "append":
        return _plain_append(s)
    return {"out": _plain_chunk(s)}


# ---------------------------------------------------------------- the plain forms
def _attend(q, k, v, seen):
    """q [u][g][n][128], k, v [u][t][128] in fp32; row i sees the first seen[u][i] keys."""
    u, g, n, _ = q.shape
    t = k.shape[1]
    x = (q.reshape(u, g * n, D) @ k.transpose(1, 2).contiguous()).view(u, g, n, t)
    x *= 1 / math.sqrt(D)
    x.masked_fill_((torch.arange(t, device=k.device) >= seen[..., None])[:, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    return (x.view(u, g * n, t) @ v).view(u, g, n, D) / total


def _plain_prompt(s):
    case = s["case"]
    b, i = s["places"]
    B, H, G, L = case["batch"], case["kv_heads"], case["heads"] // case["kv_heads"], max(s["lens"])

    def padded(x, heads):
        y = torch.zeros((B, L, heads, D), dtype=torch.float32, device=x.device)
        y[b, i] = x.float()
        return y

    q = padded(s["q"], H * G).view(B, L, H, G, D).permute(0, 2, 3, 1, 4).reshape(B * H, G, L, D)
    k = padded(s["k"], H).transpose(1, 2).reshape(B * H, L, D)
    v = padded(s["v"], H).transpose(1, 2).reshape(B * H, L, D)
    seen = torch.arange(1, L + 1, device=q.device).expand(B * H, L)
    o = _attend(q, k, v, seen).view(B, H, G, L, D).permute(0, 3, 1, 2, 4).reshape(B, L, H * G, D)
    return o[b, i].to(s["q"].dtype)


def _plain_chunk(s):
    case, (b, i) = s["case"], s["places"]
    B, H, G, n = case["batch"], case["kv_heads"], case["heads"] // case["kv_heads"], max(s["news"])
    T = -(-(case["tokens"] + n) // P) * P

    def rows(which, new):
        st = s["store"][which]
        x = torch.zeros((B * H * st["blocks"], P, D), dtype=torch.float32, device="cuda")
        for bits in (INT8, INT4, INT2):
            at, codes, scale, zero = st[bits]
            x[at] = codes.float() * scale.float() + zero.float()
        at, cent, ids = st[CENTROID]
        x[at] = torch.gather(cent.float(), 1, ids.long()[..., None].expand(-1, -1, D))
        x[st[MEAN][0]] = st[MEAN][1].float()
        x[st[EXACT][0]] = st[EXACT][1].float()
        y = torch.zeros((B, H, T, D), dtype=torch.float32, device="cuda")
        y[:, :, :st["blocks"] * P] = x.view(B, H, -1, D)
        if s["store"]["kept"] is not None:  # residual rows override their tokens
            y.view(B * H, T, D).scatter_(1, s["store"]["kept"][..., None].expand(-1, -1, D), st["rows"].float())
        y[b, :, s["start"][b] + i] = new.float()
        return y.view(B * H, T, D)

    q = torch.zeros((B, n, H * G, D), dtype=torch.float32, device="cuda")
    q[b, i] = s["q"].float()
    q = q.view(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B * H, G, n, D)
    seen = (s["start"][:, None] + torch.arange(1, n + 1, device="cuda")).repeat_interleave(H, 0)
    o = _attend(q, rows("k", s["k"]), rows("v", s["v"]), seen)
    return o.view(B, H, G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, H * G, D)[b, i].half()


def _plain_append_state(s, k, v):
    """The cache's rows, its arena of exact records (key and value slots in turn, the blocks of
    the cached tokens before the opened ones), boxes and value norms, and the places the new
    tokens touch."""
    case, lens, news = s["case"], s["lens"], s["news"]
    B, H, T0 = case["batch"], case["kv_heads"], case["tokens"]
    cap = max(-(-(t + n) // P) for t, n in zip(lens, news))
    old = [-(-t // P) for t in lens]
    end = [-(-(t + n) // P) for t, n in zip(lens, news)]
    slot = np.zeros((B, H, cap), np.int64)
    at = 0
    for lo, hi in (([0] * B, old), (old, end)):
        for b in range(B):
            for h in range(H):
                slot[b, h, lo[b]:hi[b]] = at + np.arange(hi[b] - lo[b])
                at += hi[b] - lo[b]
    rows = torch.zeros((2, B, H, cap * P, D), dtype=torch.float16, device="cuda")
    for b, t in enumerate(lens):
        rows[0, b, :, :t], rows[1, b, :, :t] = k[b, :, :t], v[b, :, :t]
    s["rows"] = rows
    s["slot"] = torch.from_numpy(slot).cuda()
    s["records"] = torch.zeros(at * 2 * 2 * P * D, dtype=torch.uint8, device="cuda")
    s["certificate"] = torch.zeros((B, H, cap, 4), dtype=torch.float32, device="cuda")
    page = case["page"]
    npages = -(-((T0 + (cap - -(-T0 // P)) * P) // page) // 64) * 64 if page else 0
    s["boxes"] = torch.zeros((B, H, npages * 2 * D), dtype=torch.int16, device="cuda")
    block = np.arange(cap)

    def pairs(of):
        b, i = np.nonzero(of)
        return torch.from_numpy(b).cuda(), torch.from_numpy(i).cuda()

    lens, ends = np.array(lens)[:, None], np.array(lens)[:, None] + np.array(news)[:, None]
    whole = pairs(block * P < lens)
    _plain_write(s, whole)
    s["touched"] = pairs((block >= lens // P) & (block * P < ends))
    if page:
        p = np.arange(npages)
        _plain_boxes(s, pairs((p + 1) * page <= lens))
        s["pages"] = pairs(((p + 1) * page > lens) & ((p + 1) * page <= ends))


def _plain_write(s, blocks):
    """The records and value norms of blocks (b, i) of every KV head."""
    b, i = blocks
    slot = s["slot"][b, :, i].reshape(-1)
    B, H = s["slot"].shape[:2]
    x = s["rows"].view(2, B, H, -1, P, D)[:, b, :, i].transpose(0, 1).reshape(2, -1, P, D)
    # 16-token pages, then for each of 64 lanes its 32 operand values
    k = x[0].view(-1, 4, 16, 4, 4, 8).permute(0, 1, 4, 2, 3, 5).reshape(-1, P * D)
    v = x[1].view(-1, 4, 4, 4, 8, 16).permute(0, 1, 2, 5, 4, 3).reshape(-1, P * D)
    out = s["records"].view(torch.float16).view(-1, 2, P * D)
    out[slot, 0] = k
    out[slot, 1] = v
    norm = x[1].float().square().sum(-1).sqrt().amax(-1).view(len(b), H)
    s["certificate"][b, :, i, 2] = norm


def _plain_boxes(s, pages):
    """The key boxes of pages (b, p) of every KV head."""
    b, p = pages
    B, H = s["slot"].shape[:2]
    page = s["case"]["page"]
    x = s["rows"][0].view(B, H, -1, page, D)[b, :, p]
    bx = s["boxes"].view(torch.float16).view(B, H, -1, D, 64, 2)
    bx[b, :, p // 64, :, p % 64] = torch.stack([x.amin(2), x.amax(2)], -1)


def _plain_append(s):
    b, i = s["places"]
    at = s["start"][b] + i
    s["rows"][0][b, :, at] = s["k"]
    s["rows"][1][b, :, at] = s["v"]
    _plain_write(s, s["touched"])
    out = {"records": s["records"], "certificate": s["certificate"]}
    if s["case"]["page"]:
        _plain_boxes(s, s["pages"])
        out["boxes"] = s["boxes"]
    return out


# ---------------------------------------------------------------- the graded records of the plain forms
def _f16(x):
    """fp64 rounded once to fp16 (by way of fp32 rounded to odd), as fp64."""
    f = x.float()
    w = f.double()
    i = f.view(torch.int32)
    i = torch.where(w.abs() > x.abs(), i - 1, i)  # towards zero
    i = torch.where(i.view(torch.float32).double() != x, i | 1, i)
    return i.view(torch.float32).half().double()


def _nearest(x, c):
    return torch.stack([(x - c[:, j:j + 1]).square().sum(-1) for j in range(c.shape[1])], -1).argmin(-1)


def _lloyd(x):
    """x [n][64][128]: four centroids (deterministic k-means of at most ten rounds) and the ids."""
    c = x[:, ::16].clone()
    for _ in range(10):
        hot = torch.nn.functional.one_hot(_nearest(x, c), 4).double()
        count = hot.sum(1)[..., None]
        c = torch.where(count > 0, hot.transpose(1, 2).contiguous() @ x / count.clamp(min=1), c)
    c = _f16(c)
    return c, _nearest(x, c)


def _scalar(x, bits, axis):
    """Codes, scale and zero of one group per channel (axis 1) or per token (axis 2)."""
    top = (1 << bits) - 1
    z, hi = x.amin(axis, keepdim=True), x.amax(axis, keepdim=True)
    scale = _f16((hi - z) / top)
    z = _f16(z)
    code = torch.where(scale > 0, torch.round((x - z) / torch.where(scale > 0, scale, 1.0)).clamp(0, top), 0.0)
    return code, scale, z


def _blocks(x):
    """[u][T][128] as blocks [u * n][64][128], the last one of each filled with zeros."""
    u, t, _ = x.shape
    n = -(-t // P)
    return torch.nn.functional.pad(x, (0, 0, 0, n * P - t)).view(u * n, P, D)


def _store(case, seed, k, v):
    """The graded cache as plain tables: the blocks of each level, and what it stores of them."""
    B, H, T = case["batch"], case["kv_heads"], case["tokens"]
    levels = torch.from_numpy(_level_table(case).reshape(-1).astype(np.int64)).cuda()
    out = {"kept": None}
    err = None
    for which, x in (("k", k), ("v", v)):
        x = _blocks(x.view(B * H, T, D))
        axis = 2 if which == "v" and case["per_token"] else 1
        st = {"blocks": -(-T // P)}
        back = x.clone() if which == "v" and _kept(case) else None  # for the value errors
        for bits in (INT8, INT4, INT2):
            at = torch.nonzero(levels == bits)[:, 0]
            parts = [[y if j else y.to(torch.uint8) for j, y in enumerate(_scalar(x[p].double(), bits, axis))]
                     for p in at.split(2048)]
            st[bits] = (at, torch.cat([p[0] for p in parts]), torch.cat([p[1].half() for p in parts]),
                        torch.cat([p[2].half() for p in parts]))
        at = torch.nonzero(levels == CENTROID)[:, 0]
        parts = [_lloyd(x[p].double()) for p in at.split(512)]
        st[CENTROID] = (at, torch.cat([p[0].half() for p in parts]), torch.cat([p[1].to(torch.uint8) for p in parts]))
        at = torch.nonzero(levels == MEAN)[:, 0]
        st[MEAN] = (at, torch.cat([_f16(x[p].double().mean(1, keepdim=True)).half() for p in at.split(2048)]))
        at = torch.nonzero(levels == EXACT)[:, 0]
        st[EXACT] = (at, x[at])
        out[which] = st
        if _kept(case):
            if which == "v":
                err = _value_errors(st, x, levels).view(B * H, -1)[:, :T]
    if _kept(case):
        score = _mass(case, seed).view(B * H, T).double() * err
        out["kept"] = torch.sort(score, descending=True, stable=True).indices[:, :_kept(case)].sort().values
        take = out["kept"][..., None].expand(-1, -1, D)
        out["k"]["rows"] = torch.gather(k.view(B * H, T, D), 1, take)
        out["v"]["rows"] = torch.gather(v.view(B * H, T, D), 1, take)
    return out


def _value_errors(st, x, levels):
    """Squared error of every value row as its level stores it."""
    err = torch.zeros(x.shape[:2], dtype=torch.float64, device=x.device)

    def put(at, value):
        for p in range(0, len(at), 2048):
            err[at[p:p + 2048]] = (x[at[p:p + 2048]].double() - value(slice(p, p + 2048))).square().sum(-1)

    for bits in (INT8, INT4, INT2):
        at, codes, scale, zero = st[bits]
        put(at, lambda p: codes[p].double() * scale[p].double() + zero[p].double())
    at, cent, ids = st[CENTROID]
    put(at, lambda p: torch.gather(cent[p].double(), 1, ids[p].long()[..., None].expand(-1, -1, D)))
    at, mean = st[MEAN]
    put(at, lambda p: mean[p].double())
    return err


# ---------------------------------------------------------------- the work of one pass
_BLOCK_BYTES = {EXACT: 16384, INT8: 512 + 8192, INT4: 512 + 4096, INT2: 512 + 2048, CENTROID: 1040, MEAN: 256}


def work(case):
    H, Hq = case["kv_heads"], case["heads"]
    lens = _lengths(case)
    if case["kind"] == "prompt":
        return {"bytes": sum(lens) * 4 * D * (Hq + H), "flops": 4 * Hq * D * sum(t * (t + 1) // 2 for t in lens)}
    news = _news(case)
    rows = 2 * 2 * D * H * sum(news)  # keys and values of the new tokens
    if case["kind"] == "append":
        pages = sum((t + n) // case["page"] - t // case["page"] for t, n in zip(lens, news)) if case["page"] else 0
        return {"bytes": 2 * rows + H * pages * 4 * D, "flops": 2 * D * H * sum(news)}
    active = [(t, n) for t, n in zip(lens, news) if n]
    read = H * sum(2 * _BLOCK_BYTES[int(x)] for t, _ in active for x in _levels(case["ladder"], t)[:t // P])
    read += 2 * 2 * D * H * sum(t % P for t, _ in active) + rows  # the partial blocks' rows and the new ones
    read += H * len(active) * _kept(case) * (2 * 2 * D + 4)
    pairs = sum(n * t + n * (n + 1) // 2 for t, n in active)
    if case["kind"] == "verify":
        read += rows  # written as well
    return {"bytes": read + 4 * D * Hq * sum(news), "flops": 4 * Hq * D * pairs}


# ---------------------------------------------------------------- the same in 64 bits
def _softmax_rows(q, k, v, first):
    """q [n][128] in fp64, row i at position first + i // heads in the outer loop: sees keys up to it."""
    w = q @ k.transpose(0, 1).contiguous() / math.sqrt(D)
    pos = torch.arange(k.shape[0], device=k.device)
    w = torch.softmax(w.masked_fill_(pos[None, :] > first[:, None], -math.inf), -1)
    return w @ v


def _prompt_exact(case, seed):
    q, k, v = (x.double() for x in _prompt_rows(case, seed))
    H, G = case["kv_heads"], case["heads"] // case["kv_heads"]
    out = torch.zeros_like(q)
    at = 0
    for t in _lengths(case):
        pos = torch.arange(t, device="cuda")
        for h in range(H):
            kh, vh = k[at:at + t, h].contiguous(), v[at:at + t, h].contiguous()
            for g in range(h * G, h * G + G):
                for lo in range(0, t, 4096):
                    hi = min(t, lo + 4096)
                    out[at + lo:at + hi, g] = _softmax_rows(q[at + lo:at + hi, g].contiguous(), kh[:hi], vh[:hi],
                                                            pos[lo:hi])
        at += t
    return out


def _rebuilt(x, levels, per_token=False):
    """x [blocks][64][128] fp64; every block as its level stores it."""
    y = x.clone()
    levels = torch.as_tensor(np.ascontiguousarray(levels).astype(np.int64), device=x.device)
    for lv in (INT8, INT4, INT2, CENTROID, MEAN):
        for part in torch.nonzero(levels == lv)[:, 0].split(512):
            if not len(part):
                continue
            b = x[part]
            if lv == MEAN:
                y[part] = _f16(b.sum(1, keepdim=True) / P).expand_as(b)
            elif lv == CENTROID:
                c, ids = _lloyd(b)
                y[part] = torch.stack([c[j][ids[j]] for j in range(len(part))])
            else:
                code, scale, zero = _scalar(b, lv, 2 if per_token else 1)
                y[part] = zero + scale * code
    return y


def _chunk_exact(case, seed):
    k, v = _cached(case, seed)
    qn, kn, vn = (x.double() for x in _new_rows(case, seed))
    H, G = case["kv_heads"], case["heads"] // case["kv_heads"]
    mass = _mass(case, seed) if _kept(case) else None
    out = torch.zeros_like(qn)
    at = 0
    for b, (t, n) in enumerate(zip(_lengths(case), _news(case))):
        if not n:
            continue
        lv = _levels(case["ladder"], t)
        pos = t + torch.arange(n, device="cuda")
        for h in range(H):
            ks, vs = k[b, h, :t].double(), v[b, h, :t].double()
            kr = _rebuilt(_blocks(ks[None]), lv).view(-1, D)[:t]
            vr = _rebuilt(_blocks(vs[None]), lv, case["per_token"]).view(-1, D)[:t]
            if mass is not None:
                score = mass[b, h].double() * (vs - vr).square().sum(-1)
                kept = torch.sort(score, descending=True, stable=True).indices[:_kept(case)]
                kr[kept], vr[kept] = ks[kept], vs[kept]
            kr, vr = torch.cat([kr, kn[at:at + n, h]]), torch.cat([vr, vn[at:at + n, h]])
            for g in range(h * G, h * G + G):
                out[at:at + n, g] = _softmax_rows(qn[at:at + n, g].contiguous(), kr, vr, pos)
        at += n
    return out


def _append_exact(case, seed):
    """The value norms of every block; the records and boxes are copies and comparisons."""
    _, v = _cached(case, seed)
    _, _, vn = _new_rows(case, seed)
    lens, news = _lengths(case), _news(case)
    cap = max(-(-(t + n) // P) for t, n in zip(lens, news))
    cert = torch.zeros((case["batch"], case["kv_heads"], cap, 4), dtype=torch.float64, device="cuda")
    at = 0
    for b, (t, n) in enumerate(zip(lens, news)):
        x = torch.cat([v[b, :, :t], vn[at:at + n].transpose(0, 1)], 1).double()
        norms = _blocks(x).norm(dim=-1).amax(-1).view(case["kv_heads"], -1)
        cert[b, :, :norms.shape[1], 2] = norms
        at += n
    out = {"records": None, "certificate": cert}
    if case["page"]:
        out["boxes"] = None
    return out


def exact(case, seed):
    if case["kind"] == "prompt":
        return {"out": _prompt_exact(case, seed)}
    if case["kind"] == "append":
        return _append_exact(case, seed)
    return {"out": _chunk_exact(case, seed)}
