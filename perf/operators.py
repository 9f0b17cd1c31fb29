"""The operators around the attention of a decoder, as cases to be timed: what makes its queries and keys, what keeps
them, and what reads them back.

A case names one operator, its sizes and its options; ``run`` computes it in elementary torch operations in 32 bits, or,
where ``own`` is set, with the library's calls.

Operators
  rotate        dfss_qk_norm_rotate: norm of every head's query and key, rotated to its position, from the rows of a
                fused projection into the layout of the attention calls
  rotate_grad   dfss_qk_norm_rotate_backward: gradients of the projection's queries and keys and of the norms' weights
  append        dfss_cache_append: new keys (norm and rotation on the way) and values into a paged cache of 8 bits
  attend        dfss_attention_cached, or dense_attention_cached where N is 0: queries over that cache

The cache holds e4m3 codes [pages, heads, page, d] and one power of two for each page and head, the scale s =
2^ceil(log2(amax / 448)), at least 2^-64, of what the page holds.  Tokens appended to a page that holds earlier ones can
only raise it; the earlier codes are then rounded again.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False
EPS = 1e-6


def _rotate(name, B, L, Hq, Hk, d, dtype="bf16", norm=True, rot=None, interleaved=False, grad=False):
    return {"name": name, "op": "rotate_grad" if grad else "rotate", "B": B, "L": L, "Hq": Hq, "Hk": Hk, "d": d,
            "dtype": dtype, "norm": norm, "rot": d if rot is None else rot, "interleaved": interleaved}


def _append(name, B, most, max_len, Hk, d, page, norm=True, interleaved=False):
    return {"name": name, "op": "append", "B": B, "most": most, "max_len": max_len, "Hk": Hk, "d": d, "page": page,
            "norm": norm, "interleaved": interleaved}


def _attend(name, B, most, max_len, Hq, Hk, d, page, N, M, causal=True):
    return {"name": name, "op": "attend", "B": B, "most": most, "max_len": max_len, "Hq": Hq, "Hk": Hk, "d": d,
            "page": page, "N": N, "M": M, "causal": causal}


def listed():
    return [
        # one step of generation for eight sequences: launch and host time
        _rotate("rotate_one_token", 8, 1, 12, 12, 64),
        # prompts of a model with large heads and shared keys
        _rotate("rotate_prompts", 4, 2048, 16, 4, 128),
        # a training step on short sequences, float data, neighbouring elements paired, part of the head rotated
        _rotate("rotate_grad_float", 16, 512, 12, 12, 64, dtype="f32", rot=32, interleaved=True, grad=True),
        # a training step of the model with large heads
        _rotate("rotate_grad_large_head", 4, 2048, 16, 16, 128, grad=True),
        # one token for each of 64 sequences into its half-filled page
        _append("append_one_token", 64, 1, 4096, 8, 128, 64),
        # prompts of different lengths, appended in one call, in small pages
        _append("append_prompts", 8, 2048, 2048, 16, 64, 16, interleaved=True),
        # one new query of one sequence: the smallest call
        _attend("attend_one_sequence", 1, 1, 4096, 12, 12, 64, 64, 2, 4),
        # generation for 64 sequences of different lengths, four queries to a key head, small pages
        _attend("attend_batch", 64, 1, 4096, 32, 8, 128, 16, 2, 4),
        # many short sequences with a key head to each query head, full attention
        _attend("attend_dense", 128, 1, 2048, 16, 16, 64, 32, 0, 0),
        # few sequences of great length, full attention
        _attend("attend_long_dense", 4, 1, 32768, 32, 8, 128, 128, 0, 0),
        # four drafted tokens a sequence are looked at together; 1:2
        _attend("attend_draft", 24, 4, 2500, 12, 4, 64, 32, 1, 2),
        # the next part of long prompts against what the cache holds of them
        _attend("attend_prompt_part", 4, 512, 4096, 16, 4, 128, 64, 2, 4),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: an operator, heads and sizes over their ranges, and as many sequences as keep it below the largest
    listed case of the operator."""
    op = rng.choice(["rotate", "rotate_grad", "append", "append", "attend", "attend", "attend", "attend"])
    d = rng.choice([64, 128])
    Hk = rng.choice([1, 2, 3, 4, 8, 12, 16])
    Hq = Hk * rng.choice([1, 1, 2, 3, 4, 8])
    if op in ("rotate", "rotate_grad"):
        L = rng.choice([1, _log_uniform(rng, 2, 64), _log_uniform(rng, 64, 4096)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = (4 * 2048 * 32 * 128) // ((Hq + Hk) * d * (2 if dtype == "f32" else 1))
        B = _log_uniform(rng, 1, max(1, min(256, rows // L)))
        rot = rng.choice([d, d, 32, d // 2, 0])
        c = _rotate("", B, L, Hq, Hk, d, dtype, rng.choice([True, True, rot == 0]), rot, rng.choice([False, True]),
                    op == "rotate_grad")
    elif op == "append":
        page = rng.choice([16, 32, 64, 128])
        most = rng.choice([1, _log_uniform(rng, 2, 32), _log_uniform(rng, 32, 2048)])
        max_len = max(most, _log_uniform(rng, 16, 8192))
        B = _log_uniform(rng, 1, max(1, min(128, (16 * 2048 * 8 * 64) // (most * Hk * d), (1 << 28) // (max_len * Hk * d))))
        c = _append("", B, most, max_len, Hk, d, page, rng.choice([True, False]), rng.choice([False, True]))
    else:
        page = rng.choice([16, 32, 64, 128])
        N, M = rng.choice([(2, 4), (2, 4), (1, 2), (0, 0)])
        most = rng.choice([1, 1, 1, _log_uniform(rng, 2, 16), _log_uniform(rng, 16, 512)])
        max_len = max(most, _log_uniform(rng, 16, 32768))
        B = min((1 << 28) // (max_len * Hk * d), (4 * 512 * 16 * 4096) // (most * Hq * max_len), 192)
        if B < 1:
            most, B = 1, 1
        c = _attend("", _log_uniform(rng, 1, B), most, max_len, Hq, Hk, d, page, N, M, rng.choice([True, True, False]))
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------


def _counts(B, most):
    """Tokens of every sequence, by the case alone (they are the outputs' shape): between half of the most and the
    most, which the first sequence has."""
    n = np.random.default_rng(1000 * B + most).integers((most + 1) // 2, most + 1, B)
    n[0] = most
    return n.astype(np.int32)


def _angles(n_pos, rot):
    """cos and sin of the position times 10000^(-2 i / rot), from 64 bits: far positions lose their angle in 32."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-2.0 * i / max(rot, 1))
    return a.cos().float(), a.sin().float()


def _pages(g, n_pages, Hk, page, d):
    """Codes and scales of pages that hold normal values, of another width in every page and head."""
    x = torch.randn((n_pages, Hk, page, d), generator=g, device="cuda")
    x *= torch.exp2(torch.rand((n_pages, Hk, 1, 1), generator=g, device="cuda") * 2 - 1)
    scale = _scale_of(x.abs().amax((2, 3)))
    x /= scale[:, :, None, None]
    return x.to(torch.float8_e4m3fn).view(torch.uint8), scale


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    h = np.random.default_rng(seed)
    state = {"c": c}
    if c["op"] in ("rotate", "rotate_grad"):
        t = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        B, L, Hq, Hk, d = c["B"], c["L"], c["Hq"], c["Hk"], c["d"]
        # rows of the projection: queries, keys and values of a token
        state["qkv"] = torch.randn((B, L, (Hq + 2 * Hk) * d), generator=g, device="cuda").to(t)
        # one new token stands somewhere in its sequence, a prompt starts at position 0
        start = h.integers(0, 4096, (B, 1)) if L == 1 else np.zeros((B, 1), np.int64)
        state["pos"] = torch.from_numpy((start + np.arange(L)).astype(np.int32)).cuda()
        state["cos"], state["sin"] = _angles(max(4096, L), c["rot"])
        state["w"] = [(1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(t) for _ in range(2)] if c["norm"] else [None, None]
        if c["op"] == "rotate_grad":
            state["dY"] = [torch.randn((B * H, L, d), generator=g, device="cuda").to(t) for H in (Hq, Hk)]
        return state
    B, Hk, d, page = c["B"], c["Hk"], c["d"], c["page"]
    n = _counts(B, c["most"])
    # lengths with the new tokens: any length that holds them, the longest among them
    length = np.maximum(h.integers((c["max_len"] + 1) // 2, c["max_len"] + 1, B), n)
    length[0] = c["max_len"]
    if c["op"] == "append" and c["most"] == c["max_len"]:
        length = n.copy()                       # whole prompts
    W = -(-c["max_len"] // page)
    table = h.permutation(B * W + 3)[:B * W].reshape(B, W)
    table[np.arange(W) * page >= length[:, None]] = -1          # pages that are not in use
    state["n"] = n
    state["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()
    state["len"] = torch.from_numpy(length.astype(np.int32)).cuda()
    state["table"] = torch.from_numpy(table.astype(np.int32)).cuda()
    state["k"], state["k_scale"] = _pages(g, B * W + 3, Hk, page, d)
    state["v"], state["v_scale"] = _pages(g, B * W + 3, Hk, page, d)
    T = int(n.sum())
    if c["op"] == "append":
        state["kv"] = torch.randn((T, 2 * Hk * d), generator=g, device="cuda").bfloat16()
        state["w"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16() if c["norm"] else None
        state["cos"], state["sin"] = _angles(c["max_len"], d)
    else:
        state["Q"] = torch.randn((T, c["Hq"], d), generator=g, device="cuda").bfloat16()
    return state


# ---- the operators in their plain form -------------------------------------------------------------------------


def _scale_of(amax):
    """The power of two that brings values up to amax to 448 or less."""
    m, e = torch.frexp(amax)                   # amax = m 2^e with m in [0.5, 1); 448 = 0.875 * 2^9
    k = (e - 9 + (m > 0.875).int()).clamp(min=-64)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, k, -64))


def _partner(x, rot, interleaved):
    """Every rotated element's other one, with the sign that it takes: (-x2, x1) for (x1, x2)."""
    r = x[..., :rot]
    if interleaved:
        return torch.stack((-r[..., 1::2], r[..., 0::2]), -1).flatten(-2)
    return torch.cat((-r[..., rot // 2:], r[..., :rot // 2]), -1)


def _spread(a, interleaved):
    """The table's columns at the elements that they turn."""
    return a.repeat_interleave(2, -1) if interleaved else torch.cat((a, a), -1)


def _turned(z, cos, sin, interleaved):
    """z with its first elements rotated; cos, sin broadcast over the heads."""
    rot = 2 * cos.shape[-1]
    if rot == 0:
        return z
    y = z[..., :rot] * _spread(cos, interleaved) + _partner(z, rot, interleaved) * _spread(sin, interleaved)
    return torch.cat((y, z[..., rot:]), -1)


def _normed(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _plain_rotate(x, w, cos, sin, interleaved):
    B, L, H, d = x.shape
    y = _turned(_normed(x.float(), w), cos[:, :, None], sin[:, :, None], interleaved)
    return y.transpose(1, 2).reshape(B * H, L, d).to(x.dtype)


def _plain_rotate_grad(dy, x, w, cos, sin, interleaved):
    B, L, H, d = x.shape
    dz = _turned(dy.float().view(B, H, L, d).transpose(1, 2), cos[:, :, None], -sin[:, :, None], interleaved)
    if w is None:
        return dz.to(x.dtype), None
    xf = x.float()
    r = torch.rsqrt(xf.square().mean(-1, keepdim=True) + EPS)
    g = dz * w.float()
    dx = r * (g - xf * (r.square() * (g * xf).mean(-1, keepdim=True)))
    return dx.to(x.dtype), (dz * xf * r).sum((0, 1, 2))


def _plain_store(cache, scale, x, at, slot, partial, old_slots, page):
    """x [T, Hk, d] into cache at pages `at`, slots `slot`; partial: pages that hold `old_slots` earlier tokens."""
    amax = torch.zeros_like(scale).index_reduce_(0, at, x.abs().amax(-1), "amax")
    fresh = torch.zeros(scale.shape[0], dtype=torch.bool, device=x.device)
    fresh[at] = True
    new = _scale_of(amax)
    grown = torch.maximum(new[partial], scale[partial])
    old = cache[partial].view(torch.float8_e4m3fn).float() * (scale[partial] / grown)[:, :, None, None]
    keep = torch.arange(page, device=x.device)[None, None, :, None] < old_slots[:, None, None, None]
    cache[partial] = torch.where(keep, old.to(torch.float8_e4m3fn).view(torch.uint8), cache[partial])
    new[partial] = grown
    scale.copy_(torch.where(fresh[:, None], new, scale))
    cache[at, :, slot] = (x / scale[at][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    c, page, Hk, d = s["c"], s["c"]["page"], s["c"]["Hk"], s["c"]["d"]
    K, V = s["kv"].view(-1, 2, Hk, d).float().unbind(1)
    cu, length = s["cu"].long(), s["len"].long()
    t = torch.arange(K.shape[0], device=K.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    i = length[b] - (cu[b + 1] - t)                       # the token's place in its sequence
    at, slot = s["table"].long()[b, i // page], i % page
    first = length - (cu[1:] - cu[:-1])                   # of every sequence's new tokens
    has = first % page > 0
    partial = s["table"].long().gather(1, (first // page)[:, None])[:, 0][has]
    K = _turned(_normed(K, s["w"]), s["cos"][i][:, None], s["sin"][i][:, None], c["interleaved"])
    _plain_store(s["k"], s["k_scale"], K, at, slot, partial, (first % page)[has], page)
    _plain_store(s["v"], s["v_scale"], V, at, slot, partial, (first % page)[has], page)


def _plain_read(cache, scale, table):
    """[B, Hk, W * page, d] of every sequence's pages."""
    at = table.long().clamp(min=0)
    x = cache[at].view(torch.float8_e4m3fn).float() * scale[at][..., None, None]
    B, W, Hk, page, d = x.shape
    return x.transpose(1, 2).reshape(B, Hk, W * page, d)


def _kept(S, N, M):
    """Which scores are among the N largest of their run of M; equal ones: the lower index."""
    r = S.unflatten(-1, (-1, M))
    a, b = r[..., :, None], r[..., None, :]
    lower = torch.ones((M, M), dtype=torch.bool, device=S.device).tril(-1)
    return (((b > a) | ((b == a) & lower)).sum(-1) < N).flatten(-2)


def _plain_attend(s):
    c, Hk, d = s["c"], s["c"]["Hk"], s["c"]["d"]
    G, most, dev = c["Hq"] // Hk, c["most"], s["Q"].device
    K, V = _plain_read(s["k"], s["k_scale"], s["table"]), _plain_read(s["v"], s["v_scale"], s["table"])
    B, L = K.shape[0], K.shape[2]
    cu, length = s["cu"].long(), s["len"].long()
    n = cu[1:] - cu[:-1]
    i = torch.arange(most, device=dev)
    row = (cu[:-1, None] + i).clamp(max=s["Q"].shape[0] - 1)
    Q = s["Q"][row].float().view(B, most, Hk, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hk, most * G, d)
    S = (Q @ K.transpose(-1, -2) * d ** -0.5).view(B, Hk, most, G, L)
    last = torch.where(i < n[:, None], length[:, None] - n[:, None] + i, 0) if c["causal"] else (length[:, None] - 1).expand(B, most)
    S = S.masked_fill((torch.arange(L, device=dev) > last[..., None])[:, None, :, None], -math.inf)
    if c["N"]:
        S = S.masked_fill(~_kept(S, c["N"], c["M"]), -math.inf)
    P = (S - S.amax(-1, keepdim=True).clamp(min=-1e30)).exp()
    P = P / P.sum(-1, keepdim=True).clamp(min=1e-30)
    O = (P.view(B, Hk, most * G, L) @ V).view(B, Hk, most, G, d).permute(0, 2, 1, 3, 4).reshape(B, most, c["Hq"], d)
    return O[i < n[:, None]].bfloat16()


def _split(s):
    """Queries and keys of the projection's rows."""
    c = s["c"]
    rows = s["qkv"].view(c["B"], c["L"], c["Hq"] + 2 * c["Hk"], c["d"])
    return rows[:, :, :c["Hq"]], rows[:, :, c["Hq"]:c["Hq"] + c["Hk"]]


def run(state):
    s, c = state, state["c"]
    if own:
        return _own(s, c)
    if c["op"] == "append":
        _plain_append(s)
        return _cache_of(s)
    if c["op"] == "attend":
        return _plain_attend(s)
    cos, sin = s["cos"][s["pos"].long()], s["sin"][s["pos"].long()]
    x = _split(s)
    if c["op"] == "rotate":
        return [_plain_rotate(x[i], s["w"][i], cos, sin, c["interleaved"]) for i in (0, 1)]
    return [_plain_rotate_grad(s["dY"][i], x[i], s["w"][i], cos, sin, c["interleaved"]) for i in (0, 1)]


def _cache_of(s):
    return {"k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn),
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ---- the library's calls ---------------------------------------------------------------------------------------


@functools.lru_cache(maxsize=None)
def _shape(*sizes):
    """The shape that a program keeps for its calls."""
    from paper_2203_00091_amd import Shape
    return Shape(*sizes)


def _own(s, c):
    import paper_2203_00091_amd as dfss

    B, d = c["B"], c["d"]
    if c["op"] in ("rotate", "rotate_grad"):
        Q, K = _split(s)
        shape = _shape(B, c["Hq"], c["L"], c["L"], d, 1, 2, dfss.DFSS_F32 if c["dtype"] == "f32" else dfss.DFSS_BF16)
        rotary = dfss.Rotary(s["cos"], s["sin"], s["pos"], c["interleaved"]) if c["rot"] else None
        if c["op"] == "rotate":
            return list(dfss.dfss_qk_norm_rotate(Q, K, s["w"][0], s["w"][1], rotary, shape, EPS))
        dQ, dK, dwq, dwk = dfss.dfss_qk_norm_rotate_backward(s["dY"][0], s["dY"][1], Q, K, s["w"][0], s["w"][1], rotary, shape, EPS)
        return [(dQ, dwq), (dK, dwk)]
    cache = dfss.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["len"])
    if c["op"] == "append":
        K, V = s["kv"].view(-1, 2, c["Hk"], d).unbind(1)
        rotary = dfss.Rotary(s["cos"], s["sin"], None, c["interleaved"])
        dfss.dfss_cache_append(K, V, s["cu"], cache, s["w"], rotary, _shape(B, c["Hk"], c["most"], c["max_len"], d), EPS)
        return _cache_of(s)
    shape = _shape(B, c["Hq"], c["most"], c["max_len"], d, c["N"], c["M"])
    call = dfss.dfss_attention_cached if c["N"] else dfss.dense_attention_cached
    return call(s["Q"], s["cu"], cache, shape, d ** -0.5, c["causal"])


# ---- work ------------------------------------------------------------------------------------------------------


def work(case):
    """Every input read once and every output written once (pages that are not touched are neither); of lengths and
    counts between half of and all the most, the mean."""
    c = case
    if c["op"] in ("rotate", "rotate_grad"):
        elem = 4 if c["dtype"] == "f32" else 2
        values = c["B"] * c["L"] * (c["Hq"] + c["Hk"]) * c["d"]
        norm_reads = 1 if c["op"] == "rotate" or not c["norm"] else 2
        return {"bytes": elem * values * (1 + norm_reads) + 4 * c["B"] * c["L"] * (1 + c["rot"] // 2 * 2 // max(1, c["B"])),
                "flops": values * (16 if c["op"] == "rotate_grad" else 8)}
    mean_n = c["most"] if c["most"] == 1 or c["B"] == 1 else 0.75 * c["most"]
    if c["op"] == "append":
        values = c["B"] * mean_n * c["Hk"] * c["d"]
        return {"bytes": values * 2 * (2 + 1) + c["B"] * mean_n * 4 * c["d"], "flops": values * 12}
    mean_len = c["max_len"] if c["B"] == 1 else 0.75 * c["max_len"]
    seen = c["B"] * c["Hq"] * mean_n * (mean_len - (mean_n / 2 if c["causal"] else 0))
    share = c["N"] / c["M"] if c["N"] else 1.0
    return {"bytes": 2 * c["B"] * mean_len * c["Hk"] * (c["d"] + 4 / c["page"]) + 4 * c["B"] * mean_n * c["Hq"] * c["d"],
            "flops": 2 * seen * c["d"] * (1 + share)}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------


def _pairs(rot, interleaved):
    """Index of the first and of the second element of every rotated pair."""
    i = torch.arange(rot // 2, device="cuda")
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _exact_rotation(z, cos, sin, interleaved):
    y = z.clone()
    if cos.shape[-1]:
        a, b = _pairs(2 * cos.shape[-1], interleaved)
        y[..., a] = z[..., a] * cos - z[..., b] * sin
        y[..., b] = z[..., b] * cos + z[..., a] * sin
    return y


def _values(codes):
    """What e4m3 codes stand for: sign, four bits of exponent (bias 7), three of fraction."""
    u = codes.to(torch.int32)
    e, f = (u >> 3) & 15, (u & 7).double()
    v = torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.exp2((e - 10).double()))
    return torch.where(u >= 128, -v, v)


def _nearest(q):
    """q at the nearest value of e4m3, ties to the even one."""
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(q / step) * step


def _exact_store(cache, scale, x, table, length, n, page):
    """Sequence by sequence and page by page."""
    values, scale, at = _values(cache), scale.double().clone(), 0
    for b in range(len(n)):
        start, end = int(length[b]) - int(n[b]), int(length[b])
        for p in range(start // page, -(-end // page)):
            lo, hi = max(start, p * page), min(end, (p + 1) * page)
            new, id = x[at + lo - start:at + hi - start].transpose(0, 1), int(table[b, p])
            amax = new.abs().amax((1, 2))
            want = torch.exp2(torch.ceil(torch.log2(amax / 448)).clamp(min=-64))
            if lo > p * page:
                grown = torch.maximum(scale[id], want)
                old = values[id, :, :lo - p * page]
                values[id, :, :lo - p * page] = _nearest(old * (scale[id] / grown)[:, None, None])
                want = grown
            scale[id] = want
            values[id, :, lo - p * page:hi - p * page] = _nearest(new / want[:, None, None])
        at += int(n[b])
    return values, scale


def exact(case, seed):
    c, s = dict(case), prepare(case, seed)
    d = c["d"]
    if c["op"] in ("rotate", "rotate_grad"):
        B, L, inter = c["B"], c["L"], c["interleaved"]
        cos, sin = (s[k].double()[s["pos"].long()][:, :, None] for k in ("cos", "sin"))
        out = []
        for i, x in enumerate(_split(s)):
            x, H = x.double(), x.shape[2]
            w = None if s["w"][i] is None else s["w"][i].double()
            r = (x.pow(2).sum(-1, keepdim=True) / d + EPS).pow(-0.5)
            if c["op"] == "rotate":
                y = _exact_rotation(x if w is None else x * r * w, cos, sin, inter)
                out.append(y.permute(0, 2, 1, 3).reshape(B * H, L, d))
                continue
            dz = _exact_rotation(s["dY"][i].double().view(B, H, L, d).permute(0, 2, 1, 3), cos, -sin, inter)
            if w is None:
                out.append((dz, None))
                continue
            xhat = x * r
            out.append((r * (dz * w - xhat * (dz * w * xhat).sum(-1, keepdim=True) / d), (dz * xhat).flatten(0, 2).sum(0)))
        return out
    n, length, table = s["n"], s["len"].cpu(), s["table"].cpu()
    if c["op"] == "append":
        if sum(-(-int(x) // c["page"]) + 1 for x in n) > 20000:
            return None
        K, V = s["kv"].double().view(-1, 2, c["Hk"], d).unbind(1)
        pos = torch.cat([torch.arange(int(l) - int(m), int(l)) for l, m in zip(length, n)]).cuda()
        if s["w"] is not None:
            K = K / (K.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * s["w"].double()
        K = _exact_rotation(K, s["cos"].double()[pos][:, None], s["sin"].double()[pos][:, None], c["interleaved"])
        k, ks = _exact_store(s["k"], s["k_scale"], K, table, length, n, c["page"])
        v, vs = _exact_store(s["v"], s["v_scale"], V, table, length, n, c["page"])
        return {"k": k, "v": v, "k_scale": ks, "v_scale": vs}
    G, at, out = c["Hq"] // c["Hk"], 0, []
    for b in range(c["B"]):
        m, l = int(n[b]), int(length[b])
        ids = table[b, :-(-l // c["page"])].long().cuda()
        K, V = ((_values(s[x][ids]) * s[x + "_scale"].double()[ids][..., None, None]).transpose(0, 1).flatten(1, 2)[:, :l]
                for x in ("k", "v"))
        O = []
        for h in range(c["Hk"]):
            q = s["Q"][at:at + m, h * G:(h + 1) * G].double().reshape(m * G, d)
            S = q @ K[h].T / math.sqrt(d)
            if c["causal"]:
                for i in range(m):
                    S[i * G:(i + 1) * G, l - m + i + 1:] = -math.inf
            if c["N"]:
                M = c["M"]
                R = torch.nn.functional.pad(S, (0, -l % M), value=-math.inf).unflatten(1, (-1, M))
                order = torch.sort(R, dim=-1, descending=True, stable=True).indices
                R = R.scatter(-1, order[..., c["N"]:], -math.inf)
                S = R.flatten(1)[:, :l]
            P = torch.softmax(S, -1)
            O.append((P @ V[h]).view(m, G, d))
        out.append(torch.cat(O, 1))
        at += m
    return torch.cat(out)
