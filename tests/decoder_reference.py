"""Plain 64-bit forms of the operators around a decoder's attention, on the CPU, one row, page or query at a time."""
import math

import torch


def rotate(z, cos, sin, interleaved):
    """z [..., d]; cos, sin [..., rot/2] of the row's position."""
    y, half = z.clone(), cos.shape[-1]
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y[..., a] = z[..., a] * cos - z[..., b] * sin
    y[..., b] = z[..., b] * cos + z[..., a] * sin
    return y


def norm(x, w, eps):
    return x if w is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w


def norm_rotate(x, w, table, pos, eps):
    """x [B, L, H, d] -> the same, normed and rotated.  table: (cos, sin, interleaved) or None; pos [B, L]."""
    z = norm(x.double(), None if w is None else w.double(), eps)
    if table is None:
        return z
    cos, sin, interleaved = table
    p = pos.long().clamp(0, cos.shape[0] - 1)
    return rotate(z, cos.double()[p][:, :, None], sin.double()[p][:, :, None], interleaved)


def codes_to_values(c):
    """e4m3: sign, 4 bits of exponent (bias 7), 3 of fraction."""
    u = c.to(torch.int32)
    e, f = (u >> 3) & 15, (u & 7).double()
    v = torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.exp2((e - 10).double()))
    v = torch.where(u & 127 == 127, torch.full_like(v, math.nan), v)
    return torch.where(u >= 128, -v, v)


def nearest(q):
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(q / step) * step


def scale_of(amax):
    """Least power of two s >= 2^-64 with amax / s <= 448."""
    k = -64
    while amax > 448 * 2.0 ** k:
        k += 1
    return 2.0 ** k


def append(values, scale, x, table, length, counts, page, max_len, n_pages):
    """x [tokens, Hk, d] (as they are to be kept) into values [n_pages, Hk, page, d] (of codes) and scale [n_pages, Hk], which
    are changed; returns the exact values of what was written, NaN elsewhere."""
    exact, at = torch.full_like(values, math.nan), 0
    limit = min(max_len, table.shape[1] * page)
    for b, n in enumerate(counts):
        start = int(length[b]) - n
        for p in range(max(start, 0) // page, (max(start + n, 0) + page - 1) // page):
            lo, hi = max(start, 0, p * page), min(start + n, limit, (p + 1) * page)
            if lo >= hi or not 0 <= int(table[b, p]) < n_pages:
                continue
            id = int(table[b, p])
            new = x[at + lo - start:at + hi - start].transpose(0, 1)      # [Hk, tokens, d]
            for h in range(x.shape[1]):
                s = scale_of(float(new[h].abs().max()))
                if lo > p * page:
                    old = float(scale[id, h])
                    if old >= s:
                        s = old
                    else:
                        values[id, h, :lo - p * page] = nearest(values[id, h, :lo - p * page] * (old / s))
                scale[id, h] = s
                exact[id, h, lo - p * page:hi - p * page] = new[h] / s
                values[id, h, lo - p * page:hi - p * page] = nearest(new[h] / s)
        at += n
    return exact


def attention(Q, counts, K, V, seen, length, max_len, N, M, scale, causal):
    """Q [tokens, H, d]; K, V [B][Hk, keys, d] of every sequence, seen [B][keys] (its page exists), 64 bits.  Returns O, sum p |v|
    and, per query and head, by how little the closest choice was made (inf without pruning)."""
    O, A, gap, at = torch.zeros_like(Q, dtype=torch.float64), torch.zeros_like(Q, dtype=torch.float64), torch.full(Q.shape[:2], math.inf, dtype=torch.float64), 0
    H = Q.shape[1]
    for b, n in enumerate(counts):
        G = H // K[b].shape[0]
        for i in range(n):
            keys = min(int(length[b]), max_len)
            if causal:
                keys = max(0, min(keys, int(length[b]) - n + i + 1))
            if keys == 0:
                continue
            k, v = (x[b][:, :keys].repeat_interleave(G, 0) for x in (K, V))
            S = (k @ Q[at + i].double()[:, :, None])[..., 0]
            S[:, ~seen[b][:keys]] = -math.inf
            if N:
                R = torch.nn.functional.pad(S, (0, -keys % M), value=-math.inf).unflatten(1, (-1, M))
                order = torch.sort(R, dim=-1, descending=True, stable=True)
                if N < M:
                    close = (order.values[..., N - 1] - order.values[..., N]).nan_to_num(nan=math.inf, posinf=math.inf)
                    close[close == 0] = math.inf        # ties are decided by the index
                    gap[at + i] = close.amin(1)
                S = R.scatter(-1, order.indices[..., N:], -math.inf).flatten(1)[:, :keys]
            m = S.amax(1, keepdim=True)
            P = torch.where(S == -math.inf, 0.0, torch.exp((S - m.clamp(min=-1e300)) * scale))
            total = P.sum(1, keepdim=True)
            P = torch.where(total > 0, P / total.clamp(min=1e-300), 0.0)
            O[at + i] = (P[:, None] @ torch.where(seen[b][:keys, None], v, 0.0))[:, 0]
            A[at + i] = (P[:, None] @ torch.where(seen[b][:keys, None], v, 0.0).abs())[:, 0]
        at += n
    return O, A, gap


def append_at_once(values, scale, x, table, length, counts, page, max_len, n_pages):
    """As append, all heads of a page at a time."""
    exact, at = torch.full_like(values, math.nan), 0
    limit = min(max_len, table.shape[1] * page)
    for b, n in enumerate(counts):
        start = int(length[b]) - n
        for p in range(max(start, 0) // page, (max(start + n, 0) + page - 1) // page):
            lo, hi, id = max(start, 0, p * page), min(start + n, limit, (p + 1) * page), int(table[b, p])
            if lo >= hi or not 0 <= id < n_pages:
                continue
            new = x[at + lo - start:at + hi - start].transpose(0, 1)
            m, e = torch.frexp(new.abs().amax((1, 2)))      # m 2^e with m in [0.5, 1); 448 = 0.875 * 2^9
            s = torch.where(m > 0, torch.ldexp(torch.ones_like(m), (e - 9 + (m > 0.875).int()).clamp(min=-64)), 2.0 ** -64)
            if lo > p * page:
                s = torch.maximum(s, scale[id])
                values[id, :, :lo - p * page] = nearest(values[id, :, :lo - p * page] * (scale[id] / s)[:, None, None])
            scale[id] = s
            exact[id, :, lo - p * page:hi - p * page] = new / s[:, None, None]
            values[id, :, lo - p * page:hi - p * page] = nearest(new / s[:, None, None])
        at += n
    return exact


def attention_at_once(Q, counts, K, V, seen, length, max_len, N, M, scale, causal):
    """As attention, all queries of a sequence at a time."""
    O, A, gap, at = torch.zeros_like(Q, dtype=torch.float64), torch.zeros_like(Q, dtype=torch.float64), torch.full(Q.shape[:2], math.inf, dtype=torch.float64), 0
    H = Q.shape[1]
    for b, n in enumerate(counts):
        G, keys, rows = H // K[b].shape[0], min(int(length[b]), max_len), slice(at, at + n)
        at += n
        if n == 0 or keys <= 0:
            continue
        k, v = (x[:, :keys].repeat_interleave(G, 0) for x in (K[b], torch.where(seen[b][:, None], V[b], 0.0)))
        S = Q[rows].double().transpose(0, 1) @ k.transpose(1, 2)                    # [H, n, keys]
        hidden = ~seen[b][:keys].expand(n, keys)
        if causal:
            hidden = hidden | (torch.arange(keys) > int(length[b]) - n + torch.arange(n)[:, None])
        S = S.masked_fill(hidden, -math.inf)
        if N:
            R = torch.nn.functional.pad(S, (0, -keys % M), value=-math.inf).unflatten(-1, (-1, M))
            order = torch.sort(R, dim=-1, descending=True, stable=True)
            if N < M:
                close = (order.values[..., N - 1] - order.values[..., N]).nan_to_num(nan=math.inf, posinf=math.inf)
                close[close == 0] = math.inf
                gap[rows] = close.amin(-1).T
            S = R.scatter(-1, order.indices[..., N:], -math.inf).flatten(-2)[..., :keys]
        m = S.amax(-1, keepdim=True)
        P = torch.where(S == -math.inf, 0.0, torch.exp((S - m.clamp(min=-1e300)) * scale))
        P = P / P.sum(-1, keepdim=True).clamp(min=1e-300)
        O[rows], A[rows] = (P @ v).transpose(0, 1), (P @ v.abs()).transpose(0, 1)
    return O, A, gap
