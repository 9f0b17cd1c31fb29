"""The decoder's calls with offsets that are none of a batch's, among rows that are nobody's; and generation against a prompt."""
import math

import decoder_reference as ref
import pytest
import test_gpu_cached_attention as cached
import torch
from test_gpu_cached_attention import DEV, MODES, Append, Attend

import paper_2203_00091_amd as dfss
from paper_2203_00091_amd import Cache, Rotary, Shape

pytestmark = pytest.mark.gpu


def _among(rows, filler):
    """The rows within a larger array, 64 rows of the filler on each side: (the array, its part)."""
    out = torch.full((rows.shape[0] + 128, *rows.shape[1:]), filler, dtype=rows.dtype, device=DEV)
    out[64:-64] = rows
    return out, out[64:-64]


# offsets as given, for T rows, and as they are cut: below 0, beyond the rows, and decreasing; every row is one sequence's
def _offsets(T, n):
    return [-3, n, T + 90, 5], [0, n, T, T]


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d, first, second", [(64, 2, 4), (128, 40, 20), (64, 100, 240), (128, 3, 70)])
def test_attention_cuts_offsets(first, second, d, mode):
    a = Attend(d, 16, 1, 2, [(300, first), (257, second), (90, 0)], 90)
    T = first + second
    given, cut = (torch.tensor(c, dtype=torch.int32, device=DEV) for c in _offsets(T, first))
    want = a.call(*mode)
    assert torch.equal(a.cu, cut)
    q, a.Q = _among(a.Q.contiguous(), math.nan)
    o, O = _among(torch.full((T, 2, d), 7.0, dtype=torch.bfloat16, device=DEV), 7.0)
    a.cu = given
    a.call(*mode, O=O)
    assert torch.equal(O, want) and bool((o[:64] == 7).all()) and bool((o[-64:] == 7).all())
    a.check(O, *mode)
    # fewer queries to a sequence than it has: the others' rows stay
    O.fill_(7)
    f = dfss.dfss_attention_cached if mode[0] else dfss.dense_attention_cached
    f(a.Q, a.cu, a.cache, Shape(3, 2, min(first, 3), a.max_len, d, mode[0] or 2, mode[1] or 4), a.scale, O=O)
    for at, n in ((0, first), (first, second)):
        k = min(n, 3, first)
        assert bool(O[at:at + k].ne(7).any()) and bool((O[at + k:at + n] == 7).all())
    assert bool((o[:64] == 7).all()) and bool((o[-64:] == 7).all())


@pytest.mark.parametrize("case", [(16, 64, 3, [(5, 40), (16, 33), (9, 0)], True, 64, False), (64, 128, 2, [(60, 7), (0, 130), (3, 0)], False, 0, False),
                                  (32, 128, 13, [(1, 1), (31, 2), (7, 0)], True, 128, True)], ids=str)
def test_append_cuts_offsets(case):
    """Codes and scales as with the offsets that they are cut to, NaN rows on both sides; pages that are nobody's stay."""
    a = Append(case, 91)
    T, Hk = a.T, a.Hk
    given, cut = _offsets(T, a.counts[0])
    want = a.call()
    _, rows = _among(a.rows, math.nan)
    cache = Cache(*(x.to(DEV) for x in (a.k, a.v, a.k_scale, a.v_scale, a.table)), torch.tensor(a.lengths, dtype=torch.int32).to(DEV))
    rotary = Rotary(a.angles[0].to(DEV), a.angles[1].to(DEV), None, a.interleaved) if a.rot else None
    s = Shape(3, Hk, 1, a.max_len, a.d)
    w = None if a.w is None else a.w.to(DEV)

    def call(cu):
        dfss.dfss_cache_append(rows[:, 1:1 + Hk], rows[:, 1 + Hk:], torch.tensor(cu, dtype=torch.int32, device=DEV), cache, w, rotary, s, cached.EPS)

    call(given)
    for name in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(cache, name), getattr(want, name)), name
    a.check(cache)
    # offsets that decrease between sequences: whose rows a page has is open, but they are rows, and in pages that a sequence has
    before = [x.clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    call([0, T, 1, T])
    call([T, 0, -5, T])
    mine = torch.zeros(a.n_pages, dtype=torch.bool)
    mine[a.table[a.table >= 0].long()] = True
    for x, y in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        assert torch.equal(x[~mine], y[~mine])
    assert bool(cache.k_scale.isfinite().all()) and bool(cache.v_scale.isfinite().all())


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d, page", [(64, 16), (128, 64)])
def test_generation_is_what_a_prompt_at_once_is(d, page, mode):
    """Norm, append and attention token by token, and for all tokens in one call each.  The values keep every page's scale at that of its
    first token (a normed row of +-1 rotated: 1 to 1.42; V: one element of 1.5, the others smaller), so the caches are the same bits."""
    L, Hq, Hk = 201, 4, 2
    g = torch.Generator().manual_seed(92)
    qkv = torch.randn((L, Hq + 2 * Hk, d), generator=g)
    qkv[:, Hq:Hq + Hk] = qkv[:, Hq:Hq + Hk].sign() + (qkv[:, Hq:Hq + Hk] == 0)
    qkv[:, Hq + Hk:] = qkv[:, Hq + Hk:].clamp(-1.4, 1.4)
    qkv[:, Hq + Hk:, 0] = 1.5
    qkv = qkv.bfloat16().to(DEV)
    w = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    angle = torch.arange(L, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    cos, sin = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    W = -(-L // page)
    table = torch.randperm(W, generator=g).int()[None].to(DEV)

    def new():
        codes = [torch.full((W, Hk, page, d), cached.NOTHING, dtype=torch.uint8, device=DEV) for _ in range(2)]
        return (*codes, *(torch.ones((W, Hk), device=DEV) for _ in range(2)))

    def run(data, at, n):
        """Tokens at .. at + n - 1."""
        x, pos = qkv[at:at + n], torch.arange(at, at + n, dtype=torch.int32, device=DEV)[None]
        cache = Cache(*data, table, torch.tensor([at + n], dtype=torch.int32, device=DEV))
        s = Shape(1, Hq, n, L, d, mode[0] or 2, mode[1] or 4)
        Q, _ = dfss.dfss_qk_norm_rotate(x[None, :, :Hq], None, w, None, Rotary(cos, sin, pos), Shape(1, Hq, n, n, d))
        dfss.dfss_cache_append(x[:, Hq:Hq + Hk], x[:, Hq + Hk:], None, cache, w, Rotary(cos, sin), Shape(1, Hk, n, L, d))
        f = dfss.dfss_attention_cached if mode[0] else dfss.dense_attention_cached
        return Q, f(Q.transpose(0, 1), None, cache, s, d ** -0.5)

    one, many, parts = new(), new(), new()
    steps = [run(one, t, 1) for t in range(L)]
    Q, O = run(many, 0, L)
    chunks = [run(parts, at, n) for at, n in ((0, 7), (7, 90), (97, 1), (98, L - 98))]
    for got in (steps, chunks):
        assert torch.equal(torch.cat([q for q, _ in got], 1), Q)
    for a, b, c in zip(one, many, parts):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert bool((many[2] == 2.0 ** -8).all()) and bool((many[3] == 2.0 ** -8).all())
    ids = table[0].cpu().long()
    K, V = ((ref.codes_to_values(x.cpu()[ids]).nan_to_num(nan=0.0) * 2.0 ** -8).transpose(0, 1).reshape(Hk, W * page, d)[:, :L] for x in many[:2])
    want, amount, gap = ref.attention_at_once(Q.transpose(0, 1).cpu(), [L], [K], [V], [torch.ones(L, dtype=torch.bool)], [L], L, *mode, d ** -0.5, True)
    half, clear = torch.finfo(torch.bfloat16).eps / 2, gap > 1e-4      # (as in Attend.check)
    assert float(clear.double().mean()) > 0.9
    tol = half * want.abs() + (half + 1e-5) * (amount + want.abs()) * 1.01
    for got in (O, torch.cat([o for _, o in steps]), torch.cat([o for _, o in chunks])):
        assert float(((got.cpu().double() - want).abs() - tol)[clear].max()) <= 0


@pytest.mark.parametrize("B", [64, 65, 4096, 4097, 5000])
def test_append_finds_its_sequence_among_many(B):
    """One token to most sequences, none to some, and a prompt here and there."""
    a = Append((16, 64, 1, [((5 * i) % 33, 0 if i % 5 == 2 else 40 if i % 701 == 63 else 1) for i in range(B)], False, 0, False), 93)
    cache = a.call()
    for x, codes, scale, got, got_scale in ((a.rows[:, 1:2], a.k, a.k_scale, cache.k, cache.k_scale), (a.rows[:, 2:], a.v, a.v_scale, cache.v, cache.v_scale)):
        values, want = ref.codes_to_values(codes), scale.double().clone()
        ref.append_at_once(values, want, x.cpu().double(), a.table, a.lengths, a.counts, 16, a.max_len, a.n_pages)
        assert torch.equal(got_scale.cpu().double(), want)
        assert torch.equal(ref.codes_to_values(got.cpu()).nan_to_num(nan=999.0), values.nan_to_num(nan=999.0))
