"""The paged cache of 8 bits: what dfss_cache_append leaves in it, and attention over it, against plain forms in 64 bits."""
import math

import decoder_reference as ref
import pytest
import torch

import paper_2203_00091_amd as dfss
from paper_2203_00091_amd import Cache, Rotary, Shape

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6
NOTHING = 0x7F      # the code of a NaN: what no call may read a value from


def _table(g, lengths, page, n_pages, width):
    """Every sequence's pages, in no order; -1 where it has none."""
    order, t, at = torch.randperm(n_pages, generator=g).tolist(), torch.full((len(lengths), width), -1, dtype=torch.int32), 0
    for b, n in enumerate(lengths):
        for p in range((n + page - 1) // page):
            t[b, p] = order[at]
            at += 1
    return t


def _filled(g, n_pages, Hk, page, d, integers=False):
    """Codes of normal values (or of small integers) and scales that differ by page and head, as they are kept."""
    x = torch.randint(-3, 4, (n_pages, Hk, page, d), generator=g).float() if integers else torch.randn((n_pages, Hk, page, d), generator=g) * 100
    scale = torch.ones(n_pages, Hk) if integers else torch.exp2(torch.randint(-8, -4, (n_pages, Hk), generator=g).float())
    # (beyond 464 the conversion gives a NaN, which no cache holds as a value: one of these, at 465.5, would be 1 in 2e5)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _clear_behind(codes, table, lengths, page):
    """NaN codes in every page that is nobody's and behind every sequence's last token."""
    keep = torch.zeros(codes.shape[0], page, dtype=torch.bool)
    for b, n in enumerate(lengths):
        for p in range((n + page - 1) // page):
            if 0 <= int(table[b, p]) < codes.shape[0]:
                keep[int(table[b, p]), :min(page, n - p * page)] = True
    codes[~keep[:, None, :, None].expand_as(codes)] = NOTHING


# ---- appending ---------------------------------------------------------------------------------------------------

APPENDS = [
    # page, d, Hk, [(tokens before, new tokens)], norm, rot, interleaved
    (16, 64, 1, [(0, 1)], True, 64, False),
    (64, 128, 3, [(0, 0), (5, 1), (63, 1), (64, 1), (127, 2), (0, 64)], True, 128, False),
    (16, 128, 2, [(0, 15), (0, 16), (0, 17), (15, 1), (15, 2), (16, 100), (3, 0), (7, 200)], False, 32, True),
    (32, 64, 5, [(31, 33), (1, 95), (0, 31), (0, 0)], True, 48, False),
    (128, 128, 2, [(100, 300), (0, 129), (127, 1)], True, 128, True),
    (128, 64, 2, [(130, 70), (0, 1)], False, 0, False),
    (64, 128, 2, [(5, 60)] + [(10, 1)] * 69, True, 64, False),      # a prompt among single tokens
    (64, 64, 12, [(10, 3)] * 70, True, 64, False),          # more sequences than lanes
]


class Append:
    def __init__(self, case, seed, size=1.0, uniform=False):
        page, d, Hk, sequences, norm, rot, interleaved = case
        g = torch.Generator().manual_seed(seed)
        self.page, self.d, self.Hk = page, d, Hk
        self.before, self.counts = [a for a, _ in sequences], [n for _, n in sequences]
        self.lengths = [a + n for a, n in sequences]
        width = (max(self.lengths) + page - 1) // page + 1
        self.n_pages = sum((n + page - 1) // page for n in self.lengths) + 2
        self.table = _table(g, self.lengths, page, self.n_pages, width)
        self.max_len = width * page
        self.k, self.k_scale = _filled(g, self.n_pages, Hk, page, d)
        self.v, self.v_scale = _filled(g, self.n_pages, Hk, page, d)
        for c in (self.k, self.v):
            _clear_behind(c, self.table, self.before, page)
        T = sum(self.counts)
        rows = torch.randn((T, 2 * Hk + 1, d), generator=g) * torch.exp2(torch.randint(-3, 4, (T, 2 * Hk + 1, 1), generator=g).float()) * size
        self.rows = rows.bfloat16().to(DEV)
        self.w = (1 + 0.3 * torch.randn(d, generator=g)).bfloat16() if norm else None
        self.rot, self.interleaved, self.angles = rot, interleaved, None
        if rot:
            a = torch.rand((self.max_len, rot // 2), generator=g, dtype=torch.float64) * 6.3
            self.angles = (a.cos().float(), a.sin().float())
        self.pos = None
        self.uniform = uniform
        self.T = T

    def call(self, k=None, table=None, lengths=None, max_len=None):
        cache = Cache(*(x.to(DEV) for x in (self.k, self.v, self.k_scale, self.v_scale)),
                      (self.table if table is None else table).to(DEV), torch.tensor(self.lengths if lengths is None else lengths, dtype=torch.int32).to(DEV))
        rotary = Rotary(self.angles[0].to(DEV), self.angles[1].to(DEV), None if self.pos is None else self.pos.int().to(DEV), self.interleaved) if self.rot else None
        cu = None if self.uniform else torch.tensor([0] + self.counts).cumsum(0).int().to(DEV)
        s = Shape(len(self.counts), self.Hk, self.counts[0] if self.uniform else 1, max_len or self.max_len, self.d)
        dfss.dfss_cache_append(self.rows[:, 1:1 + self.Hk], self.rows[:, 1 + self.Hk:], cu, cache, None if self.w is None else self.w.to(DEV), rotary, s, EPS)
        return cache

    def check(self, cache, table=None, lengths=None, max_len=None):
        table, lengths = self.table if table is None else table, self.lengths if lengths is None else lengths
        K, V = self.rows[:, 1:1 + self.Hk].cpu(), self.rows[:, 1 + self.Hk:].cpu().double()
        pos = self.pos if self.pos is not None else torch.cat([torch.arange(n) + l - n for l, n in zip(lengths, self.counts)])
        angles = None if self.angles is None else (*self.angles, self.interleaved)
        K = ref.norm_rotate(K[None], self.w, angles, pos[None], EPS)[0]
        # of every value, how far 32 bits on the way may move it (the amount is the rotated pair's)
        for x, codes, scale, got, got_scale in ((K, self.k, self.k_scale, cache.k, cache.k_scale), (V, self.v, self.v_scale, cache.v, cache.v_scale)):
            values, want_scale = ref.codes_to_values(codes), scale.double().clone()
            exact = ref.append(values, want_scale, x, table, lengths, self.counts, self.page, max_len or self.max_len, self.n_pages)
            assert torch.equal(got_scale.cpu().double(), want_scale)
            have = ref.codes_to_values(got.cpu())
            new = ~exact.isnan()
            # half a step of e4m3, at the place where the value lies
            half = torch.exp2(torch.floor(torch.log2(exact[new].abs().clamp(min=2.0 ** -6))) - 4)
            assert bool(((have[new] - exact[new]).abs() <= half * (1 + 1e-5) + 1e-6 * 448).all())
            # nearly all are the nearest value's code: the others lie on a border, up to 32-bit arithmetic
            assert float((have[new] != values[new]).double().mean()) <= 1e-4
            same = torch.where(new, 0, have.nan_to_num(nan=999.0)) == torch.where(new, 0, values.nan_to_num(nan=999.0))
            assert bool(same.all())     # earlier tokens (rounded again where the scale grew), and all that is not touched


@pytest.mark.parametrize("size", [2.0 ** -9, 1.0, 2.0 ** 9])
@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append(case, size):
    """New values much smaller than, like, and much larger than what the pages hold."""
    a = Append(case, 21, size)
    a.check(a.call())


def test_append_the_same_count_to_every_sequence():
    a = Append((32, 128, 2, [(0, 40), (31, 40), (32, 40), (60, 40)], True, 64, False), 22, uniform=True)
    a.check(a.call())


def test_append_at_positions_of_the_callers():
    a = Append((16, 64, 2, [(3, 20), (0, 2)], True, 64, False), 23)
    a.pos = torch.randint(-2, a.max_len + 3, (a.T,), generator=torch.Generator().manual_seed(3))
    a.check(a.call())


def test_append_without_a_place():
    """No page, no room, before the first place: such tokens are not kept, and nothing else changes."""
    a = Append((16, 128, 2, [(10, 30), (0, 40), (20, 25), (0, 12)], False, 0, False), 24)
    t = a.table.clone()
    t[0, 1], t[2, 2] = a.n_pages, -7
    a.check(a.call(table=t), table=t)
    lengths = [40, 33, 45, 5]              # more new tokens than tokens: the first ones have no place
    a.check(a.call(lengths=lengths), lengths=lengths)
    a.check(a.call(max_len=30), max_len=30)
    negative = [40, -5, 45, 12]
    assert torch.equal(a.call(lengths=negative).k[a.table[1, 0].item()], a.k[a.table[1, 0].item()].to(DEV))


def test_append_zeros_and_the_border_of_a_scale():
    a = Append((16, 64, 1, [(0, 3), (0, 1), (0, 1)], False, 0, False), 25)
    a.rows[:3] = 0
    a.rows[3] = 448.0           # exactly what a scale of 1 holds
    a.rows[4] = 450.0           # (the next bfloat16) needs 2
    c = a.call()
    assert c.k_scale[a.table[:, 0].long()].flatten().tolist() == [2.0 ** -64, 1.0, 2.0]
    assert ref.codes_to_values(c.v[a.table[1, 0].item(), 0, 0].cpu()).eq(448).all()
    assert ref.codes_to_values(c.v[a.table[2, 0].item(), 0, 0].cpu()).eq(224).all()     # 225 lies between 224 and 240
    a.check(c)


# ---- attention ---------------------------------------------------------------------------------------------------


class Attend:
    def __init__(self, d, page, Hk, G, sequences, seed, integers=False, bad=(), shared=False, uniform=False, size=1.0):
        """sequences: (tokens, queries); bad: (sequence, entry of its table) without a page; shared: all have the first page
        of the first."""
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.counts = [a for a, _ in sequences], [n for _, n in sequences]
        self.d, self.page, self.Hk, self.H = d, page, Hk, Hk * G
        width = max((max(self.lengths) + page - 1) // page, 1)
        n_pages = sum((max(n, 0) + page - 1) // page for n in self.lengths) + 3
        self.table = _table(g, self.lengths, page, n_pages, width)
        if shared:
            self.table[:, 0] = self.table[0, 0]
        for b, p in bad:
            self.table[b, p] = n_pages + 5 if p % 2 else -1
        self.k, self.k_scale = _filled(g, n_pages, Hk, page, d, integers)
        self.v, self.v_scale = _filled(g, n_pages, Hk, page, d, integers)
        for c in (self.k, self.v):
            _clear_behind(c, self.table, self.lengths, page)
        T = sum(self.counts)
        q = torch.randint(-2, 3, (T, self.H + 3, d), generator=g).float() if integers else torch.randn((T, self.H + 3, d), generator=g) * size
        self.Q = q.bfloat16().to(DEV)[:, 1:1 + self.H]
        self.uniform, self.max_q, self.max_len = uniform, max(max(self.counts), 1), max(max(self.lengths), 1)
        self.scale = 0.25 if integers else d ** -0.5
        self.cache = Cache(*(x.to(DEV) for x in (self.k, self.v, self.k_scale, self.v_scale)), self.table.to(DEV),
                           torch.tensor(self.lengths, dtype=torch.int32).to(DEV))
        self.cu = None if uniform else torch.tensor([0] + self.counts).cumsum(0).int().to(DEV)

    def shape(self, N, M, max_len=None):
        return Shape(len(self.counts), self.H, self.max_q, max_len or self.max_len, self.d, N or 2, M or 4)

    def call(self, N, M, causal=True, max_len=None, **kw):
        f = dfss.dfss_attention_cached if N else dfss.dense_attention_cached
        return f(self.Q, self.cu, self.cache, self.shape(N, M, max_len), self.scale, causal, **kw)

    def reference(self, N, M, causal=True, max_len=None):
        K, V, seen = [], [], []
        for b, n in enumerate(self.lengths):
            e = (max(n, 0) + self.page - 1) // self.page
            ids = self.table[b, :e].long()
            ok = (ids >= 0) & (ids < self.k.shape[0])
            at = ids.clamp(0, self.k.shape[0] - 1)
            for out, c, s in ((K, self.k, self.k_scale), (V, self.v, self.v_scale)):
                x = ref.codes_to_values(c[at]).nan_to_num(nan=0.0) * s.double()[at][..., None, None]
                out.append(x.transpose(0, 1).reshape(self.Hk, e * self.page, self.d)[:, :max(n, 0)])
            seen.append(ok.repeat_interleave(self.page)[:max(n, 0)])
        return ref.attention(self.Q.cpu().double(), self.counts, K, V, seen, [max(n, 0) for n in self.lengths], max_len or self.max_len, N, M, self.scale, causal)

    def check(self, O, N, M, causal=True, max_len=None, all_rows=False):
        want, amount, gap = self.reference(N, M, causal, max_len)
        clear = gap > 1e-4 * (0 if all_rows else 1)     # a choice by less than 32 bits of the scores hold may go either way
        assert float(clear.double().mean()) > 0.9 or want.numel() < 2000
        # O is rounded to bfloat16, and so is every weight, in the sum as in the product: half a step of |O| for the first,
        # half a step of sum p |v| and of |O| for the second; 1e-5 for 32-bit sums and exponentials; weights below 2^-126, the
        # least normal number, are 0: 10000 keys x 2^-126 x |v| <= 448 is 6e-32
        half = torch.finfo(torch.bfloat16).eps / 2
        tol = half * want.abs() + (half + 1e-5) * (amount + want.abs()) * 1.01 + 6e-32
        off = ((O.cpu().double() - want).abs() - tol)[clear]
        assert bool(O.isfinite().all())
        assert off.numel() == 0 or float(off.max()) <= 0


MODES = [(2, 4), (1, 2), (0, 0)]
RAGGED = [(1, 1), (2, 1), (3, 3), (15, 1), (16, 5), (17, 2), (63, 1), (64, 64), (65, 7), (0, 0), (130, 0), (200, 33), (700, 3), (5, 5)]


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_lengths(d, page, mode):
    a = Attend(d, page, 2, 3, RAGGED, 31)
    for causal in (True, False):
        a.check(a.call(*mode, causal), *mode, causal)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 16, 17, 40])
def test_shared_heads(d, G, mode):
    a = Attend(d, 32, 1 if G > 16 else 3, G, [(100, 1), (333, 1), (31, 1), (1, 1)], 32, uniform=True)
    a.check(a.call(*mode), *mode)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_ties_are_decided_by_the_lower_key(d, mode):
    """Small integers: scores are exact and hundreds of them equal."""
    a = Attend(d, 16, 2, 2, [(257, 9), (90, 1), (33, 33), (1030, 2)], 33, integers=True)
    a.check(a.call(*mode), *mode, all_rows=True)
    a.check(a.call(*mode, causal=False), *mode, causal=False, all_rows=True)


@pytest.mark.parametrize("mode", MODES, ids=str)
def test_many_queries(mode):
    for d, page in ((64, 64), (128, 16)):
        a = Attend(d, page, 2, 4, [(300, 130), (513, 513), (128, 77), (40, 1)], 34)
        a.check(a.call(*mode), *mode)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_long_sequences_are_shared(d, mode):
    """Several workgroups to a sequence; short ones among long ones; any contents of the workspace."""
    a = Attend(d, 64, 2, 2, [(9000, 1), (40, 1), (0, 1), (4500, 1), (257, 1)], 35, uniform=True)
    need = dfss.dfss_cached_workspace_bytes(a.shape(*mode), a.cache)
    assert need > 0
    got = [a.call(*mode, ws=torch.full((need,), fill, dtype=torch.uint8, device=DEV)) for fill in (0, 255)]
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], a.call(*mode))
    a.check(got[0], *mode)
    b = Attend(d, 16, 1, 3, [(2700, 40), (1100, 7)], 36)
    assert dfss.dfss_cached_workspace_bytes(b.shape(*mode), b.cache) > 0
    b.check(b.call(*mode), *mode)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("longest, least", [(6000, 6000), (6000, 1), (6000, 0), (5200, 4000)])
def test_few_shares_to_a_sequence(longest, least, mode):
    """Sixteen sequences on a chip that holds 32 shares of them: all alike, most of them empty or of one key, and all but alike."""
    lengths = [longest if least == longest or b % 5 == 3 else least + 29 * b * (least > 1) for b in range(16)]
    a = Attend(128, 64, 8, 4, [(n, 1) for n in lengths], 53, uniform=True)
    assert dfss.dfss_cached_workspace_bytes(a.shape(*mode), a.cache) > 0
    a.check(a.call(*mode), *mode)


@pytest.mark.parametrize("mode", MODES, ids=str)
def test_rows_that_see_nothing(mode):
    """No tokens, more queries than tokens (the first ones stand before the first key), and pages that are none."""
    a = Attend(64, 16, 1, 2, [(0, 3), (4, 9), (70, 2), (33, 1), (16, 1), (-4, 2)], 37, bad=[(2, 1), (2, 3), (3, 0), (3, 2), (4, 0)])
    O = a.call(*mode)
    a.check(O, *mode, all_rows=True)
    assert not O[:3].any() and not O[3:8].any() and not O[15].any() and O[8:12].any()
    b = Attend(128, 128, 2, 1, [(300, 2), (140, 1)], 38, bad=[(0, 0), (0, 2), (1, 1)])
    b.check(b.call(*mode), *mode)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("queries", [1, 4, 70])
def test_pages_that_are_none_and_a_page_nobody_names(queries, page, d, mode):
    """Rows of every size of tile, the first of them before the first key; what lies in a page that no sequence names, its
    scales included, is nobody's."""
    a = Attend(d, page, 2, 5, [(0, queries), (queries // 2 + 1, queries), (260, queries), (130, 1), (-3, 1)], 50,
               bad=[(2, 0), (2, 2), (2, 3), (3, 1)])
    spare = next(i for i in range(1, a.k.shape[0]) if not bool((a.table == i).any()))
    for x in (a.k, a.v, a.k_scale, a.v_scale):
        x[spare] = x[0]
    a.table[a.table == 0] = spare
    want = a.reference(*mode)[0]
    a.check(O := a.call(*mode), *mode)      # (the cache on the device is as it was, with page 0 in its place)
    for x in (a.k, a.v):
        x[0] = 0x7F                         # no number
    a.k_scale[0], a.v_scale[0] = math.inf, math.nan
    a.cache = Cache(*(x.to(DEV) for x in (a.k, a.v, a.k_scale, a.v_scale)), a.table.to(DEV), a.cache.len)
    assert torch.equal(a.reference(*mode)[0], want) and torch.equal(a.call(*mode), O)


@pytest.mark.parametrize("mode", MODES, ids=str)
def test_the_call_sees_no_more_keys_than_it_names(mode):
    a = Attend(64, 32, 2, 1, [(200, 1), (90, 1), (150, 1)], 39, uniform=True)
    a.check(a.call(*mode, causal=False, max_len=100), *mode, causal=False, max_len=100)


def test_a_page_of_several_sequences():
    a = Attend(128, 64, 2, 2, [(100, 1), (170, 1), (64, 1)], 40, shared=True, uniform=True)
    a.check(a.call(2, 4), 2, 4)


@pytest.mark.parametrize("mode", MODES, ids=str)
def test_scores_far_apart(mode):
    """A few keys carry all the weight; the reference is raised again and again."""
    a = Attend(64, 16, 1, 4, [(400, 1), (1000, 5)], 41, size=8.0)
    a.check(a.call(*mode), *mode)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("scale", [2.0 ** -14, 1.0, 64.0])
@pytest.mark.parametrize("queries", [1, 100])
def test_any_scale(queries, scale, mode):
    """Nearly equal weights, and one key with all of it: equal scores are exact ones of whole numbers."""
    for d, page in ((64, 64), (128, 16)):
        a = Attend(d, page, 1, 4, [(300, queries), (130, queries)], 47, integers=True)
        a.scale = scale
        a.check(a.call(*mode), *mode, all_rows=True)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("scale, size", [(2.0 ** -100, 1.0), (2.0 ** 100, 2.0 ** -102)])
@pytest.mark.parametrize("queries", [1, 100])
def test_the_least_and_largest_scales(queries, scale, size, mode):
    """Level weights of what is seen and none of what is hidden; and scaled scores as usual from very small ones."""
    for d, page in ((64, 64), (128, 16)):
        a = Attend(d, page, 1, 4, [(300, queries), (130, queries), (2, 1)], 49, integers=True)
        a.scale, a.Q = scale, a.Q * size
        a.check(a.call(*mode), *mode, all_rows=True)


def test_rows_of_no_sequence_stay():
    a = Attend(64, 16, 1, 2, [(50, 3), (20, 1)], 42)
    a.Q = torch.cat((a.Q, a.Q))
    O = torch.full((8, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    a.call(2, 4, O=O)
    assert bool((O[4:] == 7).all())
    a.Q = a.Q[:4]
    a.check(O[:4], 2, 4)
    # fewer queries to a sequence than it has: the others are not computed
    O.fill_(7)
    s = Shape(2, 2, 2, 50, 64, 2, 4)
    whole = a.call(2, 4)
    dfss.dfss_attention_cached(a.Q, a.cu, a.cache, s, a.scale, O=O[:4])
    assert torch.equal(O[[0, 1, 3]], whole[[0, 1, 3]]) and bool((O[2] == 7).all())


def test_offsets_that_are_cut():
    """Offsets outside the rows, or decreasing: nothing outside the arrays is read or written."""
    a = Attend(64, 16, 1, 1, [(40, 2), (40, 2), (40, 2)], 43)
    O = torch.full((6, 1, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    a.cu = torch.tensor([-3, 2, 1, 90], dtype=torch.int32, device=DEV)
    a.call(2, 4, O=O)
    assert O.isfinite().all()


def test_the_whole_step_captured_with_sequences_that_grow():
    """A decoder's step -- queries normed and rotated, keys and values appended, attention -- in one graph whose cache has room to
    grow, against the same calls made one by one; and its result against the plain form over what the cache holds."""
    B, Hq, Hk, d, page, room = 3, 8, 2, 64, 16, 2048
    g = torch.Generator().manual_seed(44)
    width = room // page
    angles = torch.rand((room, d // 2), generator=g, dtype=torch.float64) * 6.3
    rotary_tables = (angles.cos().float().to(DEV), angles.sin().float().to(DEV))
    table = torch.randperm(B * width, generator=g).int().view(B, width).to(DEV)
    length = torch.tensor([0, 700, 15], dtype=torch.int32, device=DEV)
    codes = [torch.randint(0, 120, (B * width, Hk, page, d), generator=g).to(torch.uint8).to(DEV) for _ in range(2)]
    scales = [torch.full((B * width, Hk), 2.0 ** -8, device=DEV) for _ in range(2)]
    w = (1 + 0.2 * torch.randn(2, d, generator=g)).bfloat16().to(DEV)
    qkv = torch.empty((B, 1, Hq + 2 * Hk, d), dtype=torch.bfloat16, device=DEV)
    s, sk = Shape(B, Hq, 1, room, d, 2, 4), Shape(B, Hk, 1, room, d)
    pos = torch.empty((B, 1), dtype=torch.int32, device=DEV)

    def step(codes, scales, length, ws):
        length += 1
        torch.sub(length[:, None], 1, out=pos)
        cache = Cache(*codes, *scales, table, length)
        Q, _ = dfss.dfss_qk_norm_rotate(qkv[:, :, :Hq], None, w[0], None, Rotary(*rotary_tables, pos), s, EPS)
        dfss.dfss_cache_append(qkv[:, 0, Hq:Hq + Hk], qkv[:, 0, Hq + Hk:], None, cache, w[1], Rotary(*rotary_tables), sk, EPS)
        return cache, dfss.dfss_attention_cached(Q.view(B, Hq, d), None, cache, s, d ** -0.5, ws=ws), Q

    need = dfss.dfss_cached_workspace_bytes(s, Cache(*codes, *scales, table, length))
    ws = [torch.empty(max(need, 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    other = [c.clone() for c in codes], [x.clone() for x in scales], length.clone()
    qkv.normal_()
    warm = [c.clone() for c in codes], [x.clone() for x in scales], length.clone()
    step(*warm, ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, O, _ = step(codes, scales, length, ws[0])
    for k in range(20):
        qkv.copy_(torch.randn(qkv.shape, generator=g) * 2.0 ** (k % 5 - 2))
        graph.replay()
        torch.cuda.synchronize()
        cache, eager, Q = step(*other, ws[1])
        assert torch.equal(O, eager) and torch.equal(length, other[2])
        assert all(torch.equal(a, b) for a, b in zip(codes + scales, other[0] + other[1]))
    n = length.tolist()
    K, V, seen = [], [], []
    for b in range(B):
        ids = table[b].cpu().long()
        for out, c, x in ((K, codes[0], scales[0]), (V, codes[1], scales[1])):
            v = ref.codes_to_values(c.cpu()[ids]).nan_to_num(nan=0.0) * x.cpu().double()[ids][..., None, None]
            out.append(v.transpose(0, 1).reshape(Hk, room, d)[:, :n[b]])
        seen.append(torch.ones(n[b], dtype=torch.bool))
    want, amount, gap = ref.attention(Q.view(B, Hq, d).cpu(), [1] * B, K, V, seen, n, room, 2, 4, d ** -0.5, True)
    half = torch.finfo(torch.bfloat16).eps / 2
    clear = gap > 1e-5
    off = (O.cpu().double() - want).abs() - half * want.abs() - (half + 1e-5) * (amount + want.abs()) * 1.01
    assert clear.any() and float(off[clear].max()) <= 0


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_through_the_cache_and_through_the_plain_calls(d):
    """The cache's contents are bfloat16 numbers: over the same keys and values the library's other calls say the same."""
    a = Attend(d, 64, 4, 1, [(512, 128)], 45)
    ids = a.table[0].long()
    K, V = ((ref.codes_to_values(c[ids]) * s.double()[ids][..., None, None]).transpose(0, 1).reshape(4, 512, d) for c, s in ((a.k, a.k_scale), (a.v, a.v_scale)))
    assert torch.equal(K.bfloat16().double(), K)
    Q = a.Q.transpose(0, 1).contiguous()
    want = dfss.dfss_attention_causal(Q, K.bfloat16().to(DEV), V.bfloat16().to(DEV), None, Shape(1, 4, 128, 512, d), a.scale)
    got = a.call(2, 4).transpose(0, 1)
    # each of the two is within two roundings of the weights and one of O (test_lengths); near ties may differ
    off = (got.double() - want.double()).norm() / want.double().norm()
    assert float(off) < 2 * 3 * torch.finfo(torch.bfloat16).eps / 2


def test_another_stream():
    a = Attend(128, 32, 2, 2, [(3000, 1), (20, 1)], 46, uniform=True)
    want, side = a.call(2, 4), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = a.call(2, 4)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("B, most, queries", [(6, 1 << 23, 1), (6, 1 << 23, 5), (320, 1 << 17, 1), (320, 1 << 17, 5)])
def test_calls_that_outgrow_the_last_cache(B, most, queries, page, d, mode):
    """Room for more keys than the last-level cache holds, in a cache of as many pages (most: bytes of K for each sequence and key
    head); keys shared by workgroups and not."""
    B = B * 128 // d if B > 6 else B
    a = Attend(d, page, 2, 4, [((37 * i + 3) % 301, queries) for i in range(B)], 51)
    max_len = (most if B <= 6 else most * 5 // 4 * d // 128) // d
    n = -(-(192 << 20) // (2 * 2 * d * page))
    at = torch.randperm(n, generator=torch.Generator().manual_seed(52))[:a.k.shape[0]].to(DEV)
    big = []
    for x in (a.k, a.v):
        big.append(torch.full((n, 2, page, d), NOTHING, dtype=torch.uint8, device=DEV).index_copy_(0, at, x.to(DEV)))
    for x in (a.k_scale, a.v_scale):
        big.append(torch.ones((n, 2), device=DEV).index_copy_(0, at, x.to(DEV)))
    table = torch.full((B, -(-max_len // page)), -1, dtype=torch.int32, device=DEV)
    table[:, :a.table.shape[1]] = torch.where(a.table.to(DEV) >= 0, at[a.table.to(DEV).clamp(min=0).long()].int(), -1)
    assert min(B * max_len, n * page) * 2 * 2 * d >= 192 << 20
    a.cache = Cache(*big, table, a.cache.len)
    a.check(a.call(*mode, max_len=max_len), *mode)


def test_pages_behind_four_gigabytes():
    """Places in a cache that 32 bits do not hold: the same tokens in the first and in the last pages."""
    page, Hk, d = 128, 8, 128
    n_pages = (1 << 32) // (page * Hk * d) + 16
    free, _ = torch.cuda.mem_get_info()
    if free < 3 * n_pages * page * Hk * d:
        pytest.skip("too little memory")
    k, v = (torch.empty((n_pages, Hk, page, d), dtype=torch.uint8, device=DEV) for _ in range(2))
    k_scale, v_scale = (torch.empty((n_pages, Hk), device=DEV) for _ in range(2))
    length = torch.tensor([300, 300], dtype=torch.int32, device=DEV)
    table = torch.tensor([[2, 0, 1], [n_pages - 2, n_pages - 1, n_pages - 3]], dtype=torch.int32, device=DEV)
    cache = Cache(k, v, k_scale, v_scale, table, length)
    g = torch.Generator().manual_seed(48)
    rows = torch.randn((300, 2 * Hk, d), generator=g).bfloat16().to(DEV).repeat(2, 1, 1)
    dfss.dfss_cache_append(rows[:, :Hk], rows[:, Hk:], None, cache, None, None, Shape(2, Hk, 300, 300, d))
    assert torch.equal(k[table[0, 2].item(), :, :44], k[table[1, 2].item(), :, :44]) and torch.equal(v[table[0, 0].item()], v[table[1, 0].item()])
    for queries in (1, 130):
        Q = torch.randn((queries, 2 * Hk, d), generator=g).bfloat16().to(DEV).repeat(2, 1, 1)
        for f in (dfss.dfss_attention_cached, dfss.dense_attention_cached):
            O = f(Q, None, cache, Shape(2, 2 * Hk, queries, 300, d, 2, 4), d ** -0.5)
            assert torch.equal(O[:queries], O[queries:]) and bool(O.isfinite().all()) and O.any()
