"""The calls over a paged cache where a value lies next to a border: of two codes, of two scales, of a choice, of what 32 bits hold."""
import decoder_reference as ref
import pytest
import test_gpu_cached_attention as cached
import torch
from test_gpu_cached_attention import DEV, MODES, Append, Attend

import paper_2203_00091_amd as dfss
from paper_2203_00091_amd import Cache, Rotary, Shape

pytestmark = pytest.mark.gpu


# ---- appending ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_a_key_next_to_the_border_of_two_codes(d, interleaved):
    """A rotated key 2^-40 above or below the middle of two codes takes the nearer one, though 32 bits would put it on the middle; and
    one as little above what a scale holds takes the next scale."""
    ties = [1.0625 + i / 8 for i in range(8)]                       # middles of the codes 1, 1.125 .. 2
    cos = torch.tensor([ties * 2, [1.75] * 16])                     # [position, pair]
    sin = torch.full((2, 16), 2.0 ** -40)
    first, second = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
    K = torch.zeros(8, 1, d)
    for t, (x1, x2, most) in enumerate([(1, 1, 448), (1, -1, 448), (-1, 1, 448), (-1, -1, 448), (256, 256, 1), (256, -256, 1), (256, 0, 1), (-256, -256, 1)]):
        K[t, 0, first], K[t, 0, second], K[t, 0, d - 1] = x1, x2, most
    pos = torch.tensor([0] * 4 + [1] * 4)
    table = torch.arange(8, dtype=torch.int32).flip(0)[:, None].contiguous()      # a page to each token: a scale of its own
    codes = [torch.zeros(8, 1, 16, d, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.ones(8, 1, device=DEV) for _ in range(2)]
    cache = Cache(*codes, *scales, table.to(DEV), torch.ones(8, dtype=torch.int32, device=DEV))
    rows = K.bfloat16().to(DEV)
    dfss.dfss_cache_append(rows, rows, None, cache, None, Rotary(cos.to(DEV), sin.to(DEV), pos.int().to(DEV), interleaved), Shape(8, 1, 1, 16, d))
    exact = ref.norm_rotate(K[None], None, (cos, sin, interleaved), pos[None], 0.0)[0]
    want = torch.tensor([ref.scale_of(float(exact[t].abs().max())) for t in range(8)])
    assert want.tolist() == [1, 1, 1, 1, 2, 2, 1, 2]     # 448 and 2^-32 more; (256, 0) turns into 448 and 2^-32
    assert scales[0].flatten().flip(0).tolist() == want.tolist()
    got = ref.codes_to_values(codes[0].cpu())[:, 0, 0].flip(0)
    assert torch.equal(got, ref.nearest(exact[:, 0] / want[:, None]))


def test_no_offset_to_the_mean_of_squares(monkeypatch):
    """eps = 0 with rows that are not zero: what a wave holds besides them is nobody's."""
    monkeypatch.setattr(cached, "EPS", 0.0)
    for d, page in ((64, 16), (128, 64)):
        a = Append((page, d, 5, [(0, 1), (5, 1), (3, 2), (page - 1, 1), (0, page + 3), (7, 40)], True, d, False), 60)
        a.check(a.call())


# ---- attention ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("scale", [2.0 ** -90, 2.0 ** -100])
@pytest.mark.parametrize("lengths, queries", [([1, 40, 130, 300, 9000], 1), ([1, 40, 130, 300, 9000], 20), ([1, 40, 130, 300, 6000], 150)])
def test_large_scores_under_a_small_scale(lengths, queries, scale, sign, mode):
    """Scaled scores beyond 2^22 (raw ones to 2^122), all below 0 or all above it.  One key is 64 above the others, so O is its value: the
    others weigh e^-64."""
    for d, page in ((64, 64), (128, 16)):
        a = Attend(d, page, 1, 2, [(n, 1) for n in lengths], 63)
        counts = [min(n, queries) for n in lengths]
        a.counts, a.max_q = counts, max(counts)
        a.cu = torch.tensor([0] + counts).cumsum(0).int().to(DEV)
        # q . k = 2^22 (sign + j 2^-22) / scale with j = -64, or 0 for the best key: both parts, and their sum, are 32-bit numbers
        Q = torch.zeros(sum(counts), 2, d)
        Q[..., 0], Q[..., 1] = sign * 2.0 ** 10 / scale, -1 / scale * 2.0 ** -12
        K = torch.zeros(a.k.shape[0], 1, page, d)
        K[..., 0], K[..., 1] = 2.0 ** 12, 64 * 2.0 ** 12
        best = [(n - 1) // 3 if i % 2 else 0 for i, n in enumerate(lengths)]
        for b, j in enumerate(best):
            K[int(a.table[b, j // page]), 0, j % page, 1] = 0
        a.k, a.k_scale = (K / 2.0 ** 12).to(torch.float8_e4m3fn).view(torch.uint8), torch.full(a.k_scale.shape, 2.0 ** 12)
        a.Q, a.scale = Q.bfloat16().to(DEV), scale
        a.cache = Cache(*(x.to(DEV) for x in (a.k, a.v, a.k_scale, a.v_scale)), a.table.to(DEV), a.cache.len)
        O, at = a.call(*mode, causal=False).cpu().double(), 0
        for b, (n, j) in enumerate(zip(counts, best)):
            id = int(a.table[b, j // page])
            v = ref.codes_to_values(a.v[id, 0, j % page]) * float(a.v_scale[id, 0])
            assert torch.equal(O[at:at + n], v.expand(n, 2, d)), (d, b)
            at += n


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("size", [2.0 ** -10, 2.0 ** -16, 2.0 ** -30])
@pytest.mark.parametrize("queries", [1, 20, 150])
def test_small_scores_are_told_apart(queries, size, mode):
    """The larger score wins by however little, in calls of few rows and of many: exact scores with ties, and any."""
    for d, page in ((64, 64), (128, 16)):
        a = Attend(d, page, 1, 4, [(300, queries), (130, min(queries, 130))], 61, integers=True)
        a.Q = a.Q * size
        a.check(a.call(*mode), *mode, all_rows=True)
        b = Attend(d, page, 2, 2, [(300, queries), (130, min(queries, 130))], 62, size=size)
        want, amount, gap = b.reference(*mode)
        # 32 bits: d products, each rounded once on its way into the sum, of |q| |k| altogether (|k| <= 448 x 2^-5)
        clear = gap > d * 2.0 ** -24 * 14 * b.Q.cpu().double().abs().sum(-1)
        assert float(clear.double().mean()) > 0.5
        half = torch.finfo(torch.bfloat16).eps / 2          # (as in Attend.check)
        tol = half * want.abs() + (half + 1e-5) * (amount + want.abs()) * 1.01
        assert float(((b.call(*mode).cpu().double() - want).abs() - tol)[clear].max()) <= 0
