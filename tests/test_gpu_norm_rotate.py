"""dfss_qk_norm_rotate and its gradients against their formulas in 64 bits."""
import decoder_reference as ref
import pytest
import torch

import paper_2203_00091_amd as dfss
from paper_2203_00091_amd import Rotary, Shape

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6
DTYPES = {"bf16": (torch.bfloat16, dfss.DFSS_BF16), "f32": (torch.float32, dfss.DFSS_F32)}


def _angles(n_pos, rot):
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    return a.cos().float(), a.sin().float()


class Setup:
    def __init__(self, B, L, Hq, Hk, d, rot, interleaved, weights, dtype, seed, pos="random", n_pos=97):
        g = torch.Generator().manual_seed(seed)
        t, code = DTYPES[dtype]
        self.s = Shape(B, Hq, L, L, d, 1, 2, code)
        # rows of a projection: queries, keys, values; some rows are much larger than others
        qkv = torch.randn((B, L, Hq + 2 * Hk, d), generator=g) * torch.exp2(torch.randint(-6, 7, (B, L, Hq + 2 * Hk, 1), generator=g).float())
        self.qkv = qkv.to(t).to(DEV)
        self.x = [self.qkv[:, :, :Hq], self.qkv[:, :, Hq:Hq + Hk]]
        self.w = [(1 + 0.3 * torch.randn(d, generator=g)).to(t).to(DEV) if c in weights else None for c in "qk"]
        self.rotary = self.table = None
        self.pos = torch.arange(L).expand(B, L)
        if rot:
            cos, sin = _angles(n_pos, rot)
            if pos == "random":      # also positions that the table does not hold
                self.pos = torch.randint(-3, n_pos + 4, (B, L), generator=g)
            self.table = (cos, sin, interleaved)
            self.rotary = Rotary(cos.to(DEV), sin.to(DEV), self.pos.int().to(DEV) if pos == "random" else None, interleaved)
        self.dy = [torch.randn((B * H, L, d), generator=g).to(t).to(DEV) for H in (Hq, Hk)]
        self.heads, self.half = (Hq, Hk), torch.finfo(t).eps / 2

    def forward(self, **kw):
        return dfss.dfss_qk_norm_rotate(self.x[0], self.x[1], self.w[0], self.w[1], self.rotary, self.s, EPS, **kw)

    def backward(self, **kw):
        return dfss.dfss_qk_norm_rotate_backward(self.dy[0], self.dy[1], self.x[0], self.x[1], self.w[0], self.w[1], self.rotary, self.s, EPS, **kw)

    def reference(self, i):
        return ref.norm_rotate(self.x[i].cpu(), None if self.w[i] is None else self.w[i].cpu(), self.table, self.pos, EPS)

    def by_token(self, y, i):
        """[B * H, L, d] as [B, L, H, d]."""
        return y.cpu().double().view(self.s.B, self.heads[i], self.s.Lq, self.s.d).transpose(1, 2)


# 32-bit arithmetic on the way: the row's sum (a tree of at most 8 + 4 levels), mean, root, reciprocal, two products with the
# weight, the rotation's two: below 20 roundings of 2^-24 each, relative to the largest element of the row's pair
ARITHMETIC = 20 * 2.0 ** -24

CASES = [
    # B, L, Hq, Hk, d, rot, interleaved, weights
    (1, 1, 1, 1, 64, 64, False, "qk"),
    (1, 1, 12, 12, 128, 128, True, "qk"),
    (2, 7, 5, 3, 64, 16, False, "qk"),
    (3, 5, 16, 4, 128, 48, False, "q"),
    (2, 33, 33, 1, 64, 48, True, "k"),
    (2, 9, 3, 2, 128, 96, False, ""),
    (1, 13, 4, 4, 128, 0, False, "qk"),
    (2, 300, 9, 2, 64, 32, True, "qk"),       # many tokens: several heads of a token in one wave
    (3, 257, 16, 4, 128, 128, False, "qk"),
    (1, 601, 5, 1, 128, 112, False, "qk"),
    (1, 520, 12, 12, 64, 64, False, ""),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case, dtype):
    s = Setup(*case, dtype, seed=11)
    out = s.forward()
    for i in (0, 1):
        assert out[i].shape == (s.s.B * s.heads[i], s.s.Lq, s.s.d)
        y, want = s.by_token(out[i], i), s.reference(i)
        tol = s.half * want.abs() + ARITHMETIC * want.abs().amax(-1, keepdim=True) * 1.5
        assert bool(((y - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(case, dtype):
    s = Setup(*case, dtype, seed=12)
    ws = torch.full((dfss.dfss_qk_norm_workspace_bytes(s.s),), 255, dtype=torch.uint8, device=DEV)
    got = s.backward(ws=ws)
    again = s.backward()
    for i in (0, 1):
        x = s.x[i].cpu().double().requires_grad_()
        w = None if s.w[i] is None else s.w[i].cpu().double().requires_grad_()
        y = ref.norm_rotate(x, w, s.table, s.pos, EPS)
        dy = s.by_token(s.dy[i], i)
        (y * dy).sum().backward()
        dx = got[i].cpu().double()
        r = 1 if w is None else (x.detach().square().mean(-1, keepdim=True) + EPS).rsqrt()
        most = 1 if w is None else w.detach().abs().max()
        # relative to the largest that a term of dx can be: r w dz, and x r times the mean of g x r
        tol = s.half * x.grad.abs() + 2 * ARITHMETIC * r * most * dy.abs().amax(-1, keepdim=True) * 2 * s.s.d ** 0.5
        assert bool(((dx - x.grad).abs() <= tol).all())
        assert torch.equal(got[i], again[i])
        if w is None:
            assert got[2 + i] is None
            continue
        terms = (dy.abs().amax(-1, keepdim=True) * 1.5 * (x.detach() * r).abs()).sum((0, 1, 2))
        assert bool(((got[2 + i].cpu().double() - w.grad).abs() <= 2 * ARITHMETIC * terms).all())
        assert torch.equal(got[2 + i], again[2 + i])


@pytest.mark.parametrize("d, rot, interleaved", [(64, 64, False), (128, 96, True), (128, 0, False)])
def test_gradients_against_differences(d, rot, interleaved):
    """The forward call's own slope along a direction of x and of w."""
    s = Setup(2, 5, 3, 2, d, rot, interleaved, "qk", "f32", seed=13)
    s.qkv.copy_(torch.randn(s.qkv.shape, generator=torch.Generator().manual_seed(5)))
    dQ, dK, dwq, dwk = s.backward()
    g = torch.Generator().manual_seed(14)
    v = torch.randn(s.qkv.shape, generator=g).to(DEV)
    u = [torch.randn(d, generator=g).to(DEV) for _ in range(2)]
    H, h = s.heads, 2.0 ** -7
    want = [(dQ.double() * v[:, :, :H[0]]).sum() + (dwq.double() * u[0]).sum(), (dK.double() * v[:, :, H[0]:H[0] + H[1]]).sum() + (dwk.double() * u[1]).sum()]
    ends = []
    base, w = s.qkv.clone(), [x.clone() for x in s.w]
    for sign in (1, -1):
        s.qkv.copy_(base + sign * h * v)
        s.w = [x + sign * h * y for x, y in zip(w, u)]
        ends.append([y.double() for y in s.forward()])
    for i in (0, 1):
        slope = ((ends[0][i] - ends[1][i]) / (2 * h) * s.dy[i].double()).sum()
        # third derivatives times h^2 / 6 = 1e-5, and 2^-20 / h of rounding, over a few thousand terms of order one
        assert abs(float(slope - want[i])) <= 2e-2 + 1e-3 * abs(float(want[i])), (float(slope), float(want[i]))


def test_places_for_the_results():
    """Results where the inputs were, in a layout of the caller's, and without keys: the same bits."""
    s = Setup(2, 40, 6, 2, 64, 32, False, "qk", "bf16", seed=15)
    Q, K = s.forward()
    rows = torch.zeros((2, 40, 11, 64), dtype=torch.bfloat16, device=DEV)
    s.forward(Qo=rows[:, :, 1:7], Ko=rows[:, :, 8:10])
    assert torch.equal(rows[:, :, 1:7].transpose(1, 2).reshape(12, 40, 64), Q)
    assert torch.equal(rows[:, :, 8:10].transpose(1, 2).reshape(4, 40, 64), K)
    assert not rows[:, :, [0, 7, 10]].any()
    alone, none = dfss.dfss_qk_norm_rotate(s.x[0], None, s.w[0], None, s.rotary, s.s, EPS)
    assert none is None and torch.equal(alone, Q)
    grads = s.backward()
    dQ, dK, dwq, dwk = dfss.dfss_qk_norm_rotate_backward(s.dy[0], None, s.x[0], None, s.w[0], None, s.rotary, s.s, EPS)
    assert dK is None and dwk is None and torch.equal(dQ, grads[0])
    values = s.qkv[:, :, 8:].clone()
    into = torch.zeros_like(s.qkv)      # the gradient of the whole projection's rows
    s.backward(dQ=into[:, :, :6], dK=into[:, :, 6:8])
    assert torch.equal(into[:, :, :6], grads[0]) and torch.equal(into[:, :, 6:8], grads[1]) and not into[:, :, 8:].any()
    s.forward(Qo=s.x[0], Ko=s.x[1])
    assert torch.equal(s.x[0].transpose(1, 2).reshape(12, 40, 64), Q) and torch.equal(s.qkv[:, :, 8:], values)


def test_zero_rows_and_the_tokens_own_places():
    s = Setup(2, 30, 3, 1, 128, 128, False, "qk", "f32", seed=16, pos=None)
    s.qkv[1, 4] = 0
    Q, K = s.forward()
    assert not Q.view(2, 3, 30, 128)[1, :, 4].any()
    assert bool(((s.by_token(Q, 0) - s.reference(0)).abs() <= 2 * ARITHMETIC * s.reference(0).abs().amax(-1, keepdim=True)).all())
    dQ, dK, _, _ = s.backward()
    assert bool(dQ.isfinite().all()) and bool(dK.isfinite().all())


def test_captured_and_on_another_stream():
    s = Setup(2, 300, 6, 2, 64, 64, False, "qk", "bf16", seed=17)
    want, grads = s.forward(), s.backward()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert all(torch.equal(a, b) for a, b in zip(s.forward(), want))
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        out, back = s.forward(), s.backward()
    first = s.qkv.clone()
    for k in range(3):
        s.qkv.copy_(first if k != 1 else -first)
        graph.replay()
        torch.cuda.synchronize()
        eager = list(s.forward()) + list(s.backward())
        assert all(torch.equal(a, b) for a, b in zip(list(out) + list(back), eager))
    assert all(torch.equal(a, b) for a, b in zip(list(out) + list(back), list(want) + list(grads)))


def test_strides_that_32_bits_do_not_hold():
    far = (1 << 31) + 64
    if torch.cuda.mem_get_info()[0] < 3 * 2 * far:
        pytest.skip("too little memory")
    buffer = torch.empty(far + 4096, dtype=torch.bfloat16, device=DEV)
    Q = buffer.as_strided((2, 3, 2, 64), (far, 128, 64, 1))
    x = torch.randn((2, 3, 2, 64), generator=torch.Generator().manual_seed(18)).bfloat16().to(DEV)
    Q.copy_(x)
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    s = Shape(2, 2, 3, 3, 64, 1, 2)
    want, _ = dfss.dfss_qk_norm_rotate(x, None, w, None, None, s)
    got, _ = dfss.dfss_qk_norm_rotate(Q, None, w, None, None, s)
    assert torch.equal(got, want)
    dfss.dfss_qk_norm_rotate(x, None, w, None, None, s, Qo=Q)
    assert torch.equal(Q.transpose(1, 2).reshape(4, 3, 64), want)


def test_many_tokens_and_heads():
    """Every element against the same rows in another shape: more waves than the chip holds, and fewer."""
    x = torch.randn((4, 1500, 24, 64), generator=torch.Generator().manual_seed(19)).bfloat16().to(DEV)
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    cos, sin = (t.to(DEV) for t in _angles(1500, 64))
    whole, _ = dfss.dfss_qk_norm_rotate(x, None, w, None, Rotary(cos, sin), Shape(4, 24, 1500, 1500, 64, 1, 2))
    for b, t, h in ((0, 0, 0), (3, 1499, 23), (1, 777, 5)):
        at = torch.tensor([[t]], dtype=torch.int32, device=DEV)
        one, _ = dfss.dfss_qk_norm_rotate(x[b:b + 1, t:t + 1, h:h + 1], None, w, None, Rotary(cos, sin, at), Shape(1, 1, 1, 1, 64, 1, 2))
        assert torch.equal(one[0, 0], whole.view(4, 24, 1500, 64)[b, h, t])


def test_calls_that_outgrow_the_last_cache():
    """What is read and written past the caches, in both directions: the formula without rotation, and with it the same rows in
    another shape."""
    B, L, H, Hk, d = 4, 2048, 16, 17, 128
    g = torch.Generator(device=DEV).manual_seed(20)
    rnd = lambda *n: torch.randn(n, generator=g, device=DEV).bfloat16()
    X, dY, w = (rnd(B, L, H, d), rnd(B, L, Hk, d)), (rnd(B, L, H, d), rnd(B, L, Hk, d)), (rnd(d), rnd(d))
    s = Shape(B, H, L, L, d, 1, 2)
    got = dfss.dfss_qk_norm_rotate_backward(*dY, *X, *w, None, s, EPS)
    half = torch.finfo(torch.bfloat16).eps / 2
    for i in (0, 1):
        dw, terms = torch.zeros(d, dtype=torch.float64, device=DEV), torch.zeros(d, dtype=torch.float64, device=DEV)
        for b in range(B):
            x, dz, f = X[i][b].double(), dY[i][b].double(), w[i].double()
            r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
            mean = (dz * f * x).mean(-1, keepdim=True)
            want, amount = r * (dz * f - x * r * r * mean), r * ((dz * f).abs() + (x * r * r).abs() * (dz * f * x).abs().mean(-1, keepdim=True))
            # one rounding to bfloat16, and at most 32 in 32 bits on the way to each of the amounts
            assert bool(((got[i][b].double() - want).abs() <= half * want.abs() + 2.01 * 32 * 2.0 ** -24 * amount).all())
            dw += (dz * x * r).sum((0, 1))
            terms += (dz * x * r).abs().sum((0, 1))
        # a term has fewer than 32 roundings, and passes fewer than 128 additions: 8192 x 17 rows over 512 workgroups of 16 rows side by
        # side are 18, then 2 and 2 in the workgroup and 16 and 5 over all of them
        assert bool(((got[2 + i].double() - dw).abs() <= 160 * 2.0 ** -24 * terms).all())
    rotary = Rotary(*(t.to(DEV) for t in _angles(L, d)))
    whole = dfss.dfss_qk_norm_rotate(*X, *w, rotary, s, EPS)
    for b in range(B):
        one = dfss.dfss_qk_norm_rotate(*(x[b:b + 1] for x in X), *w, rotary, Shape(1, H, L, L, d, 1, 2), EPS)
        assert all(torch.equal(x.view(B, -1, L, d)[b], y) for x, y in zip(whole, one))
