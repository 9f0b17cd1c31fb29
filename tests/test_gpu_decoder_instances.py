"""Every instance of the decoder's kernels (test_decoder_instances.py says that the cases reach them) against the plain forms in 64 bits."""
import decoder_cases as cases
import decoder_reference as ref
import pytest
import test_gpu_cached_attention as cached
import torch
from test_gpu_cached_attention import DEV, MODES, Append, Attend
from test_gpu_norm_rotate import ARITHMETIC, DTYPES

import paper_2203_00091_amd as dfss
from paper_2203_00091_amd import Rotary, Shape

pytestmark = pytest.mark.gpu


@pytest.fixture
def at_once(monkeypatch):
    monkeypatch.setattr(ref, "attention", ref.attention_at_once)


ATTEND = [(d, *case[1:]) for case, _ in cases.ATTEND for d in ((64, 128) if case[0] == 0 else case[:1])]


@pytest.mark.parametrize("mode", MODES, ids=str)
@pytest.mark.parametrize("page, causal", [(16, False), (64, True)])
@pytest.mark.parametrize("case", ATTEND, ids=str)
def test_attention(at_once, case, page, causal, mode):
    d, Hk, G, B, queries, longest = case
    shared = cases.attend_plan(*case)[2]
    a = Attend(d, page, Hk, G, list(zip(cases.attend_lengths(B, longest), cases.attend_counts(B, queries))), 80)
    assert (dfss.dfss_cached_workspace_bytes(a.shape(*mode), a.cache) > 0) == bool(shared)
    O = a.call(*mode, causal)
    a.check(O, *mode, causal)
    if shared:      # the workspace's contents are nobody's, and two calls in a row on one are two calls
        ws = torch.full((dfss.dfss_cached_workspace_bytes(a.shape(*mode), a.cache),), 255, dtype=torch.uint8, device=DEV)
        assert torch.equal(a.call(*mode, causal, ws=ws), O) and torch.equal(a.call(*mode, causal, ws=ws), O)


@pytest.mark.parametrize("case", [c for c, _ in cases.APPEND], ids=str)
def test_append(case):
    """Every code is the nearest one: what is left of 64 bits on the way, 2^-43, comes between a value and a border once in 10^11."""
    d, page, Hk, B, new = case
    rot = (d, d // 2, 0)[Hk % 3]
    a = Append((page, d, Hk, cases.append_sequences(page, B, new), Hk % 2 == 1, rot, B % 4 == 2), 81, uniform=isinstance(new, int))
    cache = a.call()
    K, V = a.rows[:, 1:1 + Hk].cpu(), a.rows[:, 1 + Hk:].cpu().double()
    pos = torch.cat([torch.arange(n) + l - n for l, n in zip(a.lengths, a.counts)])
    K = ref.norm_rotate(K[None], a.w, None if a.angles is None else (*a.angles, a.interleaved), pos[None], cached.EPS)[0]
    for x, codes, scale, got, got_scale in ((K, a.k, a.k_scale, cache.k, cache.k_scale), (V, a.v, a.v_scale, cache.v, cache.v_scale)):
        values, want_scale = ref.codes_to_values(codes), scale.double().clone()
        ref.append_at_once(values, want_scale, x, a.table, a.lengths, a.counts, page, a.max_len, a.n_pages)
        assert torch.equal(got_scale.cpu().double(), want_scale)
        assert torch.equal(ref.codes_to_values(got.cpu()).nan_to_num(nan=999.0), values.nan_to_num(nan=999.0))


@pytest.mark.parametrize("case", [c for c, _ in cases.NORM], ids=str)
def test_norm_and_its_gradients(case):
    dtype, d, B, L, Hq, Hk = case
    t, code = DTYPES[dtype]
    half, eps = torch.finfo(t).eps / 2, cached.EPS
    g = torch.Generator(device=DEV).manual_seed(82)
    rows = torch.randn((B, L, Hq + Hk + 1, d), generator=g, device=DEV).to(t)
    x = [rows[:, :, :Hq], rows[:, :, Hq:Hq + Hk]]
    dy = [torch.randn((B * H, L, d), generator=g, device=DEV).to(t) for H in (Hq, Hk)]
    w = [(1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(t) for _ in range(2)]
    rot, interleaved = (d, d // 2)[Hq % 2], Hk % 2 == 0
    angle = torch.rand((97, rot // 2), generator=g, device=DEV, dtype=torch.float64) * 6.3
    cos, sin, pos = angle.cos().float(), angle.sin().float(), torch.randint(0, 97, (B, L), generator=g, device=DEV)
    s, rotary = Shape(B, Hq, L, L, d, 1, 2, code), Rotary(cos, sin, pos.int(), interleaved)
    out = dfss.dfss_qk_norm_rotate(*x, *w, rotary, s, eps)
    grads = dfss.dfss_qk_norm_rotate_backward(*dy, *x, *w, rotary, s, eps)
    for i, H in enumerate((Hq, Hk)):
        for b in range(B):      # (64-bit forms of one batch element at a time)
            at, one = slice(b, b + 1), slice(b * H, (b + 1) * H)
            xd, wd = x[i][at].double(), w[i].double()
            want = ref.norm_rotate(x[i][at], w[i], (cos, sin, interleaved), pos[at], eps)
            y = out[i][one].double().view(1, H, L, d).transpose(1, 2)
            # (tolerances as in test_gpu_norm_rotate.py)
            assert bool(((y - want).abs() <= half * want.abs() + ARITHMETIC * want.abs().amax(-1, keepdim=True) * 1.5).all())
            dyd = dy[i][one].double().view(1, H, L, d).transpose(1, 2)
            dz = ref.rotate(dyd, cos.double()[pos[at]][:, :, None], -sin.double()[pos[at]][:, :, None], interleaved)
            r = (xd.square().mean(-1, keepdim=True) + eps).rsqrt()
            want = r * (dz * wd - xd * r.square() * (dz * wd * xd).mean(-1, keepdim=True))
            tol = half * want.abs() + 2 * ARITHMETIC * r * wd.abs().max() * dyd.abs().amax(-1, keepdim=True) * 2 * d ** 0.5
            assert bool(((grads[i][at].double() - want).abs() <= tol).all())
            part, most = (dz * xd * r).sum((0, 1, 2)), (dyd.abs().amax(-1, keepdim=True) * 1.5 * (xd * r).abs()).sum((0, 1, 2))
            dw, terms = (part, most) if b == 0 else (dw + part, terms + most)
        assert bool(((grads[2 + i].double() - dw).abs() <= 2 * ARITHMETIC * terms).all())
