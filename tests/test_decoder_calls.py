"""What the calls around a decoder's attention refuse, on the host, before anything is launched (no GPU), and the plain forms that
the GPU tests compare with, against torch."""
import ctypes

import decoder_reference as ref
import pytest
import torch

import paper_2203_00091_amd as dfss
from paper_2203_00091_amd import Shape
from paper_2203_00091_amd import binding

OK, NULL, SHAPE, UNSUP, WS = 0, 1, 2, 3, 4


class Host:
    """Arguments that every call would take; the memory is the host's and never touched."""

    def __init__(self):
        self.buf = ctypes.create_string_buffer(4096)
        self.a = (ctypes.addressof(self.buf) + 255) // 256 * 256
        self.lib = dfss.load_library()

    def rows(self, H=4, batch=0, token=256, head=64, data=None):
        return binding._ROWS.pack(self.a if data is None else data, H, batch, token, head)

    def rotary(self, **kw):
        r = dict(cos=self.a, sin=self.a, pos=0, n_pos=10, rot=64, interleaved=0) | {k: v or 0 for k, v in kw.items()}
        return binding._ROTARY.pack(*r.values())

    def cache(self, **kw):
        c = {k: self.a for k in ("k", "v", "k_scale", "v_scale", "table", "len")} | dict(n_pages=8, Hk=2, page=64, width=4)
        return binding._CACHE.pack(*(c | {k: v or 0 for k, v in kw.items()}).values())


@pytest.fixture
def host():
    return Host()


BAD_ROWS = [(dict(data=0), NULL), (dict(H=0), SHAPE), (dict(token=100), SHAPE), (dict(head=-64), SHAPE), (dict(batch=3), SHAPE),
            (dict(token=1 << 42), SHAPE)]


def _bad_rows(host):
    return [(host.rows(**kw), want) for kw, want in BAD_ROWS] + [(host.rows(data=host.a + 2), SHAPE)]


def test_norm_rotate_refuses(host):
    s, a = Shape(2, 4, 8, 8, 64), host.a

    def call(Q=None, K="same", wq=a, wk=a, rot=None, shape=s, eps=1e-6, Qo=None, Ko="same", back=False, ws=a, n=1 << 30, dw=a):
        Q, Qo = Q or host.rows(), Qo or host.rows()
        K, Ko = host.rows(H=2) if K == "same" else K, host.rows(H=2) if Ko == "same" else Ko
        if back:
            return host.lib.dfss_qk_norm_rotate_backward(Qo, Ko, Q, K, wq, wk, rot, shape.c() if shape else None, eps, Q, K, dw, dw, ws, n, None)
        return host.lib.dfss_qk_norm_rotate(Q, K, wq, wk, rot, shape.c() if shape else None, eps, Qo, Ko, None)

    for back in (False, True):
        assert call(shape=None, back=back) == NULL
        assert call(K=None, back=back) == NULL and call(Ko=None, back=back) == NULL
        for r, want in _bad_rows(host):
            assert call(Q=r, back=back) == want and call(Qo=r, back=back) == want
            assert call(K=r, back=back) == want and call(Ko=r, back=back) == want
        assert call(Q=host.rows(H=3), back=back) == SHAPE and call(Ko=host.rows(H=3), back=back) == SHAPE
        assert call(wq=a + 2, back=back) == SHAPE and call(wk=a + 4, back=back) == SHAPE
        for bad, want in ((Shape(0, 4, 8, 8, 64), SHAPE), (Shape(2, 4, 0, 8, 64), SHAPE), (Shape(2, 4, 8, 8, 96), UNSUP),
                          (Shape(2, 4, 8, 8, 64, 1, 2, dfss.DFSS_F32_BF16X3), UNSUP), (Shape(1 << 13, 4, 1 << 13, 8, 64), SHAPE)):
            assert call(shape=bad, back=back) == want, bad
        for eps in (-1e-6, float("nan"), float("inf")):
            assert call(eps=eps, back=back) == UNSUP
        for kw, want in ((dict(cos=None), NULL), (dict(sin=None), NULL), (dict(n_pos=0), SHAPE), (dict(rot=0), SHAPE), (dict(rot=24), SHAPE),
                         (dict(rot=80), SHAPE), (dict(cos=a + 4), SHAPE), (dict(sin=a + 8), SHAPE), (dict(pos=a + 2), SHAPE)):
            assert call(rot=host.rotary(**kw), back=back) == want, kw
    assert call(back=True, ws=None) == NULL and call(back=True, ws=a + 16) == SHAPE
    need = dfss.dfss_qk_norm_workspace_bytes(s)
    assert need > 0 and call(back=True, n=need - 1) == WS
    assert call(back=True, dw=None) == NULL and call(back=True, dw=a + 2) == SHAPE
    assert dfss.dfss_qk_norm_workspace_bytes(Shape(1, 1, 1, 1, 96)) == 0


BAD_CACHES = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=None), NULL), (dict(v_scale=None), NULL), (dict(table=None), NULL),
              (dict(len=None), NULL), (dict(n_pages=0), SHAPE), (dict(Hk=0), SHAPE), (dict(page=48), SHAPE), (dict(page=256), SHAPE),
              (dict(page=8), SHAPE), (dict(width=0), SHAPE), (dict(width=3), SHAPE)]     # (3 pages of 64 hold fewer than Lk tokens)


def test_append_refuses(host):
    s, a = Shape(3, 2, 5, 256, 64), host.a

    def call(K=None, V=None, rows=15, cu=a, cache=None, w=a, rot=None, shape=s, eps=1e-6):
        return host.lib.dfss_cache_append(K or host.rows(H=2), V or host.rows(H=2), rows, cu, cache or host.cache(), w, rot, shape.c() if shape else None, eps, None)

    assert call(shape=None) == NULL
    for r, want in _bad_rows(host):
        assert call(K=r) == want and call(V=r) == want
    assert call(K=host.rows(H=3)) == SHAPE and call(V=host.rows(H=1)) == SHAPE and call(shape=Shape(3, 4, 5, 256, 64)) == SHAPE
    for kw, want in BAD_CACHES + [(dict(k=a + 8), SHAPE), (dict(len=a + 2), SHAPE), (dict(table=a + 1), SHAPE), (dict(k_scale=a + 2), SHAPE)]:
        assert call(cache=host.cache(**kw)) == want, kw
    assert call(rows=0) == SHAPE and call(rows=-1) == SHAPE and call(rows=1 << 28) == SHAPE
    assert call(cu=None, rows=14) == SHAPE and call(cu=a + 2) == SHAPE and call(w=a + 2) == SHAPE
    assert call(eps=-1.0) == UNSUP and call(rot=host.rotary(rot=128)) == SHAPE
    for bad, want in ((Shape(3, 2, 5, 256, 80), UNSUP), (Shape(3, 2, 5, 256, 64, 1, 2, dfss.DFSS_F32), UNSUP), (Shape(0, 2, 5, 256, 64), SHAPE),
                      (Shape(3, 2, 0, 256, 64), SHAPE), (Shape(3, 2, 5, 257, 64), SHAPE)):
        assert call(shape=bad) == want, bad


def test_attention_refuses(host):
    s, a = Shape(3, 4, 5, 256, 64), host.a

    def call(dense, Q=None, rows=15, cu=a, cache=None, shape=s, scale=0.125, O=a, ws=a, n=1 << 40):
        f = host.lib.dense_attention_cached if dense else host.lib.dfss_attention_cached
        return f(Q or host.rows(), rows, cu, cache or host.cache(), shape.c() if shape else None, scale, 1, O, ws, n, None)

    for dense in (False, True):
        assert call(dense, shape=None) == NULL and call(dense, O=None) == NULL and call(dense, O=a + 8) == SHAPE
        for r, want in _bad_rows(host):
            assert call(dense, Q=r) == want
        for kw, want in BAD_CACHES:
            assert call(dense, cache=host.cache(**kw)) == want, kw
        assert call(dense, Q=host.rows(H=3), shape=Shape(3, 3, 5, 256, 64)) == SHAPE      # no whole group of heads
        assert call(dense, Q=host.rows(H=2)) == SHAPE and call(dense, rows=0) == SHAPE and call(dense, cu=None, rows=16) == SHAPE
        for scale in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** -101, 2.0 ** 101, 1e-40):
            assert call(dense, scale=scale) == UNSUP
        for bad, want in ((Shape(3, 4, 5, 256, 96), UNSUP), (Shape(3, 4, 5, 256, 64, 1, 2, dfss.DFSS_F32_BF16X3), UNSUP), (Shape(3, 4, 5, 300, 64), SHAPE),
                          (Shape(1 << 10, 4, 1 << 20, 256, 64), SHAPE)):
            assert call(dense, shape=bad) == want, bad
        big = host.cache(width=1 << 12)
        long = Shape(3, 4, 1, 1 << 18, 64)
        need = dfss.load_library().dfss_cached_workspace_bytes(long.c(), big)
        assert need > 0 and call(dense, shape=long, cache=big, rows=3, ws=None) == NULL
        assert call(dense, shape=long, cache=big, rows=3, n=need - 1) == WS and call(dense, shape=long, cache=big, rows=3, ws=a + 64) == SHAPE
    for n, m in ((3, 4), (2, 2), (0, 0)):
        assert call(False, shape=Shape(3, 4, 5, 256, 64, n, m)) == UNSUP
    assert dfss.load_library().dfss_cached_workspace_bytes(Shape(3, 4, 5, 300, 64).c(), host.cache()) == 0


def test_binding_refuses_what_the_library_cannot_see():
    z = torch.zeros
    q = z(2, 8, 4, 64, dtype=torch.bfloat16)
    s = Shape(2, 4, 8, 8, 64, 1, 2)
    with pytest.raises(ValueError, match="current device"):
        dfss.dfss_qk_norm_rotate(q, None, None, None, None, s)
    with pytest.raises(ValueError, match="expected torch.bfloat16"):
        dfss.dfss_qk_norm_rotate(q.float(), None, None, None, None, s)
    with pytest.raises(ValueError, match="current device"):
        dfss.Rotary(z(4, 32), z(4, 32))
    with pytest.raises(ValueError, match="rot/2"):
        dfss.Rotary(z(4), z(4))
    with pytest.raises(ValueError, match="table"):
        dfss.Cache(z(4, 2, 16, 64, dtype=torch.uint8), z(4, 2, 16, 64, dtype=torch.uint8), z(4, 2), z(4, 2), z(3), z(3))
    with pytest.raises(ValueError, match="current device"):
        dfss.dfss_cache_append(q[0], q[0], None, None, None, None, s)


def test_binding_refuses_no_sequences_and_another_devices_workspace():
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):
        dfss.dfss_qk_norm_rotate(q, None, None, None, None, Shape(0, 4, 4, 4, 64, 1, 2))

    class Elsewhere:      # (one device here: a tensor's answers, of one that is not the current)
        is_cuda, device = True, "another"
        is_contiguous = staticmethod(lambda: True)
        data_ptr = staticmethod(lambda: 256)
        get_device = staticmethod(lambda: -1)

    from paper_2203_00091_amd.binding import _scratch
    assert _scratch(None) is None
    with pytest.raises(ValueError, match="current device, got one on another"):
        _scratch(Elsewhere())
    with pytest.raises(ValueError, match="device tensor"):
        _scratch(torch.zeros(256, dtype=torch.uint8))


# ---- the plain forms themselves ----


def test_codes_and_rounding_of_the_reference():
    every = torch.arange(256, dtype=torch.uint8)
    mine, theirs = ref.codes_to_values(every), every.view(torch.float8_e4m3fn).double()
    assert torch.equal(mine.nan_to_num(nan=-1.0), theirs.nan_to_num(nan=-1.0))
    x = torch.cat((torch.linspace(-448, 448, 9001), torch.linspace(-0.05, 0.05, 2001)))
    assert torch.equal(ref.nearest(x.double()), x.to(torch.float8_e4m3fn).double())
    for m, want in ((0.0, 2.0 ** -64), (448.0, 1.0), (448.5, 2.0), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7)):
        assert ref.scale_of(m) == want


def test_attention_of_the_reference_without_pruning():
    g = torch.Generator().manual_seed(1)
    Q, K, V = (torch.randn(n, h, 16, generator=g, dtype=torch.float64) for n, h in ((5, 4), (9, 2), (9, 2)))
    k, v = K.transpose(0, 1), V.transpose(0, 1)
    O, _, _ = ref.attention(Q, [5], [k], [v], [torch.ones(9, dtype=torch.bool)], [9], 9, 0, 0, 0.25, True)
    mask = torch.ones(5, 9).tril(4) == 0
    S = (Q.transpose(0, 1) @ k.repeat_interleave(2, 0).transpose(1, 2) * 0.25).masked_fill(mask, -torch.inf)
    assert torch.allclose(O.transpose(0, 1), S.softmax(-1) @ v.repeat_interleave(2, 0), atol=1e-12)


def test_norm_and_rotation_of_the_reference():
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn(1, 3, 2, 8, generator=g, dtype=torch.float64), torch.randn(8, generator=g, dtype=torch.float64)
    assert torch.allclose(ref.norm(x, w, 1e-6), torch.nn.functional.rms_norm(x, (8,), w, 1e-6))
    a = torch.rand(4, 2, generator=g, dtype=torch.float64)
    pos = torch.tensor([[3, 0, 2]])
    for interleaved in (False, True):
        y = ref.norm_rotate(x, None, (a.cos(), a.sin(), interleaved), pos, 1e-6)
        first, second = ((x[..., 0:4:2], x[..., 1:4:2]) if interleaved else (x[..., :2], x[..., 2:4]))
        turned = torch.complex(first, second) * torch.polar(torch.ones_like(a), a)[pos][:, :, None]
        got = (y[..., 0:4:2], y[..., 1:4:2]) if interleaved else (y[..., :2], y[..., 2:4])
        assert torch.allclose(got[0], turned.real) and torch.allclose(got[1], turned.imag) and torch.equal(y[..., 4:], x[..., 4:])
