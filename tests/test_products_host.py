"""Refusals of the 8-bit products and the gated block: every check happens before the GPU is touched."""
import pytest
import torch

from paper_2303_02191_amd import binding as B
from paper_2303_02191_amd import pipeline as pl

A, W, Y, S = 0x1000000, 0x2000000, 0x4000000, 0x8000000  # never dereferenced: every case fails validation first


def _status(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except B.RtossError as e:
        assert e.args[0]
        return e.status
    return B.OK


def test_quantize_rows_refusals():
    f = B.rtoss_quantize_rows
    assert _status(f, A, 5, 4, 8, Y, S) == B.EDTYPE
    assert _status(f, A, B.F32, -1, 8, Y, S) == B.EINVAL
    assert _status(f, A, B.F32, 1 << 31, 8, Y, S) == B.ESHAPE
    assert _status(f, A, B.F32, 4, 0, Y, S) == B.ESHAPE
    assert _status(f, A, B.F32, 4, (1 << 24) + 1, Y, S) == B.ESHAPE
    assert _status(f, A, B.F32, 4, 8, Y, S, x_ld=7) == B.ESHAPE
    assert _status(f, A, B.F32, 4, 8, Y, S, q_ld=1 << 31) == B.ESHAPE
    assert _status(f, A, B.F32, 4, 8, Y, S, x_ld=-8) == B.EINVAL
    for bad in ((0, Y, S), (A, 0, S), (A, Y, 0), (A + 2, Y, S), (A, Y, S + 2)):
        assert _status(f, bad[0], B.F32, 4, 8, bad[1], bad[2]) == B.EINVAL
    assert _status(f, A, B.F32, 4, 8, A + 64, S) == B.EINVAL  # overlap
    assert _status(f, A, B.F32, 4, 8, Y, A + 124) == B.EINVAL
    assert _status(f, 0, B.F32, 0, 8, 0, 0) == B.OK


def test_matmul_i8_refusals():
    def f(a=A, sa=S, w=W, y=Y, e=None, **kw):
        d = dict(M=4, N=8, K=16, a_ld=0, w_ld=0, out_dt=B.BF16)
        d.update(kw)
        return _status(B.rtoss_matmul_i8, B.MatmulDesc(**d), a, sa, w, e, y)

    assert _status(B.rtoss_matmul_i8, None, A, S, W, None, Y) == B.EINVAL
    assert f(out_dt=3) == B.EDTYPE
    assert f(M=-1) == B.EINVAL and f(M=1 << 31) == B.ESHAPE
    assert f(N=0) == B.ESHAPE and f(K=0) == B.ESHAPE
    assert f(K=1 << 17) == B.ESHAPE  # 2^17 * 128 * 128 = 2^31
    assert f(a_ld=15) == B.ESHAPE and f(w_ld=-1) == B.EINVAL
    assert f(a=0) == B.EINVAL and f(w=0) == B.EINVAL and f(y=0) == B.EINVAL and f(y=Y + 1) == B.EINVAL and f(sa=S + 1) == B.EINVAL
    assert f(y=A + 32) == B.EINVAL and f(y=W + 64) == B.EINVAL
    assert f(M=0, a=0, y=0) == B.OK
    for e in (B.EpilogueDesc(act=3), B.EpilogueDesc(scale_dev=S + 2), B.EpilogueDesc(bias_dev=S + 1), B.EpilogueDesc(residual_dev=S + 1),
              B.EpilogueDesc(residual_dev=Y), B.EpilogueDesc(y_ld=-1)):
        assert f(e=e) == B.EINVAL
    for e in (B.EpilogueDesc(y_ld=7), B.EpilogueDesc(residual_ld=7)):
        assert f(e=e) == B.ESHAPE


def _gated(**kw):
    d = dict(M=4, K=16, F=8, dt=B.BF16, act=B.ACT_SILU, x_ld=0, w_ld=0, h_ld=0)
    d.update(kw)
    return B.GatedDesc(**d)


def test_gated_refusals():
    def f(x=A, wg=W, wu=W + 4096, h=Y, gate=None, up=None, **kw):
        return _status(B.rtoss_gated_ff, _gated(**kw), x, wg, wu, h, gate, up)

    def f8(x=A, sa=S, wg=W, sg=S, wu=W + 4096, su=S, h=Y, **kw):
        return _status(B.rtoss_gated_ff_i8, _gated(**kw), x, sa, wg, sg, wu, su, h)

    for g in (f, f8):
        assert g(dt=4) == B.EDTYPE and g(act=3) == B.EINVAL and g(act=-1) == B.EINVAL
        assert g(M=-2) == B.EINVAL and g(K=0) == B.ESHAPE and g(F=0) == B.ESHAPE
        assert g(x_ld=15) == B.ESHAPE and g(w_ld=15) == B.ESHAPE and g(h_ld=7) == B.ESHAPE
        assert g(x=0) == B.EINVAL and g(wg=0) == B.EINVAL and g(wu=0) == B.EINVAL and g(h=0) == B.EINVAL and g(h=Y + 1) == B.EINVAL
        assert g(h=A + 16) == B.EINVAL  # overlap
        assert g(M=0, x=0, h=0) == B.OK
    assert _status(B.rtoss_gated_ff, None, A, W, W, Y) == B.EINVAL
    assert f(x=A + 1) == B.EINVAL and f(gate=S) == B.EINVAL and f(up=S) == B.EINVAL
    assert f(gate=S, up=S + 16) == B.EINVAL and f(gate=Y, up=S) == B.EINVAL and f(gate=S, up=A) == B.EINVAL
    assert f8(sa=S + 2) == B.EINVAL and f8(K=1 << 17) == B.ESHAPE


def test_gated_backward_refusals():
    P = [0x10000000 + i * 0x100000 for i in range(10)]  # dh x wg wu gate up | dx dwg dwu | workspace

    def f(change=None, ws_bytes=None, **kw):
        p = list(P)
        for i, v in (change or {}).items():
            p[i] = v
        d = _gated(**kw)
        return _status(B.rtoss_gated_ff_backward, d, *p, B.rtoss_gated_ff_backward_size(_gated()) if ws_bytes is None else ws_bytes)

    assert B.rtoss_gated_ff_backward_size(_gated()) >= 2 * 4 * 8 * 2
    assert B.rtoss_gated_ff_backward_size(_gated(M=0)) >= 0
    assert _status(B.rtoss_gated_ff_backward_size, _gated(K=0)) == B.ESHAPE
    assert B.lib().rtoss_gated_ff_backward_size(_gated(), None) == B.EINVAL
    assert f(act=7) == B.EINVAL and f(dt=9) == B.EDTYPE and f(h_ld=3) == B.ESHAPE
    for i in range(6):
        assert f({i: 0}) == B.EINVAL
    assert f({7: 0}) == B.EINVAL and f({8: 0}) == B.EINVAL  # one weight gradient without the other
    for i in range(9):
        assert f({i: P[i] + 1}) == B.EINVAL
    assert f(ws_bytes=8) == B.ENOSPACE
    assert f({9: 0}) == B.EINVAL and f({9: P[9] + 128}) == B.EINVAL
    assert f({6: P[0]}) == B.EINVAL and f({7: P[1]}) == B.EINVAL and f({8: P[7]}) == B.EINVAL and f({9: P[6]}) == B.EINVAL
    assert f({6: 0, 7: 0, 8: 0}) == B.OK  # nothing asked for


def test_pipeline_refuses_host_tensors():
    x, w = torch.zeros(4, 16), torch.zeros(8, 16)
    q, s = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    wq, sw = torch.zeros(8, 16, dtype=torch.int8), torch.zeros(8)
    for call in (lambda: pl.quantize_rows(x), lambda: pl.matmul_i8(q, s, wq, sw), lambda: pl.gated_ff(x, w, w),
                 lambda: pl.gated_ff_i8(q, s, wq, sw, wq, sw), lambda: pl.gated_ff_backward(x, x, w, w, x, x)):
        with pytest.raises(AssertionError, match="GPU"):
            call()
    with pytest.raises(TypeError):
        pl.quantize_rows("x")
