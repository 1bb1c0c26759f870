"""Results that lie over operands, scales or each other are refused before the GPU is touched, also where a matrix is a slice of a wider buffer."""
import pytest

from paper_2303_02191_amd import binding as B

A, W, Y, S = 0x10000000, 0x20000000, 0x40000000, 0x80000000  # never dereferenced: every case fails validation first
M, N, K, LD = 40, 24, 64, 256


def _status(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except B.RtossError as e:
        assert "overlap" in e.args[0]
        return e.status
    return B.OK


def matmul(a=A, sa=S, w=W, y=Y, e=None, **kw):
    d = dict(M=M, N=N, K=K, a_ld=0, w_ld=0, out_dt=B.F32)
    d.update(kw)
    return _status(B.rtoss_matmul_i8, B.MatmulDesc(**d), a, sa, w, e, y)


@pytest.mark.parametrize("at", [0, M * N * 4 - 4, -(N * 4 - 4)])
def test_scales_and_bias_under_the_result(at):
    assert matmul(e=B.EpilogueDesc(scale_dev=Y + at)) == B.EINVAL
    assert matmul(e=B.EpilogueDesc(bias_dev=Y + at)) == B.EINVAL
    g = B.GatedDesc(M, K, N, B.F32, B.ACT_SILU, 0, 0, 0)
    for scales in ((S, Y + at, S), (S, S, Y + at)):
        assert _status(B.rtoss_gated_ff_i8, g, A, scales[0], W, scales[1], W + 65536, scales[2], Y) == B.EINVAL


@pytest.mark.parametrize("at", [0, M * N * 4 - 4, -(M * 4 - 4)])
def test_scales_of_the_rows_under_the_result(at):
    assert matmul(sa=Y + at) == B.EINVAL
    g = B.GatedDesc(M, K, N, B.F32, B.ACT_SILU, 0, 0, 0)
    assert _status(B.rtoss_gated_ff_i8, g, A, Y + at, W, S, W + 65536, S, Y) == B.EINVAL


@pytest.mark.parametrize("row", [0, 7, M - 1])
@pytest.mark.parametrize("at", [0, N * 4 - 1])
def test_a_result_in_a_wider_buffer_over_a_plain_operand(row, at):
    """y's row begins at an operand's last byte, or an operand at the last byte of y's row."""
    y_row = Y + row * LD * 4
    e = B.EpilogueDesc(y_ld=LD)
    assert matmul(a=y_row + at, e=e) == B.EINVAL
    assert matmul(w=y_row + at, e=e) == B.EINVAL
    assert matmul(sa=y_row + at // 4 * 4, e=e) == B.EINVAL
    assert matmul(e=B.EpilogueDesc(y_ld=LD, residual_dev=y_row + at // 4 * 4)) == B.EINVAL


def test_slices_of_one_buffer_that_share_columns():
    e = B.EpilogueDesc(y_ld=LD, residual_dev=Y + (N - 1) * 4, residual_ld=LD)
    assert matmul(e=e) == B.EINVAL
    e = B.EpilogueDesc(y_ld=LD, residual_dev=Y - (3 * LD + N - 1) * 4, residual_ld=LD)
    assert matmul(e=e) == B.EINVAL
    for h in (0, (K - 1) * 4, (LD - N + 1) * 4, -(N - 1) * 4, (5 * LD + 3) * 4):
        g = B.GatedDesc(M, K, N, B.F32, B.ACT_SILU, LD, 0, LD)
        assert _status(B.rtoss_gated_ff, g, Y, W, W + 65536, Y + h) == B.EINVAL
    for q in (0, K - 1, 4 * LD - K + 1):
        assert _status(B.rtoss_quantize_rows, A, B.F32, M, K, A + q, S, x_ld=LD, q_ld=4 * LD) == B.EINVAL


def test_gradients_over_slices():
    P = [0x10000000 + i * 0x100000 for i in range(10)]  # dh x wg wu gate up | dx dwg dwu | workspace
    g = B.GatedDesc(M, K, N, B.F32, B.ACT_SILU, LD, LD, LD)
    size = B.rtoss_gated_ff_backward_size(g)

    def f(i, at):
        p = list(P)
        p[i] = at
        return _status(B.rtoss_gated_ff_backward, g, *p, size)

    for i in (6, 7, 8):
        for j, rows in ((0, M), (1, M), (2, N), (3, N)):
            assert f(i, P[j] + (rows - 1) * LD * 4) == B.EINVAL
    assert f(9, P[1] + 256) == B.EINVAL
