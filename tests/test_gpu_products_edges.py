"""The 8-bit products and the gated block at the edges of their range: pitches at the limit, values that are not finite, sums of one to a few
products in fp32, the activation of the backward pass against the forward's, what is written of a workspace.  Tolerances count half steps, 2^-24 of the value in
fp32, one for each rounding."""
import pytest
import torch

from paper_2303_02191_amd import binding as B
from paper_2303_02191_amd import pipeline as pl
from test_gpu_products import DT, U, check, codes, equal, gen, half_step, least, normal, whole

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------
# pitches past 2^31 - 1 elements
# ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("which", ["y", "residual"])
def test_matmul_i8_refuses_results_further_apart_than_pitches_go(which):
    """Two rows 2^31 + 8 elements apart: no pitch that the library takes."""
    g = gen(1)
    N, apart = 24, (1 << 31) + 8
    buf = torch.zeros(apart + N, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((2, N), (apart, 1))
    a, w = codes(g, (2, 16)), codes(g, (N, 16))
    near = torch.zeros(2, N, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.RtossError, match=which + "_ld"):
        pl.matmul_i8(a, None, w, None, **{which: far, "y" if which == "residual" else "residual": near})
    assert not buf.any() and not near.any()
    one = buf.as_strided((1, N), (apart, 1))  # (a row alone has no pitch)
    equal(pl.matmul_i8(a[:1], None, w, None, y=one), (a[:1].double() @ w.double().t()).float().to(torch.bfloat16))


def test_matmul_i8_of_the_largest_pitch():
    g = gen(2)
    N, apart = 24, (1 << 31) - 1
    buf = torch.zeros(apart + N, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((2, N), (apart, 1))
    a, w, r = codes(g, (2, 16)), codes(g, (N, 16)), whole(g, (2, N), 9, torch.bfloat16)
    want = ((a.double() @ w.double().t()).float() + r.float()).to(torch.bfloat16)
    equal(pl.matmul_i8(a, None, w, None, residual=r, y=far), want)
    far.copy_(r)
    equal(pl.matmul_i8(a, None, w, None, residual=far), want)


# ---------------------------------------------------------------------------------------------------------
# values that are not finite
# ---------------------------------------------------------------------------------------------------------
def same(got, want, what):
    """Equal, NaN where NaN is wanted."""
    bad = ~((got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), "%s: %d of %d, first at %s: got %r, want %r" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item())


def all_pairs(g, u, dh, t):
    """Every combination of the values, one to a column."""
    return [v.reshape(1, -1).to("cuda", t) for v in torch.cartesian_prod(*(torch.tensor(v) for v in (g, u, dh))).t()]


@pytest.mark.parametrize("a", [0, 1, 2])
@pytest.mark.parametrize("dt", list(DT))
def test_gradients_keep_nan_and_infinities(dt, a):
    """One row and x = 1: the gradients of the weights are dg and du.  dg = dh u act'(g) and du = dh act(g) in IEEE arithmetic, the slope of a NaN a NaN.
    Whole numbers, so that nothing is rounded; with SiLU only what is not finite is compared."""
    inf, nan = float("inf"), float("nan")
    t = DT[dt]
    gate, up, dh = all_pairs([nan, 1.0, 2.0, -1.0, 0.0] + ([inf, -inf] if a < 2 else []), [1.0, -2.0, 0.0, inf, nan], [1.0, -2.0, 0.0, inf, -inf, nan], t)
    F = gate.shape[1]
    x, w = torch.ones(1, 1, dtype=t, device="cuda"), torch.ones(F, 1, dtype=t, device="cuda")
    G, V, H = gate.double(), up.double(), dh.double()
    if a == 0:
        act, slope = G, torch.ones_like(G)
    elif a == 1:
        act, slope = torch.where(G < 0, 0.0, G), torch.where(G > 0, 1.0, torch.where(G <= 0, 0.0, nan))
    else:
        s = torch.sigmoid(G)
        act, slope = G * s, s * (1 + G * (1 - s))
    dg, du = (H * V * slope).t(), (H * act).t()
    dx, dwg, dwu = pl.gated_ff_backward(dh, x, w, w, gate, up, act=a)
    for got, want, what in ((dwg, dg, "dw_gate"), (dwu, du, "dw_up")):
        if a == 2:
            got, want = torch.where(got.isfinite(), 0.0, got), torch.where(want.isfinite(), 0.0, want)
        same(got, want.to(t), what)
    assert dx.isnan().all()  # (NaN enters the row's sum)


def same_where_not_finite(got, want, what):
    t = got.dtype
    same(torch.where(got.isfinite(), 0.0, got.float()), torch.where(want.isfinite(), 0.0, want).float(), what)
    assert got.dtype == t


# slices of every width, a tile for every wave (fp32), tiles (16 bits); K from below a stage to several
SPOILT = [(40, 96, 130), (10, 9, 20), (33, 1030, 96), (300, 520, 387), (1500, 16, 2801), (600, 256, 520), (1030, 640, 2100)]


@pytest.mark.parametrize("pitch", [0, 3])
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("M,K,F", SPOILT)
def test_gated_ff_of_operands_that_are_not_finite(M, K, F, dt, pitch):
    """A sum with an infinite operand is infinite, of both signs or with a NaN a NaN, in every type; all others have the bits that they have without."""
    g = gen(500 + M + pitch)
    t = DT[dt]
    inf, nan = float("inf"), float("nan")
    x, wg, wu = (normal(g, (rows, K + pitch)).to(t)[:, :K] for rows in (M, F, F))
    clean = pl.gated_ff(x, wg, wu, act=1, keep=True)
    x[2, 5], x[7, 0], x[8, 3], x[8, K - 1], x[9, K - 1] = inf, -inf, inf, -inf, nan
    wg[4, 1] = inf
    h, gate, up = pl.gated_ff(x, wg, wu, act=1, keep=True)
    G, V = (x.double().cpu() @ w.double().cpu().t() for w in (wg, wu))
    for got, want, what in ((gate, G, "gate"), (up, V, "up"), (h, torch.relu(G) * V, "h")):
        same_where_not_finite(got.cpu(), want, what)
    rows = [m for m in range(M) if m not in (2, 7, 8, 9)]
    cols = [f for f in range(F) if f != 4]
    for got, want, what in zip((h, gate, up), clean, ("h", "gate", "up")):
        equal(got[rows][:, cols], want[rows][:, cols], what)


@pytest.mark.parametrize("pitch", [0, 3])
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("M,K,F", SPOILT + [(20, 70, 3333), (4100, 33, 20)])
def test_gradients_of_operands_that_are_not_finite(M, K, F, dt, pitch):
    """The same of the gradients (dg = dh u, du = dh g)."""
    g = gen(600 + M + pitch)
    t = DT[dt]
    inf, nan = float("inf"), float("nan")
    x, wg, wu = (normal(g, (rows, K + pitch)).to(t)[:, :K] for rows in (M, F, F))
    gate, up = normal(g, (M, F)).to(t), normal(g, (M, F)).to(t)
    dh = normal(g, (M, F + pitch)).to(t)[:, :F]
    clean = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    dh[2, 3], dh[5, F - 1], dh[6, 0], dh[6, 7] = inf, -inf, nan, inf
    x[8, 1], wu[4, 2] = inf, -inf
    got = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    dg, du = (dh.float() * up.float()).to(t).double().cpu(), (dh.float() * gate.float()).to(t).double().cpu()
    X, G, V = (v.double().cpu() for v in (x, wg, wu))
    for a, b, what in zip(got, (dg @ G + du @ V, dg.t() @ X, du.t() @ X), ("dx", "dw_gate", "dw_up")):
        same_where_not_finite(a.cpu(), b, what)
    rows = [m for m in range(M) if m not in (2, 5, 6)]
    channels = [f for f in range(F) if f not in (0, 3, 7, F - 1)]
    cols = [k for k in range(K) if k not in (1, 2)]
    equal(got[0][rows][:, cols], clean[0][rows][:, cols], "dx")
    for a, b, what in zip(got[1:], clean[1:], ("dw_gate", "dw_up")):
        equal(a[channels][:, cols], b[channels][:, cols], what)


# ---------------------------------------------------------------------------------------------------------
# short sums in fp32
# ---------------------------------------------------------------------------------------------------------
def short_sum_tolerance(n, size):
    """What fp32 arithmetic keeps to: n products and n - 1 additions, a rounding each, so n half steps of the sum of magnitudes.  Of bf16 parts (h of the
    first 8 bits, what is left m below 2^-7, l below 2^-16 of the value) the roundings of the sums that m enters come on top, 2^-7 and 2^-6 half steps
    each, and the dropped l l, 2^-8: below 2^-4 for each product."""
    return n * U * (1 + 2.0 ** -4) * size


@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 8, 16, 32])
@pytest.mark.parametrize("pitch", [0, 3])
def test_gated_ff_f32_short_sums(n, pitch):
    g = gen(100 + n)
    M, F = 200, 700
    x, wg, wu = (normal(g, (rows, n + pitch))[:, :n] for rows in (M, F, F))
    _, gate, up = pl.gated_ff(x, wg, wu, keep=True)
    X = x.double()
    for got, w, what in ((gate, wg.double(), "gate"), (up, wu.double(), "up")):
        check(got, X @ w.t(), short_sum_tolerance(n, X.abs() @ w.abs().t()), what)


@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 8, 16, 32])
@pytest.mark.parametrize("K,F", [(120, 300), (36, 2000), (1030, 2100)])
def test_gradients_f32_of_few_rows(n, K, F):
    """dg = dh u and du = dh g, rounded once, are the operands; sums of n products (weights)."""
    g = gen(200 + n + K)
    x, wg, wu = normal(g, (n, K)), normal(g, (F, K)), normal(g, (F, K))
    gate, up, dh = (normal(g, (n, F)) for _ in range(3))
    _, dwg, dwu = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    X = x.double()
    for got, d, what in ((dwg, (dh * up).double(), "dw_gate"), (dwu, (dh * gate).double(), "dw_up")):
        check(got, d.t() @ X, short_sum_tolerance(n, d.abs().t() @ X.abs()), what)


@pytest.mark.parametrize("F", [1, 2, 3, 4, 8])
@pytest.mark.parametrize("M,K", [(70, 200), (3000, 260)])
def test_gradients_f32_of_few_channels(M, K, F):
    """The gradient of the rows: sums of 2 F products."""
    g = gen(300 + F + M)
    x, wg, wu = normal(g, (M, K)), normal(g, (F, K)), normal(g, (F, K))
    gate, up, dh = (normal(g, (M, F)) for _ in range(3))
    dx, _, _ = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    dg, du = (dh * up).double(), (dh * gate).double()
    size = dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs()
    check(dx, dg @ wg.double() + du @ wu.double(), short_sum_tolerance(2 * F, size), "dx")


def test_gradients_f32_take_the_activation_of_the_forward_pass():
    """du = dh act(g) with the act(g) of the forward pass, bit for bit: u = 1 and dh = 1, sums of one product by 1."""
    g = gen(400)
    v = torch.cat([normal(g, (3000, 1), 3.0), torch.linspace(-100, 100, 1001, device="cuda")[:, None]])
    F = v.shape[0]
    one, zero = torch.ones_like(v), torch.zeros_like(v)
    x, wg, wu = torch.ones(1, 2, device="cuda"), torch.cat([v, zero], 1), torch.cat([zero, one], 1)
    h, gate, up = pl.gated_ff(x, wg, wu, keep=True)
    equal(gate, v.t())
    equal(up, one.t())
    _, dwg, dwu = pl.gated_ff_backward(torch.ones(1, F, device="cuda"), x, wg, wu, gate, up)
    equal(dwu[:, :1], h.t(), "du")


# ---------------------------------------------------------------------------------------------------------
# slices side by side
# ---------------------------------------------------------------------------------------------------------
def test_operands_and_results_side_by_side_in_one_buffer():
    g = gen(450)
    M, K, N = 37, 48, 40
    buf = torch.zeros(M, 2 * N + K, device="cuda")
    res, y, x = buf[:, :N], buf[:, N:2 * N], buf[:, 2 * N:]
    res.copy_(whole(g, (M, N), 9))
    x.copy_(whole(g, (M, K), 2))
    a, w = codes(g, (M, K)), codes(g, (N, K))
    before = buf.clone()
    assert pl.matmul_i8(a, None, w, None, residual=res, out_dt=B.F32, y=y) is y
    equal(y, (a.double() @ w.double().t()).float() + before[:, :N])
    wg, wu = whole(g, (N, K), 1), whole(g, (N, K), 1)
    pl.gated_ff(x, wg, wu, act=0, h=y)
    equal(y, ((x.double() @ wg.double().t()) * (x.double() @ wu.double().t())).float())
    equal(buf[:, :N], before[:, :N])
    equal(buf[:, 2 * N:], before[:, 2 * N:])
    one = torch.zeros(4 * M * K, dtype=torch.uint8, device="cuda")  # every row's codes in a gap of the rows
    rows = one.view(torch.bfloat16).view(M, 2 * K)
    q = one.view(torch.int8).view(M, 4 * K)[:, 2 * K:3 * K]
    rows[:, :K].copy_(x)
    _, s = pl.quantize_rows(rows[:, :K], q=q)
    equal(q.float() * s[:, None], q.float() * (x.abs().amax(1) / 127)[:, None])
    equal(q, torch.where(x.abs().amax(1, keepdim=True) > 0, x * 127 / x.abs().amax(1, keepdim=True), 0.0).double().round().to(torch.int8))


# ---------------------------------------------------------------------------------------------------------
# workspaces of gradients whose sums are shared by workgroups, and gradients far from 1
# ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("wanted", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,F", [(20, 70, 3333), (8192, 64, 40), (1500, 60, 1600), (130, 64, 9000)])
def test_workspaces_of_shared_sums(M, K, F, dt, wanted):
    """Counters and parts behind dg and du, in memory that holds anything; nothing is written behind the size asked for."""
    g = gen(460 + M)
    t = DT[dt]
    x, wg, wu = whole(g, (M, K), 2, t), whole(g, (F, K), 1, t), whole(g, (F, K), 1, t)
    gate, up, dh = (whole(g, (M, F), 2, t) for _ in range(3))
    n = B.rtoss_gated_ff_backward_size(B.GatedDesc(M, K, F, {"f32": B.F32, "bf16": B.BF16}[dt], B.ACT_NONE, 0, 0, 0))
    pitch = -(-F // (16 // t.itemsize)) * 16  # bytes
    assert n > 2 * (-(-M * pitch // 256) * 256), "this shape shares no sums"
    dg, du = dh.double() * up.double(), dh.double() * gate.double()
    want = [(dg @ wg.double() + du @ wu.double()).to(t), (dg.t() @ x.double()).to(t), (du.t() @ x.double()).to(t)]
    space = torch.empty(n + (1 << 20), dtype=torch.uint8, device="cuda")
    for fill in (201, 0, 255):
        space.fill_(fill)
        space[n:] = 77
        got = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0, rows=wanted[0], weights=wanted[1], workspace=space[:n])
        assert (space[n:] == 77).all()
        for a, b, asked in zip(got, want, (wanted[0], wanted[1], wanted[1])):
            assert (a is not None) == asked
            if asked:
                equal(a, b, "fill %d" % fill)


@pytest.mark.parametrize("scale", [2.0 ** -20, 2.0 ** -12, 2.0 ** 8])
def test_gradients_f16_far_from_one(scale):
    """dh at other scales: dg and du are rounded to fp16, among its subnormal numbers too, half a step each."""
    g = gen(470)
    t = torch.float16
    M, K, F = 70, 96, 130
    x, wg, wu = normal(g, (M, K)).to(t), normal(g, (F, K), K ** -0.5).to(t), normal(g, (F, K), K ** -0.5).to(t)
    gate, up, dh = normal(g, (M, F)).to(t), normal(g, (M, F)).to(t), (normal(g, (M, F)) * scale).to(t)
    dx, dwg, dwu = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    dg, du = dh.double() * up.double(), dh.double() * gate.double()
    eg, eu = ((half_step(t) + U) * v.abs() + least(t) for v in (dg, du))
    X, W, V = x.double(), wg.double(), wu.double()

    def close(got, want, error, size, n, what):
        tol = error + 2 * (n + 4) * U * size
        check(got, want, tol + half_step(t) * (want.abs() + tol) + least(t), what)

    close(dx, dg @ W + du @ V, eg @ W.abs() + eu @ V.abs(), (dg.abs() + eg) @ W.abs() + (du.abs() + eu) @ V.abs(), 2 * F, "dx")
    close(dwg, dg.t() @ X, eg.t() @ X.abs(), (dg.abs() + eg).t() @ X.abs(), M, "dw_gate")
    close(dwu, du.t() @ X, eu.t() @ X.abs(), (du.abs() + eu).t() @ X.abs(), M, "dw_up")


# ---------------------------------------------------------------------------------------------------------
# shapes of tensors
# ---------------------------------------------------------------------------------------------------------
def test_one_row_as_a_vector_and_channels_of_one():
    g = gen(480)
    K, F = 72, 50
    x, wg, wu, dh = whole(g, (K,), 2), whole(g, (F, K), 1), whole(g, (F, K), 1), whole(g, (F,), 2)
    q, s = pl.quantize_rows(x)
    assert q.shape == (K,) and s.shape == ()
    equal(q, (x.double() * 127 / x.abs().max()).round().to(torch.int8))
    y = pl.matmul_i8(q, s, codes(gen(1), (F, K)), None, out_dt=B.F32)
    equal(y, (q.double() @ codes(gen(1), (F, K)).double().t()).float() * s)
    h, gate, up = pl.gated_ff(x, wg, wu, act=1, keep=True)
    assert h.shape == gate.shape == up.shape == (F,)
    G, V = wg.double() @ x.double(), wu.double() @ x.double()
    equal(h, (torch.relu(G) * V).float())
    dx, dwg, dwu = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    dg, du = dh.double() * V, dh.double() * G
    equal(dx, (dg @ wg.double() + du @ wu.double()).float())
    equal(dwg, (dg[:, None] * x.double()).float())
    equal(dwu, (du[:, None] * x.double()).float())
    column = whole(g, (1, 40), 2).t()  # [40, 1] of rows one element apart, its last stride 40
    w = whole(g, (F, 1), 2)
    equal(pl.gated_ff(column, w, w, act=0), (column.double() * w[:, 0].double()).square().float())
    one = torch.zeros(3, 1, 5, K, device="cuda")[:, :, ::2]  # rows 2 K apart within a block, the blocks 5 K: no constant pitch
    with pytest.raises(AssertionError, match="distance"):
        pl.quantize_rows(one)


def test_workspaces_that_do_not_fit_are_refused():
    g = gen(481)
    x, w, t = whole(g, (20, 70), 2), whole(g, (3333, 70), 1), whole(g, (20, 3333), 2)
    n = B.rtoss_gated_ff_backward_size(B.GatedDesc(20, 70, 3333, B.F32, B.ACT_NONE, 0, 0, 0))
    space = torch.empty(n + 512, dtype=torch.uint8, device="cuda")
    for bad in (space[:n - 1], space[128:128 + n]):
        with pytest.raises(B.RtossError, match="workspace"):
            pl.gated_ff_backward(t, x, w, w, t, t, act=0, workspace=bad)
    for bad in (space[:n].view(torch.int8), torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError, match="workspace"):
            pl.gated_ff_backward(t, x, w, w, t, t, act=0, workspace=bad)
