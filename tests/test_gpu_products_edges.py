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
    """One row and x = 1: the gradients of the weights are dg and du.  dg = dh u act'(g) and du = dh act(g) in IEEE arithmetic, the slope of a NaN a NaN
    (fp32: infinite dg and du are operands, and make NaN).  Whole numbers, so that nothing is rounded; with SiLU only what is not finite is compared."""
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
        if dt == "f32":
            want = torch.where(want.isinf(), nan, want)
        if a == 2:
            got, want = torch.where(got.isfinite(), 0.0, got), torch.where(want.isfinite(), 0.0, want)
        same(got, want.to(t), what)
    assert dx.isnan().all()  # (NaN enters the row's sum)
