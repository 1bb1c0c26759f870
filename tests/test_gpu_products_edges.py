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
