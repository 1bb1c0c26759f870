"""Every kernel of the products (product_variants.py) on small whole numbers: every product and sum is exact in 32 bits, so results must equal the rounded
reference bit for bit, whatever the order of the additions.  Between the rows lies NaN, or codes of other values."""
import pytest
import torch

from paper_2303_02191_amd import pipeline as pl

from product_variants import MORE_TILES, VARIANTS
from product_routes import BACK, GATED, GATED_I8, I8
from test_gpu_products import ABI, DT, codes, equal, gen, inside, whole

pytestmark = pytest.mark.gpu

TYPES = {"i8": ("f32", "f16", "bf16"), "16": ("f16", "bf16"), "f32": ("f32",)}


def product(g, dt, M, K, N, pitch):
    """The sums are exact; scales and residual of whole numbers and a power of two, so that the rest is too, but for its roundings to fp32."""
    a, w = inside(codes(g, (M, K)), pitch, 77)[0], inside(codes(g, (N, K)), pitch, 55)[0]
    sa, sw, bias, residual = whole(g, (M,), 2) * 2.0 ** -6, whole(g, (N,), 2), whole(g, (N,), 3), whole(g, (M, N), 3, DT[dt])
    y = pl.matmul_i8(a, sa, w, sw, bias=bias, act=1, residual=residual, out_dt=ABI[dt])
    v = (a.double() @ w.double().t()).float() * sa[:, None] * sw + bias
    equal(y, (torch.relu(v) + residual.float()).to(DT[dt]))


def gated(g, dt, M, K, F, pitch):
    t = DT[dt]
    x = inside(whole(g, (M, K), 2, t), pitch, float("nan"))[0]
    wg, wu = (inside(whole(g, (F, K), 1, t), pitch, float("nan"))[0] for _ in range(2))
    G, V = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    h, gate, up = pl.gated_ff(x, wg, wu, act=1, keep=True)
    equal(gate, G.to(t), "gate")
    equal(up, V.to(t), "up")
    equal(h, (torch.relu(G) * V).float().to(t), "h")
    equal(pl.gated_ff(x, wg, wu, act=1), h, "h alone")


def gated_i8(g, dt, M, K, F, pitch):
    a = inside(codes(g, (M, K)), pitch, 77)[0]
    wg, wu = (inside(codes(g, (F, K)), pitch, 55)[0] for _ in range(2))
    sa, sg, su = whole(g, (M,), 1) * 2.0 ** -12, whole(g, (F,), 1), whole(g, (F,), 1)
    h = pl.gated_ff_i8(a, sa, wg, sg, wu, su, act=1, out_dt=ABI[dt])
    G, V = ((a.double() @ w.double().t()).float() * sa[:, None] * s for w, s in ((wg, sg), (wu, su)))
    equal(h, (torch.relu(G) * V).to(DT[dt]))


def gradients(g, dt, M, K, F, pitch):
    """dg and du are at most 4, sums of up to 2 * 16384 products of at most 8."""
    t = DT[dt]
    x = inside(whole(g, (M, K), 2, t), pitch, float("nan"))[0]
    wg, wu = (inside(whole(g, (F, K), 2, t), pitch, float("nan"))[0] for _ in range(2))
    dh = inside(whole(g, (M, F), 2, t), pitch, float("nan"))[0]
    gate, up = whole(g, (M, F), 2, t), whole(g, (M, F), 2, t)
    dg, du = dh.double() * up.double(), dh.double() * gate.double()
    want = ((dg @ wg.double() + du @ wu.double()).to(t), (dg.t() @ x.double()).to(t), (du.t() @ x.double()).to(t))
    for rows, weights in ((True, True), (True, False), (False, True)):
        got = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0, rows=rows, weights=weights)
        for a, b, what in zip(got, want, ("dx", "dw_gate", "dw_up")):
            if a is not None:
                equal(a, b, "%s of %d %d" % (what, rows, weights))


CHECKS = {I8: product, GATED: gated, GATED_I8: gated_i8, BACK: gradients}


@pytest.mark.parametrize("kernel,cls,what,shapes", VARIANTS, ids=["%s-%s" % v[:2] for v in VARIANTS])
def test_variant(kernel, cls, what, shapes):
    for shape in shapes:
        for dt in TYPES[cls]:
            print(kernel, dt, shape, flush=True)
            CHECKS[what](gen(sum(shape)), dt, *shape)


@pytest.mark.parametrize("shape", [v[2] for v in MORE_TILES])
def test_gradients_of_more_tiles_than_a_launch_has(shape):
    """268 million rows of one channel in fp32.  One row of x in 1024 is not zero: sums of at most 262208 * 8."""
    M, K, F, pitch = shape
    g = gen(K)
    x = torch.zeros(M, K + pitch, device="cuda")[:, :K]
    x[5::1024] = whole(g, (len(range(5, M, 1024)), K), 2)
    x[-1] = 1.0
    wg, wu = whole(g, (F, K + pitch), 2)[:, :K], whole(g, (F, K + pitch), 2)[:, :K]
    dh = torch.randint(-2, 3, (M, F + pitch), generator=g, device="cuda", dtype=torch.int8).float()[:, :F]
    gate, up = (torch.randint(-2, 3, (M, F), generator=g, device="cuda", dtype=torch.int8).float() for _ in range(2))
    dx, dwg, dwu = pl.gated_ff_backward(dh, x, wg, wu, gate, up, act=0)
    dg, du = dh * up, dh * gate
    assert torch.equal(dx, dg * wg + du * wu)
    for got, d in ((dwg, dg), (dwu, du)):
        equal(got, torch.stack([(d[:, 0] * x[:, k]).sum(dtype=torch.float64) for k in range(K)])[None].float())
