"""The products' dispatch, replayed without a GPU: product_variants.py names the kernel each of its calls launches, and together they launch
every one that the library holds, so that a change of an estimate cannot empty a GPU test unnoticed."""
import pytest

from paper_2303_02191_amd import binding as B

import product_routes as routes
from product_variants import MORE_TILES, VARIANTS

TYPES = {"i8": (B.F32, B.F16, B.BF16), "16": (B.F16, B.BF16), "f32": (B.F32,)}


def without_types(kernel):
    """'product_tiles<i8,f32,0,256,128,0>' -> ('product_tiles<0,256,128,0>', 'i8')"""
    name, args = kernel[:-1].split("<")
    args = args.split(",")
    types = [a for a in args if a in ("i8", "f32", "f16", "bf16")]
    return "%s<%s>" % (name, ",".join(a for a in args if a not in types)), "i8" if "i8" in types else "f32" if types[0] == "f32" else "16"


@pytest.mark.parametrize("cls", list(TYPES))
def test_every_call_takes_the_kernel_that_the_list_names(cls):
    calls, want = [], []
    for kernel, c, what, shapes in VARIANTS:
        if c == cls:
            for shape in shapes:
                for dt in TYPES[cls]:
                    calls.append((what, dt, *shape))
                    want.append((kernel, cls))
    if cls == "f32":
        for rows, weights, shape in MORE_TILES:
            calls += [(routes.BACK, B.F32, *shape, 1, 0), (routes.BACK, B.F32, *shape, 0, 1)]
            want += [(rows, cls), (weights, cls)]
    got = [[without_types(k) for k in ks] for ks in routes.kernels(calls)]
    assert [(c, g, w) for c, g, w in zip(calls, got, want) if w not in g] == []


def test_the_list_covers_the_library():
    held = {without_types(k) for k in routes.library_kernels() if k.startswith("product_")}
    listed = {v[:2] for v in VARIANTS} | {(k, "f32") for v in MORE_TILES for k in v[:2]}
    assert held == listed


def test_row_codes_and_slopes_reach_every_kernel():
    calls = [(routes.CODES, dt, 3, K, 1, 0) for dt in TYPES["i8"] for K in (1, 128, 129, 256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 32769)]
    got = {k for ks in routes.kernels(calls) for k in ks}
    assert got == {k for k in routes.library_kernels() if k.startswith("quantize_rows")}


def test_launches_stay_within_the_lds_they_declare():
    calls = [(what, dt, *shape) for _, cls, what, shapes in VARIANTS for shape in shapes for dt in TYPES[cls]]
    calls += [(routes.BACK, B.F32, *shape) for _, _, shape in MORE_TILES]
    calls += [(what, B.BF16, M, K, N, 0) for what in (routes.I8, routes.GATED, routes.GATED_I8, routes.BACK)
              for M, K, N in ((2 ** 31 - 1, 1, 1), (1, 2 ** 17 - 1, 2 ** 24), (2 ** 28, 16, 2 ** 10), (0, 5, 7))]
    wrong = []
    for c, launches in zip(calls, routes.launches(calls)):
        for kernel, groups, lanes, lds, limit in launches:
            if not (0 < groups * lanes < 2 ** 32 and lds <= limit <= 160 * 1024):
                wrong.append((c, kernel, groups, lanes, lds, limit))
    assert wrong == []


def test_one_gradient_alone_takes_the_kernels_of_both():
    """... so that it has the same bits: no kernel that both together do not launch."""
    for cls, shape in (("f32", (130, 264, 200, 0)), ("16", (2000, 512, 700, 3)), ("16", (8192, 4096, 10944, 0)), ("16", (4100, 33, 20, 0))):
        for dt in TYPES[cls]:
            both, rows, weights = routes.kernels([(routes.BACK, dt, *shape, r, w) for r, w in ((1, 1), (1, 0), (0, 1))])
            assert set(rows) <= set(both) and set(weights) <= set(both) and set(rows) | set(weights) == set(both)
