"""Which kernels a call of the products launches (products_probe.cpp): no GPU needed."""
import functools
import os
import re
import subprocess
import tempfile

from conftest import ROOT

from paper_2303_02191_amd import binding as B
from paper_2303_02191_amd import build

I8, GATED, GATED_I8, BACK, CODES = range(5)
_TYPES = {"rtoss::f16_t": "f16", "rtoss::bf16_t": "bf16", "float": "f32", "signed char": "i8"}


@functools.lru_cache(None)
def _probe():
    exe = os.path.join(tempfile.mkdtemp(prefix="rtoss_products_"), "products_probe")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-isystem", os.path.join(rocm, "include"),
                           "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "products_probe.cpp"), "-o", exe, "-rdynamic", build.LIB,
                           "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-ldl", "-Wl,-rpath," + build.HERE, "-Wl,-rpath," + os.path.join(rocm, "lib")])
    names = {}
    for line in subprocess.check_output(["nm", "-C", build.LIB], text=True).splitlines():
        m = re.match(r"([0-9a-f]+) . void rtoss::(?:\(anonymous namespace\)::)?(?!__device_stub__)(\w+)_kernel<(.*?)>\(", line)
        if m and m.group(2) in ("product_slices", "product_slices_back", "product_tiles", "quantize_rows", "gated_slopes"):
            args = [_TYPES.get(a, a) for a in m.group(3).split(", ")]
            names[int(m.group(1), 16)] = "%s<%s>" % (m.group(2), ",".join(args))
    return exe, names


def launches(calls):
    """calls: tuples (what, dt, M, K, N, pitch[, rows, weights]).  Returns for each the list of its launches (kernel, workgroups, lanes, dynamic LDS bytes,
    their limit), the kernel as 'product_slices<i8,f32,0,0,16,16,8,false>', or the status of a call that was refused."""
    exe, names = _probe()
    text = "".join("%d %d %d %d %d %d %d %d\n" % (*c[:6], *(map(int, c[6:]) if len(c) > 6 else (1, 1))) for c in calls)
    out = []
    for line in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines():
        status, *rest = line.split()
        found = [(names[int(rest[i], 16)], *map(int, rest[i + 1:i + 5])) for i in range(0, len(rest), 5)]
        out.append(found if int(status) == B.OK else int(status))
    assert len(out) == len(calls)
    return out


def kernels(calls):
    return [r if isinstance(r, int) else [l[0] for l in r] for r in launches(calls)]


def library_kernels():
    return set(_probe()[1].values())
