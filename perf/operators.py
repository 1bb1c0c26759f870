"""The 8-bit products and the gated feed-forward block: what they are timed on.

A case is a dict of plain values.  `kind` says which pass it is (M rows, K input channels, N or F output channels):

  i8        y = act(s_a[m] * s_w[n] * sum_k a[m][k] w[n][k] + bias[n]) + residual, 8-bit operands; `dynamic`: from 16- or 32-bit
            rows that are quantized within the pass
  ff        h = act(x Wg^T) * (x Wu^T), one pass over x; `keep`: both projections are kept for the backward pass
  ff_back   gradients of x, Wg and Wu from those of h
  ff_i8     the gated block on rows that are quantized within the pass, and 8-bit weights
  block_i8  a feed-forward block as it is served: quantized rows, gated block, quantized rows, product plus the residual
"""
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------------------------------------------------
# cases.  F is eight thirds of K, as gated blocks have it, rounded up to a multiple of 64.
# ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one generated token through a square projection: the smallest call, latency and the weights' bytes
        {"name": "i8_token", "kind": "i8", "dynamic": True, "dt": "bf16", "out": "bf16", "M": 1, "K": 4096, "N": 4096, "act": 0,
         "bias": False, "residual": True, "pitch": 0},
        # a small batch through a layer of odd sizes, rows inside a wider buffer, 32-bit results
        {"name": "i8_odd_f32out", "kind": "i8", "dynamic": True, "dt": "f16", "out": "f32", "M": 77, "K": 1021, "N": 1003, "act": 2,
         "bias": True, "residual": False, "pitch": 3},
        # a 1x1 layer of a detector (256 -> 256 channels on 8 x 80 x 80 positions) with folded norm and SiLU
        {"name": "i8_positions", "kind": "i8", "dynamic": True, "dt": "f16", "out": "f16", "M": 51200, "K": 256, "N": 256, "act": 2,
         "bias": True, "residual": False, "pitch": 0},
        # a long prompt through a wide layer, activations quantized before (shared by several layers)
        {"name": "i8_large", "kind": "i8", "dynamic": False, "dt": "bf16", "out": "bf16", "M": 8192, "K": 8192, "N": 8192, "act": 0,
         "bias": False, "residual": True, "pitch": 0},
        # eight sequences generating, gated block in 8 bits
        {"name": "ff_i8_decode", "kind": "ff_i8", "dt": "bf16", "out": "bf16", "M": 8, "K": 4096, "F": 10944, "act": 2, "pitch": 0},
        # a prompt through the whole served block
        {"name": "block_i8_prefill", "kind": "block_i8", "dt": "bf16", "out": "bf16", "M": 2048, "K": 4096, "F": 10944, "act": 2, "pitch": 0},
        # one token, 16-bit weights
        {"name": "ff_token", "kind": "ff", "dt": "f16", "M": 1, "K": 2048, "F": 5504, "act": 2, "keep": False, "pitch": 0},
        # a ragged batch of prompts, no backward pass
        {"name": "ff_prefill", "kind": "ff", "dt": "bf16", "M": 1000, "K": 4096, "F": 10944, "act": 2, "keep": False, "pitch": 0},
        # a small model trained in full precision
        {"name": "ff_train_f32", "kind": "ff", "dt": "f32", "M": 512, "K": 1024, "F": 2752, "act": 2, "keep": True, "pitch": 0},
        # a training step's forward pass
        {"name": "ff_train_large", "kind": "ff", "dt": "bf16", "M": 8192, "K": 4096, "F": 10944, "act": 2, "keep": True, "pitch": 0},
        # gradients at odd sizes, another activation
        {"name": "ff_back_odd", "kind": "ff_back", "dt": "f16", "M": 333, "K": 520, "F": 1387, "act": 1, "pitch": 0},
        # a training step's backward pass
        {"name": "ff_back_large", "kind": "ff_back", "dt": "bf16", "M": 8192, "K": 4096, "F": 10944, "act": 2, "pitch": 0},
    ]


def _size(rng, low, high):
    """Spread over the logarithm; every other one a multiple of 64, where there is one."""
    v = int(round(low * (high / low) ** rng.random()))
    if rng.random() < 0.5 and high >= 64:
        v = max(64, v // 64 * 64)
    return min(v, high)


def draw(rng):
    kind = rng.choice(["i8", "i8", "ff", "ff", "ff_back", "ff_back", "ff_i8", "block_i8"])
    M = int(round(8192 ** rng.random()))
    c = {"kind": kind, "dt": rng.choice(["f32", "f16", "bf16", "bf16"]), "M": M, "act": rng.choice([0, 1, 2, 2]),
         "pitch": rng.choice([0, 0, 0, 8, 3])}
    if kind == "i8":
        c["K"], c["N"] = _size(rng, 16, 8192), _size(rng, 16, 10944)
        c["dynamic"] = rng.random() < 0.6
        c["out"] = rng.choice(["f32", "f16", "bf16", "bf16"])
        c["bias"], c["residual"] = rng.random() < 0.5, rng.random() < 0.5
        return c
    c["K"], c["F"] = _size(rng, 16, 4096), _size(rng, 16, 10944)
    if kind == "ff":
        c["keep"] = rng.random() < 0.5
    elif kind == "block_i8":  # (16-bit: the block quantizes its own hidden values, whose last bits pick a code now and then)
        c["dt"] = c["out"] = rng.choice(["f16", "bf16"])
    elif kind == "ff_i8":
        c["out"] = rng.choice(["f32", "f16", "bf16", "bf16"])
    return c


# ---------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------
def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std


def _rows(gen, M, K, dt, pitch):
    """Activations: normal with a few channels of much larger values, in a buffer `pitch` elements wider than a row."""
    x = _normal(gen, (M, K + pitch))
    outlier = torch.rand(K + pitch, generator=gen, device="cuda") < 0.01
    x *= torch.where(outlier, 12.0, 1.0)
    return x.to(DTYPES[dt])[:, :K]


def _codes(v):
    """8-bit codes and scales of rows that a program holds already."""
    top = v.abs().amax(dim=1, keepdim=True)
    return (v * (127.0 / top)).round().to(torch.int8), (top / 127.0).reshape(-1)


def _weight(gen, rows, cols):
    return _normal(gen, (rows, cols), cols ** -0.5)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c, s = case, {"case": dict(case)}
    M, K = c["M"], c["K"]
    kind = c["kind"]
    if kind == "i8":
        s["w"], s["ws"] = _codes(_weight(gen, c["N"], K))
        s["bias"] = _normal(gen, (c["N"],)) if c["bias"] else None
        s["residual"] = _normal(gen, (M, c["N"])).to(DTYPES[c["out"]]) if c["residual"] else None
        if c["dynamic"]:
            s["x"] = _rows(gen, M, K, c["dt"], c["pitch"])
        else:
            s["q"], s["qs"] = _codes(_rows(gen, M, K, "f32", 0))
    elif kind in ("ff_i8", "block_i8"):
        s["x"] = _rows(gen, M, K, c["dt"], c["pitch"])
        s["wg"], s["wgs"] = _codes(_weight(gen, c["F"], K))
        s["wu"], s["wus"] = _codes(_weight(gen, c["F"], K))
        if kind == "block_i8":
            s["wd"], s["wds"] = _codes(_weight(gen, K, c["F"]))
    else:
        dt = DTYPES[c["dt"]]
        s["x"] = _normal(gen, (M, K + c["pitch"])).to(dt)[:, :K]
        s["wg"], s["wu"] = _weight(gen, c["F"], K).to(dt), _weight(gen, c["F"], K).to(dt)
        if kind == "ff_back":
            s["gate"], s["up"] = _normal(gen, (M, c["F"])).to(dt), _normal(gen, (M, c["F"])).to(dt)
            s["dh"] = _normal(gen, (M, c["F"])).to(dt)
    return s


# ---------------------------------------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits, the codes of quantized rows in 64 (a value next to a border between two codes)
# ---------------------------------------------------------------------------------------------------------
def _act(v, act):
    return v if act == 0 else torch.clamp_min(v, 0.0) if act == 1 else v / (1.0 + torch.exp(-v))


def _act_slope(v, act):
    if act == 0:
        return torch.ones_like(v)
    if act == 1:
        return (v > 0).to(v.dtype)
    s = 1.0 / (1.0 + torch.exp(-v))
    return s * (1.0 + v * (1.0 - s))


def _quantized(x):
    v = x.double()
    top = v.abs().amax(dim=1, keepdim=True)
    codes = torch.where(top > 0, v * 127.0 / top, torch.zeros_like(v)).round()
    return codes.float(), (top / 127.0).float()


def _product_i8(q, qs, w, ws, act, bias, residual, out):
    y = (q @ w.float().t()) * qs * ws
    y = _act(y if bias is None else y + bias, act)
    return (y if residual is None else y + residual.float()).to(out)


def _plain(s):
    c = s["case"]
    kind, act = c["kind"], c["act"]
    if kind == "i8":
        q, qs = _quantized(s["x"]) if c["dynamic"] else (s["q"].float(), s["qs"].reshape(-1, 1))
        return {"y": _product_i8(q, qs, s["w"], s["ws"], act, s["bias"], s["residual"], DTYPES[c["out"]])}
    if kind in ("ff_i8", "block_i8"):
        q, qs = _quantized(s["x"])
        g, u = (q @ s["wg"].float().t()) * qs * s["wgs"], (q @ s["wu"].float().t()) * qs * s["wus"]
        h = (_act(g, act) * u).to(DTYPES[c["out"]])
        if kind == "ff_i8":
            return {"h": h}
        q, qs = _quantized(h)
        return {"y": _product_i8(q, qs, s["wd"], s["wds"], 0, None, s["x"], DTYPES[c["out"]])}
    dt = DTYPES[c["dt"]]
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    if kind == "ff":
        g, u = x @ wg.t(), x @ wu.t()
        h = (_act(g, act) * u).to(dt)
        return {"h": h, "gate": g.to(dt), "up": u.to(dt)} if c["keep"] else {"h": h}
    g, u, dh = s["gate"].float(), s["up"].float(), s["dh"].float()
    du, dg = dh * _act(g, act), dh * u * _act_slope(g, act)
    return {"dx": (dg @ wg + du @ wu).to(dt), "dwg": (dg.t() @ x).to(dt), "dwu": (du.t() @ x).to(dt)}


def _own(s):
    from paper_2303_02191_amd import binding as B
    from paper_2303_02191_amd import pipeline as pl
    c = s["case"]
    kind, act = c["kind"], c["act"]
    out = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}[c.get("out", c["dt"])]
    if kind == "i8":
        q, qs = pl.quantize_rows(s["x"]) if c["dynamic"] else (s["q"], s["qs"])
        return {"y": pl.matmul_i8(q, qs, s["w"], s["ws"], bias=s["bias"], act=act, residual=s["residual"], out_dt=out)}
    if kind in ("ff_i8", "block_i8"):
        q, qs = pl.quantize_rows(s["x"])
        h = pl.gated_ff_i8(q, qs, s["wg"], s["wgs"], s["wu"], s["wus"], act=act, out_dt=out)
        if kind == "ff_i8":
            return {"h": h}
        q, qs = pl.quantize_rows(h)
        return {"y": pl.matmul_i8(q, qs, s["wd"], s["wds"], residual=s["x"], out_dt=out)}
    if kind == "ff":
        if not c["keep"]:
            return {"h": pl.gated_ff(s["x"], s["wg"], s["wu"], act=act)}
        h, gate, up = pl.gated_ff(s["x"], s["wg"], s["wu"], act=act, keep=True)
        return {"h": h, "gate": gate, "up": up}
    dx, dwg, dwu = pl.gated_ff_backward(s["dh"], s["x"], s["wg"], s["wu"], s["gate"], s["up"], act=act)
    return {"dx": dx, "dwg": dwg, "dwu": dwu}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c = case
    M, K, e = c["M"], c["K"], BYTES[c["dt"]]
    kind = c["kind"]
    if kind == "i8":
        N, o = c["N"], BYTES[c["out"]]
        moved = (M * K * e if c["dynamic"] else M * K + 4 * M) + N * K + 4 * N + M * N * o
        return {"bytes": moved + (4 * N if c["bias"] else 0) + (M * N * o if c["residual"] else 0), "flops": 2 * M * N * K}
    F = c["F"]
    if kind == "ff_i8":
        return {"bytes": M * K * e + 2 * F * K + 8 * F + M * F * BYTES[c["out"]], "flops": 4 * M * K * F}
    if kind == "block_i8":
        return {"bytes": 2 * M * K * e + 3 * F * K + 8 * F + 4 * K, "flops": 6 * M * K * F}
    if kind == "ff":
        return {"bytes": (M * K + 2 * F * K + (3 if c["keep"] else 1) * M * F) * e, "flops": 4 * M * K * F}
    return {"bytes": (2 * M * K + 4 * F * K + 3 * M * F) * e, "flops": 8 * M * K * F}


# ---------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    activation = {0: lambda t: t, 1: torch.relu, 2: lambda t: t * torch.sigmoid(t)}[case["act"]]
    kind = case["kind"]

    def codes(t):
        peak = t.abs().max(dim=1, keepdim=True).values
        return torch.nan_to_num(torch.round(127.0 * t / peak), nan=0.0), peak / 127.0

    def channels(a, a_scale, w, w_scale):
        return torch.matmul(a, w.transpose(0, 1)) * (a_scale * w_scale.reshape(1, -1))

    if kind == "i8":
        a, a_scale = codes(d["x"]) if case["dynamic"] else (d["q"], d["qs"].reshape(-1, 1))
        return {"y": activation(channels(a, a_scale, d["w"], d["ws"]) + d.get("bias", 0.0)) + d.get("residual", 0.0)}
    if kind in ("ff_i8", "block_i8"):
        a, a_scale = codes(d["x"])
        h = activation(channels(a, a_scale, d["wg"], d["wgs"])) * channels(a, a_scale, d["wu"], d["wus"])
        if kind == "ff_i8":
            return {"h": h}
        a, a_scale = codes(h.to(DTYPES[case["out"]]).double())
        return {"y": channels(a, a_scale, d["wd"], d["wds"]) + d["x"]}
    if kind == "ff":
        gate, up = torch.matmul(d["x"], d["wg"].transpose(0, 1)), torch.matmul(d["x"], d["wu"].transpose(0, 1))
        h = activation(gate) * up
        return {"h": h, "gate": gate, "up": up} if case["keep"] else {"h": h}
    gate = d["gate"].requires_grad_(True)
    act_of_gate = activation(gate)
    (slope,) = torch.autograd.grad(act_of_gate.sum(), gate)
    through_gate, through_up = d["dh"] * d["up"] * slope, d["dh"] * act_of_gate.detach()
    return {"dx": torch.matmul(through_gate, d["wg"]) + torch.matmul(through_up, d["wu"]),
            "dwg": torch.matmul(through_gate.transpose(0, 1), d["x"]), "dwu": torch.matmul(through_up.transpose(0, 1), d["x"])}
