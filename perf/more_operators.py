"""Timed operators of a feed-forward block in the pass that the V step's gradient comes from: what stands between a student's
4-bit products.

  norm        y = (r - mean) / sqrt(var + eps) w + b of each row of r = x + residual, with the mean or without
  norm_grad   its gradients by the row, by w and by b
  gated       h = f(x_hat wg_hat^T) (x_hat wu_hat^T), two products on 4-bit matrices with the activation between them
  gated_grad  its gradients by both products (from the 4-bit matrices again) and by x
  block       a whole block's forward pass: residual and norm into 4 bits, gated products into 4 bits, the product that follows

Block formats: "e8m0_32" has 32 elements to a power-of-two scale, "e4m3_16" has 16 to an 8-bit float scale, times one
scale of the whole matrix where there is one.  Elements are e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives.
Codes lie two to a byte, the even column in the lower half, in rows of a multiple of 16 bytes; scales lie in tiles of
128 rows x 4 blocks, byte 16 (r % 32) + 4 (r / 32) + b of a tile, tiles of a strip of 128 rows one after the other and
as many as 256 columns need.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = {"e8m0_32": 32, "e4m3_16": 16}
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
LARGEST_PRODUCT = 4096 * 8192 * 28672
LARGEST_AREA = 16384 * 8192


# ---- cases ---------------------------------------------------------------------------------------------------
def _norm(name, rows, cols, kind, dtype, out, weight="f32", residual=False, pad=0):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "kind": kind, "dtype": dtype, "out": out, "weight": weight,
            "residual": residual, "pad": pad}


def _norm_grad(name, rows, cols, kind, dtype, out, weight="f32", residual=False, pad=0):
    return {"name": name, "op": "norm_grad", "rows": rows, "cols": cols, "kind": kind, "dtype": dtype, "out": out,
            "weight": weight, "residual": residual, "pad": pad}


def _gated(name, tokens, cols, rows, fmt, act, out, tensor_scale=False):
    return {"name": name, "op": "gated", "tokens": tokens, "cols": cols, "rows": rows, "fmt": fmt, "act": act, "out": out,
            "tensor_scale": tensor_scale}


def _gated_grad(name, tokens, cols, rows, fmt, act, tensor_scale=False):
    return {"name": name, "op": "gated_grad", "tokens": tokens, "cols": cols, "rows": rows, "fmt": fmt, "act": act,
            "tensor_scale": tensor_scale}


def _block(name, tokens, cols, rows, fmt, act, kind, tensor_scale=False):
    return {"name": name, "op": "block", "tokens": tokens, "cols": cols, "rows": rows, "fmt": fmt, "act": act, "kind": kind,
            "tensor_scale": tensor_scale}


def listed():
    return [
        # the norm ahead of a layer for one generated token: latency alone
        _norm("norm_token_bf16", 1, 4096, "rms", "bf16", "bf16", residual=True),
        # a training batch at the width of the largest model, the residual stream in 16 bits
        _norm("norm_batch_bf16", 4096, 8192, "layer", "bf16", "bf16", weight="bf16", residual=True),
        # activations cut out of a wider array, rows of no alignment
        _norm("norm_ragged_f16", 2047, 5001, "layer", "f16", "f32", pad=7),
        # its backward pass: the gradient of the residual joins, the weights' gradient is summed over the batch
        _norm_grad("norm_grad_batch_bf16", 4096, 8192, "rms", "bf16", "bf16", residual=True),
        # a few calibration rows, odd everywhere, in 32 bits
        _norm_grad("norm_grad_ragged_f32", 333, 5119, "layer", "f32", "f32", pad=1),
        # generation: one token through the two projections of a feed-forward block
        _gated("gated_token_e8m0", 1, 4096, 11008, "e8m0_32", "silu", "bf16"),
        # a long prompt or a training batch through the largest ones
        _gated("gated_prompt_e8m0", 4096, 8192, 28672, "e8m0_32", "silu", "bf16"),
        # a short prompt, odd everywhere, the finer format
        _gated("gated_ragged_e4m3", 333, 5119, 13823, "e4m3_16", "gelu_tanh", "f32", tensor_scale=True),
        # backward of a training batch
        _gated_grad("gated_grad_batch_e8m0", 2048, 4096, 11008, "e8m0_32", "silu"),
        # backward of a few calibration tokens, odd everywhere
        _gated_grad("gated_grad_ragged_e4m3", 77, 5119, 4095, "e4m3_16", "gelu", tensor_scale=True),
        # the whole block for one generated token
        _block("block_token_e8m0", 1, 4096, 11008, "e8m0_32", "silu", "rms"),
        # and for a training batch
        _block("block_batch_e4m3", 2048, 4096, 11008, "e4m3_16", "silu", "rms", tensor_scale=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "gated", "gated", "gated_grad", "gated_grad", "block"])
    if op in ("norm", "norm_grad"):
        cols = _log(rng, 64, 20000)
        if rng.random() < 0.5:
            cols = (cols + 63) // 64 * 64
        rows = _log(rng, 1, LARGEST_AREA // cols // (2 if op == "norm_grad" else 1))
        make = _norm if op == "norm" else _norm_grad
        return _drawn(make("", rows, cols, rng.choice(["layer", "rms"]), rng.choice(sorted(DTYPE)), rng.choice(sorted(DTYPE)),
                           rng.choice(["f32", "f32", "bf16", "f16"]), rng.random() < 0.5, rng.choice([0, 0, 0, 1, 8, 13])))
    fmt = rng.choice(sorted(BLOCK))
    scaled = fmt == "e4m3_16"
    cols, rows = _log(rng, 33, 16384), _log(rng, 16, 28672)
    tokens = rng.choice([rng.randint(1, 16), _log(rng, 1, 8192)])
    tokens = max(1, min(tokens, LARGEST_PRODUCT // (2 * cols * rows)))
    act = rng.choice(["silu", "gelu", "gelu_tanh"])
    if op == "gated":
        return _drawn(_gated("", tokens, cols, rows, fmt, act, rng.choice(["bf16", "f16", "f32"]), scaled))
    if op == "gated_grad":
        return _drawn(_gated_grad("", min(tokens, 4096), cols, rows, fmt, act, scaled))
    return _drawn(_block("", min(tokens, 4096), cols, rows, fmt, act, rng.choice(["layer", "rms"]), scaled))


def _drawn(case):
    del case["name"]
    return case


def work(case):
    op = case["op"]
    if op in ("norm", "norm_grad"):
        n, c = case["rows"] * case["cols"], case["cols"]
        size, out, w = SIZE[case["dtype"]], SIZE[case["out"]], SIZE[case["weight"]]
        vectors = (2 if case["kind"] == "layer" else 1) * c
        if op == "norm":  # x (residual, sum), y, weights, statistics
            return {"bytes": n * (size * (3 if case["residual"] else 1) + out) + vectors * w + 8 * case["rows"], "flops": 8 * n}
        # x, dy, (dresidual,) dx, weights, their gradients, statistics
        return {"bytes": n * (size + out * (3 if case["residual"] else 2)) + c * w + vectors * 4 + 8 * case["rows"],
                "flops": 14 * n}
    t, c, r = case["tokens"], case["cols"], case["rows"]
    held = lambda n: n // 2 + n // BLOCK[case["fmt"]]  # noqa: E731
    if op == "gated":
        return {"bytes": held(t * c) + 2 * held(r * c) + t * r * SIZE[case["out"]], "flops": 4 * t * c * r}
    if op == "gated_grad":
        return {"bytes": held(t * c) + 2 * held(r * c) + 6 * t * r + 2 * t * c, "flops": 8 * t * c * r}
    return {"bytes": 6 * t * c + 4 * c + 3 * held(r * c) + 2 * t * c, "flops": 6 * t * c * r}


# ---- inputs --------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _heavy(gen, rows, cols, std):
    """Normally distributed with a gain per column, as activations have it."""
    return _normal(gen, rows, cols) * (std * torch.exp(0.5 * _normal(gen, 1, cols)))


def _tensor_scale(x):
    return (x.abs().amax() / (6.0 * 448.0)).reshape(1).float()


def _held(gen, rows, cols, fmt, std, scaled):
    """A matrix held in 4 bits: codes and scales as they lie in memory."""
    x = _heavy(gen, rows, cols, std)
    return _hold(x, fmt, _tensor_scale(x) if scaled else None)


def _rows(gen, rows, cols, pad, dtype, std=1.0, offset=0.0):
    """Rows of `cols` elements cut out of wider ones."""
    wide = torch.empty(rows, cols + pad, dtype=DTYPE[dtype], device="cuda")[:, :cols]
    return wide.copy_(_heavy(gen, rows, cols, std).add_(offset))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 29)
    op = case["op"]
    if op in ("norm", "norm_grad"):
        rows, cols, pad, dtype, layer = case["rows"], case["cols"], case["pad"], case["dtype"], case["kind"] == "layer"
        state = {"case": case, "x": _rows(gen, rows, cols, pad, dtype, offset=0.3),
                 "weight": (1.0 + 0.2 * _normal(gen, cols)).to(DTYPE[case["weight"]]),
                 "bias": (0.1 * _normal(gen, cols)).to(DTYPE[case["weight"]]) if layer else None}
        if op == "norm":
            state["residual"] = _rows(gen, rows, cols, pad, dtype, offset=0.3) if case["residual"] else None
            state["total"] = torch.empty(rows, cols, dtype=DTYPE[dtype], device="cuda") if case["residual"] else None
            state["y"] = torch.empty(rows, cols, dtype=DTYPE[case["out"]], device="cuda")
            state["stats"] = torch.empty(rows, 2, device="cuda")
            return state
        out = case["out"]
        state["stats"] = torch.cat([torch.stack(_statistics(part.double(), layer), dim=1) for part in state["x"].split(1024)]).float()
        state["dy"] = _rows(gen, rows, cols, pad, out, std=1e-2)
        state["dres"] = _rows(gen, rows, cols, pad, out, std=1e-2) if case["residual"] else None
        state["dx"] = torch.empty(rows, cols + pad, dtype=DTYPE[out], device="cuda")[:, :cols]
        state["dweight"] = torch.empty(cols, device="cuda")
        state["dbias"] = torch.empty(cols, device="cuda") if layer else None
        return state
    t, c, r, fmt = case["tokens"], case["cols"], case["rows"], case["fmt"]
    state = {"case": case}
    # (the two projections of a block share a tensor scale)
    wg, wu = _heavy(gen, r, c, 0.02), _heavy(gen, r, c, 0.02)
    ts = torch.maximum(_tensor_scale(wg), _tensor_scale(wu)) if case["tensor_scale"] else None
    state["wg"], state["wu"] = _hold(wg, fmt, ts), _hold(wu, fmt, ts)
    if op != "block":
        state["x"] = _held(gen, t, c, fmt, 1.0, case["tensor_scale"])
    if op == "gated":
        state["h"] = torch.empty(t, r, dtype=DTYPE[case["out"]], device="cuda")
        return state
    if op == "gated_grad":
        state["dh"] = (1e-3 * _normal(gen, t, r)).bfloat16()
        pitch = (r + 7) // 8 * 8
        state["dgate"] = torch.empty(t, pitch, dtype=torch.bfloat16, device="cuda")[:, :r]
        state["dup"] = torch.empty(t, pitch, dtype=torch.bfloat16, device="cuda")[:, :r]
        state["dx"] = torch.empty(t, c, dtype=torch.bfloat16, device="cuda")
        return state
    state["x"], state["residual"] = _rows(gen, t, c, 0, "bf16", offset=0.1), _rows(gen, t, c, 0, "bf16")
    state["weight"] = 1.0 + 0.2 * _normal(gen, c)
    state["bias"] = 0.1 * _normal(gen, c) if case["kind"] == "layer" else None
    state["wd"] = _held(gen, c, r, fmt, 0.02, case["tensor_scale"])
    # activations' tensor scales come from earlier batches
    state["scale_x"] = torch.tensor([12.0 / (6 * 448)], device="cuda") if case["tensor_scale"] else None
    state["scale_h"] = torch.tensor([0.05 * c / (6 * 448)], device="cuda") if case["tensor_scale"] else None
    for name, cols in (("xq", c), ("hq", r)):
        state[name] = {"codes": torch.zeros(t, _code_pitch(cols), dtype=torch.uint8, device="cuda"),
                       "scales": torch.zeros(_scale_bytes(t, cols, fmt), dtype=torch.uint8, device="cuda")}
    state["total"], state["y"] = (torch.empty(t, c, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return state


# ---- one pass ------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        return _run_own(state, case, op)
    if op == "norm":
        total = state["x"] if state["residual"] is None else (state["x"].float() + state["residual"].float()).to(state["x"].dtype)
        y, stats = _norm_plain(total.float(), case["kind"] == "layer", state["weight"], state["bias"])
        out = {"y": y.to(DTYPE[case["out"]]), "stats": stats}
        return out if state["residual"] is None else {**out, "total": total}
    if op == "norm_grad":
        return _norm_grad_plain(state, case)
    if op == "gated":
        h, _, _, _ = _gated_plain(state["x"], state, case)
        return h.to(DTYPE[case["out"]])
    if op == "gated_grad":
        _, a, b, wu = _gated_plain(state["x"], state, case)
        f, slope = _activation(a, case["act"])
        dh = state["dh"].float()
        dgate, dup = (dh * b * slope).bfloat16(), (dh * f).bfloat16()
        # (the second call's inputs are what the first has written)
        dx = dgate.float() @ _unpacked(state["wg"], case["fmt"]) + dup.float() @ wu
        return {"dgate": dgate, "dup": dup, "dx": dx.bfloat16()}
    fmt, layer = case["fmt"], case["kind"] == "layer"
    total = (state["x"].float() + state["residual"].float()).bfloat16()
    xn, _ = _norm_plain(total.float(), layer, state["weight"], state["bias"])
    xq = _hold(xn, fmt, state["scale_x"])
    h, _, _, _ = _gated_plain(xq, state, case)
    hq = _hold(h, fmt, state["scale_h"])
    return {"total": total, "y": (_unpacked(hq, fmt) @ _unpacked(state["wd"], fmt).T).bfloat16()}


def _run_own(state, case, op):
    from paper_2405_14852_b200 import binding as B

    kinds = {"layer": B.PVT_NORM_LAYER, "rms": B.PVT_NORM_RMS}
    if op == "norm":
        n = B.make_norm(state["x"], state["weight"], state["bias"], kind=kinds[case["kind"]], eps=EPS, residual=state["residual"])
        B.pvt_norm_apply(n, y=state["y"], total=state["total"], stats=state["stats"])
        out = {"y": state["y"], "stats": state["stats"]}
        return out if state["residual"] is None else {**out, "total": state["total"]}
    if op == "norm_grad":
        n = B.make_norm(state["x"], state["weight"], state["bias"], kind=kinds[case["kind"]], eps=EPS)
        if "workspace" not in state:  # kept as long as the layer is
            state["workspace"] = B.new_norm_workspace(n)
        B.pvt_norm_grad(n, state["stats"], state["dy"], state["dx"], dresidual=state["dres"], dweight=state["dweight"],
                        dbias=state["dbias"], workspace=state["workspace"])
        out = {"dx": state["dx"], "dweight": state["dweight"]}
        return out if state["dbias"] is None else {**out, "dbias": state["dbias"]}
    fmt = B.PVT_MX_E8M0_32 if case["fmt"] == "e8m0_32" else B.PVT_MX_E4M3_16
    act = {"silu": B.PVT_ACT_SILU, "gelu": B.PVT_ACT_GELU, "gelu_tanh": B.PVT_ACT_GELU_TANH}[case["act"]]

    def held(m):
        return B.make_mx(m["codes"], m["scales"], m["rows"], m["cols"], fmt, tensor_scale=m["tensor_scale"])

    wg, wu = held(state["wg"]), held(state["wu"])
    if op == "gated":
        B.pvt_mx_gated(held(state["x"]), wg, wu, h=state["h"], activation=act)
        return state["h"]
    if op == "gated_grad":
        B.pvt_mx_gated_grad(held(state["x"]), wg, wu, state["dh"], state["dgate"], state["dup"], activation=act)
        B.pvt_mx_gated_grad_input(state["dgate"], state["dup"], wg, wu, state["dx"])
        return {"dgate": state["dgate"], "dup": state["dup"], "dx": state["dx"]}
    t, c, r = case["tokens"], case["cols"], case["rows"]
    xq = B.make_mx(state["xq"]["codes"], state["xq"]["scales"], t, c, fmt, tensor_scale=state["scale_x"])
    hq = B.make_mx(state["hq"]["codes"], state["hq"]["scales"], t, r, fmt, tensor_scale=state["scale_h"])
    n = B.make_norm(state["x"], state["weight"], state["bias"], kind=kinds[case["kind"]], eps=EPS, residual=state["residual"])
    B.pvt_norm_apply(n, quantized=xq, total=state["total"])
    B.pvt_mx_gated(xq, wg, wu, quantized=hq, activation=act)
    B.pvt_mx_product(hq, held(state["wd"]), state["y"])
    return {"total": state["total"], "y": state["y"]}


# ---- plain forms ---------------------------------------------------------------------------------------------
def _statistics(r, layer):
    """Mean (0 where there is none) and 1 / sqrt(var + eps) of each row."""
    mean = r.mean(dim=1) if layer else torch.zeros_like(r[:, 0])
    d = r - mean[:, None]
    return mean, 1.0 / torch.sqrt((d * d).mean(dim=1) + EPS)


def _norm_plain(r, layer, weight, bias):
    mean, rstd = _statistics(r, layer)
    y = (r - mean[:, None]) * rstd[:, None] * weight.float()
    return y if bias is None else y + bias.float(), torch.stack((mean, rstd), dim=1)


def _norm_grad_plain(state, case):
    layer = case["kind"] == "layer"
    mean, rstd = state["stats"][:, :1], state["stats"][:, 1:]
    xh, dy = (state["x"].float() - mean) * rstd, state["dy"].float()
    g = dy * state["weight"].float()
    dx = g - xh * (g * xh).mean(dim=1, keepdim=True)
    if layer:
        dx = dx - g.mean(dim=1, keepdim=True)
    dx = dx * rstd
    if state["dres"] is not None:
        dx = dx + state["dres"].float()
    out = {"dx": dx.to(DTYPE[case["out"]]), "dweight": (dy * xh).sum(dim=0)}
    return {**out, "dbias": dy.sum(dim=0)} if layer else out


def _activation(a, act):
    """f(a) and its derivative."""
    if act == "gelu":
        phi = 0.5 * torch.erfc(a * -math.sqrt(0.5))
        return a * phi, phi + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return a * s, s * (1.0 + a * (1.0 - s))
    # gelu_tanh: (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), u = k (a + c a^3)
    k, c = math.sqrt(2.0 / math.pi), 0.044715
    s = 1.0 / (1.0 + torch.exp(-2.0 * k * (a + c * a * a * a)))
    return a * s, s + 2.0 * k * a * s * (1.0 - s) * (1.0 + 3.0 * c * a * a)


def _gated_plain(x, state, case):
    """h, both products and the second one's weights."""
    fmt = case["fmt"]
    xv, wu = _unpacked(x, fmt), _unpacked(state["wu"], fmt)
    a, b = xv @ _unpacked(state["wg"], fmt).T, xv @ wu.T
    return _activation(a, case["act"])[0] * b, a, b, wu


def _hold(x, fmt, ts):
    """A matrix held in 4 bits: codes and scales as they lie in memory."""
    codes, scales = _pack(*_quantise(x, fmt, ts), fmt)
    return {"codes": codes, "scales": scales, "tensor_scale": ts, "rows": x.shape[0], "cols": x.shape[1]}


def _code_pitch(cols):
    return (cols + 31) // 32 * 16


def _scale_tiles(cols, fmt):
    return (cols + 255) // 256 * (256 // BLOCK[fmt] // 4)


def _scale_bytes(rows, cols, fmt):
    return (rows + 127) // 128 * _scale_tiles(cols, fmt) * 512


def _element(y):
    """Code of the element nearest to y, ties to the even code, the largest where y is beyond it."""
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(y.dtype)
    a = (torch.round(a / step) * step).clamp_(max=6.0)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, 0.5 * a + 4))
    return code.to(torch.uint8) | ((y < 0).to(torch.uint8) << 3)


def _quantise(x, fmt, tensor_scale):
    """Codes [rows, cols] and scale bytes [rows, blocks]."""
    rows, cols = x.shape
    b = BLOCK[fmt]
    nb = (cols + b - 1) // b
    x = torch.nn.functional.pad(x.float(), (0, nb * b - cols)).view(rows, nb, b)
    amax = x.abs().amax(dim=2)
    if fmt == "e8m0_32":
        e = (torch.frexp(amax)[1] - 3).clamp(min=-127)  # the largest element's exponent is 2
        e = torch.where(amax > 0, e, torch.full_like(e, -127))
        # (a power of two is exact, and so is its product; two steps keep 2^127 out of the way of small blocks)
        half = e // 2
        y = torch.ldexp(torch.ldexp(x, -half[..., None]), (half - e)[..., None])
        scales = (e + 127).to(torch.uint8)
    else:
        ts = 1.0 if tensor_scale is None else tensor_scale.double()
        s = amax.double() / (6.0 * ts)
        e = (torch.frexp(s)[1] - 1).clamp(min=-6).double()
        n = torch.round(s * torch.exp2(3 - e))  # in units of the last place, ties to even
        s = (n * torch.exp2(e - 3)).clamp(max=448.0)
        y = torch.where(s[..., None] > 0, x.double() / (s * ts)[..., None], 0.0)
        e = torch.where(s >= 2.0 ** -6, torch.frexp(s)[1] - 1, torch.full_like(s, -7).int())
        scales = torch.where(e < -6, s * 512, (e + 7) * 8 + (s * torch.exp2(3.0 - e) - 8)).to(torch.uint8)
    return _element(y).view(rows, nb * b)[:, :cols], scales


def _values(codes, scales, fmt, tensor_scale):
    """What codes and scale bytes stand for, in 32 bits."""
    rows, cols = codes.shape
    mag = (codes & 7).float()
    mag = torch.where(mag < 4, 0.5 * mag, torch.where(mag < 6, mag - 2, 2 * mag - 8))
    v = torch.where(codes > 7, -mag, mag)
    s = scales.float()
    if fmt == "e8m0_32":
        s = torch.exp2(s - 127)
    else:
        e, m = torch.floor(s / 8), s % 8
        s = torch.where(e > 0, torch.exp2(e - 10) * (8 + m), m * 2.0 ** -9)
    v = v * s.repeat_interleave(BLOCK[fmt], dim=1)[:, :cols]
    return v if tensor_scale is None else (v.double() * tensor_scale.double()).float()


def _pack(codes, scales, fmt):
    """As they lie in memory."""
    rows, cols = codes.shape
    pitch = _code_pitch(cols)
    codes = torch.nn.functional.pad(codes, (0, 2 * pitch - cols))
    codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    strips, tiles = (rows + 127) // 128, _scale_tiles(cols, fmt)
    s = torch.nn.functional.pad(scales, (0, 4 * tiles - scales.shape[1], 0, 128 * strips - rows))
    s = s.view(strips, 4, 32, tiles, 4).permute(0, 3, 2, 1, 4)  # strip, tile, row in 32, 32 rows, block
    return codes.contiguous(), s.reshape(-1).contiguous()


def _unpacked(m, fmt):
    rows, cols = m["rows"], m["cols"]
    codes = torch.stack((m["codes"] & 15, m["codes"] >> 4), dim=2).view(rows, -1)[:, :cols]
    strips, tiles = (rows + 127) // 128, _scale_tiles(cols, fmt)
    s = m["scales"].view(strips, tiles, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(128 * strips, 4 * tiles)
    nb = (cols + BLOCK[fmt] - 1) // BLOCK[fmt]
    return _values(codes, s[:rows, :nb], fmt, m["tensor_scale"])


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_scales(x, fmt, ts):
    """Scale of every block of x [rows, blocks, elements] from its definition."""
    largest = x.abs().amax(dim=2)
    if fmt == "e8m0_32":
        exponent = torch.floor(torch.log2(largest))
        exponent = torch.where(torch.exp2(exponent) > largest, exponent - 1, exponent)
        exponent = torch.where(torch.exp2(exponent + 1) <= largest, exponent + 1, exponent)
        return torch.exp2(torch.clamp(exponent - 2, min=-127))
    floats = torch.tensor([m * 2.0 ** -9 for m in range(8)] +
                          [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1], dtype=torch.float64,
                          device=x.device)
    want = largest / (6.0 * ts)
    above = torch.searchsorted(floats, want.contiguous()).clamp(1, len(floats) - 1)
    lo, hi = floats[above - 1], floats[above]
    to_lo, to_hi = want - lo, hi - want
    up = (to_hi < to_lo) | ((to_hi == to_lo) & (above % 2 == 0))
    return torch.where(up, hi, lo)


def _exact_held(m, fmt):
    """Values of a held matrix by looking every code and scale up in a table."""
    dev, rows, cols, b = m["codes"].device, m["rows"], m["cols"], BLOCK[fmt]
    element = torch.tensor(_GRID + tuple(-g for g in _GRID), dtype=torch.float64, device=dev)
    col = torch.arange(cols, device=dev)
    codes = (m["codes"][:, col // 2] >> (4 * (col % 2)).to(torch.uint8)[None, :]) & 15
    row = torch.arange(rows, device=dev)[:, None]
    block = torch.arange(-(-cols // b), device=dev)[None, :]
    tile = (row // 128) * ((cols + 255) // 256 * (64 // b)) + block // 4
    byte = m["scales"][512 * tile + 16 * (row % 32) + 4 * (row % 128 // 32) + block % 4].long()
    if fmt == "e8m0_32":
        table = [2.0 ** (n - 127) for n in range(255)] + [math.nan]
    else:
        table = [(n % 8) * 2.0 ** -9 if n < 8 else (8 + n % 8) * 2.0 ** (n // 8 - 10) for n in range(127)] + [math.nan]
    scale = torch.tensor(table, dtype=torch.float64, device=dev)[byte]
    if m["tensor_scale"] is not None:
        scale = scale * m["tensor_scale"].double()
    return element[codes.long()] * scale[:, (col // b)]


def _exact_quantised(x, fmt, ts):
    """What x (float64) stands for once it is held in 4 bits, by the borders between elements."""
    rows, cols = x.shape
    b = BLOCK[fmt]
    ts = 1.0 if ts is None else ts.double()
    whole, out = -(-cols // b) * b, torch.empty_like(x)
    for at in range(0, rows, 2048):
        part = torch.zeros(min(2048, rows - at), whole, dtype=torch.float64, device=x.device)
        part[:, :cols] = x[at:at + 2048]
        blocks = part.view(part.shape[0], -1, b)
        scale = (_exact_scales(blocks, fmt, ts) * ts)[..., None]
        size, best = blocks.abs(), torch.zeros_like(blocks)
        for n in range(1, 8):  # the next element from its border on, and at the border if its code is even
            border = 0.5 * (_GRID[n - 1] + _GRID[n]) * scale
            best = torch.where((size > border) | ((size == border) & (n % 2 == 0)), _GRID[n], best)
        out[at:at + 2048] = (torch.sign(blocks) * best * scale).nan_to_num(0.0).view(part.shape[0], whole)[:, :cols]
    return out


def _exact_norm(r, layer, weight, bias):
    mean = r.mean(dim=1, keepdim=True) if layer else torch.zeros_like(r[:, :1])
    var = (r * r).mean(dim=1, keepdim=True) - mean * mean
    y = (r - mean) / torch.sqrt(var + EPS) * weight.double()
    return (y if bias is None else y + bias.double()), torch.cat((mean, (var + EPS) ** -0.5), dim=1)


def _exact_gate(a, act):
    """f(a) / a and f'(a)"""
    if act == "silu":
        s = torch.sigmoid(a)
        return s, s + a * s * torch.sigmoid(-a)
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(a / 2 ** 0.5))
        return phi, phi + a * torch.exp(-a ** 2 / 2) / (2 * math.pi) ** 0.5
    t = torch.tanh((2 / math.pi) ** 0.5 * (a + 0.044715 * a ** 3))
    return (1 + t) / 2, (1 + t) / 2 + a / 2 * (1 - t ** 2) * (2 / math.pi) ** 0.5 * (1 + 3 * 0.044715 * a ** 2)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        r = state["x"].double()
        if state["residual"] is not None:  # the sum as it is kept: rounded once
            total = r + state["residual"].double()
            kept = total.to(state["x"].dtype)
            y, stats = _exact_norm(kept.double(), case["kind"] == "layer", state["weight"], state["bias"])
            return {"y": y, "stats": stats, "total": total}
        y, stats = _exact_norm(r, case["kind"] == "layer", state["weight"], state["bias"])
        return {"y": y, "stats": stats}
    if op == "norm_grad":
        layer, dy = case["kind"] == "layer", state["dy"].double()
        mean, rstd = state["stats"].double().split(1, dim=1)
        xh = (state["x"].double() - mean) * rstd
        g = dy * state["weight"].double()
        n = case["cols"]
        # the row's derivative: rstd (I - 1 1^T / n - xh xh^T / n) g
        dx = rstd * (g - ((g * xh).sum(dim=1, keepdim=True) / n) * xh - ((g.sum(dim=1, keepdim=True) / n) if layer else 0.0))
        if state["dres"] is not None:
            dx = dx + state["dres"].double()
        out = {"dx": dx, "dweight": (dy * xh).sum(dim=0)}
        return {**out, "dbias": dy.sum(dim=0)} if layer else out
    fmt = case["fmt"]
    wg, wu = _exact_held(state["wg"], fmt), _exact_held(state["wu"], fmt)
    if op == "block":
        total = state["x"].double() + state["residual"].double()
        xn, _ = _exact_norm(total.bfloat16().double(), case["kind"] == "layer", state["weight"], state["bias"])
        x = _exact_quantised(xn, fmt, state["scale_x"])
    else:
        x = _exact_held(state["x"], fmt)
    a, b = x @ wg.T, x @ wu.T
    gate, slope = _exact_gate(a, case["act"])
    if op == "gated":
        return a * gate * b
    if op == "gated_grad":
        dh = state["dh"].double()
        dgate, dup = dh * b * slope, dh * a * gate
        return {"dgate": dgate, "dup": dup, "dx": dgate @ wg + dup @ wu}
    h = _exact_quantised(a * gate * b, fmt, state["scale_h"])
    return {"total": total, "y": h @ _exact_held(state["wd"], fmt).T}
