"""Timed operators of the pass that the V step's gradient comes from: a student whose linear layers are held in
microscaled 4-bit floating point, and the loss that distils it from a teacher's top logits.

  quant    float matrix -> 4-bit codes and block scales -> the values these stand for
  product  y = x_hat w_hat^T of two such matrices
  grad     its two gradients: dx = dy w_hat (bf16), dw = dy^T x_hat (f32, what the V step takes as g)
  top      a teacher's k largest logits of each row, in order, and the logarithm of the sum of all exponentials
  distill  Kullback-Leibler loss of the student against them and its gradient, in one call or forward and backward

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
LARGEST_FLOPS = 2 * 4096 * 8192 * 28672
LARGEST_AREA = 28672 * 8192
LARGEST_LOGITS = 4096 * 32000


# ---- cases ---------------------------------------------------------------------------------------------------
def _quant(name, rows, cols, dtype, fmt, pad=0, tensor_scale=False):
    return {"name": name, "op": "quant", "rows": rows, "cols": cols, "dtype": dtype, "fmt": fmt, "pad": pad,
            "tensor_scale": tensor_scale}


def _product(name, tokens, cols, rows, fmt, out, tensor_scale=False):
    return {"name": name, "op": "product", "tokens": tokens, "cols": cols, "rows": rows, "fmt": fmt, "out": out,
            "tensor_scale": tensor_scale}


def _grad(name, tokens, cols, rows, fmt, tensor_scale=False):
    return {"name": name, "op": "grad", "tokens": tokens, "cols": cols, "rows": rows, "fmt": fmt,
            "tensor_scale": tensor_scale}


def _top(name, rows, vocab, k, dtype, temperature):
    return {"name": name, "op": "top", "rows": rows, "vocab": vocab, "k": k, "dtype": dtype, "temperature": temperature}


def _distill(name, rows, vocab, k, dtype, temperature, tail, one_call, pad=0):
    return {"name": name, "op": "distill", "rows": rows, "vocab": vocab, "k": k, "dtype": dtype,
            "temperature": temperature, "tail": tail, "one_call": one_call, "pad": pad}


def listed():
    return [
        # the activations of one generated token on their way into a 4-bit product: latency alone
        _quant("quant_token_bf16_e4m3", 1, 4096, "bf16", "e4m3_16", tensor_scale=True),
        # the weights of the largest projection, re-quantised after a training step
        _quant("quant_weights_f32_e8m0", 28672, 8192, "f32", "e8m0_32"),
        # activations cut out of a wider array, nothing a multiple of a block or of a tile
        _quant("quant_ragged_f16_e4m3", 2047, 5001, "f16", "e4m3_16", pad=7, tensor_scale=True),
        # generation: one token through a feed-forward projection
        _product("product_token_e8m0", 1, 4096, 11008, "e8m0_32", "bf16"),
        # a long prompt or a training batch through the largest projection
        _product("product_prompt_e8m0", 4096, 8192, 28672, "e8m0_32", "bf16"),
        # a short prompt, odd everywhere, scales in both formats' finer one
        _product("product_ragged_e4m3", 333, 5119, 13823, "e4m3_16", "f32", tensor_scale=True),
        # backward of a training batch through a feed-forward projection
        _grad("grad_batch_e8m0", 2048, 4096, 11008, "e8m0_32"),
        # backward of a few calibration tokens, odd everywhere
        _grad("grad_ragged_e4m3", 77, 5119, 4095, "e4m3_16", tensor_scale=True),
        # a teacher's logits over a calibration batch, kept as the 64 largest
        _top("top_batch_bf16", 4096, 32000, 64, "bf16", 1.0),
        # the logits of a few positions over a large vocabulary
        _top("top_few_f32", 3, 131071, 257, "f32", 2.0),
        # the loss of a training step and its gradient
        _distill("distill_batch_bf16", 4096, 32000, 64, "bf16", 1.0, False, True),
        # a few positions over a large vocabulary, with the rest of the teacher's mass, forward and then backward
        _distill("distill_few_f32_tail", 5, 131071, 200, "f32", 2.0, True, False, pad=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quant", "product", "product", "grad", "grad", "top", "distill", "distill"])
    fmt = rng.choice(sorted(BLOCK))
    scaled = fmt == "e4m3_16" and rng.random() < 0.6
    if op == "quant":
        cols = _log(rng, 17, 28672)
        return _drawn(_quant("", _log(rng, 1, max(1, LARGEST_AREA // cols)), cols, rng.choice(sorted(DTYPE)), fmt,
                             rng.choice([0, 0, 1, 8, 13]), scaled))
    if op == "product":
        cols, rows = _log(rng, 33, 28672), _log(rng, 16, 28672)
        tokens = rng.choice([rng.randint(1, 16), _log(rng, 1, 8192)])
        tokens = max(1, min(tokens, LARGEST_FLOPS // (2 * cols * rows)))
        return _drawn(_product("", tokens, cols, rows, fmt, rng.choice(["bf16", "f16", "f32"]), scaled))
    if op == "grad":
        cols, rows = _log(rng, 33, 28672), _log(rng, 16, 28672)
        tokens = _log(rng, 1, 4096)
        tokens = max(1, min(tokens, LARGEST_FLOPS // (4 * cols * rows)))
        return _drawn(_grad("", tokens, cols, rows, fmt, scaled))
    vocab, dtype = _log(rng, 500, 262144), rng.choice(sorted(DTYPE))
    rows = _log(rng, 1, max(1, LARGEST_LOGITS // vocab))
    k = _log(rng, 1, min(1024, vocab // 8))
    if op == "top":
        return _drawn(_top("", rows, vocab, k, dtype, rng.choice([1.0, 2.0, 0.7])))
    return _drawn(_distill("", rows, vocab, k, dtype, rng.choice([1.0, 2.0, 0.7]), rng.random() < 0.5, rng.random() < 0.5,
                           rng.choice([0, 0, 1, 8])))


def _drawn(case):
    del case["name"]
    return case


def work(case):
    op = case["op"]
    size = {"f32": 4, "f16": 2, "bf16": 2}
    if op == "quant":
        n = case["rows"] * case["cols"]
        held = n // 2 + n // BLOCK[case["fmt"]]
        return {"bytes": n * (size[case["dtype"]] + 4) + 2 * held, "flops": 4 * n}
    if op in ("product", "grad"):
        t, c, r = case["tokens"], case["cols"], case["rows"]
        held = lambda n: n // 2 + n // BLOCK[case["fmt"]]  # noqa: E731
        if op == "product":
            return {"bytes": held(t * c) + held(r * c) + t * r * size[case["out"]], "flops": 2 * t * c * r}
        return {"bytes": held(t * c) + held(r * c) + t * r * 2 + t * c * 2 + r * c * 4, "flops": 4 * t * c * r}
    n, k = case["rows"] * case["vocab"], case["rows"] * case["k"]
    if op == "top":
        return {"bytes": n * size[case["dtype"]] + 8 * k + 4 * case["rows"], "flops": 3 * n}
    reads = 1 if case["one_call"] else 2
    return {"bytes": n * size[case["dtype"]] * (reads + 1) + reads * 8 * k + 12 * case["rows"], "flops": 5 * n}


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
    ts = _tensor_scale(x) if scaled else None
    codes, scales = _pack(*_quantise(x, fmt, ts), fmt)
    return {"codes": codes, "scales": scales, "tensor_scale": ts, "rows": rows, "cols": cols}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 17)
    op = case["op"]
    if op == "quant":
        rows, cols, fmt = case["rows"], case["cols"], case["fmt"]
        x = _heavy(gen, rows, cols + case["pad"], 0.02).to(DTYPE[case["dtype"]])[:, :cols]
        return {"case": case, "x": x, "tensor_scale": _tensor_scale(x) if case["tensor_scale"] else None,
                "codes": torch.zeros(rows, _code_pitch(cols), dtype=torch.uint8, device="cuda"),
                "scales": torch.zeros(_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda"),
                "values": torch.empty(rows, cols, device="cuda")}
    if op in ("product", "grad"):
        t, c, r, fmt = case["tokens"], case["cols"], case["rows"], case["fmt"]
        state = {"case": case, "x": _held(gen, t, c, fmt, 1.0, case["tensor_scale"]),
                 "w": _held(gen, r, c, fmt, 0.02, case["tensor_scale"])}
        if op == "product":
            state["y"] = torch.empty(t, r, dtype=DTYPE[case["out"]], device="cuda")
        else:
            pitch = (r + 7) // 8 * 8
            state["dy"] = (1e-3 * _normal(gen, t, pitch)).bfloat16()[:, :r]
            state["dx"] = torch.empty(t, c, dtype=torch.bfloat16, device="cuda")
            state["dw"] = torch.empty(r, c, device="cuda")
        return state
    rows, vocab, k, dtype = case["rows"], case["vocab"], case["k"], DTYPE[case["dtype"]]
    teacher = _normal(gen, rows, vocab).mul_(2.5)
    if op == "top":
        return {"case": case, "logits": teacher.to(dtype), "idx": torch.empty(rows, k, dtype=torch.int32, device="cuda"),
                "val": torch.empty(rows, k, device="cuda"), "lse": torch.empty(rows, device="cuda")}
    val, idx = torch.topk(teacher, k, dim=1)
    lse = torch.logsumexp(teacher.double() / case["temperature"], dim=1).float()
    weight = (torch.rand(rows, device="cuda", generator=gen) > 0.1).float() / rows  # padding has no weight
    student = torch.empty(rows, vocab + case["pad"], dtype=dtype, device="cuda")[:, :vocab]
    student.copy_(teacher.mul_(0.9).add_(_normal(gen, rows, vocab)))
    return {"case": case, "logits": student, "idx": idx.int(), "val": val.contiguous(),
            "lse": lse if case["tail"] else None, "weight": weight, "loss": torch.empty(rows, device="cuda"),
            "stats": torch.empty(rows, 8, device="cuda"), "grad": torch.empty(rows, vocab, dtype=dtype, device="cuda")}


# ---- one pass ------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        return _run_own(state, case, op)
    if op == "quant":
        codes, scales = _quantise(state["x"], case["fmt"], state["tensor_scale"])
        return _values(codes, scales, case["fmt"], state["tensor_scale"])
    if op == "product":
        return (_unpacked(state["x"], case["fmt"]) @ _unpacked(state["w"], case["fmt"]).T).to(DTYPE[case["out"]])
    if op == "grad":
        dy = state["dy"].float()
        return {"dx": (dy @ _unpacked(state["w"], case["fmt"])).bfloat16(), "dw": dy.T @ _unpacked(state["x"], case["fmt"])}
    if op == "top":
        return _top_plain(state["logits"], case["k"], case["temperature"])
    return _distill_plain(state, case)


def _run_own(state, case, op):
    from paper_2405_14852_b200 import binding as B

    def held(m):
        return B.make_mx(m["codes"], m["scales"], m["rows"], m["cols"], fmt, tensor_scale=m["tensor_scale"])

    if op in ("quant", "product", "grad"):
        fmt = B.PVT_MX_E8M0_32 if case["fmt"] == "e8m0_32" else B.PVT_MX_E4M3_16
    if op == "quant":
        m = B.make_mx(state["codes"], state["scales"], case["rows"], case["cols"], fmt, tensor_scale=state["tensor_scale"])
        B.pvt_mx_quantize(m, state["x"])
        B.pvt_mx_dequant(m, state["values"])
        return state["values"]
    if op == "product":
        B.pvt_mx_product(held(state["x"]), held(state["w"]), state["y"])
        return state["y"]
    if op == "grad":
        B.pvt_mx_grad_input(state["dy"], held(state["w"]), state["dx"])
        B.pvt_mx_grad_weight(state["dy"], held(state["x"]), state["dw"])
        return {"dx": state["dx"], "dw": state["dw"]}
    if op == "top":
        B.pvt_distill_top(state["logits"], state["idx"], state["val"], state["lse"], temperature=case["temperature"])
        return {"idx": state["idx"], "val": state["val"], "lse": state["lse"]}
    d = B.make_distill(state["logits"], state["idx"], state["val"], teacher_lse=state["lse"], weight=state["weight"],
                       temperature=case["temperature"])
    if case["one_call"]:
        B.pvt_distill_loss(d, state["loss"], grad=state["grad"])
    else:
        B.pvt_distill_loss(d, state["loss"], stats=state["stats"])
        B.pvt_distill_grad(d, state["stats"], state["grad"])
    return {"loss": state["loss"], "grad": state["grad"]}


# ---- plain forms ---------------------------------------------------------------------------------------------
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


def _top_plain(logits, k, temperature):
    z = logits.float()
    val, idx = torch.sort(z, dim=1, descending=True, stable=True)
    top = z.amax(dim=1, keepdim=True)
    lse = top[:, 0] / temperature + torch.log(torch.exp((z - top) / temperature).sum(dim=1))
    return {"idx": idx[:, :k].int(), "val": val[:, :k].contiguous(), "lse": lse}


def _distill_plain(state, case):
    idx, t = state["idx"].long(), case["temperature"]
    x = state["logits"].float() / t
    val = state["val"].double() / t  # what the listed logits leave of the teacher's mass is a small difference
    if case["tail"]:
        p = torch.exp(val - state["lse"].double()[:, None])
        rest = (1.0 - p.sum(dim=1)).clamp(min=0.0).float()
    else:
        p = torch.exp(val - val.amax(dim=1, keepdim=True))
        p = p / p.sum(dim=1, keepdim=True)
        rest = torch.zeros_like(state["weight"])
    p = p.float()
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    listed_e = torch.gather(e, 1, idx)
    rest_e = e.scatter(1, idx, 0.0)
    rest_sum = rest_e.sum(dim=1)
    z = rest_sum + listed_e.sum(dim=1)
    logq = torch.gather(x, 1, idx) - top - torch.log(z)[:, None]
    loss = torch.where(p > 0, p * (torch.log(p) - logq), 0.0).sum(dim=1)
    loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(rest_sum / z)), 0.0)
    whole = (p.sum(dim=1) + rest)[:, None]
    grad = rest_e * (whole / z[:, None] - (rest / rest_sum)[:, None])
    grad = grad.scatter(1, idx, whole * listed_e / z[:, None] - p)
    w = state["weight"]
    grad = torch.where(w[:, None] == 0, 0.0, grad * (w[:, None] / t))
    return {"loss": torch.where(w == 0, 0.0, loss * w), "grad": grad.to(DTYPE[case["dtype"]])}


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


def _exact_values(state, case):
    x = state["x"].double()
    rows, cols = x.shape
    b = BLOCK[case["fmt"]]
    ts = 1.0 if state["tensor_scale"] is None else state["tensor_scale"].double()
    out = torch.empty_like(x)
    whole = -(-cols // b) * b
    for at in range(0, rows, 2048):
        part = torch.zeros(min(2048, rows - at), whole, dtype=torch.float64, device=x.device)
        part[:, :cols] = x[at:at + 2048]
        blocks = part.view(part.shape[0], -1, b)
        scale = (_exact_scales(blocks, case["fmt"], ts) * ts)[..., None]
        size, best = blocks.abs(), torch.zeros_like(blocks)
        for n in range(1, 8):  # the next element from its border on, and at the border if its code is even
            border = 0.5 * (_GRID[n - 1] + _GRID[n]) * scale
            best = torch.where((size > border) | ((size == border) & (n % 2 == 0)), _GRID[n], best)
        out[at:at + 2048] = (torch.sign(blocks) * best * scale).nan_to_num(0.0).view(part.shape[0], whole)[:, :cols]
    return out


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


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        return _exact_values(state, case)
    if op == "product":
        return _exact_held(state["x"], case["fmt"]) @ _exact_held(state["w"], case["fmt"]).T
    if op == "grad":
        dy = state["dy"].double()
        return {"dx": dy @ _exact_held(state["w"], case["fmt"]), "dw": dy.T @ _exact_held(state["x"], case["fmt"])}
    t = case["temperature"]
    z = state["logits"].double()
    if op == "top":
        order = torch.argsort(-z, dim=1, stable=True)[:, :case["k"]]
        return {"idx": order.int(), "val": torch.gather(z, 1, order), "lse": torch.logsumexp(z / t, dim=1)}
    logq = torch.log_softmax(z / t, dim=1)
    idx, val, w = state["idx"].long(), state["val"].double() / t, state["weight"].double()
    norm = state["lse"].double() if case["tail"] else torch.logsumexp(val, dim=1)
    logp = val - norm[:, None]
    p = logp.exp()
    loss = (p * (logp - torch.gather(logq, 1, idx))).sum(dim=1)
    target = torch.zeros_like(z).scatter_(1, idx, p)
    if case["tail"]:
        # the unlisted part is one more outcome: its gradient falls on the unlisted logits by their shares of it
        left = (1.0 - p.sum(dim=1)).clamp(min=0.0)
        others = logq.scatter(1, idx, -math.inf)
        log_left = torch.logsumexp(others, dim=1)
        loss = loss + torch.where(left > 0, left * (left.log() - log_left), 0.0)
        target = target + left[:, None] * (others - log_left[:, None]).exp()
    total = target.sum(dim=1, keepdim=True)
    grad = (total * logq.exp() - target) * (w[:, None] / t)
    return {"loss": loss * w, "grad": grad}
