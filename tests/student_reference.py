"""Plain 64-bit implementations of the 4-bit block floating point calls and of the distillation calls, from include/pvt.h
alone: tables and comparisons in float64, one element at a time in the mathematics, whole tensors in the code."""
import math

import torch

E8M0, E4M3 = 0, 1
BLOCK = {E8M0: 32, E4M3: 16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
E4M3_VALUES = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]


def scale_values(fmt, device="cpu"):
    """value of every scale byte (bytes that no scale has: NaN)"""
    if fmt == E8M0:
        t = [2.0 ** (n - 127) for n in range(255)] + [math.nan]
    else:
        t = E4M3_VALUES + [math.nan] * 129
    return torch.tensor(t, dtype=torch.float64, device=device)


def element_values(device="cpu"):
    return torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float64, device=device)


def quantize(x, fmt, tensor_scale=None):
    """codes [rows, cols] and scale bytes [rows, blocks], both int64, of a float tensor"""
    ts = 1.0 if tensor_scale is None else float(tensor_scale)
    x = x.double()
    rows, cols = x.shape
    b = BLOCK[fmt]
    nb = -(-cols // b)
    pad = torch.zeros(rows, nb * b, dtype=torch.float64, device=x.device)
    pad[:, :cols] = x
    blocks = pad.view(rows, nb, b)
    bad = ~torch.isfinite(blocks).all(dim=2)
    if not (ts > 0 and math.isfinite(ts)):
        bad = torch.ones_like(bad)
        ts = 1.0
    clean = torch.where(bad[..., None], torch.zeros_like(blocks), blocks)
    amax = clean.abs().amax(dim=2)
    table = scale_values(fmt, x.device)
    if fmt == E8M0:
        e = torch.floor(torch.log2(amax.clamp(min=1e-300)))
        e = torch.where(torch.exp2(e) > amax, e - 1, e)
        e = torch.where(torch.exp2(e + 1) <= amax, e + 1, e)
        byte = (e - 2).clamp(min=-127).long() + 127
        byte = torch.where(amax == 0, torch.zeros_like(byte), byte)
    else:
        finite = table[:127]
        want = amax / (6.0 * ts)  # (compared below without this rounding)
        byte = torch.searchsorted(finite, want.contiguous()).clamp(1, 126)
        lo, hi = finite[byte - 1], finite[byte]
        mid = 0.5 * (lo + hi) * (6.0 * ts)
        up = (amax > mid) | ((amax == mid) & (byte % 2 == 0))
        byte = torch.where(up, byte, byte - 1)
        # the quotient's own rounding may have put it one interval off
        for _ in range(2):
            above = 0.5 * (finite[byte] + finite[(byte + 1).clamp(max=126)]) * (6.0 * ts)
            byte = torch.where((byte < 126) & ((amax > above) | ((amax == above) & (byte % 2 == 1))), byte + 1, byte)
            below = 0.5 * (finite[byte] + finite[(byte - 1).clamp(min=0)]) * (6.0 * ts)
            byte = torch.where((byte > 0) & ((amax < below) | ((amax == below) & (byte % 2 == 1))), byte - 1, byte)
    d = (table[byte] * ts)[..., None]
    n = torch.zeros_like(blocks, dtype=torch.int64)
    for i in range(1, 8):
        border = 0.5 * (GRID[i - 1] + GRID[i]) * d
        n = torch.where((clean.abs() > border) | ((clean.abs() == border) & (i % 2 == 0)), torch.full_like(n, i), n)
    n = torch.where(d > 0, n, torch.zeros_like(n))
    sign = torch.signbit(blocks).long() * 8
    codes = torch.where(bad[..., None] | (d == 0), torch.zeros_like(n), n | sign)
    byte = torch.where(bad, torch.full_like(byte, 255 if fmt == E8M0 else 127), byte)
    return codes.view(rows, nb * b)[:, :cols], byte


def values(codes, scales, fmt, tensor_scale=None):
    """float64 values of codes [rows, cols] and scale bytes [rows, blocks]"""
    cols = codes.shape[1]
    block = torch.arange(cols, device=codes.device) // BLOCK[fmt]
    v = element_values(codes.device)[codes.long()] * scale_values(fmt, codes.device)[scales.long()][:, block]
    return v if tensor_scale is None else v * float(tensor_scale)


def scale_index(rows, cols, fmt, device="cpu"):
    """place of the scale byte of every (row, block)"""
    b = BLOCK[fmt]
    r = torch.arange(rows, device=device)[:, None]
    n = torch.arange(-(-cols // b), device=device)[None, :]
    tile = (r // 128) * (-(-cols // 256) * (256 // b // 4)) + n // 4
    return 512 * tile + 16 * (r % 32) + 4 * (r % 128 // 32) + n % 4


def scale_bytes(rows, cols, fmt):
    return -(-rows // 128) * -(-cols // 256) * (256 // BLOCK[fmt] // 4) * 512


def pack(codes, scales, fmt, fill=0):
    """bytes as include/pvt.h lays them out: codes [rows, pitch], scales [scale_bytes]; `fill` where no code lies"""
    rows, cols = codes.shape
    pitch = -(-cols // 32) * 16
    even = torch.nn.functional.pad(codes, (0, cols % 2))
    two = (even[:, 0::2] | (even[:, 1::2] << 4)).to(torch.uint8)
    held = torch.full((rows, pitch), fill, dtype=torch.uint8, device=codes.device)
    held[:, :two.shape[1]] = two
    at = scale_index(rows, cols, fmt, codes.device)
    s = torch.zeros(scale_bytes(rows, cols, fmt), dtype=torch.uint8, device=codes.device)
    s[at.reshape(-1)] = scales.to(torch.uint8).reshape(-1)
    return held, s


def unpack(held, s, rows, cols, fmt):
    """codes [rows, cols] and scale bytes [rows, blocks] from bytes"""
    two = held[:, :(cols + 1) // 2].long()
    codes = torch.stack((two & 15, two >> 4), dim=2).view(rows, -1)[:, :cols]
    return codes, s[scale_index(rows, cols, fmt, s.device)].long()


def top(logits, k, temperature=1.0):
    """indices, values and logsumexp per row, with the order and the exclusions of pvt_distill_top"""
    z = logits.double()
    order = torch.where(torch.isnan(z), torch.full_like(z, math.inf), z)
    rank = torch.argsort(-order, dim=1, stable=True)
    # NaN ahead of infinity, by a second stable sort
    is_nan = torch.isnan(torch.gather(z, 1, rank)).long()
    rank = torch.gather(rank, 1, torch.argsort(-is_nan, dim=1, stable=True))[:, :k]
    val = torch.gather(z, 1, rank)
    gone = val == -math.inf
    idx = torch.where(gone, torch.full_like(rank, -1), rank)
    return idx, val, torch.logsumexp(z / temperature, dim=1)


def distill(logits, idx, val, teacher_lse=None, weight=None, upstream=None, temperature=1.0):
    """loss [rows] and gradient [rows, vocab] in float64"""
    rows, vocab = logits.shape
    loss = torch.zeros(rows, dtype=torch.float64)
    grad = torch.zeros(rows, vocab, dtype=torch.float64)
    x_all = logits.double().cpu() / temperature
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        u = 1.0 if upstream is None else float(upstream[r])
        seen, p_log = [], []
        for i, v in zip(idx[r].tolist(), val[r].double().tolist()):
            if 0 <= i < vocab and i not in seen:
                seen.append(i)
                p_log.append(v / temperature)
        x = x_all[r]
        if w == 0 or not seen or max(p_log) == -math.inf or (x == -math.inf).all():
            continue
        at = torch.tensor(seen)
        lp = torch.tensor(p_log, dtype=torch.float64)
        lp = lp - (torch.logsumexp(lp, 0) if teacher_lse is None else float(teacher_lse[r]))
        p = lp.exp()
        rest = 0.0 if teacher_lse is None else max(0.0, 1.0 - float(p.sum()))
        lq = torch.log_softmax(x, 0)
        some = p > 0
        total = (p[some] * (lp[some] - lq[at][some])).sum()
        others = lq.clone()
        others[at] = -math.inf
        target = torch.zeros(vocab, dtype=torch.float64)
        target[at] = p
        if rest > 0:
            log_rest = torch.logsumexp(others, 0)
            total = total + rest * (math.log(rest) - log_rest)
            if log_rest > -math.inf:
                target = target + rest * (others - log_rest).exp()
        loss[r] = w * total
        grad[r] = w * u / temperature * ((p.sum() + rest) * lq.exp() - target)
    return loss, grad
