"""Plain 64-bit implementations of the norm and gated-product calls, from include/pvt.h alone."""
import math

import torch

LAYER, RMS = 0, 1
SILU, GELU, GELU_TANH = 0, 1, 2
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def rounding(v, dtype):
    """how far rounding v to dtype moves it, at most"""
    return v.abs() * HALF_STEP[dtype] + SMALLEST[dtype]


def norm(r, kind, eps, weight=None, bias=None):
    """y, mean, rstd of the rows of r"""
    r = r.double()
    mean = r.mean(dim=1, keepdim=True) if kind == LAYER else torch.zeros_like(r[:, :1])
    d = r - mean
    rstd = ((d * d).mean(dim=1, keepdim=True) + eps).rsqrt()
    y = d * rstd
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean, rstd


def norm_bounds(r, kind, eps, weight=None, bias=None):
    """How far binary32 results of y, mean and rstd may be from the above.

    A sum along a row has at most 8 * 8 additions in a lane, 10 in exchanges: 74 roundings of 2^-24 of the sum of magnitudes, and a
    division.  The mean's error moves every difference; the sum of squares is off by 74 + 3 roundings and the square of the mean's
    error, the root halves that; a difference, two products and an addition round once each."""
    u = 2.0 ** -24
    r = r.double()
    w = torch.ones_like(r[0]) if weight is None else weight.double()
    y, mean, rstd = norm(r, kind, eps, weight, bias)
    d_mean = 75 * u * r.abs().mean(dim=1, keepdim=True) if kind == LAYER else torch.zeros_like(mean)
    d_rstd = rstd * (40 * u + 3 * u + 0.5 * d_mean ** 2 * rstd ** 2)
    scaled = (r - mean) * rstd * w
    d_y = rstd * w.abs() * d_mean + scaled.abs() * (d_rstd / rstd + 4 * u) + y.abs() * u
    return 1.001 * d_y + 2.0 ** -149, 1.001 * d_mean + 2.0 ** -149, 1.001 * d_rstd


def norm_grad(x, stats, dy, kind, weight=None, dresidual=None):
    """dx, dweight, dbias"""
    mean, rstd = stats.double().split(1, dim=1)
    xh, dy = (x.double() - mean) * rstd, dy.double()
    u = dy if weight is None else dy * weight.double()
    dx = u - xh * (u * xh).mean(dim=1, keepdim=True)
    if kind == LAYER:
        dx = dx - u.mean(dim=1, keepdim=True)
    dx = dx * rstd
    if dresidual is not None:
        dx = dx + dresidual.double()
    return dx, (dy * xh).sum(dim=0), dy.sum(dim=0)


def norm_grad_bounds(x, stats, dy, kind, weight=None, dresidual=None):
    """How far binary32 results may be from the above: xh has two roundings, u one, the means at most 16 + 10 + 10 additions and
    two products more, dx four and the residual's one.  Of the weights' gradients a thread adds the rows of its block, of which
    there are at least 37 where there are as many rows (148 SMs, up to four blocks to a row); exchanges add 13 more."""
    e = 2.0 ** -24
    mean, rstd = stats.double().split(1, dim=1)
    xh, dy = (x.double() - mean) * rstd, dy.double()
    u = dy if weight is None else dy * weight.double()
    m1 = u.abs().mean(dim=1, keepdim=True) if kind == LAYER else 0.0
    m2 = (u * xh).abs().mean(dim=1, keepdim=True)
    dx, _, _ = norm_grad(x, stats, dy, kind, weight, dresidual)
    d_dx = rstd * (4 * e * u.abs() + 42 * e * m1 + 46 * e * xh.abs() * m2)
    if dresidual is not None:
        d_dx = d_dx + e * dx.abs()
    n = -(-x.shape[0] // 37) + 13
    return (1.001 * d_dx + 2.0 ** -149, 1.001 * ((n + 4) * e * (dy * xh).abs().sum(dim=0)) + 2.0 ** -149,
            1.001 * ((n + 1) * e * dy.abs().sum(dim=0)) + 2.0 ** -149)


def activation(a, act):
    """f(a) and f'(a)"""
    if act == SILU:
        s = torch.sigmoid(a)
        return a * s, s + a * s * torch.sigmoid(-a)
    if act == GELU:
        phi = 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
        return a * phi, phi + a * torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    k, c = math.sqrt(2.0 / math.pi), 0.044715
    s = torch.sigmoid(2.0 * k * (a + c * a ** 3))
    return a * s, s + a * s * torch.sigmoid(-2.0 * k * (a + c * a ** 3)) * 2.0 * k * (1.0 + 3.0 * c * a * a)


def gated(a, b, act):
    return activation(a, act)[0] * b


def products(xv, wg, wu):
    """a, b and how far binary32 sums of them may be off: (cols + 4) 2^-23 of the sum of magnitudes"""
    n = (xv.shape[1] + 4) * 2.0 ** -23
    return xv @ wg.T, xv @ wu.T, n * (xv.abs() @ wg.abs().T), n * (xv.abs() @ wu.abs().T)


def _steps(a, act):
    """Roundings of 2^-23 in f(a) / a, relative: an exponential (2 units), a sum, a quotient (2) and products; an argument's own
    rounding counts as often as it is large: |z| of the logistic function's, a^2 of the normal distribution's (whose function is
    within 4 units)."""
    if act == GELU:
        return 10 + a * a
    z = a if act == SILU else 1.6 * (a + 0.045 * a ** 3)
    return 8 + 2 * z.abs()


def gated_bound(a, b, d_a, d_b, act):
    """How far h may be off in binary32, |f'| being at most 1.13; quotients beyond 2^126 are 0."""
    f, _ = activation(a, act)
    off = 1.13 * d_a * b.abs() + f.abs() * d_b + 1.13 * d_a * d_b + _steps(a, act) * 2.0 ** -23 * (f * b).abs()
    return 1.001 * off + 2.0 ** -126 * (1 + (a * b).abs())


def gated_grad_bounds(a, b, d_a, d_b, dh, act):
    """The same for dgate and dup, |f''| being at most 1; f' is a sum of two terms of at most 1.3, one of which has a difference
    from 1 in it (2^-24 of a dz / da)."""
    f, slope = activation(a, act)
    dz = torch.ones_like(a) if act == SILU else 1.6 + 0.22 * a * a
    d_slope = 2.0 ** -23 * (1.3 * (_steps(a, act) + 4) + (a.abs() * dz if act != GELU else 0.0))
    dh = dh.double().abs()
    d_gate = dh * (b.abs() * (d_a + d_slope) + slope.abs() * d_b + d_a * d_b + 2.0 ** -22 * (b * slope).abs())
    d_up = dh * (1.13 * d_a + (_steps(a, act) + 2) * 2.0 ** -23 * f.abs())
    return 1.001 * d_gate + 2.0 ** -126, 1.001 * d_up + 2.0 ** -126
