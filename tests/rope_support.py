"""Plain 64-bit norm, rotation and gradients of queries and keys, with the bounds on
what fp32 arithmetic and one final rounding may be off."""
import torch

U = 2.0 ** -24                                        # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def pairs(rot, interleaved):
    """Index of each rotated value's other value, its pair, and its sine's sign."""
    at = torch.arange(rot)
    if interleaved:
        return at ^ 1, at // 2, torch.where(at % 2 == 0, -1.0, 1.0).double()
    h = rot // 2
    return (at + h) % max(rot, 1), at % max(h, 1), torch.where(at < h, -1.0, 1.0).double()


def turn(x, pos, freqs, interleaved, back=False):
    """x [T][H][d] (64 bits) at positions pos [T]; also |value| + |other value| of each pair,
    what the errors of the turn are relative to."""
    rot = 0 if freqs is None else 2 * freqs.numel()
    y, size = x.clone(), x.abs()
    if rot:
        other, pair, sign = pairs(rot, interleaved)
        a = (pos.double()[:, None] * freqs.double())[:, None, pair]
        s = torch.sin(a) * sign * (-1 if back else 1)
        y[..., :rot] = x[..., :rot] * torch.cos(a) + x[..., other] * s
        size[..., :rot] = x[..., :rot].abs() + x[..., other].abs()
    return y, size


def forward(x, w, pos, freqs, interleaved, eps):
    """(result, bound without the final rounding).  fp32: the sum of squares is off by at most
    13 U relative (8 products a lane, five additions), so its inverse root by 7 U and a step of the
    instruction's (2 U); three products and the fma's add 4 U; the angle's fraction is rounded once
    (pi U radians) and the sine's polynomial is off by at most 4 U: 24 U of |a| + |b| in all."""
    x = x.double()
    n = x
    if w is not None:
        n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    y, size = turn(n, pos, freqs, interleaved)
    return y, 24 * U * size


def backward(x, w, dy, pos, freqs, interleaved, eps):
    """(dx, its bound, terms of dw, their bound); as above, the products and the row's second sum
    add 13 U and 8 U, doubled to 48 U of the absolute terms."""
    g, size = turn(dy.double(), pos, freqs, interleaved, back=True)
    if w is None:
        return g, 24 * U * size, None, None
    x, w = x.double(), w.double()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    n, h = x * r, g * w
    dx = r * (h - n * (n * h).mean(-1, keepdim=True))
    tol = 48 * U * r * (size * w.abs() + n.abs() * (n.abs() * size * w.abs()).mean(-1, keepdim=True))
    return dx, tol, g * n, size * n.abs()
