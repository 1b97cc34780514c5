"""float64 oracle of normalised, rotated heads: forward, backward and the backward of that, from the closed forms

  xh = r x, r = (mean(x^2) + eps)^-1/2 (1 without a weight),  y = R (w xh)
  g = R^T dy, a = w g:  dx = r (a - (a.xh) xh / d),  dw = sum g xh
  with cotangents u on dx and uw on dw:  A = a.u, B = a.xh, C = u.xh, S = (uw g).xh,
  xt = r uw g - r ((r A + S) xh + r C a + r B u) / d + 3 r^2 B C xh / d^2
  wt = sum (r g u - r C g xh / d),  dyt = R (r w u - r C w xh / d + uw xh)

one tensor of heads [B, H, N, d] at a time.
"""
import numpy as np


def _f(x):
    return np.asarray(x, dtype=np.float64)


def turned(x, angles, interleaved):
    """x with its pairs turned by angles [B, N, pairs]."""
    n = angles.shape[-1]
    i = np.arange(n)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
    c, s = np.cos(angles)[:, None], np.sin(angles)[:, None]
    y = np.array(x, dtype=np.float64)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def angles(positions, freqs, axes):
    """[B, N, pairs] from positions [axes, B, N]."""
    return _f(positions)[np.asarray(axes)].transpose(1, 2, 0) * _f(freqs)


def run(x, angle, w=None, eps=1e-6, interleaved=False, dy=None, u=None, uw=None):
    """Dict of y; with dy also dx and dw; with u (and uw) also xt, dyt and wt (dw and wt with a weight)."""
    x = _f(x)
    d = x.shape[-1]
    if w is None:
        out = {"y": turned(x, angle, interleaved)}
        if dy is not None:
            out["dx"] = turned(_f(dy), -angle, interleaved)
        if u is not None:
            out["dyt"] = turned(_f(u), angle, interleaved)
            out["xt"] = np.zeros_like(x)
        return out
    w = _f(w)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh = r * x
    out = {"y": turned(w * xh, angle, interleaved)}
    if dy is None:
        return out
    dot = lambda p, q: (p * q).sum(-1, keepdims=True)  # noqa: E731
    g = turned(_f(dy), -angle, interleaved)
    a = w * g
    out["dx"] = r * (a - dot(a, xh) * xh / d)
    out["dw"] = (g * xh).sum((0, 1, 2))
    if u is None:
        return out
    u, uw = _f(u), _f(uw)
    A, B, C, S = dot(a, u), dot(a, xh), dot(u, xh), dot(uw * g, xh)
    out["xt"] = (r * uw * g - r * ((r * A + S) * xh + r * C * a + r * B * u) / d + 3 * r * r * B * C * xh / d ** 2)
    out["wt"] = (r * g * u - r * C * g * xh / d).sum((0, 1, 2))
    out["dyt"] = turned(r * w * u - r * C * w * xh / d + uw * xh, angle, interleaved)
    return out
