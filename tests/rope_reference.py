"""Plain 64-bit definition of the norms and rotation of heads (torch on the
CPU, none of the library's code), and the tolerance of its fp32 steps."""
from fractions import Fraction

import torch

PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def angles(positions, inv_freq):
    """Positions times frequencies, whole turns taken out exactly, [tokens, pairs]."""
    rows = []
    for p in positions:
        rows.append([float(a - 2 * PI * (a // (2 * PI))) for a in (Fraction(int(p)) * Fraction(f) for f in inv_freq)])
    return torch.tensor(rows, dtype=torch.float64).reshape(len(rows), len(inv_freq))


def rotate(x, positions, inv_freq, interleaved=False, norm=None, eps=1e-6, offset=0.0, scale=1.0):
    """Heads x [tokens, heads, dim] normalised and rotated, and how far fp32 steps may be off:
    2^-20 of the elements that a result is made of.  A norm's factor is a
    sum of D squares (up to 16 of a lane, then 2 or 3 exchanges: under 20 roundings of 2^-24, halved by the root), a
    root (2^-22) and two products (2^-23); a sine or cosine is off by 2^-23
    and by an angle of 2^-25 half turns (2^-23); two products and a sum (2^-23): below 2^-20.4 together."""
    y, rot = x.double(), 2 * len(inv_freq)
    if norm is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32)))
        y = y * (norm.double() + offset)
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    t = angles(positions, inv_freq)[:, None]
    out, tol = y.clone(), y.abs() * 2.0 ** -20
    ya, yb = y[..., a], y[..., b]
    s = float(torch.tensor(scale, dtype=torch.float32))
    out[..., a], out[..., b] = s * (ya * t.cos() - yb * t.sin()), s * (yb * t.cos() + ya * t.sin())
    tol[..., a] = tol[..., b] = abs(s) * (ya.abs() + yb.abs()) * 2.0 ** -20
    return out, tol


def frequencies(rot, theta=500000.0):
    return [theta ** (-2.0 * i / rot) for i in range(rot // 2)]


def check_bf16(got, want, tol):
    """Rounded once to bf16 (2^-8 of the value at most, 2^-134 below its normal range)."""
    assert torch.equal(got.isnan(), want.isnan())
    err = (got.double() - want).abs() - (tol * 1.01 + want.abs() * 2.0 ** -8 + 2.0 ** -134)
    bad = ~want.isnan() & ~(err <= 0)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, by {float(err[bad].max()):.3g} over the bound"


def check_codes(codes, exps, want, tol):
    """Stored rows [.., dim] of the values want: the exponent the smallest that holds the row's largest
    magnitude (as fp32 may have it), the codes within half an e4m3 step of the value (2^-4 of it, 2^-10 of the unit at least)."""
    e = exps.long()
    a, ta = want.abs().amax(-1), tol.amax(-1) * 1.01
    unit = torch.exp2(e.double() - 127)
    assert bool((a - ta <= 448 * unit)[e > 0].all())
    assert bool(((a + ta > 224 * unit) | (e == 1))[e > 0].all())
    assert bool((a[e == 0] <= ta[e == 0]).all())
    err = (codes * unit[..., None] - want).abs() - (want.abs() * 2.0 ** -4 + unit[..., None] * 2.0 ** -10 + 1.1 * tol)
    assert bool((err <= 0)[e > 0].all()), f"off by {float(err.max()):.3g} over the bound"


__all__ = ["PI", "angles", "rotate", "frequencies", "check_bf16", "check_codes"]
