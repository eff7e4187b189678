"""Inputs of the 8-bit tests and their plain implementations in float64."""
import numpy as np
import torch

CODE = {"f16": 1, "bf16": 0}
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
# half a step of a type relative to the value, and half its smallest step
HALF = {torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134),
        torch.float32: (2.0 ** -24, 2.0 ** -150)}


def strided(t, cols, offset=0):
    """t's values as rows of stride `cols`, `offset` elements into each; and the buffer, filled with 77 around them."""
    buf = torch.full((t.shape[0], cols), 77, dtype=t.dtype, device=t.device)
    view = buf[:, offset:offset + t.shape[1]]
    view.copy_(t)
    return view, buf


def untouched(buf, cols, offset=0):
    """Everything of a strided buffer outside its rows still holds 77."""
    b = buf.float().cpu()
    return bool((b[:, :offset] == 77).all() and (b[:, offset + cols:] == 77).all())


def norm64(s, g, b, layer, eps):
    """(y, error of y in 64 bits per element) of rows s as they are stored; CPU."""
    s, d = s.double(), s.shape[1]
    mean = s.mean(1, keepdim=True) if layer else torch.zeros(s.shape[0], 1, dtype=torch.float64)
    v = s - mean
    rstd = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + float(np.float32(eps)))
    u = v * rstd * g.double()
    y = u + (0 if b is None else b.double())
    # sums of d terms in any order, both sides: 2 (d + 16) 2^-53 of the mean magnitude (the
    # mean) and of the result (the root), and of the addition's operands
    err = (d + 16) * 2.0 ** -52 * (u.abs() + y.abs() + (0 if b is None else b.double().abs()) +
                                   s.abs().mean(1, keepdim=True) * rstd * g.double().abs() * (1 if layer else 0))
    return y, err


def check_rows8(q, scale, y, err, what=""):
    """q and scale (any device) against rows y in float64, themselves off by err: the scale is
    max|y| / 127 rounded to fp32, q the integer next to y / scale."""
    q, scale = q.cpu(), scale.cpu()
    top = y.abs().amax(1)
    exact = top / 127
    tiny = exact < 2.0 ** -126 * (1 + 1e-9)
    step = torch.from_numpy(np.spacing(scale.abs().clamp(min=2.0 ** -126).numpy())).double()
    off = (scale.double() - exact).abs()
    bound = step / 2 + err.amax(1) / 127 + exact * 2.0 ** -52
    assert bool(((off <= bound) | (tiny & (scale == 0))).all()), (what, (off / step).max())
    s = scale.double()[:, None]
    t = torch.where(s > 0, y / s, 0.0)
    off = (q.double() - t).abs()
    bound = 0.5 + torch.where(s > 0, err / s, 0.0) + 127 * 2.0 ** -52
    assert bool((off <= bound).all()), (what, float((off - bound).max()))
    assert int(q.to(torch.int32).abs().max()) <= 127


def gemm64(X, sx, W, sw, bias, epi, qscale, qcols, old, dt):
    """(out, tolerance) in float64.

    The integer sum is exact; it is rounded to fp32, multiplied by sx, multiplied by sw and
    added to the bias with one rounding, multiplied by qscale, added to the old value: each
    at most 2^-24 of its result.  Then one rounding to the output's type."""
    u = 2.0 ** -24
    acc = X.double() @ W.double().t()  # exact: below 2^53
    p = acc * sx.double()[:, None] * sw.double()[None]
    y = p + (0 if bias is None else bias.double()[None])
    tol = 2.01 * u * p.abs() + u * y.abs()
    if epi == 0:
        f = torch.where(torch.arange(W.shape[0], device=W.device) < qcols, float(np.float32(qscale)), 1.0)[None]
        y, tol = y * f, tol * f + u * (y * f).abs()
    elif epi == 1:
        y = y.clamp(min=0)
    elif epi == 2:
        y = y + old.double()
        tol = tol + u * y.abs()
    kind = dt if epi < 2 else torch.float32
    half, least = HALF[kind]
    if epi < 2:
        tol = tol * (1 + half) + half * y.abs() + least
    return y, tol + 2.0 ** -149


def numbers8(g, rows, cols):
    return torch.randint(-128, 128, (rows, cols), generator=g, dtype=torch.int32).to(torch.int8)
