"""Float64 definitions of the stage operators, and the error bounds their
tests use.  Plain torch on the CPU or the GPU; nothing of the library.

Bounds are per element and derived, not fitted:
- a stored bf16 value is off by at most 2^-8 of itself (8 significant bits,
  round to nearest: 1 + 2^-8 is stored as 1); fp32 by 2^-24;
- a sum of K products in fp32, in any order, by at most (K + 8) 2^-24 of the
  sum of their magnitudes, 8 for the epilogue's few additions; doubled for the
  matrix unit's own intermediate rounding;
- the activations use the hardware's exp2 and reciprocal (1 ulp each) and, for
  GELU, a published approximation of erfc good to 1.5e-7: ACT = 1e-6 of
  (1 + |z|) covers each of them and their derivatives; |act'| <= 1.13, so an
  error of z grows by at most LIP = 1.2.
"""

import math

import torch

ACT = 1e-6
LIP = 1.2


def unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


def act64(act, z):
    """(act(z), act'(z))"""
    if act == 0:
        return z, torch.ones_like(z)
    if act == 1:
        return z.clamp_min(0), (z > 0).to(z.dtype)
    if act == 2:
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == 3:
        q = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        t = torch.tanh(q)
        dq = math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * dq
    s = torch.sigmoid(z)
    return z * s, s * (1 + z * (1 - s))


def forward64(X, W, bias, act, R, gated):
    """(Y, Z, bound of Y, bound of Z)"""
    dt, k = X.dtype, X.shape[1]
    x, w = X.double(), W.double()
    z = x @ w.t()
    s = x.abs() @ w.abs().t()
    if bias is not None:
        z, s = z + bias.double(), s + bias.double().abs()
    dz = 2 * (k + 8) * 2.0 ** -24 * s
    n = W.shape[0] // 2 if gated else W.shape[0]
    a, _ = act64(act, z[:, :n])
    da = LIP * dz[:, :n] + ACT * (1 + z[:, :n].abs())
    if gated:
        u, du = z[:, n:], dz[:, n:]
        y = a * u
        dy = da * (u.abs() + du) + a.abs() * du + 2.0 ** -23 * y.abs()
    else:
        y, dy = a, da
    if R is not None:
        y = y + R.double()
        dy = dy + 2.0 ** -23 * y.abs()
    return y, z, dy + unit(dt) * (y.abs() + dy) * 1.01, dz + unit(dt) * (z.abs() + dz) * 1.01


def backward64(dY, X, W, Z, act, gated, dw_dtype=None):
    """{name: (value, bound)} of dX, dW and dbias"""
    dt = dY.dtype
    dy = dY.double()
    if Z is None:
        dz, slack = dy, torch.zeros_like(dy)
    else:
        z = Z.double()
        n = dY.shape[1]
        a, da = act64(act, z[:, :n])
        err = ACT * (1 + z[:, :n].abs()) * dy.abs()
        if gated:
            u = z[:, n:]
            dz = torch.cat((dy * u * da, dy * a), 1)
            slack = torch.cat((err * u.abs(), err), 1)
        else:
            dz, slack = dy * da, err
        slack = slack + 2.0 ** -22 * dz.abs()
    summed = (dz.abs() + slack).sum(0) * dY.shape[0] * 2.0 ** -24 + slack.sum(0)
    out = {"dbias": (dz.sum(0), summed + 2.0 ** -24 * dz.sum(0).abs())}
    if Z is not None:
        slack = slack + unit(dt) * 1.01 * (dz.abs() + slack)
    top = dz.abs() + slack
    if W is not None:
        w = W.double()
        v = dz @ w
        b = slack @ w.abs() + 2 * (dz.shape[1] + 8) * 2.0 ** -24 * (top @ w.abs())
        out["dX"] = (v, b + unit(dt) * 1.01 * (v.abs() + b))
    if X is not None:
        x = X.double()
        v = dz.t() @ x
        b = slack.t() @ x.abs() + 2 * (dz.shape[0] + 8) * 2.0 ** -24 * (top.t() @ x.abs())
        out["dW"] = (v, b + unit(dw_dtype or dt) * 1.01 * (v.abs() + b))
    return out


def within(got, want, bound, what=""):
    """Every element inside its bound (2^-126 for results that underflow)."""
    off = (got.double() - want).abs() - bound - 2.0 ** -126
    assert torch.isfinite(got).all(), what
    bad = int((off > 0).sum())
    assert bad == 0, f"{what}: {bad} of {off.numel()} outside, worst by {float(off.max()):.3g}"


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
RUN = 256


def e4m3_values():
    """The 127 magnitudes of OCP e4m3, from its definition."""
    v = []
    for c in range(127):
        e, f = c >> 3, c & 7
        v.append(f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return torch.tensor(v, dtype=torch.float64)


def decode(codes, scale, cols):
    """float64 values of 8-bit codes (rows x cols, uint8) with their scales."""
    c = codes.view(torch.uint8).long()
    v = e4m3_values().to(codes.device)
    mag = torch.where((c & 127) < 127, v[(c & 127).clamp_max(126)], torch.nan)
    wide = scale.double().repeat_interleave(RUN, 1)[:, :cols]
    return torch.where(c >= 128, -mag, mag) * wide


def adamw64(W, m, v, g, lr, b1, b2, eps, step, decay):
    """(W, m, v, sqrt v) of one step from float64 inputs"""
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    w = W * (1 - lr * decay) - lr * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + eps)
    return w, m, v, v.sqrt()
