"""Float64 definitions of the router, the exchange of rows and the distillation
loss, and the error bounds their tests use.  Plain torch; nothing of the library.

U = 2^-24 is half a step of fp32.  The hardware's exp2 is good to one ulp (2 U);
its argument x log2(e) (or x log2(e) / T) carries up to three roundings, so
e^x is off by (3 |x| + 2) U of itself.  A sum of n fp32 terms in any order is
off by n U of the sum of their magnitudes.
"""

import math

import torch

from stage_ref import unit

U = 2.0 ** -24


def exp_rel(x):
    """Relative error of e^x as the kernels compute it (x <= 0, e^-inf exact)."""
    return torch.where(torch.isfinite(x), (3 * x.abs() + 2) * U, 0.0)


# ---------------------------------------------------------------------------
# router
# ---------------------------------------------------------------------------
def plan64(logits, k):
    """(index, offsets, order, slots) by picking the first of the largest, k times."""
    x = torch.nan_to_num(logits.double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    t, e = x.shape
    number = torch.arange(e, device=x.device).expand(t, e)
    index = torch.full((t, k), -1, dtype=torch.long, device=x.device)
    for j in range(k):
        top = x.amax(1, keepdim=True)
        at = torch.where(x == top, number, e).amin(1, keepdim=True)
        index[:, j:j + 1] = torch.where(top > -math.inf, at, -1)
        x = x.scatter(1, at, -math.inf)
    flat = index.view(-1).cpu().tolist()
    runs = [[] for _ in range(e)]
    for i, expert in enumerate(flat):
        if expert >= 0:
            runs[expert].append(i)
    order = [i for r in runs for i in r]
    slots = [-1] * len(flat)
    for s, i in enumerate(order):
        slots[i] = s
    offsets = [0]
    for r in runs:
        offsets.append(offsets[-1] + len(r))
    return index, offsets, order, torch.tensor(slots).view(t, k)


def weights64(logits, index, renorm):
    """(weights, bound)"""
    x = logits.double()
    x = torch.where(torch.isnan(x), -math.inf, x)
    none = index < 0
    chosen = torch.gather(x, 1, index.clamp_min(0)).masked_fill(none, -math.inf)
    top = chosen[:, :1]
    every = chosen if renorm else x
    d = torch.where(torch.isfinite(top), every - top, -math.inf)
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    zrel = (e * exp_rel(d)).sum(1, keepdim=True) / z + (every.shape[1] + 8) * U
    dc = torch.where(none, -math.inf, chosen - top)
    w = torch.where(none, 0.0, torch.exp(dc) / z)
    return w, torch.where(none, 0.0, w * (exp_rel(dc) + zrel + 4 * U) * 1.01)


def route_bwd64(logits, index, weights, dweights, renorm):
    """(dlogits, bound) from the weights as they are stored"""
    x, live = logits.double(), index >= 0
    w = torch.where(live, weights.double(), 0.0)
    up = torch.where(live, w * dweights.double(), 0.0)
    s, size = up.sum(1, keepdim=True), up.abs().sum(1, keepdim=True)
    k = index.shape[1]
    serr = (k + 8) * U * size
    if renorm:
        v = up - w * s
        err = serr * w + 4 * U * (up.abs() + (w * s).abs())
        d, b = torch.zeros_like(x), torch.zeros_like(x)
    else:
        v, err = up, 2 * U * up.abs()
        top = x.amax(1, keepdim=True)
        e = torch.where(top > -math.inf, torch.exp(x - top), 0.0)
        z = e.sum(1, keepdim=True).clamp_min(1e-300)
        rel = torch.where(top > -math.inf, exp_rel(x - top), 0.0)
        zrel = (e * rel).sum(1, keepdim=True) / z + (x.shape[1] + 8) * U
        p = e / z
        d = -p * s
        b = p * serr + (rel + zrel + 6 * U) * d.abs()
    at = index.clamp_min(0)
    d = d.scatter_add(1, at, torch.where(live, v, 0.0))
    b = b.scatter_add(1, at, torch.where(live, err, 0.0)) + 4 * U * d.abs()
    return d, b + unit(logits.dtype) * 1.01 * (d.abs() + b)


# ---------------------------------------------------------------------------
# exchange
# ---------------------------------------------------------------------------
def combine64(Ys, slots, weights, R):
    """(Y, bound)"""
    live = slots >= 0
    w = torch.ones(slots.shape, dtype=torch.float64, device=Ys.device) if weights is None \
        else weights.double()
    rows = Ys.double()[slots.long().clamp_min(0)]
    terms = torch.where(live[:, :, None], rows * torch.where(live, w, 0.0)[:, :, None], 0.0)
    y, size = terms.sum(1), terms.abs().sum(1)
    if R is not None:
        y, size = y + R.double(), size + R.double().abs()
    b = (slots.shape[1] + 2) * U * size
    return y, b + unit(Ys.dtype) * 1.01 * (y.abs() + b)


def combine_bwd64(dY, Ys, slots, weights):
    """(dYs of each entry, its bound, dweights, its bound)"""
    live = slots >= 0
    w = torch.ones(slots.shape, dtype=torch.float64, device=dY.device) if weights is None \
        else torch.where(live, weights.double(), 0.0)
    d = dY.double()[:, None, :] * w[:, :, None]
    b = U * d.abs()
    terms = dY.double()[:, None, :] * Ys.double()[slots.long().clamp_min(0)]
    n = dY.shape[1]
    dw = torch.where(live, terms.sum(2), 0.0)
    return d, b + unit(dY.dtype) * 1.01 * (d.abs() + b), dw, (n / 64 + 16) * U * torch.where(
        live, terms.abs().sum(2), 0.0) + U * dw.abs()


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------
def distill64(S, index, teacher, temperature, alpha, labels, scale):
    """{"loss", "lse", "dS": (value, bound)}; dS both from the statistics of the
    same pass and from stored logarithms ("dS_lse")."""
    s = S.double()
    t, v = s.shape
    T = temperature
    dev = S.device
    one = torch.ones(t, dtype=torch.float64, device=dev)
    scale = one if scale is None else scale.double()
    label = torch.full((t,), -1, device=dev) if labels is None or alpha == 1 else labels.long()
    label = torch.where(label < v, label, -1)
    if index is None or index.shape[1] == 0 or alpha == 0:
        index = torch.full((t, 1), -1, device=dev)
        teacher = torch.zeros(t, 1, device=dev)
    at = torch.where((index >= 0) & (index < v), index.long(), -1)
    tt = torch.where(at >= 0, teacher.double(), -math.inf) / T
    k = at.shape[1]
    top = tt.amax(1, keepdim=True)
    soft = (top[:, 0] > -math.inf) & (scale != 0)
    hard = (label >= 0) & (scale != 0)
    live = soft | hard
    safe = torch.where(live[:, None], s, 0.0)

    # the teacher's distribution over the columns, and its relative error
    d = torch.where(soft[:, None], tt - top, -math.inf)
    pe = torch.exp(d)
    psum = pe.sum(1, keepdim=True).clamp_min(1e-300)
    p = pe / psum
    prel = exp_rel(d) + (p * exp_rel(d)).sum(1, keepdim=True) + (k + 16) * U
    col = at.clamp_min(0)
    P = torch.zeros_like(s).scatter_add_(1, col, torch.where(at >= 0, p, 0.0))
    PE = torch.zeros_like(s).scatter_add_(1, col, torch.where(at >= 0, p * prel, 0.0))

    def stats(x):
        m = x.amax(1, keepdim=True)
        e = torch.exp(x - m)
        z = e.sum(1, keepdim=True)
        rel = exp_rel(x - m)
        zrel = (e * rel).sum(1, keepdim=True) / z + (v / 64 + 64) * U
        return m, z, rel, zrel, e / z

    m, z, rel, zrel, q = stats(safe / T)
    m1, z1, rel1, zrel1, c = stats(safe)
    a_s = torch.where(soft, scale * alpha * T, 0.0)[:, None]
    a_h = torch.where(hard, scale * (1 - alpha), 0.0)[:, None]
    hot = torch.zeros_like(s).scatter_(1, label.clamp_min(0)[:, None], 1.0)
    dS = a_s * (q - P) + a_h * (c - hot)
    b = a_s.abs() * (q * (rel + zrel + 6 * U) + PE + 4 * U * P) \
        + a_h.abs() * (c * (rel1 + zrel1 + 6 * U) + 2 * U * hot) + 4 * U * dS.abs()
    lse, lse1 = m + torch.log(z), m1 + torch.log(z1)
    # a logarithm of the sum: its own relative error, two roundings, and its storage
    lerr = zrel + 4 * U * torch.log(z).abs() + 2 * U * m.abs() + U * lse.abs()
    lerr1 = zrel1 + 4 * U * torch.log(z1).abs() + 2 * U * m1.abs() + U * lse1.abs()
    again = a_s.abs() * q * (lerr + 3 * U * (safe.abs() / T + lse.abs()) + 6 * U) \
        + a_h.abs() * c * (lerr1 + 3 * U * (safe.abs() + lse1.abs()) + 6 * U)
    keep = a_s.abs() * (PE + 4 * U * P) + a_h.abs() * 2 * U * hot + 4 * U * dS.abs()
    st = unit(S.dtype) * 1.01

    # the loss
    logp = torch.where(p > 0, d - torch.log(psum), 0.0)
    x = torch.where(at >= 0, torch.gather(safe / T, 1, col) - m, 0.0)
    logz = torch.log(z)
    kl = torch.where(p > 0, p * (logp - (x - logz)), 0.0).sum(1)
    parts = p * (logp.abs() + x.abs() + logz.abs())
    klerr = (parts * (prel + (k + 16) * U)).sum(1) + (p * (zrel + prel)).sum(1) + \
        3 * U * (p * (d.nan_to_num(neginf=0.0).abs() + x.abs())).sum(1)
    ce = lse1[:, 0] - torch.gather(safe, 1, label.clamp_min(0)[:, None])[:, 0]
    ceerr = zrel1[:, 0] + 6 * U * (torch.log(z1).abs()[:, 0] + ce.abs())
    soft_part = torch.where(soft, scale * alpha * T * T * kl, 0.0)
    hard_part = torch.where(hard, scale * (1 - alpha) * ce, 0.0)
    loss = soft_part + hard_part
    lossb = torch.where(soft, (scale * alpha).abs() * T * T * klerr, 0.0) \
        + torch.where(hard, (scale * (1 - alpha)).abs() * ceerr, 0.0) \
        + 8 * U * (soft_part.abs() + hard_part.abs())
    lv = torch.stack([torch.where(soft, lse[:, 0], 0.0), torch.where(hard, lse1[:, 0], 0.0)], 1)
    lb = torch.cat([lerr, lerr1], 1)
    return {"loss": (loss, lossb), "lse": (lv, lb),
            "dS": (dS, b + st * (dS.abs() + b)),
            "dS_lse": (dS, again + keep + st * (dS.abs() + again + keep))}
