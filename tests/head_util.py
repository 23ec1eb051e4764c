"""Inputs, a plain 64-bit implementation and tolerances for the tests of the head operators.

Tolerances, from the arithmetic alone.  B = 2^-8 is the largest relative error of a rounding to bf16, u = 2^-24 of one to fp32.

  logits    x is a sum of D products of bf16 values (exact in fp32).  32 of them at a time are added by one matrix
            instruction, so at most D / 32 + 8 dependent roundings (2 u each, should the unit truncate) act on sums of at most
            S = sum |h w| + |bias|:  dx = (D / 32 + 8) 2 u S.  A wave's own sum of a row (the logits at labels and ids) has
            D / 64 + 6 of them.  The soft cap has a slope of at most 1 and adds 2^-21 cap (exponential, reciprocal and two
            operations of 1 .. 2 u, at a derivative of at most 1/2).
  lse, nll  errors of logits pass on with weights that sum to 1; the exponents' arguments (up to 128 in magnitude where a
            term counts, 128 u ln 2 each), the exponential and the sums (32 terms per lane, then trees and V / 128 / 256
            partials) give less than 2^-16 of the sum together; two roundings of the result.
  kd        the same, and each of its terms p_T (log p_T - log p_S) once more 2^-20 relative.
  G         kept as bf16 (B |G|), times a factor of the row that is off by a weighted mean of the roundings of its entries at
            the label and the teacher's ids (B |G| at most again); where it is a difference its parts w p, gs p_T, cs 1 carry the errors of the scalars.
            A soft cap's slope 1 - (x / cap)^2 changes by 2 dx / cap relative with x, and is a difference from 1 of a square
            that is off by 2^-20 at most.
  grads     |dG| passes through the second product, whose fp32 sums of n terms add (n / 32 + 8) 2 u sum |G| |w|; hidden
            states are rounded once more with the row's scale (B); the result is rounded to bf16 (B).
"""
import torch

B, U = 2.0 ** -8, 2.0 ** -24


def dev():
    return torch.device("cuda:0")


def inputs(T, V, D, k=0, bias=False, seed=0, spread=3.0, mask=0.75, device=None):
    """bf16 hidden states and weights with logits of a few units, labels that are expected to all degrees, a teacher's record."""
    device = device or dev()
    g = torch.Generator(device=device).manual_seed(1000 * seed + T + 7 * V + 31 * D + k)

    def randn(*shape):
        return torch.randn(shape, device=device, generator=g)

    w = (randn(V, D) * (spread / D ** 0.5)).to(torch.bfloat16)
    labels = torch.randint(0, V, (T,), device=device, generator=g)
    h = randn(T, D) + (6.0 / spread ** 2) * torch.rand((T, 1), device=device, generator=g) * 2 * w[labels].float()
    s = dict(hidden=h.to(torch.bfloat16), weight=w, labels=labels.to(torch.int32),
             mask=(torch.rand(T, device=device, generator=g) < mask).to(torch.uint8),
             bias=randn(V).to(torch.bfloat16) if bias else None, idx=None, val=None)
    if k:
        step = torch.randint(1, max(2, V // k), (T, 1), device=device, generator=g) if V > k else 1
        first = labels[:, None] if seed % 2 == 0 else torch.randint(0, V, (T, 1), device=device, generator=g)
        s["idx"] = ((first + step * torch.arange(k, device=device)) % V).to(torch.int32).contiguous()
        s["val"] = torch.log_softmax(2.0 * randn(T, k), 1).contiguous()
    return s


def head64(s, cap=0.0):
    """64-bit logits, the soft cap's slope and the bound on the errors of fp32 ones."""
    h, w = s["hidden"].double(), s["weight"].double()
    z, size = h @ w.T, h.abs() @ w.abs().T
    if s["bias"] is not None:
        z, size = z + s["bias"].double(), size + s["bias"].double().abs()
    dx = (h.shape[1] / 32 + 8) * 2 * U * size
    if not cap:
        return z, torch.ones_like(z), dx
    y = cap * torch.tanh(z / cap)
    return y, 1 - (y / cap) ** 2, dx + cap * 2.0 ** -21


def loss64(s, *, cap=0.0, tau=1.0, grad_scale=1.0, ce=0.0):
    """Scalars, gradients and their tolerances ({name: (value, tolerance)})."""
    x, slope, dx = head64(s, cap)
    T, V = x.shape
    on = s["mask"].bool()
    rows = torch.arange(T, device=x.device)
    lse = torch.logsumexp(x / tau, 1)
    y = s["labels"].long()
    p = torch.exp(x / tau - lse[:, None])
    d = dx.nan_to_num(0.0, 0.0, 0.0).amax(1) / tau  # of a row's logits
    out = {}

    def scalar(name, v, t):
        out[name] = (torch.where(on, v, torch.zeros_like(v)), torch.where(on, t, torch.zeros_like(t)))

    if tau == 1.0:
        scalar("lse", lse, d + 2.0 ** -16 + 4 * U * lse.abs())
        nll = lse - x[rows, y]
        scalar("nll", nll, 2 * d + 2.0 ** -16 + 4 * U * nll.abs())
    kd_w = grad_scale / tau if s["idx"] is not None else 0.0
    gw = kd_w + ce
    G = gw * p
    parts = abs(gw) * p
    if s["idx"] is not None:
        ids = s["idx"].long()
        logq = torch.log_softmax(s["val"].double() / tau, 1)
        q = logq.exp()
        terms = torch.where(q > 0, q * (logq - x.gather(1, ids) / tau + lse[:, None]), torch.zeros_like(q))
        scalar("kd", terms.sum(1), 2 * d + 2.0 ** -16 + 2.0 ** -20 * terms.abs().sum(1))
        G = G.scatter_add(1, ids, -kd_w * q)
        parts = parts.scatter_add(1, ids, abs(kd_w) * q)
    if ce:
        G[rows, y] -= ce
        parts[rows, y] += abs(ce)
    G, parts, flat = G * slope * on[:, None], parts * slope * on[:, None], parts * on[:, None]
    dG = 2 * B * G.abs() + (2 * d[:, None] + 2.0 ** -18) * parts
    if cap:
        dG = dG + 2 * d[:, None] * tau / cap * parts + 2.0 ** -20 * flat
    h, w = s["hidden"].double(), s["weight"].double()
    out["grad_hidden"] = _with_rounding(G @ w, dG @ w.abs() + (V / 32 + 8) * 2 * U * (parts @ w.abs()))
    out["grad_weight"] = _with_rounding(
        G.T @ h, (dG + B * (1 + B) * (G.abs() + dG)).T @ h.abs() + (T / 32 + 8) * 2 * U * (parts.T @ h.abs()))
    out["grad_bias"] = _with_rounding(G.sum(0), dG.sum(0) + (T + 8) * 2 * U * parts.sum(0))
    return out


def _with_rounding(v, t):
    return v, t + B * (v.abs() + t) + 2.0 ** -126


def bwd64(g, s, logits=None, cap=0.0):
    z = g.double()
    dz = torch.zeros_like(z)
    if cap:
        z = z * (1 - (logits.double() / cap) ** 2)
        dz = B * z.abs() + 8 * U * g.double().abs()
    h, w = s["hidden"].double(), s["weight"].double()
    T, V = z.shape
    a = z.abs() + dz
    return dict(grad_hidden=_with_rounding(z @ w, dz @ w.abs() + (V / 32 + 8) * 2 * U * (a @ w.abs())),
                grad_weight=_with_rounding(z.T @ h, dz.T @ h.abs() + (T / 32 + 8) * 2 * U * (a.T @ h.abs())),
                grad_bias=_with_rounding(z.sum(0), dz.sum(0) + (T + 8) * 2 * U * a.sum(0)))


def near(got, want, name=""):
    """`got` within the tolerance of `want` = (value, tolerance), with the same infinities and NaN."""
    v, t = want
    got = got.double()
    fine = torch.isfinite(v)
    same = torch.where(fine, (got - v).abs() <= t, (got == v) | (got.isnan() & v.isnan()))
    if not bool(same.all()):
        off = ((got - v).abs() / t)[fine & ~same]
        raise AssertionError(f"{name}: {int((~same).sum())} of {same.numel()} values off, the worst by "
                             f"{off.max().item() if off.numel() else float('nan'):.3g} tolerances")
