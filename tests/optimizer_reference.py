"""Plain 64-bit forms of the optimiser operators, and how far the library may be from them.

The bounds count roundings: a rounding to nearest is off by at most half a step, eps / 2 relative (binary32 2^-24,
bfloat16 2^-8).
"""
import numpy as np
import torch

U32, UB = 2.0 ** -24, 2.0 ** -8


def f32(x: float) -> float:
    return float(np.float32(x))


def momentum(m, idx, vals, scale, mu, nesterov):
    """(momentum, update) in 64 bits and the bounds of both in binary32."""
    m, g = m.double(), torch.zeros(m.numel(), dtype=torch.float64)
    g[idx.long()] = f32(scale) * vals.double()
    mu = f32(mu)
    new = mu * m + g
    # scale * val is rounded once, the fma once
    bound = U32 * (g.abs() + new.abs()) * 1.001 + 1e-44
    if not nesterov:
        return new, new, bound, bound
    u = mu * new + g
    return new, u, bound, (mu * bound + U32 * (g.abs() + u.abs())) * 1.001 + 1e-44


def view(flat, place):
    offset, rows, cols, stride = place
    return flat.as_strided((rows, cols), (stride, 1), flat.storage_offset() + offset)


def orthogonalize(u, coeffs, eps):
    """Newton-Schulz on one matrix in 64 bits (the coefficients are binary32 arguments)."""
    coeffs = [tuple(f32(v) for v in c) for c in coeffs]
    x = u.double()
    x = x / (x.norm() + f32(eps))
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for a, b, c in coeffs:
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _halves(x, scale):
    """(hi, lo) of x in binary16, at the scale that values of its kind have."""
    hi = (x * scale).half().float()
    return hi / scale, (x * scale - hi).half().float() / scale


def _product(a, b, split):
    """Product of two operands in halves, with sums in binary32."""
    p = a[0] @ b[0]
    return p + (a[0] @ b[1] + a[1] @ b[0]) if split else p


def orthogonalize_model(u, coeffs, eps, split):
    """The same in binary32 with operands in one or two halves, rounded where the definition of the precision says."""
    x = u.double()
    x = (x / (x.norm() + f32(eps))).float()
    coeffs = [tuple(f32(v) for v in c) for c in coeffs]
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for a, b, c in coeffs:
        h = _halves(x, 4096.0)
        x = h[0] + h[1]
        s = _product(h, tuple(v.t().contiguous() for v in h), split)
        d = s.diagonal().clone()
        e = _halves(s.fill_diagonal_(0.0), 2048.0)
        q = _product(e, e, split)
        t = e[0] + e[1] if split else e[0]
        p = b * t + c * ((d[:, None] + d[None]) * t + q)
        dp = b * d + c * (d * d + q.diagonal())
        x = (a + dp)[:, None] * x + _product(_halves(p.fill_diagonal_(0.0), 1024.0), h, split)
    return x.t() if tall else x


def orthogonalize_bound(u, coeffs, eps, split, out_bf16, draws=4):
    """How far (2-norm over all elements) a result may be from the exact one.  The error is a sum of very many roundings,
    carried on by the steps that follow, and no useful bound holds for all of them pulling one way.  The model above makes
    roundings of the same sizes in the same places, so its error is drawn from the same distribution: the largest of a few
    draws (inputs moved by 1e-3, which changes every rounding and hardly the matrix), times four.  To that comes the
    rounding of the result, half a step, and for matrices of so few elements other than zero that a draw may happen to be
    exact a floor of eight half steps of binary32 per step, enlarged fourfold by the steps after it.  (One element: x = 1, and
    a + (b x^2 + c x^4) is formed with four roundings of values up to |b| + |c| = 6.8, ten times the sum.)"""
    gen = torch.Generator(device=u.device).manual_seed(11)
    worst = size = 0.0
    for _ in range(draws):
        v = u.double() * (1.0 + 1e-3 * torch.randn(u.shape, generator=gen, device=u.device))
        exact = orthogonalize(v, coeffs, eps)
        worst = max(worst, float((orthogonalize_model(v, coeffs, eps, split).double() - exact).norm()))
        size = max(size, float(exact.norm()))
    floor = 8 * U32 * sum(4.0 ** k for k in range(len(coeffs))) if int((u != 0).sum()) < 64 else 0.0
    return 4.0 * worst + (UB if out_bf16 else U32) * 1.01 * size + floor * size


def orthogonalize_element_bound(u, want, coeffs, eps, split, out_bf16, draws=2):
    """How far every element of a result may be from the exact one (`want`): four times the largest error that an element of the model
    has in a few draws, as in orthogonalize_bound, and half a step of the value itself.  What the norm of a large matrix
    hides, a row's end that was not written for instance, stands out here: elements are about as large as the matrix's norm over the root of
    their number, errors before the last rounding a thousandth of that or less."""
    gen = torch.Generator(device=u.device).manual_seed(12)
    worst = 0.0
    for _ in range(draws):
        v = u.double() * (1.0 + 1e-3 * torch.randn(u.shape, generator=gen, device=u.device))
        worst = max(worst, float((orthogonalize_model(v, coeffs, eps, split).double() - orthogonalize(v, coeffs, eps)).abs().max()))
    return 4.0 * worst + (UB if out_bf16 else U32) * 1.01 * (want.abs() + 4.0 * worst)
