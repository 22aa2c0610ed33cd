"""Plain 64-bit forms of the embedding and of the losses over a vocabulary, and how far the library may be from them.

The bounds count roundings: a rounding to nearest is off by at most half a step, eps / 2 relative (binary32 2^-24,
bfloat16 2^-8).  A sum of m terms in binary32, in any order, is off by at most m roundings of the sum of its terms' sizes; twice that where the
matrix units add, whose inner additions may truncate.
"""
import math

import torch

U32, UB = 2.0 ** -24, 2.0 ** -8
TINY = 1e-37                    # what is lost where values leave binary32's normal range


def step(dtype):
    return U32 if dtype is torch.float32 else UB


def embed(table, tokens, scale):
    there = (tokens >= 0) & (tokens < table.shape[0])
    rows = table.double()[tokens.long().clamp(0, table.shape[0] - 1)] * scale
    return torch.where(there[:, None], rows, 0.0)


def embed_grad(tokens, dout, vocab, scale, old=None):
    """(gradient, sum of the sizes of its terms, number of terms of every row)"""
    there = (tokens >= 0) & (tokens < vocab)
    at, rows = tokens[there].long(), dout[there].double() * scale
    grad = torch.zeros(vocab, dout.shape[1], dtype=torch.float64, device=dout.device).index_add_(0, at, rows)
    size = torch.zeros_like(grad).index_add_(0, at, rows.abs())
    count = torch.zeros(vocab, dtype=torch.float64, device=dout.device).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    return (grad if old is None else grad + old.double()), size, count[:, None]


def embed_grad_bound(grad, size, count, dtype):
    # the sum, its product with the scale, the addition to what was there, the rounding to the gradient's type
    return (count + 1) * U32 * size + (U32 + step(dtype)) * grad.abs() * 1.01 + TINY


class Loss:
    """A loss over the vocabulary in 64 bits with bounds: x, w, and a target distribution (tokens x vocabulary, rows of zeros for
    tokens that take no part) in 64 bits; `entropy`: sum of q log q over the entries of every row; `exact_target`: the library forms
    the loss of the target from the others' share."""

    def __init__(self, x, w, target, rows, entropy, temperature, entries):
        self.rows, self.t = rows, temperature
        x = torch.where(rows[:, None], x.double(), 0.0)
        self.x, self.w, self.target = x, w.double(), target
        bf16 = w.dtype is torch.bfloat16
        self.terms = 1 if bf16 else 6                       # products a pair of operands
        z = x @ self.w.t() / temperature
        size = x.abs() @ self.w.abs().t() / temperature
        dim, vocab = w.shape[1], w.shape[0]
        # a logit: its sum, the product with 1 / temperature (itself rounded), what planes drop (2^-23 of a term at most,
        # two of the twelve roundings a place that are counted); the matrix units' inner dimension is padded with zeros, which cost nothing
        e_z = (2 * self.terms * dim + 4) * U32 * size
        self.lse = torch.logsumexp(z, 1)
        logp = z - self.lse[:, None]
        self.p = logp.exp()
        spread = (z.amax(1) - z.amin(1)).clamp(max=100.0) if vocab > 1 else torch.zeros_like(self.lse)
        # exp(a): the product with log2 e is off by |a| 2^-24, doubled, the function by two steps; sums: 32 of a lane, two
        # exchanges, the parts of the vocabulary (64 at least in each) in turn by 16 waves; the logarithm
        exp_steps = 2 * spread + 4
        sum_steps = 32 + 2 + vocab / 64 / 16 + 1 + 16 + 4
        e_top = (e_z * self.p).sum(1) + e_z.amax(1) * 1e-3  # how the logits' errors move lse: by their mean under p, to first order
        self.e_lse = 1.1 * e_top + U32 * (exp_steps + sum_steps + 4 * self.lse.abs() + 8)
        e_target = (e_z * target).sum(1) / target.sum(1).clamp(min=1e-300)
        self.loss = torch.where(rows, (entropy - (target * logp).sum(1)) * temperature ** 2, 0.0)
        of_terms = (target * logp.abs()).sum(1) + (entropy.abs() if torch.is_tensor(entropy) else 0.0)
        # (q: an exponential, a quotient, its logarithm; sums over the list)
        self.e_loss = torch.where(rows, (self.e_lse + e_target + U32 * (entries + 24) * (of_terms + self.lse.abs() + (target * z).sum(1).abs() + 1.0)
                                         ) * temperature ** 2 * 1.01, 0.0)
        self.e_lse = torch.where(rows, self.e_lse, 0.0)
        self.lse = torch.where(rows, self.lse, 0.0)
        # of a probability: relative
        self.e_p = self.p * (e_z + self.e_lse[:, None] + U32 * (2 * logp.abs().clamp(max=200.0) + 6)) * 1.05 + TINY
        self.listed, self.e_listed = z, e_z + U32 * z.abs()
        self.entries = entries

    def gradients(self, dloss, dx_dtype, dw_dtype, old=None):
        """(dx, its bound, dw, its bound)"""
        c = torch.where(self.rows, dloss.double() * self.t, 0.0)[:, None]
        dz = c * (self.p - self.target)
        # q: an exponential and a quotient, sums over the list
        e = c.abs() * (self.e_p + U32 * (self.entries + 24) * self.target) + 3 * U32 * dz.abs()
        x, w, tokens, vocab = self.x, self.w, len(self.x), len(self.w)

        def product(a, e_a, b, planes, dtype, was):
            # `a` rounded to planes of 8 bits: half a step of the last one's
            rounded = e_a + a.abs() * {1: UB, 2: 2.0 ** -16, 3: 2.0 ** -23}[planes]
            value, inner = a @ b, a.shape[1]
            bound = rounded @ b.abs() + (2 * self.terms * (3 if one and planes == 3 else 1) * inner + 64) * U32 * ((a.abs() + rounded) @ b.abs())
            if was is not None:
                value = value + was.double()
            return value, bound * 1.01 + (U32 + step(dtype)) * value.abs() * 1.01 + TINY

        one = self.terms == 1
        dx, e_dx = product(dz, e, w, 1 if one else 3, dx_dtype, None)
        planes = (1 if one else 2) if dw_dtype is torch.bfloat16 else 3
        dw, e_dw = product(dz.t().contiguous(), e.t().contiguous(), x, planes, dw_dtype, old)
        if dw_dtype is torch.bfloat16 and not one:          # (three of the six products: what is dropped is 2^-15 of a term)
            e_dw = e_dw + 2.0 ** -15 * (dz.abs().t() @ x.abs())
        return dx, e_dx, dw, e_dw


def cross_entropy(x, w, targets):
    rows = (targets >= 0) & (targets < w.shape[0])
    target = torch.zeros(len(x), len(w), dtype=torch.float64, device=x.device)
    target[rows, targets[rows].long()] = 1.0
    return Loss(x, w, target, rows, 0.0, 1.0, 1)


def distill(x, w, ids, teacher, temperature):
    there = (ids >= 0) & (ids < w.shape[0])
    u = torch.where(there, teacher.double() / temperature, -math.inf)
    rows = u.amax(1) > -math.inf
    q = torch.where(rows[:, None], torch.softmax(u, 1), 0.0)
    target = torch.zeros(len(x), len(w) + 1, dtype=torch.float64, device=x.device)
    target.scatter_add_(1, torch.where(there, ids, len(w)).long(), q)
    return Loss(x, w, target[:, :-1].contiguous(), rows, torch.special.xlogy(q, q).sum(1), temperature, ids.shape[1])
