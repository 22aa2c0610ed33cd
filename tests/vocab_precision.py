"""How many bits the losses over a vocabulary keep: inputs, in binary32, that show every product of their operands' planes, a model of the library's
arithmetic from which products can be left out, and how far results may be from the exact ones in the 2-norm.

An operand is hi + mid + lo, three bfloat16 numbers, and a product of two the six products of planes that are not below 2^-24 of it.  Every element
here is plus or minus a power of two times 1 + 179 2^-16 + 51 2^-23: hi is the power of two, mid 2.7e-3 and lo 6.1e-6 of it, all of one sign, so
without one product of planes a product of such elements, and a sum of them, is 6.1e-6 (hi lo) or 7.5e-6 (mid mid) too small, and one
with values of any other bits (dz) off by some 2e-6 to 6e-6 in the 2-norm.

Intact, logits of size up to 8 are summed in five steps of 32 places, so five roundings of at most 2^-22, half a step, 1.2e-6 in all; lse, of size 4 to
8, is rounded once more, and the exponential's argument.  Most logits are smaller, and roundings differ in sign, so that in the 2-norm errors are well below it.
  flat:   no token has much of the probability: FLAT is those five roundings
  peaked: a token that is not the target has most of it, so an error of its logit, of size 7, is one of dz in full: PEAKED is three times as much (the
          matrix units' inner sums, which may truncate; lse and the exponential)
"""
import torch

TOKENS, VOCAB, DIM = 160, 600, 160
FLAT, PEAKED = 1.2e-6, 3.6e-6
# A gradient in bfloat16 is the rounded exact one but where that lies next to the middle of two numbers: dz has 16 bits, so sums are off by some 1e-5, and of
# elements a step of 5.5e-3 apart four in a thousand go the other way, 3.5e-4 of the 2-norm; twice that.  dz rounded to bfloat16 makes it 1.6e-3.
ROUNDED = 7e-4
ALL = [(2, 0), (0, 2), (1, 1), (0, 1), (1, 0), (0, 0)]      # planes of the two operands, the smallest products first


def shaped(v):
    """Signs and powers of two of v, mantissas as above."""
    return torch.sign(v) * torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=1e-3)))) * (1 + 179 * 2.0 ** -16 + 51 * 2.0 ** -23)


def inputs(peaked, tokens=TOKENS, vocab=VOCAB, device="cpu"):
    gen = torch.Generator().manual_seed(11 + peaked)
    w = shaped(torch.randn(vocab, DIM, generator=gen))
    x = torch.randn(tokens, DIM, generator=gen)
    targets = torch.randint(0, vocab, (tokens,), generator=gen, dtype=torch.int32)
    if peaked:                                              # (the signs of a row of w: what they add to its logit is all of one sign)
        other = (targets.long() + 1 + torch.randint(0, vocab - 1, (tokens,), generator=gen)) % vocab
        x = x * 0.5 + 1.5 * torch.sign(w[other])
    x = shaped(x) * (0.0625 if peaked else 0.125)
    dloss = torch.rand(tokens, generator=gen) + 0.5
    return tuple(t.to(device) for t in (x, w, targets, dloss))


def exact(x, w, targets, dloss):
    """lse, dx and dw in 64 bits."""
    z = x.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    dz = (z - lse[:, None]).exp()
    dz[torch.arange(len(x), device=x.device), targets.long()] -= 1
    dz *= dloss.double()[:, None]
    return {"lse": lse, "dx": dz @ w.double(), "dw": dz.t().contiguous() @ x.double()}


def planes(v):
    hi = v.bfloat16().float()
    mid = (v - hi).bfloat16().float()
    return hi, mid, (v - hi - mid).bfloat16().float()


def product(a, b, pairs):
    """a b^T in binary32 from the pairs of planes."""
    a, b = planes(a), planes(b)
    total = torch.zeros(len(a[0]), len(b[0]))
    for i, j in pairs:
        for k in range(0, a[0].shape[1], 32):
            total += a[i][:, k:k + 32] @ b[j][:, k:k + 32].t()
    return total


def model(x, w, targets, dloss, sums=ALL, dz_logits=ALL, dx=ALL, dw=ALL):
    """The library's arithmetic with the plane products that are given; pairs are (w, x), (w, dz) and (x, dz)."""
    lse = torch.logsumexp(product(w, x, sums).t(), 1)
    dz = (product(w, x, dz_logits).t() - lse[:, None]).exp()
    at = torch.arange(len(x)), targets.long()
    z = (x.double() @ w.double().t())[at].float()
    dz[at] = torch.expm1(z - lse)
    dz *= dloss[:, None]
    return {"lse": lse, "dx": product(w.t(), dz, dx).t(), "dw": product(x.t(), dz.t(), dw).t()}


def off(got, want):
    """Errors: of lse the root of the mean square, of the gradients relative in the 2-norm."""
    rms = lambda v: float(v.double().pow(2).mean().sqrt())
    return {k: rms(got[k].double() - want[k]) / (1.0 if k == "lse" else rms(want[k])) for k in want}


def off_rounded(got, want):
    """How far bfloat16 results are from the rounded exact ones, relative in the 2-norm."""
    return {k: float((got[k].double() - v.bfloat16().double()).norm() / v.norm()) for k, v in want.items()}


def limit(peaked):
    return PEAKED if peaked else FLAT
