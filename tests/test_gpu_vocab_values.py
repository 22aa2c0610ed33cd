"""Values at the ends of their ranges in the losses over a vocabulary on the GPU: infinite logits, teachers' logits that a small temperature
would carry out of range."""
import math

import pytest
import torch

import vocab_reference as ref
from paper_2104_11125_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16


def _context():
    return binding.scalecom_init(64, 1, F32, device=DEV, k_max=0)


def _within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (what, float(off.max()), int(off.argmax()))


def _inputs(tokens, vocab, dim, dtype, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(tokens + vocab * 3 + dim * 5 + seed)
    w = (torch.randn(vocab, dim, generator=gen, device=DEV) * 0.2).to(dtype)
    x = torch.randn(tokens, dim, generator=gen, device=DEV).to(dtype)
    targets = torch.randint(0, vocab, (tokens,), generator=gen, device=DEV, dtype=torch.int32)
    return x, w, targets, torch.rand(tokens, generator=gen, device=DEV) + 0.1, gen


# A logit's roundings are at most twice its 64 terms' (which add up to less than 16 in size), 1.2e-4; the exponentials and the sum of 300 add 1e-5.
NEAR = 2e-4


@pytest.mark.parametrize("tokens", [3, 90])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_an_infinite_logit_at_the_target(dtype, tokens):
    """Infinity less infinity: no loss, not a perfect one.  Token 1's logit is infinite at its target only; the others' is minus infinity there, a
    probability of zero (in binary32 an infinite element may make it NaN)."""
    x, w, targets, dloss, _ = _inputs(tokens, 300, 64, dtype)
    targets[targets == 4] = 5
    x[:, 7], w[4, 7] = -1.0, math.inf
    x[1, 7], targets[1] = 1.0, 4
    ctx = _context()
    loss, lse = ctx.scalecom_cross_entropy(x, w, targets)
    assert math.isnan(float(loss[1])) and float(lse[1]) == math.inf
    if dtype is BF16:
        z = x.double() @ w.double().t()
        others = torch.arange(tokens, device=DEV) != 1
        want = torch.logsumexp(z, 1)
        assert bool(((lse - want).abs() <= NEAR)[others].all())
        assert bool(((loss - (want - z.gather(1, targets.long()[:, None])[:, 0])).abs() <= NEAR)[others].all())
    dx, dw = ctx.scalecom_cross_entropy_grad(x, w, targets, loss, lse, dloss)
    assert not bool(torch.isfinite(dx[1]).any()) and not bool(torch.isfinite(dw[4]).any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_token_in_the_vocabulary(dtype):
    """No other token shares the probability, so nothing but the target's own logit says that it is infinite."""
    x, w, targets, dloss, _ = _inputs(5, 1, 8, dtype)
    x[2, 3], w[0, 3] = math.inf, 0.5
    x[4, 0], w[0, 0] = 2e38, 64.0                           # finite, but not the product
    ctx = _context()
    loss, lse = ctx.scalecom_cross_entropy(x, w, targets)
    assert torch.isnan(loss).tolist() == [False, False, True, False, True] and bool((loss[[0, 1, 3]] == 0).all())
    dx, dw = ctx.scalecom_cross_entropy_grad(x, w, targets, loss, lse, dloss)
    assert torch.isnan(dx).all(1).tolist() == [False, False, True, False, True] and bool((dx[[0, 1, 3]] == 0).all())
    assert bool(torch.isnan(dw).all())


def test_a_target_that_cannot_be():
    """A logit of minus infinity at the target: an infinite loss; elsewhere a probability of zero."""
    x, w, targets, _, _ = _inputs(20, 100, 64, BF16)
    x[:, 5], w[7, 5] = 1.0, -math.inf
    targets[targets == 7] = 8
    targets[3] = 7
    loss, lse = _context().scalecom_cross_entropy(x, w, targets)
    want = torch.logsumexp(x.double() @ w.double().t(), 1)
    assert float(loss[3]) == math.inf and int(torch.isinf(loss).sum()) == 1 and bool(((lse - want).abs() <= NEAR).all())


@pytest.mark.parametrize("temperature", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("teacher_dtype", [F32, BF16])
def test_teachers_logits_near_the_ends_of_their_range(teacher_dtype, temperature):
    """What the temperature makes of the differences counts, also where it carries the logits themselves out of range: a list of lowest values is an even
    distribution, not an empty list, and one largest value has all of the probability."""
    tokens, vocab, dim, entries = 40, 90, 64, 6
    x, w, _, dloss, gen = _inputs(tokens, vocab, dim, F32)
    ids = torch.stack([torch.randperm(vocab, generator=gen, device=DEV)[:entries] for _ in range(tokens)]).to(torch.int32)
    teacher = (torch.randn(tokens, entries, generator=gen, device=DEV) * 2.0).to(teacher_dtype)
    lowest, largest = torch.finfo(teacher_dtype).min, torch.finfo(teacher_dtype).max
    teacher[0::4] = lowest
    teacher[1::4, 2:] = lowest
    teacher[2::4, 3] = largest
    teacher[2::8, 4] = -math.inf
    teacher[4, 1:], ids[8, 0] = -math.inf, -1
    want = ref.distill(x, w, ids, teacher, temperature)
    ctx = _context()
    loss, lse, listed = ctx.scalecom_distill(x, w, ids, teacher, temperature)
    _within(loss, want.loss, want.e_loss, "loss")
    _within(lse, want.lse, want.e_lse, "lse")
    wdx, bdx, wdw, bdw = want.gradients(dloss, F32, F32)
    dx, dw = ctx.scalecom_distill_grad(x, w, ids, teacher, temperature, lse, listed, dloss)
    _within(dx, wdx, bdx, "dx")
    _within(dw, wdw, bdw, "dw")
    # infinite and NaN logits of a teacher are no distribution; none above -infinity is no list
    teacher[3, 0], teacher[7, 5], teacher[11] = math.inf, math.nan, -math.inf
    again = ctx.scalecom_distill(x, w, ids, teacher, temperature)[0]
    odd = torch.zeros(tokens, dtype=torch.bool, device=DEV)
    odd[3] = odd[7] = True
    assert torch.equal(torch.isnan(again), odd) and float(again[11]) == 0.0
    odd[11] = True
    assert torch.equal(again[~odd], loss[~odd])
