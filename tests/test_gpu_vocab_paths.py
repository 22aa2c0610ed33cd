"""Ways through the losses over a vocabulary that a rule on the sizes takes, each against the plain form in 64 bits."""
import pytest
import torch

from test_gpu_vocab import BF16, DEV, F32, _check_entropy, _context, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,vocab,dim", [(11_000, 17_000, 40),     # three pieces of 5888 rows
                                              (44_000, 5000, 8)])       # three of 1792
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_tokens_in_small_pieces(tokens, vocab, dim, dtype):
    """Of so many tokens dz in three planes is held for fewer rows of the vocabulary than few tokens' is."""
    x, w, targets, dloss, gen = _inputs(tokens, vocab, dim, dtype)
    old = torch.randn(vocab, dim, generator=gen, device=DEV) * 0.1
    _check_entropy(_context(), x, w, targets, dloss, F32, old)


def test_a_loss_keeps_the_scratch_of_a_loss():
    """The context's own scratch after a loss of a few tokens over a large vocabulary is small; the gradient's larger one then serves both."""
    x, w, targets, dloss, _ = _inputs(8, 131_072, 128, BF16)
    ctx = _context()
    loss, lse = ctx.scalecom_cross_entropy(x, w, targets)
    ids = torch.arange(24, dtype=torch.int32, device=DEV).view(8, 3)
    ctx.scalecom_distill(x, w, ids, ids.float(), 2.0)
    small = ctx._ortho_scratch[-1].numel()
    ctx.scalecom_cross_entropy_grad(x, w, targets, loss, lse, dloss)
    large = ctx._ortho_scratch[-1].numel()
    again = ctx.scalecom_cross_entropy(x, w, targets)
    assert small < 8 << 20 < large and len(ctx._ortho_scratch) == 1 and ctx._ortho_scratch[-1].numel() == large
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
