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
