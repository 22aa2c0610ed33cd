"""Ways through the losses over a vocabulary that a rule on the sizes takes, each against the plain form in 64 bits."""
import pytest
import torch

import test_gpu_vocab as base
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


@pytest.mark.parametrize("tokens,vocab,dim", [(70_001, 700, 512), (70_001, 600, 1023)])
@pytest.mark.parametrize("dtype,dw_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_blocks_that_share_large_tiles_of_dw(tokens, vocab, dim, dtype, dw_dtype):
    """So many tokens that tiles of 256 pay off for a gradient of few rows: 21 to 42 blocks share their inner dimension."""
    base.test_cross_entropy(tokens, vocab, dim, dtype, dw_dtype)


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


# Which tiles and pieces the rules choose for an output matrix of bfloat16 that is read as it lies (seen in a trace; a change of the rules asks for other
# sizes here), and how many blocks share dx's inner dimension
@pytest.mark.parametrize("tokens,vocab,dim", [(20_000, 20_001, 1408),   # 256 throughout, three pieces; 1
                                              (1100, 33_001, 1408),     # 256 throughout, one piece, a part of a tile at every end; 8
                                              (520, 132_001, 640),      # logits and dx 256, dw 128, half a tile of columns (a binary32 dw: two pieces); 28
                                              (300, 262_274, 128),      # logits 256, dx and dw 128, two pieces; 170
                                              (200, 9001, 384)])        # 128 throughout
@pytest.mark.parametrize("dw_dtype", [BF16, F32])
def test_an_output_matrix_as_it_lies(tokens, vocab, dim, dw_dtype):
    """Rows of a wider matrix, with NaN behind their ends; the gradient's too, where nothing else is written."""
    x, w, targets, dloss, gen = _inputs(tokens, vocab, dim, BF16)
    wide = torch.full((vocab, dim + 16), float("nan"), dtype=BF16, device=DEV)
    wide[:, 8:8 + dim] = w
    into = torch.full((vocab, dim + 9), 5.0, dtype=dw_dtype, device=DEV)
    old = None
    if vocab % 2:
        old = (torch.randn(vocab, dim, generator=gen, device=DEV) * 0.1).to(dw_dtype)
        into[:, 4:4 + dim] = old
    _check_entropy(_context(), x, wide[:, 8:8 + dim], targets, dloss, dw_dtype, old, True, into[:, 4:4 + dim])
    assert bool((into[:, :4] == 5).all()) and bool((into[:, 4 + dim:] == 5).all())


# Planes of the output matrix, two pieces, logits and dx in tiles of 256: dw too, by way of the scratch (dim is no multiple of four); dw in 128
@pytest.mark.parametrize("tokens,vocab,dim", [(1100, 33_001, 1407), (300, 262_274, 128)])
@pytest.mark.parametrize("dtype,dw_dtype", [(F32, F32), (F32, BF16)])
def test_planes_of_the_output_matrix(tokens, vocab, dim, dtype, dw_dtype):
    base.test_cross_entropy(tokens, vocab, dim, dtype, dw_dtype)


@pytest.mark.parametrize("tokens,vocab,dim,entries", [(1100, 33_001, 1408, 33), (20_000, 20_001, 1408, 8), (300, 262_274, 128, 100)])
@pytest.mark.parametrize("dw_dtype,temperature", [(BF16, 1.0), (F32, 2.0)])
def test_distillation(tokens, vocab, dim, entries, dw_dtype, temperature):
    base.test_distill(tokens, vocab, dim, entries, BF16, dw_dtype, F32, temperature)
