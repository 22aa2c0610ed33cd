"""Ways through the embedding's gradient that a rule on the sizes takes, against the plain form in 64 bits (on the CPU: many additions to one row)."""
import pytest
import torch

import vocab_reference as ref
from test_gpu_embed import BF16, DEV, F32, _context, _tokens, _within

pytestmark = pytest.mark.gpu
KINDS = [(F32, F32, False), (BF16, BF16, True), (BF16, F32, True), (F32, BF16, False)]


def _check(n, vocab, dim, kind, dtype, grad_dtype, accumulate):
    gen = torch.Generator(device=DEV).manual_seed(n + vocab * 5 + dim)
    tokens = _tokens(n, vocab, gen, kind)
    dout = torch.randn(n, dim, generator=gen, device=DEV).to(dtype)
    scale = float(torch.tensor(1.7, dtype=F32))
    old = torch.randn(vocab, dim, generator=gen, device=DEV).to(grad_dtype)
    grad = _context().scalecom_embed_grad(tokens, dout, old.clone(), scale, accumulate)
    want, size, count = ref.embed_grad(tokens.cpu(), dout.cpu(), vocab, scale, old.cpu() if accumulate else None)
    _within(grad.cpu(), want, ref.embed_grad_bound(want, size, count, grad_dtype), "grad")


# One block sorts: one row of positions a wave up to 1024, four up to 4096; one, two and three digits of the token
@pytest.mark.parametrize("n", [1023, 1024, 1025, 2047, 2048, 2049, 3000, 3100, 4095, 4096])
@pytest.mark.parametrize("vocab,dim,kind", [(500, 30, "zipf"), (20_000, 12, "even"), (300_000, 3, "zipf"), (700, 513, "one")])
@pytest.mark.parametrize("dtype,grad_dtype,accumulate", [KINDS[0], KINDS[2]])
def test_positions_that_one_block_sorts(n, vocab, dim, kind, dtype, grad_dtype, accumulate):
    _check(n, vocab, dim, kind, dtype, grad_dtype, accumulate)


# 8192 batches of 16 positions times chunks of 512 columns: a wave sums two batches one behind the other.  Runs end in either batch, cross both, cross
# tiles; the last tile has 18 positions (a batch and two), 2, 16 and all 32
@pytest.mark.parametrize("n,vocab,dim", [(131_090, 40_000, 5), (131_090, 700, 8), (44_002, 3000, 1030), (131_088, 3, 16), (131_104, 131_000, 4)])
@pytest.mark.parametrize("kind", ["zipf", "one", "even"])
@pytest.mark.parametrize("dtype,grad_dtype,accumulate", KINDS)
def test_two_batches_a_wave(n, vocab, dim, kind, dtype, grad_dtype, accumulate):
    assert -(-n // 16) * -(-dim // 512) >= 8192
    _check(n, vocab, dim, kind, dtype, grad_dtype, accumulate)
