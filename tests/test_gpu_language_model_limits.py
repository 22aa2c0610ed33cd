"""The operators at the two ends of a language model at the ends of their ranges: as many tokens, as large a vocabulary and rows as long as they take."""
import pytest
import torch

import test_gpu_vocab as base
import vocab_reference as ref
from paper_2104_11125_amd import binding
from test_gpu_embed import _tokens
from test_gpu_vocab import BF16, DEV, F32, _context, _within

pytestmark = pytest.mark.gpu
TOKENS, VOCAB, DIM, LISTED = (getattr(binding, f"SCALECOM_{name}_MAX") for name in ("TOKENS", "VOCAB", "DIM", "LISTED"))


@pytest.mark.parametrize("n,vocab,dim", [(TOKENS, 9, 4), (300, VOCAB, 3), (300, 7, DIM), (TOKENS, VOCAB, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_embedding(n, vocab, dim, dtype):
    gen = torch.Generator(device=DEV).manual_seed(n + vocab + dim)
    table, tokens = torch.randn(vocab, dim, generator=gen, device=DEV).to(dtype), _tokens(n, vocab, gen, "zipf")
    tokens[1] = vocab - 1
    ctx = _context()
    out = ctx.scalecom_embed(table, tokens, 0.5)
    want = ref.embed(table, tokens, 0.5)
    _within(out, want, want.abs() * (ref.U32 + ref.step(dtype)) * 1.01 + ref.TINY, "out")
    for accumulate in (False, True):
        grad = ctx.scalecom_embed_grad(tokens, out, table.clone(), 2.0, accumulate).cpu()
        # (on the CPU: many additions to one row)
        want, size, count = ref.embed_grad(tokens.cpu(), out.cpu(), vocab, 2.0, table.cpu() if accumulate else None)
        _within(grad, want, ref.embed_grad_bound(want, size, count, dtype), "grad")


@pytest.mark.parametrize("tokens,vocab,dim", [(TOKENS, 5, 3), (3, VOCAB, 2), (130, 300, DIM), (3, 40, DIM)])
@pytest.mark.parametrize("dtype,dw_dtype", [(F32, F32), (BF16, F32)])
def test_cross_entropy(tokens, vocab, dim, dtype, dw_dtype):
    base.test_cross_entropy(tokens, vocab, dim, dtype, dw_dtype)


@pytest.mark.parametrize("tokens,vocab,dim,entries", [(TOKENS, 5, 3, 3), (TOKENS, 40, 2, 2), (3, VOCAB, 2, LISTED), (130, 300, DIM, 10)])
def test_distillation(tokens, vocab, dim, entries):
    base.test_distill(tokens, vocab, dim, entries, BF16, F32, F32, 2.0)
