"""How many bits the losses over a vocabulary and their gradients keep on the GPU, in the 2-norm over inputs that show every product of planes."""
import pytest
import torch

import vocab_precision as precision
from paper_2104_11125_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16
# tiles of 128 x 64, 128 x 128, 256 x 256 for the logits
SIZES = [(60, precision.VOCAB), (precision.TOKENS, precision.VOCAB), (600, 20_000)]


def _context():
    return binding.scalecom_init(64, 1, F32, device=DEV, k_max=0)


@pytest.mark.parametrize("tokens,vocab", SIZES)
@pytest.mark.parametrize("peaked", [False, True])
@pytest.mark.parametrize("dtype,dw_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_cross_entropy(tokens, vocab, peaked, dtype, dw_dtype):
    x, w, targets, dloss = precision.inputs(peaked, tokens, vocab, DEV)
    x, w = x.to(dtype), w.to(dtype)
    want = precision.exact(x, w, targets, dloss)
    ctx = _context()
    loss, lse = ctx.scalecom_cross_entropy(x, w, targets)
    dx, dw = ctx.scalecom_cross_entropy_grad(x, w, targets, loss, lse, dloss, True, torch.empty(w.shape, dtype=dw_dtype, device=DEV))
    got = precision.off({"lse": lse, "dx": dx, "dw": dw}, want)
    # (of 20000 tokens lse is of size 8 to 16, a step twice as large)
    limit = precision.limit(peaked) * (2 if vocab > 10_000 else 1)
    limits = {"lse": limit, "dx": limit if dtype is F32 else precision.HALVES, "dw": limit if dw_dtype is F32 else precision.HALVES}
    print(got)
    assert all(got[k] <= limits[k] for k in got), (got, limits)


@pytest.mark.parametrize("tokens,vocab", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_listed_logits(tokens, vocab, dtype):
    x, w, _, _ = precision.inputs(False, tokens, vocab, DEV)
    x, w = x.to(dtype), w.to(dtype)
    ids = torch.randint(0, vocab, (tokens, 20), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=torch.int32)
    _, lse, listed = _context().scalecom_distill(x, w, ids, torch.zeros(tokens, 20, device=DEV))
    z = x.double() @ w.double().t()
    got = precision.off({"lse": lse, "listed": listed}, {"lse": torch.logsumexp(z, 1), "listed": z.gather(1, ids.long())})
    print(got)
    assert got["listed"] <= precision.FLAT and got["lse"] <= precision.FLAT * (2 if vocab > 10_000 else 1), got
