"""How many bits the losses over a vocabulary and their gradients keep on the GPU, in the 2-norm over inputs that show every product of planes."""
import pytest
import torch

import vocab_precision as precision
from paper_2104_11125_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16
U32, UB = 2.0 ** -24, 2.0 ** -8
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
    got = {"lse": lse, "dx": dx, "dw": dw}
    # (of 20000 tokens lse is of size 8 to 16, a step twice as large)
    limit = precision.limit(peaked) * (2 if vocab > 10_000 else 1)
    for name, value in got.items():
        alone = {name: want[name]}
        off, most = (precision.off({name: value}, alone), limit) if value.dtype is F32 else (precision.off_rounded({name: value}, alone), precision.ROUNDED)
        print(off)
        assert off[name] <= most, (off, most)


@pytest.mark.parametrize("tokens,vocab,dim", [(1, 3, 64), (1, 100, 128), (2, 100, 40), (5, 60, 96), (300, 70, 128)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("entries", [0, 4])
def test_one_rounding_of_gradients(tokens, vocab, dim, dtype, entries):
    """Gradients in bfloat16 are rounded once, of few tokens too and where every token's loss counts the same, so that roundings of dz would all be alike."""
    gen = torch.Generator(device=DEV).manual_seed(tokens + vocab + dim)
    w = (torch.randn(vocab, dim, generator=gen, device=DEV) * 0.1).to(dtype)
    x = torch.randn(tokens, dim, generator=gen, device=DEV).to(dtype)
    dloss = torch.full((tokens,), 1 / 7.0, device=DEV)
    ctx = _context()
    z = x.double() @ w.double().t()
    dz = torch.softmax(z, 1)
    dw = torch.empty(vocab, dim, dtype=BF16, device=DEV)
    if entries:
        ids = torch.stack([torch.randperm(vocab, generator=gen, device=DEV)[:min(entries, vocab)] for _ in range(tokens)]).to(torch.int32)
        teacher = torch.randn(ids.shape, generator=gen, device=DEV)
        _, lse, listed = ctx.scalecom_distill(x, w, ids, teacher)
        dx, dw = ctx.scalecom_distill_grad(x, w, ids, teacher, 1.0, lse, listed, dloss, True, dw)
        dz = dz.scatter_add(1, ids.long(), -torch.softmax(teacher.double(), 1))
    else:
        targets = torch.randint(0, vocab, (tokens,), generator=gen, device=DEV, dtype=torch.int32)
        loss, lse = ctx.scalecom_cross_entropy(x, w, targets)
        dx, dw = ctx.scalecom_cross_entropy_grad(x, w, targets, loss, lse, dloss, True, dw)
        dz[torch.arange(tokens, device=DEV), targets.long()] -= 1
    dz = dz * float(dloss[0])
    # dz: half a step of its second plane, 2^-16; a probability's logit and lse, each off by twice their roundings, 2 dim of 2^-24 of terms that add up to less than
    # 0.08 dim (3e-4 for 128 places).  Sums: twice as many roundings as terms, of six products at most; the result: half a step
    error = 2.0 ** -16 + 4 * dim * U32 * 0.08 * dim
    for got, value, size, inner in ((dx, dz @ w.double(), dz.abs() @ w.double().abs(), vocab), (dw, dz.t() @ x.double(), dz.abs().t() @ x.double().abs(), tokens)):
        off = (got.double() - value).abs() - (error + (12 * inner + 64) * U32) * size - (UB if got.dtype is BF16 else U32) * value.abs() * 1.01
        assert bool((off <= 0).all()), (float(off.max()), float((got.double() - value).norm() / value.norm()))


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
