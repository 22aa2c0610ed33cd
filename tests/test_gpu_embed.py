"""The embedding and its gradient on the GPU against their plain forms in 64 bits."""
import math

import pytest
import torch

import vocab_reference as ref
from paper_2104_11125_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16


def _context(stream=None):
    return binding.scalecom_init(64, 1, F32, device=DEV, stream=stream, k_max=0)


def _within(got, want, bound, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (what, float(off.max()), int(off.argmax()))


def _tokens(n, vocab, gen, kind):
    if kind == "zipf":                                      # long runs of the first tokens
        t = (torch.rand(n, generator=gen, device=DEV, dtype=torch.float64) * math.log(vocab + 1)).exp() - 1
    elif kind == "one":
        t = torch.full((n,), vocab - 1, device=DEV)
    else:
        t = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    t = t.clamp(max=vocab - 1).to(torch.int32)
    if kind == "zipf":
        t[::9], t[4::11] = -100, vocab
    return t


@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 5, 3), (3, 7, 256), (64, 100, 257), (777, 1000, 64), (5000, 50, 515), (20, 9, 4096)])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_embed(n, vocab, dim, dtype, out_dtype):
    gen = torch.Generator(device=DEV).manual_seed(n + vocab * 5 + dim)
    table = torch.randn(vocab, dim, generator=gen, device=DEV).to(dtype)
    tokens = _tokens(n, vocab, gen, "zipf" if n > 1 else "even")
    for scale in (1.0, 0.3):
        out = _context().scalecom_embed(table, tokens, scale, torch.full((n, dim), 7.0, dtype=out_dtype, device=DEV))
        want = ref.embed(table, tokens, float(torch.tensor(scale, dtype=F32)))
        _within(out, want, want.abs() * (ref.U32 + ref.step(out_dtype)) * 1.01 + ref.TINY, "out")


GRAD_SIZES = [(1, 1, 1, "even"), (2, 3, 5, "one"), (15, 4, 300, "even"), (16, 4, 256, "one"), (17, 40, 64, "zipf"), (33, 1, 100, "one"),
              (1000, 10_000, 12, "even"), (4097, 300, 129, "zipf"), (12_288, 777, 30, "zipf"), (12_289, 511, 8, "zipf"), (12_289, 512, 8, "zipf"),
              (20_000, 5, 260, "even"), (70_001, 50_257, 16, "zipf"), (40_000, 300_000, 4, "even"), (13_000, 1, 1024, "one")]


@pytest.mark.parametrize("n,vocab,dim,kind", GRAD_SIZES)
@pytest.mark.parametrize("dtype,grad_dtype,accumulate", [(F32, F32, False), (BF16, BF16, True), (BF16, F32, True), (F32, BF16, False)])
def test_embed_grad(n, vocab, dim, kind, dtype, grad_dtype, accumulate):
    gen = torch.Generator(device=DEV).manual_seed(n + vocab * 5 + dim)
    tokens = _tokens(n, vocab, gen, kind)
    dout = torch.randn(n, dim, generator=gen, device=DEV).to(dtype)
    scale = float(torch.tensor(1.7, dtype=F32))
    flat = torch.full((vocab * dim + 16,), 7.0, dtype=grad_dtype, device=DEV)
    begin = 8 if dim % 2 else 5                             # (the flat gradient's matrix on round and odd addresses)
    grad = flat[begin:begin + vocab * dim].view(vocab, dim)
    old = None
    if accumulate:
        old = torch.randn(vocab, dim, generator=gen, device=DEV).to(grad_dtype)
        grad.copy_(old)
    _context().scalecom_embed_grad(tokens, dout, grad, scale, accumulate)
    want, size, count = ref.embed_grad(tokens, dout, vocab, scale, old)
    _within(grad, want, ref.embed_grad_bound(want, size, count, grad_dtype), "grad")
    assert bool((flat[:begin] == 7).all()) and bool((flat[begin + vocab * dim:] == 7).all())
    if accumulate:
        assert torch.equal(grad[count[:, 0] == 0], old[count[:, 0] == 0])


@pytest.mark.parametrize("n", [200, 13_000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views_at_any_place(n, dtype):
    gen = torch.Generator(device=DEV).manual_seed(n)
    vocab, dim = 60, 70
    table = torch.randn(vocab, dim + 13, generator=gen, device=DEV).to(dtype)[:, 3:3 + dim]
    tokens = _tokens(n, vocab, gen, "zipf")
    out = torch.full((n, dim + 5), 7.0, dtype=dtype, device=DEV)
    ctx = _context()
    ctx.scalecom_embed(table, tokens, 1.0, out[:, 1:1 + dim])
    assert torch.equal(out[:, 1:1 + dim].double(), ref.embed(table, tokens, 1.0))
    assert bool((out[:, 0] == 7).all()) and bool((out[:, 1 + dim:] == 7).all())
    dout = torch.randn(n, dim + 9, generator=gen, device=DEV).to(dtype)[:, 5:5 + dim]
    grad = torch.full((vocab, dim + 3), 7.0, dtype=dtype, device=DEV)
    ctx.scalecom_embed_grad(tokens, dout, grad[:, 2:2 + dim])
    want, size, count = ref.embed_grad(tokens, dout, vocab, 1.0)
    _within(grad[:, 2:2 + dim], want, ref.embed_grad_bound(want, size, count, dtype), "grad")
    assert bool((grad[:, :2] == 7).all()) and bool((grad[:, 2 + dim:] == 7).all())


def test_padding_and_nothing():
    """Rows of tokens that are none reach no gradient, whatever they hold; no tokens at all."""
    ctx = _context()
    table = torch.randn(6, 10, device=DEV)
    tokens = torch.tensor([2, -1, 6, 2, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    dout = torch.full((6, 10), math.nan, device=DEV)
    dout[0], dout[3] = 1.0, 2.0
    grad = ctx.scalecom_embed_grad(tokens, dout, torch.full((6, 10), 7.0, device=DEV))
    want = torch.zeros(6, 10, device=DEV)
    want[2] = 3.0
    assert torch.equal(grad, want)
    out = ctx.scalecom_embed(table, tokens, 2.0)
    assert torch.equal(out[0], 2 * table[2]) and bool((out[[1, 2, 4, 5]] == 0).all())
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    assert ctx.scalecom_embed(table, none).shape == (0, 10)
    grad.fill_(7.0)
    ctx.scalecom_embed_grad(none, torch.empty(0, 10, device=DEV), grad, accumulate=True)
    assert bool((grad == 7).all())
    ctx.scalecom_embed_grad(none, torch.empty(0, 10, device=DEV), grad)
    assert bool((grad == 0).all())


def test_a_nan_stays_in_its_row():
    tokens = torch.arange(40, dtype=torch.int32, device=DEV).repeat(3)
    dout = torch.ones(120, 33, device=DEV)
    dout[7, 5] = math.nan
    grad = _context().scalecom_embed_grad(tokens, dout, torch.empty(40, 33, device=DEV))
    bad = torch.zeros(40, 33, dtype=torch.bool, device=DEV)
    bad[7, 5] = True
    assert torch.equal(torch.isnan(grad), bad) and bool((grad[~bad] == 3).all())


@pytest.mark.parametrize("n", [3000, 30_000])
def test_results_do_not_vary(n):
    gen = torch.Generator(device=DEV).manual_seed(n)
    tokens, dout = _tokens(n, 500, gen, "zipf"), torch.randn(n, 100, generator=gen, device=DEV)
    ctx = _context()
    runs = [ctx.scalecom_embed_grad(tokens, dout, torch.empty(500, 100, device=DEV), 0.7) for _ in range(4)]
    assert all(torch.equal(runs[0], r) for r in runs[1:])


def test_far_rows():
    """A table and a gradient whose offsets pass 2^32 bytes and 2^31 elements."""
    vocab, dim = 1_100_000, 2048
    table = torch.zeros(vocab, dim, dtype=BF16, device=DEV)
    tokens = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], dtype=torch.int32, device=DEV)
    table[vocab - 1], table[0], table[vocab - 2] = 3.0, 1.0, 2.0
    ctx = _context()
    out = ctx.scalecom_embed(table, tokens)
    assert out[:, 0].tolist() == [3.0, 1.0, 2.0, 3.0] and torch.equal(out, out[:, :1].expand_as(out))
    ctx.scalecom_embed_grad(tokens, out, table)
    assert bool((table[vocab - 1] == 6).all()) and bool((table[0] == 1).all()) and bool((table[vocab - 2] == 2).all())
    assert float(table[1:vocab - 2].abs().amax()) == 0.0
