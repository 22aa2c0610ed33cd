"""The operators at the two ends of a language model as they are used: a tied matrix's gradient in learners' flat gradients, which
are compressed and applied; captured and replayed; on streams of their own; and what they refuse."""
import math

import numpy as np
import pytest
import torch

import oracle
import vocab_reference as ref
from gpu_util import compare_step, to_host
from paper_2104_11125_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16


def _context(numel=64, learners=1, dtype=F32, tensors=1, stream=None, k_max=0):
    return binding.scalecom_init(numel, learners, dtype, tensors, DEV, stream, k_max=k_max)


def _within(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (what, float(off.max()), int(off.argmax()))


def test_training_step_with_one_matrix_for_both_ends():
    """Predicting the next token from the last one, one matrix for both ends, three learners, two steps: the gradient of every learner against
    the formulas in 64 bits, the compression against the oracle, the weights."""
    vocab, dim, tokens, learners, scale = 300, 40, 150, 3, 6.0
    gen = torch.Generator(device=DEV).manual_seed(5)
    before, after = 3, 11                               # the matrix lies between other tensors of the flat vector
    numel = before + vocab * dim + after
    offsets, ks = [0, before, before + vocab * dim, numel], [1, vocab * dim // 50, 2]
    theta = torch.randn(numel, generator=gen, device=DEV) * 0.15
    ctx = _context(numel, learners, F32, 3, k_max=sum(ks))
    mem = [torch.zeros(numel, device=DEV) for _ in range(learners)]
    mem_ref = [m.cpu().numpy().copy() for m in mem]
    losses = []
    for step in range(2):
        table = theta[before:before + vocab * dim].view(vocab, dim)
        grads, total = [], 0.0
        for i in range(learners):
            text = torch.randint(0, vocab, (tokens + 1,), generator=gen, device=DEV, dtype=torch.int32)
            text[1::2] = (text[:-1:2] * 7 + 1) % vocab  # half of it follows a rule
            inputs, targets = text[:-1].contiguous(), text[1:].contiguous()
            targets[-9:] = -100
            inputs[-5:] = -1
            flat = torch.randn(numel, generator=gen, device=DEV)
            kept = flat.clone()
            grad = flat[before:before + vocab * dim].view(vocab, dim)
            x = ctx.scalecom_embed(table, inputs, scale)
            loss, lse = ctx.scalecom_cross_entropy(x, table, targets)
            dloss = torch.full((tokens,), 1.0 / (tokens - 9), device=DEV)
            dx, _ = ctx.scalecom_cross_entropy_grad(x, table, targets, loss, lse, dloss, True, grad)
            ctx.scalecom_embed_grad(inputs, dx, grad, scale, accumulate=True)
            want = ref.cross_entropy(x, table, targets)
            wdx, bdx, wdw, bdw = want.gradients(dloss, F32, F32)
            both, size, count = ref.embed_grad(inputs, wdx, vocab, scale, wdw)
            moved, _, _ = ref.embed_grad(inputs, bdx, vocab, scale)
            _within(grad, both, bdw + moved + ref.embed_grad_bound(both, size + moved, count, F32) + ref.U32 * wdw.abs(), "gradient")
            assert torch.equal(flat[:before], kept[:before]) and torch.equal(flat[before + vocab * dim:], kept[before + vocab * dim:])
            grads.append(flat)
            total += float(loss.sum()) / (tokens - 9)
        losses.append(total / learners)
        idx, vals = compare_step(ctx, mem, grads, mem_ref, step, 0.9, 1.0, offsets=offsets, ks=ks, what="language model")
        weights = to_host(theta).copy()
        oracle.apply_update(weights, idx.cpu().numpy(), vals.cpu().numpy(), 0.3 / learners)
        ctx.scalecom_apply_update(theta, idx, vals, 0.3 / learners)
        assert to_host(theta).tobytes() == weights.tobytes()
    assert all(math.isfinite(v) for v in losses)


def _everything(ctx, d):
    """All operators one behind the other, with outputs in d."""
    ctx.scalecom_embed(d["table"], d["ids"], 2.0, d["x"])
    ctx.scalecom_cross_entropy(d["x"], d["w"], d["targets"], d["loss"], d["lse"], scratch=d.get("scratch"))
    ctx.scalecom_cross_entropy_grad(d["x"], d["w"], d["targets"], d["loss"], d["lse"], d["dloss"], d["dx"], d["dw"], scratch=d.get("scratch"))
    ctx.scalecom_embed_grad(d["ids"], d["dx"], d["dtable"], 2.0, scratch=d.get("scratch"))
    ctx.scalecom_distill(d["x"], d["w"], d["lists"], d["teacher"], 2.0, d["loss2"], d["lse2"], d["listed"], scratch=d.get("scratch"))
    ctx.scalecom_distill_grad(d["x"], d["w"], d["lists"], d["teacher"], 2.0, d["lse2"], d["listed"], d["dloss"], d["dx2"], d["dw"], accumulate=True,
                              scratch=d.get("scratch"))


OUTPUTS = ("x", "loss", "lse", "dx", "dw", "dtable", "loss2", "lse2", "listed", "dx2")


def _inputs(seed, n, vocab, dim, dtype, entries=9):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    d = {"table": (torch.randn(vocab, dim, generator=gen, device=DEV) * 0.3).to(dtype), "w": (torch.randn(vocab, dim, generator=gen, device=DEV) * 0.2).to(dtype),
         "dloss": torch.rand(n, generator=gen, device=DEV), "teacher": torch.randn(n, entries, generator=gen, device=DEV).to(dtype)}
    for name, shape in (("ids", (n,)), ("targets", (n,)), ("lists", (n, entries))):
        d[name] = torch.randint(-vocab // 8, vocab, shape, generator=gen, device=DEV, dtype=torch.int32)
    return d


def _outputs(n, vocab, dim, dtype, entries=9):
    return {"x": torch.empty(n, dim, dtype=dtype, device=DEV), "loss": torch.empty(n, device=DEV), "lse": torch.empty(n, device=DEV),
            "dx": torch.empty(n, dim, dtype=dtype, device=DEV), "dw": torch.empty(vocab, dim, device=DEV), "dtable": torch.empty(vocab, dim, dtype=dtype, device=DEV),
            "loss2": torch.empty(n, device=DEV), "lse2": torch.empty(n, device=DEV), "listed": torch.empty(n, entries, device=DEV),
            "dx2": torch.empty(n, dim, dtype=dtype, device=DEV)}


@pytest.mark.parametrize("n,vocab,dim,dtype", [(20, 1000, 64, BF16), (200, 700, 128, BF16), (70, 300, 30, F32), (13_000, 40, 16, BF16)])
def test_captured_in_the_first_call_and_replayed(n, vocab, dim, dtype):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx, eager = _context(stream=stream), _context(stream=stream)
        d = {**_inputs(1, n, vocab, dim, dtype), **_outputs(n, vocab, dim, dtype)}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _everything(ctx, d)
    for seed in (2, 3, 4, 5):
        with torch.cuda.stream(stream):
            new = _inputs(seed, n, vocab, dim, dtype)
            for name, t in new.items():
                d[name].copy_(t)
            for name in OUTPUTS:
                d[name].fill_(float("nan"))
            graph.replay()
            got = {name: d[name].clone() for name in OUTPUTS}
            want = {**new, **_outputs(n, vocab, dim, dtype)}
            _everything(eager, want)                    # the program's own work between the replays
        torch.cuda.synchronize()
        for name in OUTPUTS:
            assert torch.equal(got[name], want[name]), (seed, name)


def test_two_contexts_at_once():
    """Two streams, two contexts, each with its own scratch, their calls under way together; the same bits as one after the other."""
    n, vocab, dim = 150, 2000, 128
    alone = []
    for seed in (7, 8):
        d = {**_inputs(seed, n, vocab, dim, BF16), **_outputs(n, vocab, dim, BF16)}
        _everything(_context(), d)
        alone.append(d)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [{**_inputs(seed, n, vocab, dim, BF16), **_outputs(n, vocab, dim, BF16)} for seed in (7, 8)]
    torch.cuda.synchronize()
    contexts = [_context(stream=s) for s in streams]
    for _ in range(3):
        for c, d in zip(contexts, both):
            _everything(c, d)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for name in OUTPUTS:
            assert torch.equal(a[name], b[name]), name


def test_a_scratch_of_the_callers_own():
    n, vocab, dim = 90, 500, 64
    lib, code = binding.lib(), binding.SCALECOM_GRAD_BF16
    need = max(lib.scalecom_vocab_scratch_bytes(n, vocab, dim, 9, code), lib.scalecom_embed_grad_scratch_bytes(n, dim))
    buffer = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device=DEV)
    begin = -buffer.data_ptr() % 256
    a, b = ({**_inputs(3, n, vocab, dim, BF16), **_outputs(n, vocab, dim, BF16)} for _ in range(2))
    a["scratch"] = buffer[begin:begin + need]
    ctx = _context()
    _everything(ctx, a)
    _everything(ctx, b)
    torch.cuda.synchronize()
    for name in OUTPUTS:
        assert torch.equal(a[name], b[name]), name
    assert bool((buffer[:begin] == 0xa5).all()) and bool((buffer[begin + need:] == 0xa5).all())


def _refused(status, call, *args, **kw):
    with pytest.raises(binding.ScaleComError) as e:
        call(*args, **kw)
    assert e.value.status == status


def test_refusals():
    ctx = _context()
    d = {**_inputs(3, 12, 50, 16, F32), **_outputs(12, 50, 16, F32)}
    before = {k: v.clone() for k, v in d.items()}
    x, w, t = d["x"], d["w"], d["targets"]
    small, odd = torch.zeros(256, dtype=torch.uint8, device=DEV), torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)[8:]
    inval, nomem = binding.SCALECOM_EINVAL, binding.SCALECOM_ENOMEM
    grad = (x, w, t, d["loss"], d["lse"], d["dloss"])
    distill = (x, w, d["lists"], d["teacher"])
    # a scratch that is too small or not aligned
    for status, s in ((nomem, small), (inval, odd)):
        _refused(status, ctx.scalecom_cross_entropy, x, w, t, d["loss"], d["lse"], scratch=s)
        _refused(status, ctx.scalecom_cross_entropy_grad, *grad, d["dx"], d["dw"], scratch=s)
        _refused(status, ctx.scalecom_distill, *distill, 1.0, d["loss2"], d["lse2"], d["listed"], scratch=s)
        _refused(status, ctx.scalecom_distill_grad, *distill, 1.0, d["lse2"], d["listed"], d["dloss"], d["dx2"], d["dw"], scratch=s)
        _refused(status, ctx.scalecom_embed_grad, d["ids"], d["dx"], d["dtable"], scratch=s)
    # numbers
    for temperature in (0.0, -1.0, math.inf, math.nan, 1e-45):
        _refused(inval, ctx.scalecom_distill, *distill, temperature)
        _refused(inval, ctx.scalecom_distill_grad, *distill, temperature, d["lse2"], d["listed"], d["dloss"])
    for scale in (math.nan, math.inf):
        _refused(inval, ctx.scalecom_embed, d["table"], d["ids"], scale)
        _refused(inval, ctx.scalecom_embed_grad, d["ids"], d["dx"], d["dtable"], scale)
    # rows that lie on each other
    spread = d["dx"][:1].expand(12, 16)
    _refused(inval, ctx.scalecom_embed_grad, d["ids"], spread, d["dtable"])
    _refused(inval, ctx.scalecom_cross_entropy, spread, w, t)
    _refused(inval, ctx.scalecom_cross_entropy_grad, *grad, spread, None)
    # outputs over inputs, or over each other
    both = torch.zeros(62, 16, device=DEV)
    _refused(inval, ctx.scalecom_embed, both[:50], d["ids"], 1.0, both[45:57])
    _refused(inval, ctx.scalecom_embed_grad, d["ids"], both[45:57], both[:50])
    _refused(inval, ctx.scalecom_cross_entropy, x, w, t, x.view(-1)[5:17], d["lse"])
    _refused(inval, ctx.scalecom_cross_entropy, x, w, t, d["loss"], d["loss"])
    _refused(inval, ctx.scalecom_cross_entropy_grad, *grad, x, None)
    _refused(inval, ctx.scalecom_cross_entropy_grad, *grad, None, w)
    _refused(inval, ctx.scalecom_cross_entropy_grad, *grad, both[:12], both[5:55])
    for name, v in before.items():
        assert torch.equal(d[name].nan_to_num(), v.nan_to_num()), name
    # the context goes on working
    _everything(ctx, d)
    assert bool(torch.isfinite(d["dw"]).all())
