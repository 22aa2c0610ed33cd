"""What the performance of the operators at the two ends of a language model is measured on: the embedding of tokens and
its gradient, and the losses over the vocabulary (cross entropy, distillation from a teacher's listed logits), which
take the last hidden states and the output matrix and never hold the logits of a whole batch.

A case names an operator, its sizes and its types.  The gradients of the two matrices go where a learner's flat gradient
has them, in its type, over what was there or added to it (a matrix that is embedding and output matrix in one).
"""
import math

import numpy
import torch

own = False                 # set by the tools: the framework's operators instead of the plain forms

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTH = {"f32": 4, "bf16": 2}
ABSENT = -100               # a position without a token or a target, an entry of a list that is not there


def listed():
    def embed(name, tokens, vocab, dim, scale, table, out):
        return {"name": name, "op": "embed", "tokens": tokens, "vocab": vocab, "dim": dim, "scale": scale, "type": table, "out": out}

    def embed_grad(name, tokens, vocab, dim, scale, dout, grad, accumulate):
        return {"name": name, "op": "embed_grad", "tokens": tokens, "vocab": vocab, "dim": dim, "scale": scale, "type": dout, "out": grad,
                "accumulate": accumulate}

    def loss(name, tokens, vocab, dim, kind, grad, train, accumulate=False, entries=0, temperature=1.0):
        return {"name": name, "op": "distill" if entries else "entropy", "tokens": tokens, "vocab": vocab, "dim": dim, "type": kind, "out": grad,
                "train": train, "accumulate": accumulate, "entries": entries, "temperature": temperature}

    return [
        # a short prompt's embedding, the smallest call: the time is a launch
        embed("embed_512", 512, 32_768, 512, 22.627417, "f32", "f32"),
        # a long batch from 32-bit weights into a 16-bit model
        embed("embed_65k", 65_536, 32_768, 1024, 1.0, "f32", "bf16"),
        # a Transformer-base's batch: few launches, many repeated tokens
        embed_grad("embed_grad_4k", 4096, 32_768, 512, 22.627417, "f32", "f32", False),
        # odd sizes, added to the output matrix's gradient (one matrix for both)
        embed_grad("embed_grad_odd", 10_007, 50_257, 771, 1.0, "f32", "f32", True),
        # a large vocabulary, 16 bits: most of the gradient is rows of zeros
        embed_grad("embed_grad_65k", 65_536, 131_072, 2048, 1.0, "bf16", "bf16", False),
        # the loss of a few tokens, for their probabilities: the output matrix is read once
        loss("entropy_8", 8, 32_768, 512, "bf16", "f32", False),
        # a training step of a Transformer-base, 16-bit activations, gradient in 32 bits
        loss("entropy_4k", 4096, 32_768, 512, "bf16", "f32", True),
        # everything in 32 bits, odd sizes, added to a gradient that is there
        loss("entropy_odd", 1003, 10_007, 333, "f32", "f32", True, accumulate=True),
        # the largest: a wide model's training step in 16 bits
        loss("entropy_8k", 8192, 131_072, 4096, "bf16", "bf16", True),
        # distillation in 32 bits, odd sizes, short lists
        loss("distill_odd", 500, 30_011, 520, "f32", "f32", True, entries=17, temperature=1.0),
        # a training step with a teacher's 64 largest logits a token
        loss("distill_2k", 2048, 32_768, 1024, "bf16", "f32", True, entries=64, temperature=2.0),
        # long lists, a large vocabulary
        loss("distill_4k", 4096, 131_072, 2048, "bf16", "bf16", True, entries=128, temperature=1.5),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["embed", "embed_grad", "entropy", "entropy", "distill", "distill"])
    kind = rng.choice(["f32", "bf16", "bf16"])
    dim = rng.choice([log_int(8, 4096), 64 * log_int(1, 64), 128 * log_int(1, 32)])
    vocab = log_int(16, 131_072)
    if op in ("embed", "embed_grad"):
        tokens = log_int(1, 65_536)
        while (tokens + vocab) * dim > (65_536 + 131_072) * 2048:
            dim = max(1, dim // 2)
        case = {"op": op, "tokens": tokens, "vocab": vocab, "dim": dim, "scale": rng.choice([1.0, 0.5, dim ** 0.5]), "type": kind,
                "out": rng.choice(["f32", "bf16"])}
        if op == "embed_grad":
            case["accumulate"] = rng.random() < 0.4
        return case
    tokens = log_int(1, 8192)
    # products of 32-bit operands are several of 16 bits
    while tokens * vocab * dim * (8 if kind == "f32" else 1) > 8192 * 131_072 * 4096:
        tokens = max(1, tokens // 2)
    return {"op": op, "tokens": tokens, "vocab": vocab, "dim": dim, "type": kind, "out": rng.choice(["f32", kind]), "train": rng.random() < 0.75,
            "accumulate": rng.random() < 0.3, "entries": min(vocab, log_int(1, 128)) if op == "distill" else 0,
            "temperature": rng.choice([1.0, 1.0, 2.0, 4.0]) if op == "distill" else 1.0}


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 7907 + 31)
    return gen


def _zipf(n, vocab, gen):
    """Tokens as texts have them: the v-th most frequent one about 1 / v as often as the first."""
    u = torch.rand(n, generator=gen, device=DEVICE, dtype=torch.float64)
    return u.mul_(math.log(vocab + 1)).exp_().sub_(1.0).clamp_(max=vocab - 1).to(torch.int32)


def _absent(n, gen):
    """An eighth of the positions: padding, or a prompt that is not learned from."""
    return torch.randperm(n, generator=gen, device=DEVICE)[:n // 8]


def _normal(shape, gen, factor, dtype):
    return torch.randn(shape, generator=gen, device=DEVICE).mul_(factor).to(dtype)


def prepare(case, seed):
    gen = _generator(seed)
    tokens, vocab, dim, kind, out = case["tokens"], case["vocab"], case["dim"], DTYPES[case["type"]], DTYPES[case["out"]]
    ids = _zipf(tokens, vocab, gen)
    ids[_absent(tokens, gen)] = ABSENT
    state = {"case": case, "ids": ids}
    if case["op"] == "embed":
        state["table"] = _normal((vocab, dim), gen, 0.02, kind)
        state["out"] = torch.empty(tokens, dim, dtype=out, device=DEVICE)
    elif case["op"] == "embed_grad":
        state["dout"] = _normal((tokens, dim), gen, 1e-3, kind)
        state["grad"] = _normal((vocab, dim), gen, 1e-3, out)
    else:
        state["w"] = _normal((vocab, dim), gen, 0.02, kind)
        if case["entries"]:
            # a teacher's largest logits, the largest first: distinct tokens all over the vocabulary
            n = case["entries"]
            steps = 1 + (torch.rand(tokens, 1, generator=gen, device=DEVICE) * (vocab // n - 1)).long()
            lists = (ids.long().clamp(min=0)[:, None] + steps * torch.arange(n, device=DEVICE)) % vocab
            fall = torch.rand(tokens, n, generator=gen, device=DEVICE).mul_(2.0 / n ** 0.5).cumsum(1)
            state["teacher"] = (12.0 - fall).to(kind)
            lists = lists.to(torch.int32)
            lists[ids < 0] = ABSENT
            if n > 2:               # every fifth list is shorter than the others
                lists[::5, n - n // 4:] = ABSENT
            state["lists"] = lists
            state["listed"] = torch.empty(tokens, n, device=DEVICE)
        # hidden states that point towards their token, some more than others
        x = torch.randn(tokens, dim, generator=gen, device=DEVICE)
        sure = torch.rand(tokens, 1, generator=gen, device=DEVICE).mul_(14.0 / 0.0004 / dim)
        state["x"] = x.addcmul_(state["w"][ids.long().clamp(min=0)].float(), sure).to(kind)
        state["loss"], state["lse"] = torch.empty(tokens, device=DEVICE), torch.empty(tokens, device=DEVICE)
        if case["train"]:
            valid = max(1, tokens - tokens // 8)
            state["dloss"] = torch.rand(tokens, generator=gen, device=DEVICE).add_(0.5).mul_(1.0 / valid)
            state["dx"] = torch.empty(tokens, dim, dtype=kind, device=DEVICE)
            state["dw"] = _normal((vocab, dim), gen, 1e-4, out)
    if own:
        from paper_2104_11125_amd import binding

        state["handle"] = binding.scalecom_init(4096, 1, torch.float32, device=DEVICE, k_max=0)
    return state


def run(state):
    return {"embed": _run_embed, "embed_grad": _run_embed_grad, "entropy": _run_entropy, "distill": _run_distill}[state["case"]["op"]](state)


def _run_embed(state):
    case, ids, table, out = state["case"], state["ids"], state["table"], state["out"]
    if own:
        state["handle"].scalecom_embed(table, ids, case["scale"], out)
    else:
        rows = table[ids.long().clamp(min=0)].float().mul_(case["scale"])
        out.copy_(rows.mul_((ids >= 0)[:, None]))
    return {"out": out}


def _run_embed_grad(state):
    case, ids, dout, grad = state["case"], state["ids"], state["dout"], state["grad"]
    if own:
        state["handle"].scalecom_embed_grad(ids, dout, grad, case["scale"], case["accumulate"])
        return {"grad": grad}
    there = ids >= 0
    full = torch.zeros(grad.shape, dtype=torch.float64, device=DEVICE)  # (a frequent token's sum is long)
    full.index_add_(0, ids[there].long(), dout[there].double())
    full.mul_(case["scale"])
    if case["accumulate"]:
        full.add_(grad)
    grad.copy_(full)
    return {"grad": grad}


def _run_entropy(state):
    case, ids, x, w, loss, lse = state["case"], state["ids"], state["x"], state["w"], state["loss"], state["lse"]
    if own:
        h = state["handle"]
        h.scalecom_cross_entropy(x, w, ids, loss, lse)
        if not case["train"]:
            return {"loss": loss, "lse": lse}
        h.scalecom_cross_entropy_grad(x, w, ids, loss, lse, state["dloss"], state["dx"], state["dw"], case["accumulate"])
        return {"loss": loss, "lse": lse, "dx": state["dx"], "dw": state["dw"]}
    there, at = ids >= 0, ids.long().clamp(min=0)
    z = x.float() @ w.float().t()
    # the target apart from the others: where it is nearly certain, what is left of it to 1 would be lost in 32 bits
    of_target = z.gather(1, at[:, None])
    z.scatter_(1, at[:, None], -torch.inf)
    top = z.amax(dim=1)
    far = (z - top[:, None]).exp().sum(dim=1).log().add_(top).sub_(of_target[:, 0])
    loss.copy_(far.clamp(min=0.0) + (-far.abs()).exp().log1p()).mul_(there)
    lse.copy_(of_target[:, 0] + loss).mul_(there)
    if not case["train"]:
        return {"loss": loss, "lse": lse}
    dz = z.sub_(lse[:, None]).exp_()
    dz.scatter_(1, at[:, None], (-loss).expm1()[:, None])
    return _gradients(state, dz.mul_((state["dloss"] * there)[:, None]), {"loss": loss, "lse": lse})


def _gradients(state, dz, out):
    state["dx"].copy_(dz @ state["w"].float())
    dw = dz.t().contiguous() @ state["x"].float()
    state["dw"].copy_(dw.add_(state["dw"]) if state["case"]["accumulate"] else dw)
    out["dx"], out["dw"] = state["dx"], state["dw"]
    return out


def _run_distill(state):
    case, lists, x, w, loss, lse, listed_ = (state["case"], state["lists"], state["x"], state["w"], state["loss"], state["lse"],
                                             state["listed"])
    t = case["temperature"]
    if own:
        h = state["handle"]
        h.scalecom_distill(x, w, lists, state["teacher"], t, loss, lse, listed_)
        if not case["train"]:
            return {"loss": loss, "lse": lse}
        h.scalecom_distill_grad(x, w, lists, state["teacher"], t, lse, listed_, state["dloss"], state["dx"], state["dw"], case["accumulate"])
        return {"loss": loss, "lse": lse, "dx": state["dx"], "dw": state["dw"]}
    there, at = lists >= 0, lists.long().clamp(min=0)
    rows = there.any(dim=1)
    q = torch.where(there, state["teacher"].float() / t, -torch.inf)
    q = (q - torch.where(rows, q.amax(dim=1), 0.0)[:, None]).exp()
    q = q / q.sum(dim=1, keepdim=True).clamp(min=1e-30)
    z = (x.float() @ w.float().t()).mul_(1.0 / t)
    top = z.amax(dim=1)
    lse.copy_((z - top[:, None]).exp().sum(dim=1).log().add_(top)).mul_(rows)
    apart = torch.where(q > 0, q.log(), 0.0) - (z.gather(1, at) - lse[:, None])
    loss.copy_((q * apart).sum(dim=1).mul_(t * t)).mul_(rows)
    if not case["train"]:
        return {"loss": loss, "lse": lse}
    dz = z.sub_(lse[:, None]).exp_()
    dz.scatter_add_(1, at, -q)
    return _gradients(state, dz.mul_((state["dloss"] * rows * t)[:, None]), {"loss": loss, "lse": lse})


def work(case):
    tokens, vocab, dim, kind, out = case["tokens"], case["vocab"], case["dim"], WIDTH[case["type"]], WIDTH[case["out"]]
    valid = tokens - tokens // 8
    if case["op"] in ("embed", "embed_grad"):
        # distinct tokens, as many as the distribution lets expect
        share = numpy.diff(numpy.log(numpy.arange(1, vocab + 2))) / math.log(vocab + 1)
        rows = float(-numpy.expm1(valid * numpy.log1p(-numpy.minimum(share, 1.0 - 1e-12))).sum())
        if case["op"] == "embed":
            return {"bytes": int(rows * dim * kind + tokens * (dim * out + 4)), "flops": valid * dim}
        written = 2 * rows * dim * out if case["accumulate"] else vocab * dim * out
        return {"bytes": int(valid * dim * kind + tokens * 4 + written), "flops": valid * dim}
    b = (valid + vocab) * dim * kind + 12 * tokens + case["entries"] * tokens * (4 + kind)
    f = 2 * valid * vocab * dim
    if case["train"]:
        b += tokens * (dim * kind + 4) + vocab * dim * out * (2 if case["accumulate"] else 1)
        f *= 3
    return {"bytes": b, "flops": f}


def exact(case, seed):
    """The outputs of run() from the definitions, in 64 bits."""
    state = prepare(case, seed)
    tokens, vocab, dim = case["tokens"], case["vocab"], case["dim"]
    if case["op"] == "embed":
        padded = torch.cat([state["table"].double() * case["scale"], torch.zeros(1, dim, dtype=torch.float64, device=DEVICE)])
        ids = state["ids"].long()
        return {"out": padded[torch.where(ids < 0, vocab, ids)]}
    if case["op"] == "embed_grad":
        grad = state["grad"].double() if case["accumulate"] else torch.zeros(vocab, dim, dtype=torch.float64, device=DEVICE)
        order = torch.argsort(state["ids"], stable=True)
        ids = state["ids"][order].long()
        order, ids = order[ids >= 0], ids[ids >= 0]
        distinct, counts = torch.unique_consecutive(ids, return_counts=True)
        ends = counts.cumsum(0).tolist()
        if len(order):
            for c in range(0, dim, 512):        # sums of sorted runs, a few columns at a time
                rows = state["dout"][:, c:c + 512].double()[order]
                sums = torch.segment_reduce(rows, "sum", lengths=counts, axis=0)
                grad[distinct, c:c + 512] += case["scale"] * sums
        assert not ends or ends[-1] == len(order)
        return {"grad": grad}
    w, x, t = state["w"].double(), state["x"].double(), case["temperature"]
    loss, lse = torch.zeros(tokens, dtype=torch.float64, device=DEVICE), torch.zeros(tokens, dtype=torch.float64, device=DEVICE)
    if case["train"]:
        dx = torch.zeros(tokens, dim, dtype=torch.float64, device=DEVICE)
        dw = state["dw"].double() if case["accumulate"] else torch.zeros(vocab, dim, dtype=torch.float64, device=DEVICE)
    for a in range(0, tokens, 1024):
        part = torch.arange(a, min(a + 1024, tokens), device=DEVICE)
        target = torch.zeros(len(part), vocab + 1, dtype=torch.float64, device=DEVICE)      # the last column takes what is absent
        if case["op"] == "entropy":
            ids = state["ids"][part].long()
            target[torch.arange(len(part), device=DEVICE), torch.where(ids < 0, vocab, ids)] = 1.0
            entropy = 0.0
        else:
            lists = state["lists"][part].long()
            teacher = state["teacher"][part].double().div(t).masked_fill(lists < 0, -torch.inf)
            q = torch.softmax(teacher, dim=1).nan_to_num(0.0)
            target.scatter_add_(1, torch.where(lists < 0, vocab, lists), q)
            entropy = torch.special.xlogy(q, q).sum(dim=1)
        target = target[:, :vocab]
        rows = target.sum(dim=1) > 0.5
        logp = torch.log_softmax(x[part] @ w.t() / t, dim=1)
        first = (x[part] * w[0]).sum(dim=1) / t
        lse[part] = torch.where(rows, first - logp[:, 0], 0.0)
        loss[part] = torch.where(rows, (entropy - (target * logp).sum(dim=1)) * t * t, 0.0)
        if case["train"]:
            dz = (logp.exp_() - target) * (torch.where(rows, state["dloss"][part].double(), 0.0) * t)[:, None]
            dx[part] = dz @ w
            dw += dz.t() @ x[part]
    out = {"loss": loss, "lse": lse}
    if case["train"]:
        out["dx"], out["dw"] = dx, dw
    return out
