"""What the performance of the optimiser operators is measured on: momentum from a compressed gradient,
orthogonalised updates, and the dense update of the weights.

A case names an operator, its sizes and its types.  Tensors lie back to back in one flat vector, as the steps of
this library take them; a matrix is followed by the vectors that belong to it (biases, or the gain and bias of a
normalisation), which the matrix operators leave alone, so most matrices do not begin on a round address.
`shapes` lists the matrices: "64x576*3" is three of 64 rows and 576 columns.
"""
import array

import torch

own = False                 # set by the tools: the framework's operators instead of the plain forms

DEVICE = "cuda:0"
MU, SCALE, EPS, DECAY = 0.95, 0.125, 1e-7, 0.999
COEFFS = (3.4445, -4.7750, 2.0315)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# the convolutions of a small residual network for 32 x 32 images, as matrices, and its classifier
SMALL_NET = "16x27,16x144*6,32x144,32x288*5,64x288,64x576*5,16x32,32x64,10x64"
# the matrices of a ResNet-50: 25.5 M elements
RESNET50 = ("64x147,64x64,64x576*3,256x64*4,64x256*2,128x256,128x1152*4,512x128*4,512x256,128x512*3,256x512,256x2304*6,"
            "1024x256*6,1024x512,256x1024*5,512x1024,512x4608*3,2048x512*3,2048x1024,512x2048*2,1000x2048")
# the projections of a Transformer-base, six encoder and six decoder layers: 44 M elements
TRANSFORMER = "512x512*72,2048x512*12,512x2048*12"
# what does not fit a tile: vectors, a few rows, a few columns, primes, one above and one below a power of two
ODD = "1x1000,7x1000,50x3,257x129,2001x65,333x777,1000x4095,511x513,1x1,1x70001"


def listed():
    def momentum(name, numel, rate, out, nesterov):
        return {"name": name, "op": "momentum", "numel": numel, "rate": rate, "out": out, "nesterov": nesterov}

    def matrices(name, op, shapes, src, out, vectors, pad=0, steps=5):
        return {"name": name, "op": op, "shapes": shapes, "src": src, "out": out, "vectors": vectors, "pad": pad, "steps": steps}

    return [
        # a small network, the smallest calls: the time is a launch
        momentum("momentum_200k", 200_003, 100, "f32", True),
        # a ResNet-50-sized vector whose update goes to the orthogonaliser in 16 bits
        momentum("momentum_25m", 25_557_032, 112, "bf16", True),
        # the largest vector of the benchmark's configurations
        momentum("momentum_1g", 1_000_000_000, 400, "bf16", False),
        # every convolution of a small network, orthogonalised in full precision: launches and latency count
        matrices("ortho_small_net", "ortho", SMALL_NET, "f32", "f32", 2),
        # a ResNet-50, all sizes from 64 x 64 to 512 x 4608 in one call, full precision
        matrices("ortho_resnet50", "ortho", RESNET50, "f32", "f32", 2),
        # a Transformer-base in 16 bits: many matrices of two sizes
        matrices("ortho_transformer", "ortho", TRANSFORMER, "bf16", "bf16", 1),
        # tensors of odd sizes, 32-bit momentum and a 16-bit result
        matrices("ortho_odd", "ortho", ODD, "f32", "bf16", 0),
        # one large matrix in full precision
        matrices("ortho_2048x8192", "ortho", "2048x8192", "f32", "f32", 0),
        # the largest: a tall projection of a wide model in 16 bits
        matrices("ortho_16384x4096", "ortho", "16384x4096", "bf16", "bf16", 0),
        # the weights of a small network: launches and latency count
        matrices("apply_small_net", "apply", SMALL_NET, "f32", "f32", 2),
        # the weights of a ResNet-50 from an update in 32 bits
        matrices("apply_resnet50", "apply", RESNET50, "f32", "f32", 2),
        # the weights of a Transformer-base from an update in 16 bits
        matrices("apply_transformer", "apply", TRANSFORMER, "bf16", "f32", 1),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["momentum", "ortho", "ortho", "ortho", "apply"])
    if op == "momentum":
        return {"op": op, "numel": log_int(5_000, 400_000_000), "rate": rng.choice([1, 25, 50, 100, 112, 155, 400]),
                "out": rng.choice(["f32", "bf16"]), "nesterov": rng.random() < 0.6}
    src, out = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
    # one matrix of any size, or up to sixty of a network; in 32 bits up to 2048 x 8192
    kind = rng.choice(["one", "few", "many"])
    short, long = {"one": (2048, 8192) if out == "f32" else (4096, 16_384), "few": (1024, 4096), "many": (384, 1536)}[kind]
    count = {"one": 1, "few": rng.randint(2, 8), "many": rng.randint(9, 60)}[kind]
    shapes = []
    for _ in range(count):
        m = log_int(1 if kind != "one" else 32, short)
        n = max(m, log_int(4, long))
        shapes.append("%dx%d" % ((m, n) if rng.random() < 0.5 else (n, m)))
    return {"op": op, "shapes": ",".join(shapes), "src": src, "out": "f32" if op == "apply" else out,
            "vectors": rng.choice([0, 1, 2]),
            # matrices that are blocks of columns of wider ones: their rows lie further apart than they are long
            "pad": rng.choice([0, 0, 0, 1, 64]), "steps": rng.choice([5, 5, 5, 4, 6])}


def _matrices(case):
    """(offset, rows, columns, row stride) of every matrix, and the length of the flat vector."""
    found, at = [], 0
    for item in case["shapes"].split(","):
        shape, _, count = item.partition("*")
        rows, cols = (int(v) for v in shape.split("x"))
        for _ in range(int(count or 1)):
            found.append((at, rows, cols, cols + case["pad"]))
            at += rows * (cols + case["pad"]) + case["vectors"] * rows
    return found, at


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 7919 + 29)
    return gen


def _momentum_values(rows, cols, gen):
    """A matrix of a momentum: a few directions that all batches share, noise, rows and columns of different size."""
    rank = min(8, rows, cols)
    x = torch.randn(rows, cols, generator=gen, device=DEVICE)
    x.addmm_(torch.randn(rows, rank, generator=gen, device=DEVICE), torch.randn(rank, cols, generator=gen, device=DEVICE), alpha=0.5)
    x.mul_(torch.randn(rows, 1, generator=gen, device=DEVICE).mul_(0.5).exp_())
    return x.mul_(torch.randn(1, cols, generator=gen, device=DEVICE).mul_(0.3).exp_()).mul_(1e-3)


def _view(flat, place):
    offset, rows, cols, stride = place
    return flat.as_strided((rows, cols), (stride, 1), flat.storage_offset() + offset)


def prepare(case, seed):
    gen = _generator(seed)
    if case["op"] == "momentum":
        numel = case["numel"]
        k = max(1, numel // case["rate"])
        state = {"case": case, "momentum": torch.randn(numel, generator=gen, device=DEVICE).mul_(1e-3),
                 "update": torch.empty(numel, dtype=DTYPES[case["out"]], device=DEVICE)}
        # ascending positions, denser towards the beginning, as where layers are compressed at different rates
        u = torch.rand(k, generator=gen, device=DEVICE, dtype=torch.float64).square_().mul_(numel)
        idx = torch.unique_consecutive(u.sort().values.to(torch.int32).clamp_(max=numel - 1))
        del u
        state["idx"], state["vals"] = idx, torch.randn(idx.numel(), generator=gen, device=DEVICE).mul_(1e-2)
        state["handle"] = _handle(numel, 1)
        return state
    places, numel = _matrices(case)
    src = torch.zeros(numel, device=DEVICE)
    for p in places:
        _view(src, p).copy_(_momentum_values(p[1], p[2], gen))
    state = {"case": case, "places": places, "src": src.to(DTYPES[case["src"]])}
    state["table"] = [array.array("q", [p[j] for p in places]) for j in range(4)]
    if case["op"] == "ortho":
        state["out"] = torch.zeros(numel, dtype=DTYPES[case["out"]], device=DEVICE)
    else:
        state["theta"] = torch.randn(numel, generator=gen, device=DEVICE).mul_(0.03)
        # steps of one size whatever the shape: an orthogonal matrix of r x c has elements of about 1 / sqrt(max(r, c))
        state["scales"] = [0.2 * 0.02 * max(p[1], p[2]) ** 0.5 for p in places]
    state["handle"] = _handle(numel, len(places))
    return state


def _handle(numel, tensors):
    if not own:
        return None
    from paper_2104_11125_amd import binding

    return binding.scalecom_init(numel, 1, torch.float32, n_tensors_max=tensors, device=DEVICE, k_max=0)


def run(state):
    return {"momentum": _run_momentum, "ortho": _run_ortho, "apply": _run_apply}[state["case"]["op"]](state)


def _run_momentum(state):
    case, m, update = state["case"], state["momentum"], state["update"]
    if own:
        state["handle"].scalecom_momentum_update(m, state["idx"], state["vals"], SCALE, MU, case["nesterov"], update)
    else:
        g = torch.zeros_like(m)
        g[state["idx"].long()] = SCALE * state["vals"]
        m.mul_(MU).add_(g)
        update.copy_(g.add_(m, alpha=MU) if case["nesterov"] else m)
    return {"momentum": m, "update": update}


def _run_ortho(state):
    case, out = state["case"], state["out"]
    if own:
        offsets, rows, cols, strides = state["table"]
        state["handle"].scalecom_orthogonalize(state["src"], offsets, rows, cols, strides, out, coeffs=[COEFFS] * case["steps"], eps=EPS)
        return {"out": out}
    same = {}                   # matrices of one shape are worked on together
    for p in state["places"]:
        same.setdefault(p[1:3], []).append(p)
    for (rows, cols), group in same.items():
        x = torch.stack([_view(state["src"], p) for p in group]).float()
        if rows > cols:
            x = x.transpose(1, 2).contiguous()
        x = x / (x.double().square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS).float()
        for _ in range(case["steps"]):
            s = x @ x.transpose(1, 2).contiguous()
            x = COEFFS[0] * x + (COEFFS[1] * s + COEFFS[2] * (s @ s)) @ x
        if rows > cols:
            x = x.transpose(1, 2)
        for p, o in zip(group, x):
            _view(out, p).copy_(o)
    return {"out": out}


def _run_apply(state):
    theta = state["theta"]
    if own:
        offsets, rows, cols, strides = state["table"]
        state["handle"].scalecom_apply_tensors(theta, state["src"], offsets, rows, cols, state["scales"], DECAY, strides)
        return {"theta": theta}
    for p, scale in zip(state["places"], state["scales"]):
        _view(theta, p).mul_(DECAY).sub_(scale * _view(state["src"], p).float())
    return {"theta": theta}


def work(case):
    width = {"f32": 4, "bf16": 2}
    if case["op"] == "momentum":
        return {"bytes": case["numel"] * (8 + width[case["out"]]) + 8 * max(1, case["numel"] // case["rate"]), "flops": 4 * case["numel"]}
    places, _ = _matrices(case)
    elements = sum(r * c for _, r, c, _ in places)
    if case["op"] == "apply":   # weight in and out, update in
        return {"bytes": elements * (8 + width[case["src"]]), "flops": 3 * elements}
    flops = 0
    for _, r, c, _ in places:   # the two symmetric products need one half of themselves
        m, n = min(r, c), max(r, c)
        flops += case["steps"] * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
    return {"bytes": elements * (width[case["src"]] + width[case["out"]]), "flops": flops}


def exact(case, seed):
    """The outputs of run() from the definitions, in 64 bits."""
    state = prepare(case, seed)
    if case["op"] == "momentum":
        m = state["momentum"].double().mul_(MU)
        at = state["idx"].long()
        g = SCALE * state["vals"].double()
        m[at] += g
        if not case["nesterov"]:
            return {"momentum": m, "update": m}
        u = MU * m
        u[at] += g
        return {"momentum": m, "update": u}
    a, b, c = COEFFS
    if case["op"] == "apply":
        theta = state["theta"].double()
        for p, scale in zip(state["places"], state["scales"]):
            v = _view(theta, p)
            v.copy_(DECAY * v - scale * _view(state["src"], p).double())
        return {"theta": theta}
    out = torch.zeros(state["out"].numel(), dtype=torch.float64, device=DEVICE)
    for p in state["places"]:
        x = _view(state["src"], p).double()
        x = x / (torch.linalg.vector_norm(x) + EPS)
        eye = torch.eye(min(p[1:3]), dtype=torch.float64, device=DEVICE)
        for _ in range(case["steps"]):
            if p[1] >= p[2]:    # on the side with the smaller Gram matrix: X (a + b X'X + c (X'X)^2)
                g = x.t() @ x
                x = x @ (a * eye + g @ (b * eye + c * g))
            else:
                g = x @ x.t()
                x = (a * eye + g @ (b * eye + c * g)) @ x
        _view(out, p).copy_(x)
    return {"out": out}
