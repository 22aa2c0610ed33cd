"""The optimiser operators on the GPU against their plain forms in 64 bits: momentum from a compressed gradient, orthogonalised
updates, the dense update of the weights, and all of them behind a compression step."""
import math

import numpy as np
import pytest
import torch

import optimizer_reference as ref
from paper_2104_11125_amd import binding

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _context(numel, tensors=1, stream=None):
    return binding.scalecom_init(max(numel, 1), 1, torch.float32, tensors, DEV, stream, k_max=0)


def _within(got, want, bound, what):
    off = (got.double().cpu() - want).abs() - bound
    assert bool((off <= 0).all()), (what, float(off.max()), int(off.argmax()))


# momentum ----------------------------------------------------------------------------------------
def _members(numel, k, gen, where):
    if where == "even":
        return torch.randperm(numel, generator=gen)[:k].sort().values
    if where == "front":
        return torch.arange(k)
    if where == "back":
        return torch.arange(numel - k, numel)
    assert where == "middle"
    return torch.arange(k) + (numel - k) // 2


@pytest.mark.parametrize("numel,k,where", [(1, 0, "even"), (1, 1, "even"), (3, 2, "even"), (4095, 41, "even"), (4096, 4096, "even"),
                                           (4097, 1, "back"), (8193, 4099, "middle"), (70_001, 700, "front"), (70_001, 0, "even"),
                                           (100_003, 70_000, "even"), (1_000_003, 10_000, "even"), (300_007, 64, "back"),
                                           (300_007, 65, "middle")])
@pytest.mark.parametrize("out,nesterov", [("f32", True), ("bf16", True), ("f32", False), ("bf16", False), (None, True)])
def test_momentum(numel, k, where, out, nesterov):
    gen = torch.Generator().manual_seed(numel * 31 + k)
    m = torch.randn(numel, generator=gen)
    idx = _members(numel, k, gen, where).to(torch.int32)
    vals = torch.randn(k, generator=gen)
    scale, mu = 0.3, 0.95
    want_m, want_u, bound_m, bound_u = ref.momentum(m, idx, vals, scale, mu, nesterov)
    ctx = _context(numel)
    # a guard behind both vectors: what lies after the last position stays as it is
    buf = torch.full((numel + 8,), 7.0, device=DEV)
    buf[:numel] = m.to(DEV)
    ubuf = torch.full((numel + 8,), 7.0, device=DEV, dtype=TYPES[out or "f32"])
    ctx.scalecom_momentum_update(buf[:numel], idx.to(DEV), vals.to(DEV), scale, mu, nesterov, None if out is None else ubuf[:numel])
    torch.cuda.synchronize()
    _within(buf[:numel], want_m, bound_m, "momentum")
    if out is not None:
        _within(ubuf[:numel], want_u, bound_u + (ref.UB * (want_u.abs() + bound_u) if out == "bf16" else 0.0), "update")
    assert bool((buf[numel:] == 7).all()) and bool((ubuf[numel if out else 0:] == 7).all())
    ctx.close()


def test_momentum_keeps_to_its_buffers_with_entries_that_are_no_positions():
    """Entries outside the vector are skipped (they lie at the ends of an ascending list), and infinities and NaN stay where they are."""
    numel = 10_000
    idx = torch.tensor([-5, -1, 0, 17, 4096, 9_999, 10_000, 2 ** 31 - 1], dtype=torch.int32)
    vals = torch.tensor([9.0, 9.0, 1.0, float("inf"), float("nan"), 2.0, 9.0, 9.0])
    ctx = _context(numel)
    m = torch.ones(numel, device=DEV)
    u = torch.empty(numel, device=DEV, dtype=torch.bfloat16)
    ctx.scalecom_momentum_update(m, idx.to(DEV), vals.to(DEV), 1.0, 0.5, True, u)
    m, u = m.cpu(), u.float().cpu()
    want = torch.full((numel,), 0.5)
    want[0], want[17], want[4096], want[9_999] = 1.5, math.inf, math.nan, 2.5
    assert torch.equal(m.nan_to_num(-1.0, 1e9), want.nan_to_num(-1.0, 1e9))
    assert math.isnan(u[4096]) and u[17] == math.inf and u[1] == 0.25 and u[0] == 1.75 and u[9_999] == 3.25
    # a list in another order stays inside its buffers, too
    torch.manual_seed(0)
    back = torch.randperm(numel).to(torch.int32).to(DEV)
    guard = torch.full((numel + 64,), 3.0, device=DEV)
    ctx.scalecom_momentum_update(guard[:numel], back, torch.ones(numel, device=DEV), 1.0, 0.5, False)
    assert bool((guard[numel:] == 3).all())
    ctx.close()


# weight update -----------------------------------------------------------------------------------
def _places(shapes, pad=0, gap=0, first=0):
    found, at = [], first
    for r, c in shapes:
        found.append((at, r, c, c + pad))
        at += r * (c + pad) + gap
    return found, at


def _split(places):
    return [[p[j] for p in places] for j in range(4)]


SHAPE_SETS = {
    "one": [(1, 1)],
    "row": [(1, 5001)],
    "column": [(777, 1)],
    "empty": [(0, 7), (5, 0), (3, 2)],
    "odd": [(7, 13), (64, 64), (129, 127), (3, 1000), (1000, 3), (65, 200), (200, 65), (1, 70_001)],
    "many": [(1 + i % 9, 1 + (7 * i) % 31) for i in range(211)],
    "large": [(513, 1025), (300, 700)],
}


@pytest.mark.parametrize("name", sorted(SHAPE_SETS))
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("pad,gap,first", [(0, 0, 0), (0, 3, 1), (5, 1, 2), (64, 0, 3)])
def test_apply_tensors(name, src, pad, gap, first):
    places, numel = _places(SHAPE_SETS[name], pad, gap, first)
    numel += 5
    gen = torch.Generator().manual_seed(numel)
    theta, update = torch.randn(numel, generator=gen), torch.randn(numel, generator=gen).to(TYPES[src])
    scales = [0.01 * (1 + s % 7) * (-1) ** s for s in range(len(places))]
    decay = 0.99
    want, bound = theta.double(), torch.zeros(numel, dtype=torch.float64)
    for p, scale in zip(places, scales):
        if p[1] * p[2]:
            v, e = ref.view(want, p), ref.view(bound, p)
            old = ref.f32(decay) * v
            v.copy_(old - ref.f32(scale) * ref.view(update, p).double())
            e.copy_(ref.U32 * (old.abs() + v.abs()) * 1.001 + 1e-44)        # two roundings
    ctx = _context(numel, len(places))
    dev = theta.to(DEV)
    offsets, rows, cols, strides = _split(places)
    ctx.scalecom_apply_tensors(dev, update.to(DEV), offsets, rows, cols, scales, decay, strides if pad else None)
    _within(dev, want, bound, name)             # (bound 0 outside the tensors: untouched)
    ctx.close()


# orthogonalised updates --------------------------------------------------------------------------
COEFFS = binding.SCALECOM_ORTHO_COEFFS


def _matrix(rows, cols, kind, gen):
    x = torch.randn(rows, cols, generator=gen)
    if kind == "low rank":
        x = 0.01 * x + torch.randn(rows, 1, generator=gen) @ torch.randn(1, cols, generator=gen)
    elif kind == "sparse":
        x = x * (torch.rand(rows, cols, generator=gen) < 0.05)
    elif kind == "scaled":
        x = x * torch.randn(rows, 1, generator=gen).exp() * 1e-6
    return x


def _check_matrices(flat, out, places, coeffs, eps, split, out_bf16):
    for p in places:
        if p[1] * p[2] == 0:
            continue
        u, got = ref.view(flat, p), ref.view(out, p).double()
        want = ref.orthogonalize(u, coeffs, eps)
        bound = ref.orthogonalize_bound(u, coeffs, eps, split, out_bf16)
        off = float((got - want).norm())
        print(f"{p[1]}x{p[2]} split {split}: off {off:.2e} of {float(want.norm()):.2e}, allowed {bound:.2e}", flush=True)
        assert off <= bound, (p, off, bound)


ORTHO_SETS = {
    "one": [(1, 1)],
    "row": [(1, 1000)],
    "column": [(333, 1)],
    "tile": [(128, 128)],
    "small": [(7, 13), (16, 27), (64, 64), (10, 64), (64, 200), (33, 500)],
    "odd": [(129, 127), (3, 700), (0, 4), (700, 3), (65, 200), (200, 65), (127, 257)],
    "mid": [(300, 520), (520, 300), (256, 384)],
    "many": [(5 + 3 * (i % 9), 4 + (11 * i) % 61) for i in range(130)],
    "long": [(1, 641), (3, 5000), (2049, 7), (16, 1300), (17, 641), (641, 64), (640, 64), (64, 640), (65, 66), (1, 3)],
    "many long": [(1 + i % 16, 700 + 13 * i) for i in range(60)] + [(700 + 13 * i, 1 + i % 16) for i in range(60)],
}


@pytest.mark.parametrize("name", ["one", "row", "column", "tile", "small", "odd", "mid", "many", "long", "many long"])
@pytest.mark.parametrize("src,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("kind", ["normal", "low rank", "sparse", "scaled"])
def test_orthogonalize(name, src, out, kind):
    pad, gap, first = (0, 0, 0) if kind == "normal" else (3, 5, 1) if kind == "low rank" else (0, 1, 2)
    places, numel = _places(ORTHO_SETS[name], pad, gap, first)
    numel += 7
    gen = torch.Generator().manual_seed(numel)
    flat = torch.full((numel,), float("nan"))           # what lies between the matrices is neither read nor written
    for p in places:
        if p[1] * p[2]:
            ref.view(flat, p).copy_(_matrix(p[1], p[2], kind, gen))
    flat = flat.to(TYPES[src])
    ctx = _context(numel, len(places))
    dev_out = torch.full((numel,), 7.0, device=DEV, dtype=TYPES[out])
    offsets, rows, cols, strides = _split(places)
    print(name, src, out, kind, flush=True)
    ctx.scalecom_orthogonalize(flat.to(DEV), offsets, rows, cols, strides if pad else None, dev_out)
    got = dev_out.cpu()
    _check_matrices(flat, got, places, COEFFS, 1e-7, out == "f32", out == "bf16")
    untouched = torch.ones(numel, dtype=torch.bool)
    for p in places:
        if p[1] * p[2]:
            ref.view(untouched, p).fill_(False)
    assert bool((got[untouched] == 7).all())
    ctx.close()


def test_orthogonalize_zero_and_non_finite_matrices():
    """A zero matrix stays zero; one with an infinity or a NaN becomes NaN; their neighbours do not notice."""
    places, numel = _places([(40, 50)] * 5 + [(200, 150)] * 4 + [(2, 3), (150, 200)])
    gen = torch.Generator().manual_seed(3)
    flat = torch.randn(numel, generator=gen)
    ref.view(flat, places[1]).zero_()
    ref.view(flat, places[2])[3, 4] = float("inf")
    ref.view(flat, places[3])[39, 49] = float("nan")
    ref.view(flat, places[5])[199, 149] = float("nan")
    ref.view(flat, places[7]).zero_()
    ref.view(flat, places[8]).mul_(1e38)                # some of its elements overflow: infinities
    ref.view(flat, places[10]).mul_(1e37)               # its squares overflow binary32, its norm does not
    ref.view(flat, places[4]).mul_(1e-30)               # far below eps
    assert bool(ref.view(flat, places[8]).isinf().any()) and bool(ref.view(flat, places[10]).isfinite().all())
    ctx = _context(numel, len(places))
    offsets, rows, cols, _ = _split(places)
    for dtype in (torch.float32, torch.bfloat16):
        out = ctx.scalecom_orthogonalize(flat.to(DEV), offsets, rows, cols, out=torch.empty(numel, device=DEV, dtype=dtype)).cpu()
        for j in (1, 7):
            assert bool((ref.view(out, places[j]) == 0).all()), j
        for j in (2, 3, 5, 8):
            assert bool(ref.view(out, places[j]).isnan().all()), j
        fine = [places[j] for j in (0, 6, 9, 10)]
        _check_matrices(flat, out, fine, COEFFS, 1e-7, dtype == torch.float32, dtype != torch.float32)
        # 1e-30 / 1e-7 of a matrix: the steps multiply it by a^5
        tiny = ref.orthogonalize(ref.view(flat, places[4]), COEFFS, 1e-7)
        got = ref.view(out, places[4]).double()
        assert float((got - tiny).norm()) <= 0.01 * float(tiny.norm())
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orthogonalize_in_place_and_other_steps(dtype):
    """The update's own buffer as the result, one to six steps with coefficients of their own."""
    places, numel = _places([(100, 300), (300, 100), (64, 64), (130, 131)], gap=3, first=1)
    gen = torch.Generator().manual_seed(4)
    flat = torch.randn(numel, generator=gen).to(dtype)
    ctx = _context(numel, len(places))
    offsets, rows, cols, _ = _split(places)
    for coeffs in ([(1.5, -0.5, 0.0)], [(3.4445, -4.7750, 2.0315)] * 6, [(1.875, -1.25, 0.375), (1.5, -0.5, 0.0)]):
        buf = flat.to(DEV)
        assert ctx.scalecom_orthogonalize(buf, offsets, rows, cols, out=buf, coeffs=coeffs) is buf
        got = buf.cpu()
        _check_matrices(flat, got, places, coeffs, 1e-7, dtype == torch.float32, dtype != torch.float32)
        again = ctx.scalecom_orthogonalize(flat.to(DEV), offsets, rows, cols, coeffs=coeffs).cpu()
        for p in places:                                # the same bits on every call
            assert torch.equal(ref.view(again, p), ref.view(got, p))
    ctx.close()


@pytest.mark.parametrize("out,rows,cols", [("f32", 1000, 1100), ("bf16", 2048, 1024), ("bf16", 1500, 4000), ("f32", 512, 8192)])
def test_orthogonalize_large(out, rows, cols):
    """Sizes with many tiles: the exact values come from the GPU in 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(rows)
    u = torch.randn(rows, cols, generator=gen, device=DEV) + torch.randn(rows, 4, generator=gen, device=DEV) @ torch.randn(4, cols, generator=gen, device=DEV)
    ctx = _context(u.numel())
    got = ctx.scalecom_orthogonalize(u.view(-1), [0], [rows], [cols], out=torch.empty(u.numel(), device=DEV, dtype=TYPES[out]))
    want = ref.orthogonalize(u, COEFFS, 1e-7)
    bound = ref.orthogonalize_bound(u, COEFFS, 1e-7, out == "f32", out == "bf16", draws=1)
    off = float((got.view(rows, cols).double() - want).norm())
    print(f"off {off:.2e} of {float(want.norm()):.2e}, allowed {bound:.2e}", flush=True)
    assert off <= bound
    ctx.close()
