"""That the bounds of vocab_precision.py see what they are for: with any one product of planes left out, anywhere, results are out of them."""
import pytest
import torch

import vocab_precision as precision


@pytest.mark.parametrize("peaked", [False, True])
def test_all_products(peaked):
    x, w, targets, dloss = precision.inputs(peaked)
    want = precision.exact(x, w, targets, dloss)
    z = x.double() @ w.double().t()
    assert 6 < float(want["lse"].min()) and float(want["lse"].max()) < 8 and float(z.abs().max()) < 8
    assert max(precision.off(precision.model(x, w, targets, dloss), want).values()) < precision.limit(peaked) / 4


@pytest.mark.parametrize("where", ["sums", "dz_logits", "dx", "dw"])
@pytest.mark.parametrize("pair", precision.ALL[:5])
def test_one_product_left_out(where, pair):
    seen = []
    for peaked in (False, True):
        given = precision.inputs(peaked)
        got = precision.off(precision.model(*given, **{where: [p for p in precision.ALL if p != pair]}), precision.exact(*given))
        seen.append(max(got.values()) > 2 * precision.limit(peaked))
    assert any(seen)


def test_a_plane_of_dz_left_out():
    """A binary32 gradient of bfloat16 operands: one plane of the operands, three of dz."""
    x, w, targets, dloss = precision.inputs(False)
    x, w = x.bfloat16().float(), w.bfloat16().float()
    want = precision.exact(x, w, targets, dloss)
    assert precision.off(precision.model(x, w, targets, dloss), want)["dw"] < precision.FLAT / 4
    for planes in ([(0, 1), (0, 0)], [(0, 2), (0, 0)]):
        assert precision.off(precision.model(x, w, targets, dloss, dw=planes), want)["dw"] > 2 * precision.FLAT


@pytest.mark.parametrize("peaked", [False, True])
def test_roundings_to_bfloat16(peaked):
    """A gradient rounded once, from dz in two planes, is inside the bound; from dz rounded to one it is not."""
    x, w, targets, dloss = precision.inputs(peaked)
    x, w = x.bfloat16().float(), w.bfloat16().float()
    want = precision.exact(x, w, targets, dloss)
    want.pop("lse")
    for planes, good in (([(0, 1), (0, 0)], True), ([(0, 0)], False)):
        got = precision.model(x, w, targets, dloss, dx=planes, dw=planes)
        off = precision.off_rounded({k: got[k].bfloat16() for k in want}, want)
        assert all((v < precision.ROUNDED / 1.5) if good else (v > 1.5 * precision.ROUNDED) for v in off.values()), off
