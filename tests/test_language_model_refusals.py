"""What the embedding and the losses over a vocabulary refuse without touching a device: null contexts, sizes that are out of range, and what
the binding sees by itself."""
import pytest
import torch

from paper_2104_11125_amd import binding

EINVAL = binding.SCALECOM_EINVAL


def test_null_context_is_refused():
    lib, p = binding.lib(), 0x10000                     # (addresses that are never read: the context is looked at first)
    assert lib.scalecom_embed(None, p, 0, 4, 4, 4, p, 2, 1.0, p, 0, 4) == EINVAL
    assert lib.scalecom_embed_grad(None, p, 2, p, 0, 4, 4, 4, 1.0, p, 0, 4, 0, p, 4096) == EINVAL
    assert lib.scalecom_cross_entropy(None, p, p, 0, 2, 4, 4, 4, 4, p, p, p, p, 4096) == EINVAL
    assert lib.scalecom_cross_entropy_grad(None, p, p, 0, 2, 4, 4, 4, 4, p, p, p, p, p, 4, p, 0, 4, 0, p, 4096) == EINVAL
    assert lib.scalecom_distill(None, p, p, 0, 2, 4, 4, 4, 4, 3, p, p, 0, 1.0, p, p, p, p, 4096) == EINVAL
    assert lib.scalecom_distill_grad(None, p, p, 0, 2, 4, 4, 4, 4, 3, p, p, 0, 1.0, p, p, p, p, 4, p, 0, 4, 0, p, 4096) == EINVAL


@pytest.mark.parametrize("n,vocab,dim,listed,dtype", [(-1, 4, 4, 0, 0), (2 ** 22 + 1, 4, 4, 0, 0), (4, 0, 4, 0, 0), (4, 2 ** 24 + 1, 4, 0, 0), (4, 4, 0, 0, 0),
                                                      (4, 4, 2 ** 16 + 1, 0, 0), (4, 4, 4, -1, 0), (4, 4, 4, 1025, 0), (4, 4, 4, 0, 2),
                                                      (2 ** 22, 4, 4, 129, 0), (2 ** 21, 2 ** 24, 4, 0, 1), (2 ** 62, 4, 4, 0, 0)])
def test_scratch_bytes_of_sizes_out_of_range(n, vocab, dim, listed, dtype):
    assert binding.lib().scalecom_vocab_scratch_bytes(n, vocab, dim, listed, dtype) == 0
    if listed == 0 and dtype == 0 and vocab == 4:
        assert binding.lib().scalecom_embed_grad_scratch_bytes(n, dim) == 0


def test_scratch_bytes():
    lib = binding.lib()
    f, g = lib.scalecom_vocab_scratch_bytes, lib.scalecom_embed_grad_scratch_bytes
    assert g(0, 4) == 256 and 16 * 1000 <= g(1000, 8) and g(65_536, 2048) <= 65_536 * (16 + 2048 * 4 / 8 + 16) + 2 ** 20
    assert f(0, 1, 1, 0, 0) > 0 and f(1, 1, 1, 0, 0) > 0 and f(1, 1, 1, 1024, 1) > 0
    assert f(4, 2 ** 24, 64, 0, 1) > 0 and f(2 ** 20, 1000, 64, 8, 0) > 0
    # no logits of a whole batch: 8192 x 131072 of them in 32 bits are 4.3 GB, in 16 bits 2.1; here dz of a piece, 1 GB at most, beside x and dx
    assert f(8192, 131_072, 4096, 0, 1) < 1.5 * 2 ** 30 + 8192 * 4096 * 16
    # what a token costs beside the pieces does not grow with the vocabulary by more than a part of a sum for every 32 to 128 tokens of it
    assert f(64, 2 ** 24, 64, 0, 1) < 2 ** 30 + 64 * 2 ** 24


class _Ctx(binding.ScaleCom):
    """A binding without a context: what it checks itself comes before any call of the library."""

    def __init__(self):
        self._ctx, self.device, self.stream = None, torch.device("cpu"), None
        self._ortho_scratch, self._ortho_captured = [], False

    def close(self):
        pass

    __del__ = close


def _raises(kind, call, *args, **kw):
    with pytest.raises(kind):
        call(*args, **kw)


def test_binding_refuses_what_does_not_fit(monkeypatch):
    def no_call():
        raise AssertionError("the library was called")

    monkeypatch.setattr(binding, "lib", no_call)
    c = _Ctx()
    w, x = torch.zeros(7, 4), torch.zeros(3, 4)
    ids, f = torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    away = torch.zeros(3, 4, device="meta")
    s = torch.zeros(64, dtype=torch.uint8)

    _raises(TypeError, c.scalecom_embed, w, ids.long())
    _raises(TypeError, c.scalecom_embed, w.half(), ids)
    _raises(TypeError, c.scalecom_embed, w, ids, 1.0, torch.zeros(3, 4, dtype=torch.float64))
    for out in (torch.zeros(3, 5), torch.zeros(2, 4), torch.zeros(12), away, torch.zeros(4, 3).t()):
        _raises(ValueError, c.scalecom_embed, w, ids, 1.0, out)
    _raises(ValueError, c.scalecom_embed, torch.zeros(28), ids)
    _raises(ValueError, c.scalecom_embed, w, torch.zeros(6, dtype=torch.int32)[::2])
    _raises(ValueError, c.scalecom_embed, w, ids.view(3, 1))

    _raises(TypeError, c.scalecom_embed_grad, ids.long(), x, w)
    _raises(TypeError, c.scalecom_embed_grad, ids, x.half(), w)
    for dout, grad in ((torch.zeros(3, 5), w), (torch.zeros(2, 4), w), (x, torch.zeros(28)), (x, torch.zeros(4, 7).t()), (away, w)):
        _raises(ValueError, c.scalecom_embed_grad, ids, dout, grad)
    _raises(ValueError, c.scalecom_embed_grad, ids, x, w, scratch=torch.zeros(64))

    for bad in (dict(x=x.bfloat16()), dict(targets=ids.long()), dict(loss=f.double()), dict(lse=f.bfloat16()), dict(x=x.half(), w=w.half())):
        _raises(TypeError, c.scalecom_cross_entropy, **{**dict(x=x, w=w, targets=ids, loss=f, lse=f.clone(), scratch=s), **bad})
    for bad in (dict(x=torch.zeros(3, 5)), dict(targets=ids[:2]), dict(loss=torch.zeros(4)), dict(lse=torch.zeros(6)[::2]), dict(x=torch.zeros(12)), dict(w=away)):
        _raises(ValueError, c.scalecom_cross_entropy, **{**dict(x=x, w=w, targets=ids, loss=f, lse=f.clone(), scratch=s), **bad})
    good = dict(x=x, w=w, targets=ids, loss=f, lse=f, dloss=f, dx=x.clone(), dw=w.clone(), scratch=s)
    for bad in (dict(dx=x.bfloat16()), dict(dw=w.half()), dict(dloss=f.double())):
        _raises(TypeError, c.scalecom_cross_entropy_grad, **{**good, **bad})
    for bad in (dict(dx=torch.zeros(2, 4)), dict(dw=torch.zeros(7, 5)), dict(dw=torch.zeros(4, 7).t()), dict(dloss=f[:2]), dict(loss=torch.zeros(1)),
                dict(dw=True, accumulate=True), dict(scratch=torch.zeros(64))):
        _raises(ValueError, c.scalecom_cross_entropy_grad, **{**good, **bad})

    lists, teacher, listed = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2), torch.zeros(3, 2)
    good = dict(x=x, w=w, ids=lists, teacher=teacher, loss=f, lse=f.clone(), listed=listed, scratch=s)
    for bad in (dict(ids=lists.long()), dict(teacher=teacher.half()), dict(listed=listed.bfloat16())):
        _raises(TypeError, c.scalecom_distill, **{**good, **bad})
    for bad in (dict(ids=ids), dict(ids=lists[:2]), dict(teacher=teacher[:, :1]), dict(listed=torch.zeros(3, 3)), dict(loss=f[:1])):
        _raises(ValueError, c.scalecom_distill, **{**good, **bad})
    good = dict(x=x, w=w, ids=lists, teacher=teacher, temperature=1.0, lse=f, listed=listed, dloss=f, dx=x.clone(), dw=w.clone(), scratch=s)
    for bad in (dict(listed=torch.zeros(2, 3)), dict(lse=f[:2]), dict(dx=w), dict(dw=True, accumulate=True)):
        _raises(ValueError, c.scalecom_distill_grad, **{**good, **bad})


def test_binding_refuses_sizes_before_a_launch():
    c = _Ctx()
    w, ids = torch.zeros(7, 0), torch.zeros(3, dtype=torch.int32)
    _raises(binding.ScaleComError, c.scalecom_embed_grad, ids, torch.zeros(3, 0), w)
    _raises(binding.ScaleComError, c.scalecom_cross_entropy, torch.zeros(3, 0), w, ids, torch.zeros(3), torch.zeros(3))
    _raises(binding.ScaleComError, c.scalecom_cross_entropy, torch.zeros(3, 4), torch.zeros(0, 4), ids, torch.zeros(3), torch.zeros(3))
    _raises(binding.ScaleComError, c.scalecom_distill, torch.zeros(1, 4), torch.zeros(5, 4), torch.zeros(1, 1025, dtype=torch.int32), torch.zeros(1, 1025), 1.0,
            torch.zeros(1), torch.zeros(1), torch.zeros(1, 1025))
