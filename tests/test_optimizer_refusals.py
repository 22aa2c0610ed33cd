"""What the optimiser operators refuse without touching a device: null contexts, sizes that are out of range, and what the
binding sees by itself."""
import ctypes

import pytest
import torch

from paper_2104_11125_amd import binding

EINVAL = binding.SCALECOM_EINVAL


def _i64(*values):
    return (ctypes.c_int64 * len(values))(*values)


def test_null_context_is_refused():
    lib = binding.lib()
    one, f = _i64(1), (ctypes.c_float * 3)(1.5, -0.5, 0.0)
    p = ctypes.c_void_p(0x10000)                        # never read: the context is looked at first
    assert lib.scalecom_momentum_update(None, p, 4, p, p, 1, 1.0, 0.9, 1, p, 0) == EINVAL
    assert lib.scalecom_orthogonalize(None, 1, 1, one, one, one, None, p, 0, p, 0, 1, f, 1e-7, p, 256) == EINVAL
    assert lib.scalecom_apply_tensors(None, p, 1, 1, one, one, one, None, p, 0, f, 1.0) == EINVAL


@pytest.mark.parametrize("rows,cols", [([-1], [4]), ([4], [-1]), ([16385], [16385]), ([1], [4194305]), ([4194305], [1]),
                                       ([2 ** 40], [1]), ([4, 4, 2 ** 62], [4, 4, 2 ** 62])])
def test_scratch_bytes_of_sizes_out_of_range(rows, cols):
    assert binding.lib().scalecom_orthogonalize_scratch_bytes(len(rows), _i64(*rows), _i64(*cols)) == 0


def test_scratch_bytes_of_other_arguments():
    f = binding.lib().scalecom_orthogonalize_scratch_bytes
    assert f(0, _i64(4), _i64(4)) == 0 and f(-3, _i64(4), _i64(4)) == 0
    assert f(1, None, _i64(4)) == 0 and f(1, _i64(4), None) == 0
    assert f(1, _i64(0), _i64(5)) == 256 and f(1, _i64(1), _i64(1)) >= 256
    assert f(1, _i64(16384), _i64(16384)) >= 16 * 16384 ** 2
    assert f(1, _i64(1), _i64(4194304)) > 0 and f(1, _i64(100), _i64(4194304)) >= 8 * 100 * 4194304
    n = 96
    many = f(n, _i64(*[512] * n), _i64(*[2048] * n))
    assert n * 8 * (512 * 2048 + 512 * 512) <= many <= 1.1 * n * 8 * (512 * 2048 + 512 * 512)


class _Ctx(binding.ScaleCom):
    """A binding without a context: what it checks itself comes before any call of the library."""

    def __init__(self):
        self._ctx, self.device, self.stream = None, torch.device("cpu"), None
        self._ortho_scratch, self._ortho_bytes = [], (None, None, 0)

    def close(self):
        pass

    __del__ = close


def test_binding_refuses_what_does_not_fit(monkeypatch):
    def no_call():
        raise AssertionError("the library was called")

    monkeypatch.setattr(binding, "lib", no_call)
    ctx = _Ctx()
    m, idx, vals = torch.zeros(8), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    for args in [(m.double(), idx, vals), (m, idx.long(), vals), (m, idx, vals.bfloat16())]:
        with pytest.raises(TypeError):
            ctx.scalecom_momentum_update(*args, 1.0, 0.9)
    for args, out in [((m, idx, vals[:1]), None), ((m, idx, vals), torch.zeros(7)), ((torch.zeros(16)[::2], idx, vals), None),
                      ((m, idx, torch.zeros(4)[::2]), None), ((m, idx, vals), torch.zeros(16)[::2])]:
        with pytest.raises(ValueError):
            ctx.scalecom_momentum_update(*args, 1.0, 0.9, True, out)
    with pytest.raises(TypeError):
        ctx.scalecom_momentum_update(m, idx, vals, 1.0, 0.9, True, torch.zeros(8, dtype=torch.float16))
    with pytest.raises(ValueError):                      # another device
        ctx.scalecom_momentum_update(torch.zeros(8, device="meta"), idx, vals, 1.0, 0.9)

    u = torch.zeros(12)
    for kw in [dict(offsets=[0, 1], rows=[3], cols=[4]), dict(offsets=[0], rows=[3], cols=[4, 4]),
               dict(offsets=[0], rows=[3], cols=[4], strides=[4, 4]), dict(offsets=[0], rows=[3], cols=[4], out=torch.zeros(11)),
               dict(offsets=[0], rows=[3], cols=[4], coeffs=[(1.5, -0.5)]),
               dict(offsets=[0], rows=[3], cols=[4], scratch=torch.zeros(4096)),
               dict(offsets=[0], rows=[3], cols=[4], scratch=torch.zeros(4096, dtype=torch.uint8)[::2])]:
        with pytest.raises(ValueError):
            ctx.scalecom_orthogonalize(u, **kw)
    with pytest.raises(ValueError):
        ctx.scalecom_orthogonalize(torch.zeros(24)[::2], [0], [3], [4])

    for kw in [dict(offsets=[0, 1], rows=[3], cols=[4], scales=[1.0]), dict(offsets=[0], rows=[3], cols=[4], scales=[1.0, 2.0]),
               dict(offsets=[0], rows=[3], cols=[4], scales=[1.0], strides=[])]:
        with pytest.raises(ValueError):
            ctx.scalecom_apply_tensors(u, torch.zeros(12), **kw)
    with pytest.raises(ValueError):
        ctx.scalecom_apply_tensors(u, torch.zeros(11), [0], [3], [4], [1.0])
    with pytest.raises(TypeError):
        ctx.scalecom_apply_tensors(u.bfloat16(), torch.zeros(12), [0], [3], [4], [1.0])


def test_binding_refuses_types_and_sizes_before_a_launch():
    ctx = _Ctx()
    with pytest.raises(TypeError):
        ctx.scalecom_orthogonalize(torch.zeros(12, dtype=torch.float16), [0], [3], [4], scratch=torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(TypeError):
        ctx.scalecom_apply_tensors(torch.zeros(12), torch.zeros(12, dtype=torch.int32), [0], [3], [4], [1.0])
    with pytest.raises(binding.ScaleComError):           # no matrices
        ctx.scalecom_orthogonalize(torch.zeros(12), [], [], [])
    with pytest.raises(binding.ScaleComError):           # too large a side
        ctx.scalecom_orthogonalize(torch.zeros(12), [0], [16385], [16385])
