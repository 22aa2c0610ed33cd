"""The scratch of the losses over a vocabulary is what the header says: it grows with the tokens as x and dx do, and dz's part of it is bounded."""
import pytest

from paper_2104_11125_amd import binding

F32, BF16 = binding.SCALECOM_GRAD_F32, binding.SCALECOM_GRAD_BF16
GB, MB, SHARED = 2 ** 30, 2 ** 20, 70 * 10 ** 6


def up_to(v, a):
    return -(-v // a) * a


def _most(n, vocab, dim, listed, dtype):
    """The header's account, with rows and columns rounded up to whole tiles and some columns behind them."""
    rows, cols, planes = up_to(max(n, 1), 256), up_to(dim, 128) + 64, 3 if dtype == F32 else 1
    piece = min(up_to(vocab, 256), 2 ** 18)
    x = rows * cols * 2 * planes
    w = min(piece * cols * 2 * planes, max(512 * MB * 1.5, 16384 * cols * 2 * planes))
    dz = min(rows * (piece + 32) * 6, max(GB, rows * 2048 * 6) + rows * 32 * 6)
    dx = rows * cols * 4 + SHARED
    dw = SHARED + (w * 2 / planes if dim % 4 else 0)
    small = 64 * rows + 4 * n * listed + 4096
    return max(x + w + dz + dx + dw, x + w + 8 * rows * (vocab // (32 if n <= 64 else 64) + 4)) + small


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 8, 64, 65, 500, 4096, 8192, 11_000, 32_768, 33_000, 65_536, 131_072, 300_000, 2 ** 20, 2 ** 22])
def test_as_the_header_states_it(n, dtype):
    f = binding.lib().scalecom_vocab_scratch_bytes
    for vocab in (1, 300, 10_007, 32_768, 131_072, 300_000, 2 ** 24):
        for dim in (1, 64, 333, 512, 4096, 4095, 65_536):
            for listed in (0, 64):
                if n * vocab > 2 ** 44 or n * listed > 2 ** 29:
                    continue
                got = f(n, vocab, dim, listed, dtype)
                assert 0 < got <= _most(n, vocab, dim, listed, dtype), (n, vocab, dim, listed, got, _most(n, vocab, dim, listed, dtype))


def test_many_tokens():
    """dz of 16384 rows of the vocabulary for all of them was 97 GB in the first of these."""
    f = binding.lib().scalecom_vocab_scratch_bytes
    assert f(2 ** 20, 131_072, 64, 0, BF16) < 15 * GB
    assert f(65_536, 131_072, 4096, 0, BF16) < 3.2 * GB
    assert f(131_072, 32_768, 4096, 0, F32) < 8.5 * GB


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_loss_alone(dtype):
    """A loss without its gradient needs x, the piece's planes of an output matrix that is not read as it lies, and parts of its sums."""
    f, both = binding.lib().scalecom_vocab_loss_scratch_bytes, binding.lib().scalecom_vocab_scratch_bytes
    planes = 3 if dtype == F32 else 1
    for n in (0, 1, 8, 64, 65, 4096, 33_000, 2 ** 20):
        for vocab in (1, 300, 131_072, 2 ** 24):
            for dim in (1, 333, 4096):
                for address, stride in ((0, dim), (16, dim + 8), (2, dim), (0, dim + 1)):
                    rows, cols = up_to(max(n, 1), 256), up_to(dim, 128) + 64
                    as_it_lies = dtype == BF16 and dim % 128 == 0 and address % 16 == 0 and stride % 8 == 0
                    w = 0 if as_it_lies else min(up_to(vocab, 256) * cols * 2 * planes, max(768 * MB, 16384 * cols * 2 * planes))
                    most = rows * cols * 2 * planes + w + 8 * rows * (vocab // (32 if n <= 64 else 64) + 4) + 64 * rows + 4096
                    got = f(n, vocab, dim, 0, address, stride, dtype)
                    assert 0 < got <= min(most, both(n, vocab, dim, 0, dtype)), (n, vocab, dim, address, stride)
    # a few tokens: 2 MB of x and 4 of parts, not the 650 MB of a gradient
    assert dtype == F32 or f(8, 131_072, 4096, 0, 0, 4096, dtype) < 8 * MB
    for bad in ((-1, 4, 4, 0, 0, 4), (4, 0, 4, 0, 0, 4), (4, 4, 2 ** 16 + 1, 0, 0, 2 ** 17), (4, 4, 4, 1025, 0, 4), (2 ** 21, 2 ** 24, 4, 0, 0, 4), (4, 4, 4, 0, 0, 3)):
        assert f(*bad, dtype) == 0
    assert f(4, 4, 4, 0, 0, 4, 2) == 0
