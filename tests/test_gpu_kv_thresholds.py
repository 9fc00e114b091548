"""Writing the 4-bit cache on the GPU where a boundary times a block's scale is too small for 32 bits: the oracle's bytes all the same."""
import numpy as np
import pytest

from oracle import kv as okv
from tests.kv_util import Case, patterns
from tests.test_gpu_kv_cache import check

pytestmark = pytest.mark.gpu

BOOKS = [
    # boundaries on both sides of zero, the innermost -5e-31 and 5e-31
    [-1.0, -0.5, -0.25, -1e-3, -1e-10, -1e-20, -1e-30, 0.0, 1e-30, 1e-20, 1e-10, 1e-3, 0.25, 0.5, 0.75, 1.0],
    # around the line from which on 64 bits are taken, 2^-40, and near the smallest numbers of bf16
    [-1.0, -2.0 ** -38, -2.0 ** -39, -2.0 ** -40, -2.0 ** -41, -2.0 ** -42, -2.0 ** -130, 0.0, 2.0 ** -133, 2.0 ** -126, 2.0 ** -42, 2.0 ** -41, 2.0 ** -40, 2.0 ** -39, 2.0 ** -38, 1.0],
    # nothing but tiny ones
    [-(2.0 ** -100)] * 4 + [-(2.0 ** -110)] * 3 + [2.0 ** -120] * 3 + [2.0 ** -90, 2.0 ** -80, 2.0 ** -70, 2.0 ** -60, 2.0 ** -50, 2.0 ** -45],
]


@pytest.mark.parametrize("book", range(len(BOOKS)))
@pytest.mark.parametrize("kv", (0, 1))
@pytest.mark.parametrize("rows", (3, 130))
def test_tiny_boundaries(book, kv, rows):
    """K's or V's codebook has them and the other's has not; blocks with scales from 2^-133 to 2^120, most of them between 2^-60 and 2^-50, hold zeros of
    both signs, the smallest numbers, and numbers on and beside every boundary."""
    print(f"tiny boundaries: book {book} kv {kv} rows {rows}", flush=True)
    c = Case(60 + book, [rows], [rows], 32, 2, 128)
    g = np.random.default_rng(61 + rows)
    c.books[kv] = patterns(BOOKS[book])
    x = [patterns(g.standard_normal((rows, 2, 128))) for _ in range(2)]
    blocks = x[kv].reshape(-1, 64)
    power = np.where(g.random(len(blocks)) < 0.7, g.integers(-60, -49, len(blocks)), g.integers(-133, 121, len(blocks)))
    scale = patterns(2.0 ** power)
    with np.errstate(under="ignore"):
        edge = patterns(np.outer(okv.bf16_value(scale), okv.boundaries(c.books[kv])))
    blocks[:, 1:16], blocks[:, 16:31], blocks[:, 31:46] = edge, edge + (edge & 0x7FFF != 0), edge - (edge & 0x7FFF != 0)
    blocks[:, 46:52], blocks[:, 52:58], blocks[:, 58:61], blocks[:, 61:64] = 0, 0x8000, 0x0001, 0x8001
    blocks[:, 0] = scale
    blocks[(blocks & 0x7FFF) > scale[:, None]] = 0
    assert (blocks == 0).any(1).all()
    check(c, *x)
