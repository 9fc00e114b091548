"""What is not finite stays with the tokens that it concerns: the outputs of all others are the same bits as without it."""
import numpy as np
import pytest

from tests.moe_util import NAN16, Experts, check_experts, patterns, run_experts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    made = {}

    def get(bits):
        if bits not in made:
            e = Experts(60 + bits, 9, 1024, 512, bits, poison=(2,))
            e.books[1][5][:] = 0x7F80                                             # an up projection of infinities
            made[bits] = e, e.on_device()
        return made[bits]
    return get


@pytest.mark.parametrize("bits", (1, 2, 3, 4))
@pytest.mark.parametrize("rows,top_k", ((5, 2), (8, 4), (16, 7), (40, 3), (128, 2)))
def test_all_others_are_the_same_bits(layers, bits, rows, top_k):
    """Four, eight and sixteen tokens at a time, with fewer of them than there is room for, and with turns of their own."""
    e, w = layers(bits)
    g = np.random.default_rng(100 * bits + rows)
    ids, gates = np.argsort(g.random((rows, 9)), axis=1)[:, :top_k].astype(np.int32), g.uniform(0.05, 0.6, (rows, top_k)).astype(np.float32)
    ids[(ids == 2) | (ids == 5)] = -1
    x = patterns(g.standard_normal((rows, 1024)))
    clean = run_experts(w, x, ids, gates)
    check_experts(e, clean, x, ids, gates, None, "nobody's experts hold no number", range(0, rows, -(-rows // 8)))
    concerned = np.zeros(rows, dtype=bool)

    def check(at, x, ids, gates, label):
        got = run_experts(w, x, ids, gates)
        concerned[:] = False
        concerned[at] = True
        assert np.array_equal(got[~concerned], clean[~concerned]), f"{label}: {np.nonzero((got != clean).any(1) & ~concerned)[0]} are others"
        value = (got[concerned].astype(np.uint32) << 16).view(np.float32)
        assert not np.isfinite(value).all(1).any(), f"{label}: finite"

    ids[0, 0], ids[3, 0] = 0, 1                                                   # (so that some expert meets them)
    clean = run_experts(w, x, ids, gates)
    bad = x.copy()
    bad[0] = NAN16
    check([0], bad, ids, gates, "a token of NaN")
    bad = x.copy()
    bad[3, 700] = 0x7F80
    check([3], bad, ids, gates, "an infinite element")
    for expert, label in ((2, "an expert of NaN"), (5, "an expert of infinities")):
        other = ids.copy()
        other[4, 0] = expert
        check([4], x, other, gates, label)
    other = gates.copy()
    other[3, 0] = np.inf
    check([3], x, ids, other, "an infinite gate")
    bad, both, other = x.copy(), ids.copy(), gates.copy()
    bad[0], bad[rows - 2, 3], both[4, 0], both[rows - 1, top_k - 1], other[3, 0] = NAN16, 0xFF80, 2, 5, np.nan
    both[rows - 2, 0] = 0
    clean = run_experts(w, x, np.where((both == 2) | (both == 5), -1, both), gates)
    check([0, rows - 2, 4, rows - 1, 3], bad, both, other, "all of it")
