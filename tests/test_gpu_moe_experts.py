"""The experts' kernels against the oracle."""
import numpy as np
import pytest
import torch

from paper_2602_15563_amd import kmq
from tests.moe_util import NAN16, Experts, check_experts, dev, host, patterns, rows_on_device, run_experts

pytestmark = pytest.mark.gpu

UNIT = {1: 512, 2: 256, 3: 128, 4: 128}


def choices(g, rows, experts, top_k):
    """Different experts for every token."""
    ids = np.argsort(g.random((rows, experts)), axis=1)[:, :top_k].astype(np.int32)
    return ids, g.uniform(0.05, 0.6, (rows, top_k)).astype(np.float32)


def tokens(g, rows, hidden):
    return patterns(g.standard_normal((rows, hidden)))


@pytest.fixture(scope="module")
def layers():
    """Made once for a size: packing on the host takes longest."""
    made = {}

    def get(*key):
        if key not in made:
            e = Experts(sum(int(k) * 31 ** i for i, k in enumerate(key)) % 10007, *key)
            made[key] = (e, e.on_device())
        return made[key]
    return get


@pytest.mark.parametrize("rows", (1, 2, 7, 16, 17, 31, 48, 64, 65, 128))
@pytest.mark.parametrize("bits", (1, 2, 3, 4))
def test_rows(layers, bits, rows):
    e, w = layers(12, 512, 512, bits)
    g = np.random.default_rng(100 * bits + rows)
    ids, gates = choices(g, rows, 12, 4)
    x, res = tokens(g, rows, 512), tokens(g, rows, 512)
    check_experts(e, run_experts(w, x, ids, gates, res), x, ids, gates, res, f"{bits} bits, {rows} rows")
    check_experts(e, run_experts(w, x, ids, gates, x_stride=520, y_stride=776), x, ids, gates, None, f"{bits} bits, {rows} rows, no residual")


@pytest.mark.parametrize("bits", (1, 2, 3, 4))
@pytest.mark.parametrize("hidden,width", ((1, 1), (1, 5), (3, 1), (9, 2), (2, 17), (5, 7), (33, 1), (1, 33), (17, 2)))
def test_sizes(layers, bits, hidden, width):
    """In whole super-blocks: fewer of them than waves, numbers that do not share evenly, rows of more than one piece of scales."""
    if bits == 1 and hidden * width > 30:
        pytest.skip("the others cover it")
    e, w = layers(3, hidden * UNIT[bits], width * UNIT[bits], bits)
    g = np.random.default_rng(hidden * 10 + width)
    for rows in (1, 5, 20):
        ids, gates = choices(g, rows, 3, 2)
        x = tokens(g, rows, e.hidden)
        check_experts(e, run_experts(w, x, ids, gates), x, ids, gates, None, f"{e.hidden} x {e.width}, {rows} rows")


@pytest.mark.parametrize("bits", (1, 2, 3, 4))
@pytest.mark.parametrize("hidden,width", ((16, 1), (1, 17), (31, 1)))
def test_few_long_rows(layers, bits, hidden, width):
    """Eight waves a row, one to four super-blocks each."""
    e, w = layers(3, hidden * UNIT[bits], width * UNIT[bits], bits)
    g = np.random.default_rng(hidden + 50 * width)
    for rows in (1, 3, 5, 8):
        ids, gates = choices(g, rows, 3, 2)
        x, res = tokens(g, rows, e.hidden), tokens(g, rows, e.hidden)
        check_experts(e, run_experts(w, x, ids, gates, res), x, ids, gates, res, f"{e.hidden} x {e.width}, {rows} rows")


@pytest.mark.parametrize("bits,hidden,width", [(b, *s) for b in (1, 2, 3, 4) for s in ((2560, 512), (512, 2560))] + [(3, 640, 384), (4, 640, 384)])
def test_many_tokens_of_many_experts(bits, hidden, width):
    """Work for every unit: up to 16 tokens at a time and more, rows of one piece and of several, numbers of them that teams do not share evenly."""
    e = Experts(bits, 4, hidden, width, bits)
    of = np.arange(40) % 4                                                       # 40 experts that are four
    pick = torch.from_numpy(of).cuda()
    w = kmq.MoeWeights(*(t[pick].contiguous() for t in e.on_device().tensors), 40, hidden, width, bits)
    g = np.random.default_rng(hidden + bits)
    ids, gates = choices(g, 70, 40, 8)
    ids[:, 7][(ids[:, :7] != 33).all(1)] = 33                                    # one that all tokens have
    x, res = tokens(g, 70, hidden), tokens(g, 70, hidden)
    got = run_experts(w, x, ids, gates, res)
    check_experts(e, got, x, of[ids].astype(np.int32), gates, res, "", range(0, 70, 6))
    assert np.array_equal(run_experts(w, x, ids, gates, res), got)


@pytest.mark.parametrize("bits", (2, 4))
@pytest.mark.parametrize("experts,top_k,rows", ((1, 1, 1), (1, 1, 40), (2, 1, 128), (64, 16, 3), (64, 16, 128), (200, 10, 9)))
def test_numbers_of_experts(layers, bits, experts, top_k, rows):
    e, w = layers(experts, 256, 256, bits)
    g = np.random.default_rng(experts + top_k)
    ids, gates = choices(g, rows, experts, top_k)
    x, res = tokens(g, rows, 256), tokens(g, rows, 256)
    mine = range(0, rows, max(1, rows // 12))
    check_experts(e, run_experts(w, x, ids, gates, res), x, ids, gates, res, f"{experts} experts, {rows} rows", mine)


@pytest.mark.parametrize("bits", (1, 2, 3, 4))
@pytest.mark.parametrize("rows,top_k", ((16, 8), (9, 16), (16, 16), (5, 13)))
def test_many_short_rows(layers, bits, rows, top_k):
    """More row blocks than run at once; experts with 4, 8 and 16 tokens and more at a time."""
    e, w = layers(128, 512, 512, bits)
    g = np.random.default_rng(rows * top_k)
    ids, gates = choices(g, rows, 128, top_k)
    ids[:, 0] = 77                                                               # one expert that all tokens have
    ids[1:, 1:][ids[1:, 1:] == 77] = 5
    x = tokens(g, rows, 512)
    got = run_experts(w, x, ids, gates)
    check_experts(e, got, x, ids, gates, None, f"{rows} rows", range(0, rows, 3))


def test_most_of_everything():
    """128 rows of 16 of 1024 experts: the longest list there is."""
    e = Experts(91, 4, 256, 128, 4)
    one = e.on_device()
    of = np.random.default_rng(1).integers(0, 4, 1024)                           # 1024 experts that are four
    pick = torch.from_numpy(of).cuda()
    w = kmq.MoeWeights(*(t[pick].contiguous() for t in one.tensors), 1024, 256, 128, 4)
    g = np.random.default_rng(2)
    ids, gates = choices(g, 128, 1024, 16)
    x, res = tokens(g, 128, 256), tokens(g, 128, 256)
    got = run_experts(w, x, ids, gates, res)
    check_experts(e, got, x, of[ids].astype(np.int32), gates, res, "", range(0, 128, 9))
    all_same = np.tile(np.arange(0, 1024, 64, dtype=np.int32), (128, 1))
    check_experts(e, run_experts(w, x, all_same, gates), x, of[all_same].astype(np.int32), gates, None, "", range(0, 128, 9))


@pytest.mark.parametrize("bits", (1, 2, 3, 4))
@pytest.mark.parametrize("rows", (16, 100, 128))
def test_all_tokens_choose_the_same(layers, bits, rows):
    e, w = layers(12, 512, 512, bits)
    g = np.random.default_rng(rows)
    ids, gates = np.tile(np.array([[11, 0, 5]], dtype=np.int32), (rows, 1)), g.uniform(0.1, 0.5, (rows, 3)).astype(np.float32)
    x = tokens(g, rows, 512)
    check_experts(e, run_experts(w, x, ids, gates), x, ids, gates, None, f"{rows} rows", range(0, rows, 7))


@pytest.mark.parametrize("bits,hidden,width", ((1, 9, 10), (2, 17, 9), (3, 17, 34), (4, 18, 9)))
def test_more_tokens_than_sixteen_over_several_pieces(layers, bits, hidden, width):
    """Experts with up to three times 16 tokens, rows of several pieces, calls that agree bit for bit."""
    e, w = layers(3, hidden * UNIT[bits], width * UNIT[bits], bits)
    g = np.random.default_rng(bits)
    ids, gates = choices(g, 40, 3, 2)
    ids[:, 0], ids[:, 1] = 1, np.where(np.arange(40) % 3 == 0, 2, 0)
    x, res = tokens(g, 40, e.hidden), tokens(g, 40, e.hidden)
    got = run_experts(w, x, ids, gates, res)
    check_experts(e, got, x, ids, gates, res, f"{e.hidden} x {e.width}", range(0, 40, 5))
    for _ in range(3):
        assert np.array_equal(run_experts(w, x, ids, gates, res), got)


@pytest.mark.parametrize("rows", (1, 9, 40))
def test_ids_that_are_none_and_experts_chosen_twice(layers, rows):
    e, w = layers(12, 512, 512, 3)
    g = np.random.default_rng(rows)
    ids, gates = choices(g, rows, 12, 6)
    ids[:, 1], ids[:, 4] = -1, 12
    ids[0, 2], ids[0, 5] = ids[0, 0], ids[0, 0]                                  # three times the same
    ids[-1, 3], gates[-1, 3] = np.int32(-2 ** 31), np.nan                        # what counts for nothing may hold anything
    ids[rows // 2, 5] = np.int32(2 ** 31 - 1)
    x, res = tokens(g, rows, 512), tokens(g, rows, 512)
    check_experts(e, run_experts(w, x, ids, gates, res), x, ids, np.nan_to_num(gates), res, "some")
    none = np.full((rows, 6), -1, dtype=np.int32)
    assert np.array_equal(run_experts(w, x, none, gates, res), res)
    assert (run_experts(w, x, none, gates) == 0).all()


def test_residual_in_its_own_place(layers):
    e, w = layers(12, 512, 512, 4)
    g = np.random.default_rng(4)
    ids, gates = choices(g, 20, 12, 3)
    x, res = tokens(g, 20, 512), tokens(g, 20, 512)
    y, ws = rows_on_device(res, 1024), torch.empty(kmq.moe_experts_workspace_bytes(w, 20, 3), dtype=torch.uint8, device="cuda")
    kmq.moe_experts(w, dev(x), 512, 20, dev(ids), dev(gates), 3, y, 1024, residual=y, residual_stride=1024, workspace=ws)
    torch.cuda.synchronize()
    got = host(y)
    assert (got[:, 512:] == NAN16).all()
    check_experts(e, got[:, :512], x, ids, gates, res)


@pytest.mark.parametrize("bits", (1, 2, 3, 4))
@pytest.mark.parametrize("rows", (6, 40))
def test_what_is_not_finite_stays_where_it_is(bits, rows):
    """Experts that nobody chose, tokens of NaN, an expert of NaN: only what they concern is not finite, the rest is as it was, bit for bit."""
    e = Experts(50 + bits, 7, 512, 512, bits, poison=(2,))
    w = e.on_device()
    g = np.random.default_rng(bits)
    ids, gates = choices(g, rows, 7, 3)
    ids[ids == 2] = -1
    x = tokens(g, rows, 512)
    clean = run_experts(w, x, ids, gates)
    check_experts(e, clean, x, ids, gates, None, "one expert is all NaN")
    bad, bad_ids = x.copy(), ids.copy()
    bad[1], bad[3, 5] = NAN16, 0x7F80
    bad_ids[4, 0] = 2
    got = run_experts(w, bad, bad_ids, gates)
    hit = np.zeros(rows, dtype=bool)
    hit[[1, 3, 4]] = True
    value = (got.astype(np.uint32) << 16).view(np.float32)
    assert np.isnan(value[[1, 4]]).all() and not np.isfinite(value[3]).all()
    check_experts(e, got, bad, bad_ids, gates, None, "beside them", np.nonzero(~hit)[0])


def test_a_token_of_nan_changes_no_other(layers):
    """The same choices, so the same sums: bit for bit."""
    for bits in (1, 2, 3, 4):
        e, w = layers(12, 512, 512, bits)
        g = np.random.default_rng(bits)
        ids, gates = choices(g, 33, 12, 4)
        x = tokens(g, 33, 512)
        bad = x.copy()
        bad[[0, 8, 32]] = NAN16
        a, b = run_experts(w, x, ids, gates), run_experts(w, bad, ids, gates)
        rest = np.setdiff1d(np.arange(33), [0, 8, 32])
        assert np.array_equal(a[rest], b[rest])
        assert (run_experts(w, x, ids, gates) == a).all(), "repeats are the same bits"


def test_infinite_centroids_and_gates(layers):
    """An infinity that a token meets makes it not finite; padding of its tile meets none of it."""
    e = Experts(71, 3, 512, 512, 4)
    e.books[0][1][-1] = 0x7F80
    e.books[2][2][0] = 0xFF80
    w = e.on_device()
    g = np.random.default_rng(1)
    x = tokens(g, 3, 512)
    ids, gates = np.array([[0], [1], [2]], dtype=np.int32), np.ones((3, 1), dtype=np.float32)
    got = run_experts(w, x, ids, gates)
    value = (got.astype(np.uint32) << 16).view(np.float32)
    check_experts(e, got, x, ids, gates, None, "beside", [0])
    assert not np.isfinite(value[1]).all() and not np.isfinite(value[2]).all()
    gates[0] = np.inf
    assert not np.isfinite((run_experts(w, x, ids, gates)[0].astype(np.uint32) << 16).view(np.float32)).any()


def test_words_beyond_32_bit_offsets():
    """An expert that starts 5 GB behind the first: one buffer serves as all three matrices."""
    size, bits, experts = 4096, 4, 640
    e = Experts(81, 1, size, size, bits)
    one = e.on_device()
    words = torch.zeros((experts, size * size // 8), dtype=torch.int32, device="cuda")
    words[-1] = one.tensors[0][0]
    books = torch.zeros((experts, 16), dtype=torch.int16, device="cuda")
    books[-1] = one.tensors[3][0]
    scales = torch.full((experts, size, size // 64), NAN16, dtype=torch.int16, device="cuda")
    scales[-1] = one.tensors[6][0].view(size, size // 64)
    w = kmq.MoeWeights(words, words, words, books, books, books, scales, scales, scales, experts, size, size, bits)
    for m in (1, 2):
        e.idx[m], e.books[m], e.scales[m] = e.idx[0], e.books[0], e.scales[0]
    g = np.random.default_rng(2)
    x = tokens(g, 2, size)
    got = run_experts(w, x, np.array([[experts - 1], [-1]], dtype=np.int32), np.ones((2, 1), dtype=np.float32))
    check_experts(e, got, x, np.array([[0], [-1]], dtype=np.int32), np.ones((2, 1), dtype=np.float32))
