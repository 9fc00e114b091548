"""Attention over the 4-bit cache (kmq_kv_attention) where the tokens go into parts that a second kernel joins: a NaN that a row sees reaches
it from any part, whichever of the two joining kernels runs."""
import numpy as np
import pytest

from oracle import kv as okv
from paper_2602_15563_amd import kmq
from paper_2602_15563_amd.tolerance import attention_bound, attention_lse_bound
from tests.kv_util import Case, patterns, run_attention

pytestmark = pytest.mark.gpu

ONE, TWO, TILE = "kv_attention", "kv_attention_two", "kv_attention_tile"
NAN = 0x7FC1


def compare(c, q, scale, label, causal=True, window=0):
    """Every row against the oracle: NaN and infinities where it has them, the bounds elsewhere.  Returns outputs, log-sum-exps and the oracle's."""
    got, lse = run_attention(c, q, q.shape[1], scale, causal, window)
    value, outs, lses = okv.bf16_value(got), np.zeros(got.shape), np.zeros(lse.shape)
    for b, n in enumerate(c.news):
        if not n:
            continue
        k, v, there = okv.sequence(c.pages, c.table[b], c.lengths[b], c.books)
        mine = slice(c.starts[b], c.starts[b + 1])
        with np.errstate(invalid="ignore", over="ignore"):
            out, want, spread, size = okv.attention(q[mine], k, v, there, c.lengths[b], scale, causal, window)
            most, far = attention_bound(out, spread, size, max(1, len(there)), c.D), attention_lse_bound(size, max(1, len(there)), c.D)
        for what, g, w, bound in (("output", value[mine], out, most), ("log-sum-exp", lse[mine], want, far)):
            assert np.array_equal(np.isnan(g), np.isnan(w)), f"{label}: sequence {b}: {int(np.isnan(g).sum())} NaN, the oracle has {int(np.isnan(w).sum())} ({what})"
            some = np.isfinite(w)
            assert np.array_equal(g[~some], w[~some], equal_nan=True), f"{label}: sequence {b}: {what}"
            assert (np.abs(g[some] - w[some]) <= bound[some]).all(), f"{label}: sequence {b}: {what}"
        outs[mine], lses[mine] = out, want
    return value, lse, outs, lses


def spoil(c, token, kv, head=0, block=0, bits=NAN):
    """The scale of a block of K (kv = 0) or V (kv = 1) of a token of the first sequence."""
    page, place = okv.place(c.table[0], c.page_size, c.num_pages, token)
    at = c.pages.places(page, place)[4][head, kv, block]
    c.pages.bytes[at], c.pages.bytes[at + 1] = bits & 0xFF, bits >> 8


def parts_of(c, q_heads):
    """Parts of the tokens, and tokens of a part (the last row's)."""
    bytes_ = kmq.kv_attention_workspace_bytes(c.cache, c.batch, q_heads)
    parts = bytes_ // (4 * c.rows * q_heads * (c.D + 2))
    steps = -(-max(c.lengths) // 32)
    return parts, 32 * max(8, -(-steps // max(parts, 1)))


# kernel, rows, tokens, head size, query heads a key head, table width (pages of 32), more than the few parts that one thread passes over
CASES = [
    (ONE, 1, 257, 128, 3, None, False), (ONE, 1, 257, 64, 3, None, False), (ONE, 1, 257, 256, 3, None, False), (ONE, 3, 1500, 256, 2, None, False),
    (ONE, 1, 3000, 64, 2, None, True), (ONE, 1, 3000, 128, 4, None, True), (ONE, 1, 3000, 256, 3, None, True), (ONE, 2, 5000, 256, 5, None, True),
    (TWO, 9, 1900, 128, 3, 64, False), (TWO, 9, 1900, 64, 3, 64, False), (TWO, 20, 2500, 128, 1, None, True), (TWO, 20, 2500, 64, 1, None, True),
    (TILE, 300, 5000, 64, 1, None, True), (TILE, 300, 4000, 128, 1, None, True), (TILE, 150, 3000, 256, 1, None, True),
    (TILE, 250, 1500, 64, 3, None, False), (TILE, 250, 1500, 128, 3, None, False), (TILE, 250, 1500, 256, 3, None, False),
]


def case(seed, kernel, rows, tokens, D, group, width):
    print(f"parts: {kernel} rows={rows} tokens={tokens} D={D} group={group} width={width}", flush=True)
    return Case(seed, [rows], [tokens], 32, 2, D, width=width)


def check_kernel(c, kernel, group, many):
    c.to_device()
    assert kmq.kernel_name_kv_attention(c.cache, c.batch, 2 * group) == kernel
    parts, tokens = parts_of(c, 2 * group)
    assert (parts > 8) == many and parts > 1
    return tokens


@pytest.mark.parametrize("kernel,rows,tokens,D,group,width,many", CASES)
@pytest.mark.parametrize("where", ("first", "last"))
def test_a_part_of_nan_scores_reaches_its_rows(kernel, rows, tokens, D, group, width, many, where):
    """Every score of a part is a NaN: of the first part for all rows, or of the newest token alone, which is the last part's only one where
    257 tokens go into two parts."""
    c = case(900 + D, kernel, rows, tokens, D, group, width)
    per = check_kernel(c, kernel, group, many)
    for t in range(per) if where == "first" else [tokens - 1]:
        spoil(c, t, 0)
    c.to_device()
    q = patterns(np.random.default_rng(901).standard_normal((rows, 2 * group, D)))
    value, lse, _, _ = compare(c, q, D ** -0.5, "a part of NaN")
    first = 0 if where == "first" else rows - 1
    assert np.isnan(value[first:, :group]).all() and np.isnan(lse[first:, :group]).all()
    assert np.isfinite(value[:, group:]).all() and np.isfinite(value[:first]).all()


@pytest.mark.parametrize("kernel,rows,tokens,D,group,width,many", CASES)
def test_a_value_that_is_nan_reaches_rows_whose_other_parts_outweigh_its_own(kernel, rows, tokens, D, group, width, many):
    """The first part's scores are so far below the others that its weight rounds to zero in 32 bits; one of its values is a NaN."""
    c = case(910 + D, kernel, rows, tokens, D, group, width)
    per = check_kernel(c, kernel, group, many)
    g = np.random.default_rng(911)
    direction = np.where(g.random(D) < 0.5, -1.0, 1.0)
    for t in range(tokens):
        page, place = okv.place(c.table[0], 32, c.num_pages, t)
        c.pages.write(page, place, patterns(np.tile(direction * (-1 if t < per else 1), (2, 1))), patterns(g.standard_normal((2, D))), c.books)
    spoil(c, 5, 1, block=D // 64 - 1)
    c.to_device()
    q = patterns(np.tile(direction, (rows, 2 * group, 1)))
    value, lse, _, _ = compare(c, q, 70.0 / D, "a NaN far below")               # scores about 140 apart: 2^-200
    assert np.isnan(value[:, :group, D - 64:]).all() and np.isfinite(value[:, group:]).all() and np.isfinite(lse).all()


@pytest.mark.parametrize("news,lengths", [([1, 1, 1], [5000, 40, 2999]), ([3, 1, 2], [3100, 2, 1700]), ([2, 0, 1], [4097, 10, 0])])
@pytest.mark.parametrize("group", (1, 7))
@pytest.mark.parametrize("window", (0, 1000))
def test_many_parts_of_wide_heads(news, lengths, group, window):
    """256 elements a head and more parts than a thread passes over, some of them empty for a sequence."""
    print(f"wide heads in many parts: news={news} lengths={lengths} group={group} window={window}", flush=True)
    c = Case(920, news, lengths, 64, 1, 256, behind=2).to_device()
    assert parts_of(c, group)[0] > 8
    compare(c, patterns(np.random.default_rng(921).standard_normal((c.rows, group, 256))), 0.07, "wide heads", window=window)
