"""Attention over the 4-bit cache (kmq_kv_attention) on the GPU where something that a row sees is not finite: it reaches the row, and no other."""
import numpy as np
import pytest

from oracle import kv as okv
from paper_2602_15563_amd import kmq
from tests.kv_util import Case, patterns, run_attention
from tests.test_gpu_kv_attention_parts import NAN, ONE, TILE, TWO, compare, spoil

pytestmark = pytest.mark.gpu

# kernel, rows, tokens, head size, query heads a key head, table width (pages of 32)
CASES = [(ONE, 1, 20, 64, 3, None), (ONE, 1, 20, 128, 3, None), (ONE, 1, 20, 256, 3, None), (ONE, 4, 70, 128, 2, None), (TWO, 9, 20, 64, 3, 64),
         (TWO, 9, 20, 128, 3, 64), (TWO, 40, 75, 128, 1, 64), (TILE, 150, 150, 64, 4, None), (TILE, 150, 150, 128, 4, None), (TILE, 150, 150, 256, 4, None)]


def make(seed, kernel, rows, tokens, D, group, width):
    print(f"not finite: {kernel} rows={rows} tokens={tokens} D={D} group={group} width={width}", flush=True)
    c = Case(seed, [rows], [tokens], 32, 2, D, width=width).to_device()
    assert kmq.kernel_name_kv_attention(c.cache, c.batch, 2 * group) == kernel
    return c


@pytest.mark.parametrize("kernel,rows,tokens,D,group,width", CASES)
@pytest.mark.parametrize("bits", (NAN, 0x7F80))
def test_a_value_of_a_token_whose_probability_rounds_to_zero(kernel, rows, tokens, D, group, width, bits):
    """Token 3's score is so far below that of token 0 that its probability is zero in 32 bits; it stands in a step that some of its tokens' columns
    do not see whole.  A NaN or an infinity among its values is one in every row that sees it."""
    c = make(940 + D, kernel, rows, tokens, D, group, width)
    g = np.random.default_rng(941)
    direction = np.where(g.random(D) < 0.5, -1.0, 1.0)
    for t in range(tokens):
        page, place = okv.place(c.table[0], 32, c.num_pages, t)
        c.pages.write(page, place, patterns(np.tile(direction * (-1 if t == 3 else 1), (2, 1))), patterns(g.standard_normal((2, D))), c.books)
    spoil(c, 3, 1, block=D // 64 - 1, bits=bits)
    c.to_device()
    q = patterns(np.tile(direction, (rows, 2 * group, 1)))
    if bits == NAN:
        value, lse, _, _ = compare(c, q, 70.0 / D, "a NaN far below")           # scores about 140 apart: 2^-200
    else:
        got, lse = run_attention(c, q, 2 * group, 70.0 / D)
        value = okv.bf16_value(got)
    first = max(0, 3 - (tokens - rows))                                          # the first row that sees token 3
    assert not np.isfinite(value[first:, :group, D - 64:]).any() and np.isfinite(value[:first]).all()
    assert np.isfinite(value[:, group:]).all() and np.isfinite(value[:, :, :D - 64]).all() and np.isfinite(lse).all()


@pytest.mark.parametrize("kernel,rows,tokens,D,group,width", CASES + [(ONE, 1, 1, 128, 2, None), (ONE, 1, 2, 64, 1, None), (ONE, 1, 700, 128, 2, None), (ONE, 1, 3000, 256, 2, None),
                                                                      (TWO, 20, 5, 128, 2, 64), (TILE, 250, 700, 128, 3, None)])
@pytest.mark.parametrize("bits", (0x7F80, 0xFF80))
def test_an_infinite_query_is_nan_in_its_head_and_row(kernel, rows, tokens, D, group, width, bits):
    """Its scores are infinite, all of one sign where its keys are few: exp(S) / sum exp(S) has no number for them.  A row that sees nothing stays zero."""
    c = make(950 + D, kernel, rows, tokens, D, group, width)
    g = np.random.default_rng(951)
    q = patterns(g.standard_normal((rows, 2 * group, D)))
    want, lse = run_attention(c, q, 2 * group, D ** -0.5)
    places = {(int(g.integers(0, rows)), int(h)) for h in g.permutation(2 * group)[:3]} | {(0, 0)}
    for r, h in places:
        q[r, h, g.integers(0, D)] = bits
    got, lse2 = run_attention(c, q, 2 * group, D ** -0.5)
    for r, h in places:
        if r >= rows - tokens:
            assert np.isnan(okv.bf16_value(got[r, h])).all() and np.isnan(lse2[r, h])
        else:
            assert (got[r, h] == 0).all() and np.isneginf(lse2[r, h])
        got[r, h], lse2[r, h] = want[r, h], lse[r, h]
    assert np.array_equal(got, want) and np.array_equal(lse2, lse)


@pytest.mark.parametrize("kernel,rows,tokens,D,group,width", CASES + [(ONE, 1, 1, 128, 2, None), (ONE, 1, 700, 64, 2, None), (ONE, 2, 3000, 256, 2, None), (TWO, 20, 300, 128, 2, 64),
                                                                      (TWO, 20, 2500, 64, 2, None), (TILE, 250, 700, 64, 3, None), (TILE, 250, 700, 256, 3, None)])
@pytest.mark.parametrize("bits", (0x7F80, NAN))
def test_a_key_that_is_not_finite_is_nan_in_every_row_that_sees_it(kernel, rows, tokens, D, group, width, bits):
    """One block's scale of one key, in tokens that all rows see, some do, or the last alone, in whole steps and at their ends, for every place in a
    tile; and in a token that lies behind the sequence or before every window, which changes nothing."""
    c = make(960 + D, kernel, rows, tokens, D, group, width)
    g = np.random.default_rng(961)
    q = patterns(g.standard_normal((rows, 2 * group, D)))
    clean = c.pages.bytes.copy()
    want, lse = run_attention(c, q, 2 * group, D ** -0.5)
    places = sorted({0, tokens - 1, max(0, tokens - rows), tokens // 2} | {int(t) for t in g.integers(0, tokens, 6)})
    for t in places:
        c.pages.bytes[:] = clean
        spoil(c, t, 0, head=1, block=int(g.integers(0, D // 64)), bits=bits)
        got, lse2 = run_attention(c.to_device(), q, 2 * group, D ** -0.5)
        first = max(0, t - (tokens - rows))
        assert np.isnan(okv.bf16_value(got[first:, group:])).all() and np.isnan(lse2[first:, group:]).all(), f"token {t}"
        assert np.array_equal(got[:, :group], want[:, :group]) and np.array_equal(lse2[:, :group], lse[:, :group]), f"token {t}: the other head"
        assert np.array_equal(got[:first], want[:first]) and np.array_equal(lse2[:first], lse[:first]), f"token {t}: rows before it"
    if tokens > rows + 20:
        c.pages.bytes[:] = clean
        want, lse = run_attention(c.to_device(), q, 2 * group, D ** -0.5, window=20)
        for t in range(0, tokens - rows - 20):
            spoil(c, t, 0, bits=bits)
        got, lse2 = run_attention(c.to_device(), q, 2 * group, D ** -0.5, window=20)
        assert np.array_equal(got, want) and np.array_equal(lse, lse2)
