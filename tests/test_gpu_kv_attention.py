"""Attention over the 4-bit cache (kmq_kv_attention) on the GPU against the 64-bit oracle: outputs within attention_bound, and the
log-sum-exp, in which a single token left out or seen twice shows, within attention_lse_bound."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from paper_2602_15563_amd import kmq
from tests.kv_util import NAN16, Case, check_attention, dev, host, patterns, run_attention

pytestmark = pytest.mark.gpu


def queries(seed, rows, heads, D, size=1.0):
    return patterns(np.random.default_rng(seed).standard_normal((rows, heads, D)) * size)


def check(seed, news, lengths, page, kv_heads, group, D, causal=True, window=0, size=1.0, scale=None, stride=None, lse=True, tiles=None, **more):
    print(f"attention seed={seed} news={news[:8]} lengths={lengths[:8]} page={page} kv={kv_heads} group={group} D={D} causal={causal} window={window}", flush=True)
    c = Case(seed, news, lengths, page, kv_heads, D, **more).to_device()
    if tiles is not None:                                        # the case is meant for one of the two kernels
        assert (kmq.kernel_name_kv_attention(c.cache, c.batch, kv_heads * group) == "kv_attention_tile") == tiles
    q = queries(seed + 1, c.rows, kv_heads * group, D, size)
    return c, q, check_attention(c, q, D ** -0.5 if scale is None else scale, causal, window, stride=stride, lse=lse, label=f"seed {seed}")


@pytest.mark.parametrize("length", (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 600))
@pytest.mark.parametrize("D", (64, 128, 256))
def test_one_token_after_few(length, D):
    check(length, [1], [length], 32, 2, 3, D, starts=False)


@pytest.mark.parametrize("group", (1, 2, 4, 5, 8, 15, 16, 17, 33))
@pytest.mark.parametrize("n", (1, 3))
def test_query_heads_a_key_head(group, n):
    check(100 + group, [n, 1], [90, 40], 64, 2, group, 64)


@pytest.mark.parametrize("D", (64, 128, 256))
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 40), (False, 33), (True, 5000)])
def test_rows_of_a_prompt(D, causal, window):
    check(200 + D + window, [150, 70], [150, 190], 32, 2, 4, D, causal, window, tiles=True)
    check(250 + D + window, [50, 20], [50, 90], 32, 2, 2, D, causal, window, tiles=False)


@pytest.mark.parametrize("causal", (True, False))
def test_rows_that_see_nothing(causal):
    """Empty sequences, more rows than tokens, and lengths of zero: rows of zeros."""
    check(300, [3, 0, 5, 1], [0, 10, 3, 1], 32, 2, 2, 64, causal)
    check(301, [1, 1], [0, 4], 32, 1, 4, 128, causal, starts=False)
    check(309, [130, 0, 60], [0, 10, 40], 32, 2, 8, 64, causal, tiles=True)


def test_rows_behind_the_last_sequence_and_strides():
    check(302, [4, 20], [40, 20], 32, 2, 2, 128, behind=9, stride=4 * 128 + 40)
    check(308, [100, 130], [140, 130], 32, 2, 4, 128, behind=9, stride=8 * 128 + 40, tiles=True)
    check(303, [1, 1, 1], [400, 1, 77], 32, 2, 2, 64, behind=40, stride=4 * 64 + 8)


def test_without_log_sum_exp():
    check(304, [2], [50], 32, 1, 1, 64, lse=False)


def test_pages_that_are_none():
    """Tokens on pages that the table does not have are passed over; so is what lies beyond the table."""
    for seed, news in ((305, [80]), (306, [1])):
        c = Case(seed, news, [200], 32, 2, 128)
        c.table[0, 1], c.table[0, 5] = -1, c.num_pages
        c.to_device()
        check_attention(c, queries(1, c.rows, 4, 128), 0.1, label="missing pages")
        c = Case(seed, news, [300], 32, 2, 128, width=4).to_device()
        check_attention(c, queries(2, c.rows, 4, 128), 0.1, label="short table")
        c = Case(seed, news, [64], 32, 2, 128)
        c.table[0, :] = -1
        c.to_device()
        check_attention(c, queries(3, c.rows, 4, 128), 0.1, label="no pages")


@pytest.mark.parametrize("seed,news,lengths", [(310, [1], [3000]), (311, [2, 1], [1500, 2100]), (312, [1] * 3, [1, 900, 2000])])
def test_tokens_split_over_workgroups(seed, news, lengths):
    c, q, _ = check(seed, news, lengths, 64, 2, 4, 128)
    assert kmq.kv_attention_workspace_bytes(c.cache, c.batch, 8) > 0


def test_many_sequences():
    """More sequences than a wave has lanes, most of them short, some empty."""
    news = [1, 0, 3, 1, 2] * 30
    lengths = [5, 9, 3, 64, 65] * 30
    check(320, news, lengths, 32, 1, 4, 64)
    check(321, [1] * 70, list(range(1, 71)), 32, 1, 2, 64, starts=False)


@pytest.mark.parametrize("size", (0.0, 8.0, 60.0))
def test_flat_and_peaked_scores(size):
    """Queries of zeros (the mean of the values), and scores so far apart that one token takes all."""
    check(330, [80], [300], 32, 2, 2, 128, size=size, tiles=True)
    check(329, [20], [300], 32, 2, 2, 128, size=size, tiles=False)
    check(331, [1], [700], 32, 2, 4, 128, size=size)


def test_negative_and_zero_scale():
    check(332, [5], [80], 32, 1, 2, 64, scale=-0.125)
    check(333, [5], [80], 32, 1, 2, 64, scale=0.0)


@pytest.mark.parametrize("n", (1, 70))
def test_maxima_that_grow_and_fall(n):
    """Keys whose scores rise along the tokens (every step a new maximum) and fall (none after the first)."""
    for order in (1, -1):
        c = Case(340, [n], [500], 32, 1, 64)
        g = np.random.default_rng(341)
        direction = g.standard_normal(64)
        at = np.arange(500)[::order] / 500
        for p in range(500):
            page, token = okv.place(c.table[0], 32, c.num_pages, p)
            k = patterns(direction * at[p] * 40 + 0.1 * g.standard_normal(64)).reshape(1, 64)
            c.pages.write(page, token, k, patterns(g.standard_normal((1, 64))), c.books)
        c.to_device()
        q = patterns(np.tile(direction, (n, 2, 1)) * g.uniform(0.5, 1.0, (n, 2, 1)))
        check_attention(c, q, 0.125, label=f"order {order}")


def test_what_lies_behind_a_sequence_does_not_matter():
    """NaN and infinite scales in the tokens that a row does not see: behind the sequence, behind the row, before its window."""
    for n, window in ((1, 0), (1, 50), (20, 30), (20, 0), (90, 50)):
        c = Case(350, [n], [100], 64, 2, 128)
        clean = c.pages.bytes.copy()
        q = queries(351, n, 4, 128)
        want, lse = run_attention(c.to_device(), q, 4, 0.1, True, window)
        first = 100 - n                                                          # the first row's position
        for p in list(range(100, 128)) + (list(range(0, first - window + 1)) if window else []):
            page, token = okv.place(c.table[0], 64, c.num_pages, p)
            sa = c.pages.places(page, token)[4]
            c.pages.bytes[sa] = 0x80 if p % 2 else 0xC1
            c.pages.bytes[sa + 1] = 0x7F                                         # infinity, NaN
        assert not np.array_equal(clean, c.pages.bytes)
        got, lse2 = run_attention(c.to_device(), q, 4, 0.1, True, window)
        assert np.array_equal(got, want) and np.array_equal(lse, lse2)
        # a token that the last row alone sees: the other rows stay as they were
        page, token = okv.place(c.table[0], 64, c.num_pages, 99)
        sa = c.pages.places(page, token)[4]
        c.pages.bytes[sa], c.pages.bytes[sa + 1] = 0x80, 0x7F
        got, lse2 = run_attention(c.to_device(), q, 4, 0.1, True, window)
        assert np.array_equal(got[:-1], want[:-1]) and np.array_equal(lse[:-1], lse2[:-1])
        assert not np.isfinite(okv.bf16_value(got[-1])).all()


def test_a_nan_query_stays_in_its_row():
    for n in (3, 70):
        c = Case(360, [n], [150], 32, 2, 64).to_device()
        q = queries(361, n, 6, 64)
        want, _ = run_attention(c, q, 6, 0.1)
        q[1, 4, 7] = 0x7FC1
        got, _ = run_attention(c, q, 6, 0.1)
        assert np.isnan(okv.bf16_value(got[1, 4])).all()
        got[1, 4] = want[1, 4]
        assert np.array_equal(got, want)


def test_the_same_call_twice_gives_the_same_bits():
    for news, lengths in (([1, 1], [2000, 900]), ([250, 3], [300, 700])):
        c = Case(370, news, lengths, 64, 2, 128).to_device()
        q = queries(371, c.rows, 8, 128)
        first = run_attention(c, q, 8, 0.09)
        again = run_attention(c, q, 8, 0.09)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


@pytest.mark.parametrize("D", (64, 128, 256))
@pytest.mark.parametrize("n", (1, 40))
def test_one_token_decides(D, n):
    """Every token in turn has the one key that matters: its value comes out, from every place of a tile, a page and a step."""
    tokens = 70
    c = Case(380 + D, [n], [tokens], 32, 1, D)
    g = np.random.default_rng(381)
    direction = np.where(g.random(D) < 0.5, -1.0, 1.0)
    values = patterns(g.standard_normal((tokens, 1, D)))
    q = patterns(np.tile(direction, (n, 4, 1)))
    for hot in range(tokens - n + 1):
        for p in range(tokens):
            page, token = okv.place(c.table[0], 32, c.num_pages, p)
            c.pages.write(page, token, patterns(direction * (30.0 if p == hot else -30.0)).reshape(1, D), values[p], c.books)
        check_attention(c.to_device(), q, 1.0, label=f"token {hot}")


def test_no_rows():
    c = Case(390, [0], [50], 32, 1, 64).to_device()
    x = torch.full((1, 64), NAN16, dtype=torch.int16, device="cuda")
    kmq.kv_attention(c.cache, c.batch, x, 64, x, 64, 1, 1.0)
    torch.cuda.synchronize()
    assert (host(x) == NAN16).all()


def test_a_workspace_larger_than_asked_for_and_one_byte_too_small():
    c = Case(391, [1], [3000], 64, 1, 64).to_device()
    need = kmq.kv_attention_workspace_bytes(c.cache, c.batch, 1)
    q, out = dev(queries(1, 1, 1, 64).reshape(1, 64)), torch.full((1, 64), NAN16, dtype=torch.int16, device="cuda")
    with pytest.raises(kmq.KmqError) as e:
        kmq.kv_attention(c.cache, c.batch, q, 64, out, 64, 1, 0.1, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 6
    torch.cuda.synchronize()
    assert (host(out) == NAN16).all()
    kmq.kv_attention(c.cache, c.batch, q, 64, out, 64, 1, 0.1, workspace=torch.empty(need + 100, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert not np.isnan(okv.bf16_value(host(out))).any()


@pytest.mark.parametrize("D", (64, 128, 256))
@pytest.mark.parametrize("window", (0, 700))
def test_pieces_of_prompts_split_over_workgroups(D, window):
    """Many rows after a long context: the tokens go into parts, some of which a row does not see."""
    c, _, _ = check(400 + D, [250, 60], [1500, 900], 64, 1, 3, D, window=window, tiles=True)
    assert kmq.kv_attention_workspace_bytes(c.cache, c.batch, 3) > 0


@pytest.mark.parametrize("group", (1, 3, 7, 16, 20))
def test_query_heads_a_key_head_in_tiles(group):
    n = 1200 // group + 37
    check(420 + group, [n, 0, 50], [n + 13, 7, 77], 32, 1, group, 64, tiles=True)


@pytest.mark.parametrize("rows", (1, 21, 200))
@pytest.mark.parametrize("window", (0, 900))
def test_more_pages_than_are_read_at_once(rows, window):
    """A sequence of 69 pages whose tokens one workgroup walks through: the bits of the same tokens on one long page."""
    heads, D, pages, n = 96, 64, 69, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    small = torch.randint(0, 256, (n * pages, heads, 2, 17 * D), dtype=torch.uint8, device="cuda", generator=g)
    small[..., 16 * D:] = (0.5 + torch.rand((n * pages, heads, 2, D // 2), device="cuda", generator=g)).to(torch.bfloat16).view(torch.uint8)
    table = torch.randperm(n * pages, device="cuda", generator=g).to(torch.int32).view(n, pages)
    long = small[table.long()].permute(0, 2, 1, 3, 4).contiguous()
    books = dev(np.sort(np.random.default_rng(6).uniform(-1, 1, (2, 16)), axis=1).astype(np.float32).view(np.uint32) >> 16).to(torch.int16)
    lengths = dev(np.array([2208 - 100 * i for i in range(n)], dtype=np.int32))
    starts = dev(np.arange(0, n * rows + 1, rows, dtype=np.int32)) if rows > 1 else None
    q = torch.randn((n * rows, 2 * heads * D), device="cuda", generator=g).to(torch.bfloat16)
    outs = []
    for data, per, tab in ((small, 32, table), (long, 32 * pages, torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1))):
        cache = kmq.KvCache(data, books, data.shape[0], per, heads, D)
        batch = kmq.KvBatch(tab, lengths, starts, n * rows)
        assert kmq.kv_attention_workspace_bytes(cache, batch, 2 * heads) == 0                # one part
        out = torch.zeros_like(q)
        kmq.kv_attention(cache, batch, q, 2 * heads * D, out, 2 * heads * D, 2 * heads, 0.2, window=window)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and bool(outs[0].isfinite().all()) and float(outs[0].float().abs().mean()) > 1e-3
