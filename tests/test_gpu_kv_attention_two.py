"""Attention over the 4-bit cache (kmq_kv_attention) where a workgroup takes two tiles of columns: more than 16 (row, query head) pairs a
key head over tables of 2048 tokens and more, on the GPU against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from paper_2602_15563_amd import kmq
from tests.kv_util import NAN16, Case, check_attention, dev, host, run_attention
from tests.test_gpu_kv_attention import queries

pytestmark = pytest.mark.gpu


def check(seed, news, lengths, page, kv_heads, group, D, causal=True, window=0, size=1.0, width=None, stride=None, lse=True, **more):
    print(f"attention, two tiles: seed={seed} news={news} lengths={lengths} page={page} kv={kv_heads} group={group} D={D} causal={causal} window={window}", flush=True)
    c = Case(seed, news, lengths, page, kv_heads, D, width=width or 2048 // page, **more).to_device()
    assert kmq.kernel_name_kv_attention(c.cache, c.batch, kv_heads * group) == "kv_attention_two"
    return c, check_attention(c, queries(seed + 1, c.rows, kv_heads * group, D, size), D ** -0.5, causal, window, stride=stride, lse=lse, label=f"seed {seed}")


@pytest.mark.parametrize("n", (17, 31, 32, 33, 47, 64, 65))
@pytest.mark.parametrize("D", (64, 128))
def test_columns(n, D):
    check(600 + n, [n], [n], 32, 2, 1, D)
    check(700 + n, [n], [n + 200], 64, 1, 1, D)


@pytest.mark.parametrize("group", (17, 24, 33, 40))
def test_query_heads_of_single_tokens(group):
    check(800 + group, [1, 1, 1], [200, 1, 77], 64, 2, group, 128, starts=False)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 40), (False, 33), (True, 5000)])
def test_masks(D, causal, window):
    check(810 + D + window, [50, 20], [50, 190], 32, 2, 3, D, causal, window)
    check(811 + D + window, [9], [500], 2048, 1, 4, D, causal, window)


@pytest.mark.parametrize("causal", (True, False))
def test_rows_that_see_nothing(causal):
    """Empty sequences, more rows than tokens, and lengths of zero: rows of zeros."""
    check(820, [30, 0, 60, 1], [0, 10, 40, 1], 32, 2, 2, 64, causal)
    check(821, [1, 1], [0, 4], 32, 1, 20, 128, causal, starts=False)


def test_sequences_that_leave_a_tile_empty_and_rows_behind():
    """Of two tiles the second has no column, or the first is not full."""
    check(822, [3, 40, 16, 0, 1], [70, 90, 16, 5, 300], 32, 2, 2, 128, behind=9, stride=4 * 128 + 40)
    check(823, [40], [50], 32, 1, 1, 64, lse=False)


def test_pages_that_are_none():
    c = Case(824, [80], [200], 32, 2, 128, width=64)
    c.table[0, 1], c.table[0, 5] = -1, c.num_pages
    c.to_device()
    check_attention(c, queries(1, c.rows, 4, 128), 0.1, label="missing pages")
    c = Case(825, [80], [2100], 32, 2, 128, width=64).to_device()
    check_attention(c, queries(2, c.rows, 4, 128), 0.1, label="short table")
    c.table[0, :] = -1
    c.to_device()
    check_attention(c, queries(3, c.rows, 4, 128), 0.1, label="no pages")


@pytest.mark.parametrize("size", (0.0, 8.0, 60.0))
def test_flat_and_peaked_scores(size):
    check(826, [30], [300], 32, 2, 2, 128, size=size)
    check(827, [30], [900], 32, 2, 2, 64, size=size)


@pytest.mark.parametrize("window", (0, 700))
@pytest.mark.parametrize("D", (64, 128))
def test_tokens_split_over_workgroups(D, window):
    c, _ = check(830 + D, [30, 7], [2500, 900], 64, 2, 3, D, window=window, width=40)
    assert kmq.kv_attention_workspace_bytes(c.cache, c.batch, 6) > 0


def test_what_a_row_does_not_see_does_not_matter():
    """NaN and infinite scales behind the sequence, before the first row's window, and in the last row's token."""
    for n, window in ((20, 30), (20, 0), (33, 50)):
        c = Case(840, [n], [100], 64, 2, 128, width=32)

        def spoil(tokens):
            for p in tokens:
                page, token = okv.place(c.table[0], 64, c.num_pages, p)
                sa = c.pages.places(page, token)[4]
                c.pages.bytes[sa], c.pages.bytes[sa + 1] = 0x80 if p % 2 else 0xC1, 0x7F      # infinity, NaN

        q = queries(841, n, 4, 128)
        want, lse = run_attention(c.to_device(), q, 4, 0.1, True, window)
        assert kmq.kernel_name_kv_attention(c.cache, c.batch, 4) == "kv_attention_two"
        spoil(list(range(100, 128)) + (list(range(100 - n - window + 1)) if window else []))
        got, lse2 = run_attention(c.to_device(), q, 4, 0.1, True, window)
        assert np.array_equal(got, want) and np.array_equal(lse, lse2)
        spoil([99])
        got, lse2 = run_attention(c.to_device(), q, 4, 0.1, True, window)
        assert np.array_equal(got[:-1], want[:-1]) and np.array_equal(lse[:-1], lse2[:-1])
        assert not np.isfinite(okv.bf16_value(got[-1])).all()


def test_captured_and_replayed_with_other_lengths():
    c, _ = check(850, [20, 12], [300, 90], 64, 2, 2, 128)
    q = dev(queries(851, c.rows, 4, 128).reshape(c.rows, 512))
    out, lse = torch.empty((c.rows, 512), dtype=torch.int16, device="cuda"), torch.empty((c.rows, 4), dtype=torch.float32, device="cuda")
    space = torch.empty(max(1, kmq.kv_attention_workspace_bytes(c.cache, c.batch, 4)), dtype=torch.uint8, device="cuda")

    def call():
        kmq.kv_attention(c.cache, c.batch, q, 512, out, 512, 4, 0.1, workspace=space)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lengths in ([300, 90], [20, 1700], [64, 0]):
        c.batch.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        call()
        torch.cuda.synchronize()
        want = host(out).copy()
        out.fill_(NAN16)
        graph.replay()
        torch.cuda.synchronize()
        assert (host(out) == want).all()
