"""Heads, cache and attention as a program uses them: between the products of a decoder layer, over prompts and generated tokens, in
captured graphs that are replayed for other tokens and lengths, on streams of their own."""
import numpy as np
import pytest
import torch

import oracle
from oracle import kv as okv
from paper_2602_15563_amd import kmq, synth
from paper_2602_15563_amd.tolerance import arithmetic_bound, attention_bound, attention_lse_bound
from tests.kv_util import NAN16, Case, check_attention, dev, host, patterns

pytestmark = pytest.mark.gpu

HIDDEN, NQ, NK, D, BITS, EPS = 512, 4, 2, 64, 3, 1e-5
WIDTH = (NQ + 2 * NK) * D


class Layer:
    """QKV product, append, attention, output product: rows in, rows out, everything kept on the device."""

    def __init__(self, seed, case):
        self.c = case
        g = np.random.default_rng(seed)
        self.idx = [synth.make_indices(seed, i, n, k, BITS) for i, (n, k) in enumerate(((WIDTH, HIDDEN), (HIDDEN, NQ * D)))]
        self.cb = [synth.make_codebook(seed, i, n, BITS) for i, n in enumerate((WIDTH, HIDDEN))]
        self.packed = [oracle.pack(i, BITS) for i in self.idx]
        self.W = [(dev(p), dev(c)) for p, c in zip(self.packed, self.cb)]
        self.gq, self.gk = patterns(1 + 0.2 * g.standard_normal(D)), patterns(1 + 0.2 * g.standard_normal(D))
        self.freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
        self.dev = [dev(x) for x in (self.gq, self.gk, self.freq)]

    def prepare(self, batch):
        rows = batch.rows
        new = lambda w: torch.full((rows, w), NAN16, dtype=torch.int16, device="cuda")  # noqa: E731
        need = kmq.kv_attention_workspace_bytes(self.c.cache, batch, NQ)
        return dict(batch=batch, x=new(HIDDEN), qkv=new(WIDTH), q=new(NQ * D), o=new(NQ * D), y=new(HIDDEN),
                    lse=torch.full((rows, NQ), float("nan"), device="cuda"), ws=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))

    def product(self, i, x, y, n, k):
        for m in range(0, x.shape[0], kmq.MAX_BATCH):
            part = x[m:m + kmq.MAX_BATCH]
            kmq.gemm_smallbatch_noalloc(*self.W[i], part, y[m:m + kmq.MAX_BATCH], n, k, part.shape[0], BITS)

    def run(self, s):
        self.product(0, s["x"], s["qkv"], WIDTH, HIDDEN)
        gq, gk, freq = self.dev
        kmq.kv_append(self.c.cache, s["batch"], s["qkv"], WIDTH, s["q"], NQ * D, NQ, inv_freq=freq, rotary_dim=D, q_gain=gq, k_gain=gk, eps=EPS)
        kmq.kv_attention(self.c.cache, s["batch"], s["q"], NQ * D, s["o"], NQ * D, NQ, D ** -0.5, lse=s["lse"], workspace=s["ws"])
        self.product(1, s["o"], s["y"], HIDDEN, NQ * D)

    def check(self, s, x, news, lengths):
        """Every stage against the oracle, each from the device's own input to it; the cache's bytes throughout."""
        c = self.c
        qkv, q, o, y = (host(s[k]) for k in ("qkv", "q", "o", "y"))
        rows = x.shape[0]

        def product(i, got, inputs, k):
            for m in range(0, rows, 16):
                want, size, _ = oracle.gemm(self.packed[i], self.cb[i], inputs[m:m + 16], k, BITS)
                assert (np.abs(synth.bf16_to_f64(got[m:m + 16]) - want) <= arithmetic_bound(size, want, k)).all()
        product(0, qkv, x, HIDDEN)
        heads = qkv.reshape(rows, NQ + 2 * NK, D)
        c.news, c.lengths, c.rows = list(news), list(lengths), rows
        c.starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        pos = np.array([c.position(r)[1] for r in range(rows)])
        turned = [okv.round_bf16(okv.turn(heads[:, a:b], pos, self.freq, D, False, True, gain, EPS)) for a, b, gain in ((0, NQ, self.gq), (NQ, NQ + NK, self.gk))]
        assert np.array_equal(q.reshape(rows, NQ, D), turned[0])
        for r, page, token in c.places():
            c.pages.write(page, token, turned[1][r], heads[r, NQ + NK:], c.books)
        c.check_pages()
        for b, n in enumerate(news):
            mine = slice(c.starts[b], c.starts[b + 1])
            if n:
                k, v, there = okv.sequence(c.pages, c.table[b], lengths[b], c.books)
                out, lse, spread, size = okv.attention(q.reshape(rows, NQ, D)[mine], k, v, there, lengths[b], D ** -0.5)
                assert (np.abs(okv.bf16_value(o.reshape(rows, NQ, D)[mine]) - out) <= attention_bound(out, spread, size, len(there), D)).all()
                assert (np.abs(s["lse"].cpu().numpy()[mine] - lse) <= attention_lse_bound(size, len(there), D)).all()
        product(1, y, o, NQ * D)


def grow(c, table_rows):
    """A page table of `table_rows` sequences with all pages dealt out."""
    per = c.num_pages // table_rows
    c.table = np.arange(table_rows * per, dtype=np.int32).reshape(table_rows, per)[:, ::-1].copy()
    c.width = per


def test_prompts_then_tokens_through_a_layer():
    """Two prompts, then a second piece of one of them beside a token of the other, then tokens of both."""
    c = Case(1, [1, 1], [1, 1], 32, NK, D, spare=16)
    grow(c, 2)
    c.to_device()
    layer = Layer(2, c)
    g = np.random.default_rng(3)
    lengths = np.zeros(2, dtype=np.int64)
    for news in ([70, 33], [1, 40], [1, 1], [1, 1], [0, 2]):
        lengths += news
        starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        batch = kmq.KvBatch(dev(c.table), dev(lengths.astype(np.int32)), dev(starts), int(starts[-1]))
        s = layer.prepare(batch)
        x = patterns(g.standard_normal((batch.rows, HIDDEN)))
        s["x"].copy_(dev(x))
        layer.run(s)
        torch.cuda.synchronize()
        layer.check(s, x, news, lengths)


def test_a_captured_step_replayed_for_other_tokens():
    """One captured step of three sequences replayed while they grow across pages, eager work and synchronisation between; a second
    graph with buffers of its own, the two replayed in turn, against eager runs of the same steps."""
    c = Case(4, [1] * 3, [1] * 3, 32, NK, D, spare=24)
    grow(c, 3)
    c.to_device()
    layer = Layer(5, c)
    g = np.random.default_rng(6)
    table = dev(c.table)
    lengths = [dev(np.array([30, 1, 95], dtype=np.int32)) for _ in range(2)]
    states = [layer.prepare(kmq.KvBatch(table, m)) for m in lengths]
    stream = torch.cuda.Stream()
    graphs = []
    for s in states:                                             # captured on a stream of its own, after a run that makes what is lazily made
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            layer.run(s)
        torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer.run(s)
        graphs.append(graph)
    torch.cuda.synchronize()
    c.pages_d.copy_(torch.from_numpy(c.pages.bytes))
    at = np.array([30, 1, 95])
    for step in range(6):
        s, graph = states[step % 2], graphs[step % 2]
        x = patterns(g.standard_normal((3, HIDDEN)))
        s["x"].copy_(dev(x))
        lengths[step % 2].copy_(dev(at.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        layer.check(s, x, [1] * 3, at)
        eager = layer.prepare(kmq.KvBatch(table, dev(at.astype(np.int32))))
        eager["x"].copy_(dev(x))
        before = c.pages_d.clone()
        layer.run(eager)
        torch.cuda.synchronize()
        for k in ("qkv", "q", "o", "y", "lse"):
            assert torch.equal(eager[k], s[k]), f"step {step}: {k} differs from the eager run"
        assert torch.equal(before, c.pages_d)                     # the same tokens written again
        at = at + 1


def test_calls_on_two_streams_at_once():
    """Two attentions over one cache, each with a workspace of its own, at the same time on two streams."""
    c = Case(7, [1, 1], [3000, 2000], 64, 2, 128).to_device()
    g = np.random.default_rng(8)
    q = [patterns(g.standard_normal((2, 8, 128))) for _ in range(2)]
    want = [check_attention(c, x, 0.09)[0] for x in q]
    need = kmq.kv_attention_workspace_bytes(c.cache, c.batch, 8)
    assert need > 0
    streams = [torch.cuda.Stream() for _ in range(2)]
    qd, outs = [dev(x.reshape(2, -1)) for x in q], [torch.zeros((2, 1024), dtype=torch.int16, device="cuda") for _ in range(2)]
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                kmq.kv_attention(c.cache, c.batch, qd[i], 1024, outs[i], 1024, 8, 0.09, workspace=spaces[i])
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        assert np.array_equal(host(out).reshape(2, 8, 128), w)


@pytest.mark.parametrize("rows", (1, 40))
def test_pages_beyond_32_bit_offsets(rows):
    """A cache of more than 4 GiB whose sequence uses its first and its last pages: the same bytes and results as a small cache's."""
    heads, D, page = 8, 128, 1024
    size = kmq.kv_page_bytes(page, heads, D)
    many = (1 << 32) // size + 3
    g = np.random.default_rng(9)
    small = Case(10, [rows], [2500], page, heads, D, spare=0)
    small.to_device()
    big_pages = torch.zeros(many * size, dtype=torch.uint8, device="cuda")
    table = np.array([[many - 1, 0, many - 2]], dtype=np.int32)
    for i, p in enumerate(small.table[0]):
        at = int(table[0, i]) * size
        big_pages[at:at + size] = small.pages_d[int(p) * size:(int(p) + 1) * size]
    cache = kmq.KvCache(big_pages, dev(small.books), many, page, heads, D)
    batch = kmq.KvBatch(dev(table), dev(np.array([2500], dtype=np.int32)), dev(small.starts), rows)
    k, v = (dev(patterns(g.standard_normal((rows, heads * D)))) for _ in range(2))
    q = dev(patterns(g.standard_normal((rows, 2 * heads * D))))
    results = []
    for c, b in ((small.cache, small.batch), (cache, batch)):
        kmq.kv_write(c, b, k, heads * D, v, heads * D)
        back = [torch.zeros_like(k), torch.zeros_like(v)]
        kmq.kv_read(c, b, back[0], heads * D, back[1], heads * D)
        out, need = torch.zeros_like(q), kmq.kv_attention_workspace_bytes(c, b, 2 * heads)
        kmq.kv_attention(c, b, q, 2 * heads * D, out, 2 * heads * D, 2 * heads, 0.1, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        results.append((*back, out))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    for i, p in enumerate(small.table[0]):
        at = int(table[0, i]) * size
        assert torch.equal(big_pages[at:at + size], small.pages_d[int(p) * size:(int(p) + 1) * size])
