"""Norm, router, experts, norm as a program uses them: one after the other, in captured graphs that are replayed for other tokens, on
streams of their own, two at once."""
import numpy as np
import pytest
import torch

from oracle import moe as omoe
from oracle.kv import bf16_value, round_bf16
from paper_2602_15563_amd import kmq
from tests.moe_util import Experts, check_experts, dev, host, patterns

pytestmark = pytest.mark.gpu

HIDDEN, WIDTH, EXPERTS, TOP_K, EPS = 512, 512, 24, 4, 1e-6


class Layer:
    def __init__(self, seed, bits):
        g = np.random.default_rng(seed)
        self.e = Experts(seed, EXPERTS, HIDDEN, WIDTH, bits)
        self.w = self.e.on_device()
        self.router, self.bias = patterns(g.standard_normal((EXPERTS, HIDDEN)) / 23), (0.1 * g.standard_normal(EXPERTS)).astype(np.float32)
        self.gains = [patterns(1 + 0.2 * g.standard_normal(HIDDEN)) for _ in range(3)]
        self.dev = [dev(t) for t in (self.router, self.bias, *self.gains)]

    def buffers(self, rows):
        new = lambda: torch.zeros((rows, HIDDEN), dtype=torch.int16, device="cuda")  # noqa: E731
        need = max(kmq.moe_route_workspace_bytes(rows, EXPERTS, HIDDEN), kmq.moe_experts_workspace_bytes(self.w, rows, TOP_K))
        return dict(rows=rows, x=new(), residual=new(), first=new(), h=new(), y=new(), second=new(), last=new(),
                    ids=torch.zeros((rows, TOP_K), dtype=torch.int32, device="cuda"), gates=torch.zeros((rows, TOP_K), dtype=torch.float32, device="cuda"),
                    ws=torch.empty(need, dtype=torch.uint8, device="cuda"))

    def run(self, b):
        router, bias, before, after, gain = self.dev
        rows = b["rows"]
        kmq.block_norm(b["x"], HIDDEN, rows, HIDDEN, b["first"], HIDDEN, b["h"], HIDDEN, residual=b["residual"], residual_stride=HIDDEN, pre_gain=before, eps=EPS)
        kmq.moe_route(b["h"], HIDDEN, rows, router, EXPERTS, HIDDEN, b["ids"], b["gates"], TOP_K, sigmoid=True, bias=bias, groups=6, top_groups=3, scale=1.5,
                      workspace=b["ws"])
        kmq.moe_experts(self.w, b["h"], HIDDEN, rows, b["ids"], b["gates"], TOP_K, b["y"], HIDDEN, workspace=b["ws"])
        kmq.block_norm(b["y"], HIDDEN, rows, HIDDEN, b["second"], HIDDEN, b["last"], HIDDEN, residual=b["first"], residual_stride=HIDDEN, post_gain=after,
                       pre_gain=gain, eps=EPS)

    def fill(self, b, seed):
        g = np.random.default_rng(seed)
        x, r = patterns(g.standard_normal((b["rows"], HIDDEN))), patterns(2 * g.standard_normal((b["rows"], HIDDEN)))
        b["x"].copy_(dev(x))
        b["residual"].copy_(dev(r))
        return x, r

    def check(self, b, x, r):
        """Every stage against the oracle, each from the device's own input to it."""
        first, h, y, second, last = (host(b[k]) for k in ("first", "h", "y", "second", "last"))
        ids, gates = b["ids"].cpu().numpy(), b["gates"].cpu().numpy()
        before, after, gain = self.gains
        same = lambda got, want: np.array_equal(got, round_bf16(want))  # noqa: E731
        s, n = omoe.block_norm(x, r, pre_gain=before, eps=EPS)
        assert same(first, s) and same(h, n)
        want, exact = omoe.route(h, self.router, TOP_K, sigmoid=True, bias=self.bias, groups=6, top_groups=3, scale=1.5)
        assert np.array_equal(ids, want) and (np.abs(gates - exact) <= 2.0 ** -23 * exact).all()
        check_experts(self.e, y, h, ids, gates)
        s, n = omoe.block_norm(y, first, post_gain=after, pre_gain=gain, eps=EPS, post_norm=True)
        assert same(second, s) and same(last, n)
        return [bf16_value(last), ids, gates]


@pytest.fixture(scope="module")
def layer():
    return Layer(5, 3)


@pytest.mark.parametrize("rows", (1, 3, 16, 40, 128))
def test_stages(layer, rows):
    b = layer.buffers(rows)
    x, r = layer.fill(b, rows)
    layer.run(b)
    torch.cuda.synchronize()
    layer.check(b, x, r)


@pytest.mark.parametrize("rows", (1, 20))
def test_captured_and_replayed_for_other_tokens(layer, rows):
    b, e = layer.buffers(rows), layer.buffers(rows)
    layer.fill(b, 0)
    layer.run(b)                                              # before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(b)
    for seed in range(1, 5):
        x, r = layer.fill(b, seed)
        layer.fill(e, seed)
        graph.replay()
        layer.run(e)                                          # the program's own work between replays
        torch.cuda.synchronize()
        for k in ("first", "h", "ids", "gates", "y", "second", "last"):
            assert torch.equal(b[k], e[k]), f"replay {seed}: {k}"
        layer.check(b, x, r)


def test_two_streams_at_once(layer):
    sets = [layer.buffers(rows) for rows in (17, 5)]
    data = [layer.fill(b, 30 + i) for i, b in enumerate(sets)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(sets, streams):
            with torch.cuda.stream(s):
                layer.run(b)
    torch.cuda.synchronize()
    for b, (x, r) in zip(sets, data):
        layer.check(b, x, r)


def test_two_graphs_share_a_workspace(layer):
    """One after the other on one stream, a workspace may serve both."""
    sets = [layer.buffers(rows) for rows in (9, 30)]
    big = max((b["ws"] for b in sets), key=lambda t: t.numel())
    for b in sets:
        b["ws"] = big
    graphs = []
    for b in sets:
        layer.fill(b, 1)
        layer.run(b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer.run(b)
        graphs.append(g)
    for turn in range(3):
        data = [layer.fill(b, 50 + turn) for b in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for b, (x, r) in zip(sets, data):
            layer.check(b, x, r)
