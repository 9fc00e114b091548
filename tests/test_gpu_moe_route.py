"""The router against the oracle: the same experts, and their weights to the rounding to 32 bits."""
import numpy as np
import pytest
import torch

from oracle import moe as omoe
from paper_2602_15563_amd import kmq
from tests.moe_util import dev, patterns, rows_on_device

pytestmark = pytest.mark.gpu


def inputs(seed, rows, experts, width):
    g = np.random.default_rng(seed)
    return patterns(g.standard_normal((rows, width))), patterns(g.standard_normal((experts, width)) / np.sqrt(width)), (0.2 * g.standard_normal(experts)).astype(np.float32)


def run(x, w, top_k, bias=None, stride=None, **how):
    rows, width = x.shape
    experts = w.shape[0]
    ids = torch.full((rows + 1, top_k), -7, dtype=torch.int32, device="cuda")
    gates = torch.full((rows + 1, top_k), -7.0, dtype=torch.float32, device="cuda")
    need = kmq.moe_route_workspace_bytes(rows, experts, width)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")               # NaNs: what is read is written first
    kmq.moe_route(rows_on_device(x, stride), stride or width, rows, dev(w), experts, width, ids, gates, top_k, bias=dev(bias) if bias is not None else None,
                  workspace=ws[:need], **how)
    torch.cuda.synchronize()
    ids, gates = ids.cpu().numpy(), gates.cpu().numpy()
    assert (ids[rows:] == -7).all() and (gates[rows:] == -7).all() and (ws[need:] == 0xFF).all(), "something behind the outputs was written"
    return ids[:rows], gates[:rows]


def check(x, w, top_k, label="", stride=None, **how):
    """Weights: a rounding to 32 bits (2^-24 of the weight); what 64 bits leave, thousands of 2^-53, is nothing beside it."""
    ids, gates = run(x, w, top_k, stride=stride, **how)
    want, exact = omoe.route(x, w, top_k, **how)
    assert np.array_equal(ids, want), f"{label}: rows {np.nonzero((ids != want).any(1))[0][:5]} have other experts"
    bad = ~(np.abs(gates - exact) <= (2.0 ** -24 + 2.0 ** -40) * np.abs(exact) + 2.0 ** -149)
    assert np.array_equal(np.isnan(gates), np.isnan(exact)) and not (bad & ~np.isnan(exact)).any(), f"{label}: {int(bad.sum())} weights off"
    return ids, gates


@pytest.mark.parametrize("rows", (1, 2, 16, 17, 33, 64, 65, 130))
@pytest.mark.parametrize("experts,width,top_k", ((8, 512, 2), (64, 2048, 6), (128, 1000, 8), (256, 520, 16)))
def test_rows(rows, experts, width, top_k):
    x, w, bias = inputs(rows * experts, rows, experts, width)
    check(x, w, top_k, f"softmax {rows}")
    check(x, w, top_k, f"sigmoid {rows}", sigmoid=True, bias=bias, scale=2.5, stride=width + 24)


@pytest.mark.parametrize("experts", (1, 2, 15, 17, 63, 65, 129, 200, 384, 511, 513, 1000, 1024))
def test_numbers_of_experts(experts):
    x, w, bias = inputs(experts, 5, experts, 264)
    for top_k in {1, min(5, experts), min(16, experts)}:
        check(x, w, top_k, f"{experts} {top_k}", normalise=False)
        check(x, w, top_k, f"{experts} {top_k}", sigmoid=True, bias=bias)


@pytest.mark.parametrize("width", (8, 16, 24, 56, 64, 72, 248, 1032, 7168, 16392, 65536))
def test_widths(width):
    x, w, bias = inputs(width, 3, 40, width)
    check(x, w, 4, f"{width}")
    check(x, w, 4, f"{width}", bias=bias, stride=width + 8)


@pytest.mark.parametrize("experts,groups,top_groups,top_k", ((256, 8, 4, 8), (64, 64, 7, 7), (64, 32, 3, 6), (96, 4, 1, 16), (1024, 16, 2, 16), (160, 8, 8, 6), (6, 3, 2, 4)))
@pytest.mark.parametrize("sigmoid", (False, True))
def test_groups(experts, groups, top_groups, top_k, sigmoid):
    x, w, bias = inputs(experts + groups, 21, experts, 512)
    check(x, w, top_k, groups=groups, top_groups=top_groups, sigmoid=sigmoid)
    check(x, w, top_k, groups=groups, top_groups=top_groups, sigmoid=sigmoid, bias=bias, scale=0.5)


def test_equal_values_go_to_the_lower_index():
    x, w, _ = inputs(5, 9, 48, 512)
    x[0] = 0                                                                     # all alike
    w[3], w[17], w[40] = w[44], w[44], w[44]                                     # four the same
    w[20] = w[21]
    for how in (dict(), dict(sigmoid=True), dict(groups=4, top_groups=2), dict(groups=48, top_groups=11), dict(sigmoid=True, bias=np.full(48, -np.inf, np.float32))):
        ids, _ = check(x, w, 11, str(how), **how)
    assert (ids == np.arange(11)).all()


def test_what_is_not_finite():
    x, w, bias = inputs(6, 8, 24, 128)
    x[0, 3], x[1, 4], x[2] = 0x7FC0, 0x7F80, 0xFF80
    w[5, 9] = 0x7FC0                                                             # an expert that is a NaN for every token
    w[7, 1] = 0x7F80
    bias[2], bias[11], bias[12] = np.inf, -np.inf, np.nan
    for how in (dict(), dict(sigmoid=True), dict(sigmoid=True, bias=bias), dict(bias=bias, groups=4, top_groups=3), dict(sigmoid=True, groups=12, top_groups=12, normalise=False)):
        check(x, w, 16, str(how), **how)
    w[:] = 0xFF80                                                                # sigmoid of minus infinity: weights of zero
    x[:] = 0x3F80
    _, gates = check(x, w, 4, "zeros", sigmoid=True)
    assert (gates == 0).all()


def test_far_scores():
    x, w, _ = inputs(8, 6, 33, 256)
    w[::2] = patterns(30 * np.random.default_rng(1).standard_normal((17, 256)))  # logits of hundreds: most of the softmax is nothing
    check(x, w, 5)
    check(x, w, 5, sigmoid=True, bias=np.linspace(0, 1, 33).astype(np.float32))


def test_many_rows():
    x, w, bias = inputs(9, 5000, 72, 256)
    check(x, w, 6, sigmoid=True, bias=bias, groups=9, top_groups=4)


def test_a_row_is_the_same_in_every_batch():
    x, w, _ = inputs(10, 128, 128, 2048)
    ids, gates = run(x, w, 8)
    for rows in (1, 7, 20, 100):
        i, g = run(x[:rows], w, 8)
        assert np.array_equal(i, ids[:rows])
        assert (np.abs(g - gates[:rows]) <= 2.0 ** -23 * gates[:rows]).all()
    again = run(x, w, 8)
    assert np.array_equal(again[0], ids) and np.array_equal(again[1], gates)
