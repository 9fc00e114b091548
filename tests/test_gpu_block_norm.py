"""Norms around a block against the oracle: bit for bit, as both compute in 64 bits and round to 32 and to bf16."""
import numpy as np
import pytest
import torch

from oracle import moe as omoe
from oracle.kv import bf16_value, round_bf16
from paper_2602_15563_amd import kmq
from tests.moe_util import NAN16, dev, host, patterns, rows_on_device

pytestmark = pytest.mark.gpu


def inputs(seed, rows, width, gate="none"):
    g = np.random.default_rng(seed)
    gates = {"none": None, "channel": lambda: g.standard_normal(width), "rows": lambda: g.standard_normal((rows, width))}[gate]
    return dict(x=patterns(g.standard_normal((rows, width)) * 3), residual=patterns(g.standard_normal((rows, width)) * 5), gate=patterns(gates()) if gates else None,
                post_gain=patterns(1 + 0.3 * g.standard_normal(width)), pre_gain=patterns(1 + 0.3 * g.standard_normal(width)))


def run(d, out=True, normed=True, stride=None, in_place=(), **how):
    """(out, normed) patterns; rows have NaN between their ends and the stride, and there is a row of NaN behind the last.  in_place: which of
    the outputs go to the place of which input."""
    rows, width = d["x"].shape
    stride = stride or width
    x, res = rows_on_device(d["x"], stride, 1), rows_on_device(d["residual"], stride, 1) if d.get("residual") is not None else None
    places = {"x": x, "residual": res}
    new = lambda: torch.full((rows + 1, stride), NAN16, dtype=torch.int16, device="cuda")  # noqa: E731
    o = places[dict(in_place)["out"]] if "out" in dict(in_place) else new() if out else None
    n = places[dict(in_place)["normed"]] if "normed" in dict(in_place) else new() if normed else None
    gate = d.get("gate")
    kmq.block_norm(x, stride, rows, width, o, stride, n, stride, residual=res, residual_stride=stride, gate=dev(gate) if gate is not None else None,
                   gate_stride=width if gate is not None and gate.ndim == 2 else 0, post_gain=dev(d["post_gain"]) if d.get("post_gain") is not None else None,
                   pre_gain=dev(d["pre_gain"]) if d.get("pre_gain") is not None else None, **how)
    torch.cuda.synchronize()
    got = []
    for t in (o, n):
        if t is None:
            got.append(None)
            continue
        h = host(t)
        assert (h[rows:] == NAN16).all() and (h[:, width:] == NAN16).all(), "something behind the rows was written"
        got.append(h[:rows, :width])
    return got


def check(d, got, label="", **how):
    post = how.pop("post_norm", None)
    how = {k: v for k, v in how.items() if k not in ("out", "normed", "stride", "in_place")}
    want = omoe.block_norm(d["x"], d.get("residual"), d.get("gate"), d.get("post_gain"), d.get("pre_gain"),
                           post_norm=d.get("post_gain") is not None if post is None else post, **how)
    for name, g, w in zip(("out", "normed"), got, want):
        if g is None:
            continue
        w = round_bf16(w)
        same = (g == w) | (np.isnan(bf16_value(g)) & np.isnan(bf16_value(w)))
        assert same.all(), f"{label} {name}: {int((~same).sum())} of {same.size} differ"


@pytest.mark.parametrize("rows", (1, 3, 700))
@pytest.mark.parametrize("width", (8, 16, 504, 512, 520, 1000, 2048, 4096, 5120, 8192, 8200, 16392, 24584, 32768))
def test_widths(width, rows):
    if rows * width > 700 * 5120:
        rows = 37
    d = inputs(width + rows, rows, width, "rows" if width % 16 else "none")
    for how in (dict(eps=1e-6), dict(eps=0.5, scale=0.5, residual_scale=-2.0, stride=width + 8)):
        check(d, run(d, **how), f"{rows} x {width} {how}", **how)


@pytest.mark.parametrize("gate", ("none", "channel", "rows"))
@pytest.mark.parametrize("sigmoid", (False, True))
@pytest.mark.parametrize("post", ("gain", "unit", "no"))
def test_forms(gate, sigmoid, post):
    d = inputs(7, 13, 1032, gate)
    how = dict(eps=1e-5, gate_sigmoid=sigmoid, post_norm=post != "no", scale=1.5)
    if post == "unit":
        d["post_gain"] = None
    for missing in ((), ("residual",), ("pre_gain",), ("residual", "pre_gain")):
        e = {**d, **{m: None for m in missing}}
        check(e, run(e, **how), f"without {missing}", **how)
    check(d, run(d, out=False, **how), "no out", **how)
    check(d, run(d, normed=False, **how), "no norm", **how)


@pytest.mark.parametrize("places", ((("out", "residual"),), (("out", "x"),), (("normed", "x"),), (("out", "residual"), ("normed", "x"))))
@pytest.mark.parametrize("post_norm", (False, True))
@pytest.mark.parametrize("shape", ((5, 512), (300, 4104)))
def test_in_place(places, post_norm, shape):
    d = inputs(11, *shape)
    how = dict(eps=1e-6, post_norm=post_norm, in_place=places, stride=shape[1] + 16)
    check(d, run(d, **how), str(places), **how)


def test_what_is_not_finite_and_the_ends_of_the_range():
    d = inputs(3, 12, 264, "rows")
    x, r, g = d["x"], d["residual"], d["gate"]
    x[0, 5], x[1, 6], x[2, 7] = 0x7F80, 0xFF80, 0x7FC0
    r[3, 8], r[4, 9] = 0x7F80, 0x7FC0
    g[5, 1], g[6, 2], g[7, 3] = 0x7F80, 0xFF80, 0x7FC0
    x[8] = 0                                                                     # a row of zeros, and no eps below
    x[9], r[9] = 0x7F7F, 0                                                       # the largest numbers
    x[10], r[10] = 0x0001, 0x0001                                                # the smallest
    x[11], r[11] = 0x8000, 0x8000                                                # minus zeros
    for how in (dict(eps=1e-6), dict(eps=0.0), dict(eps=0.0, post_norm=False), dict(eps=1e-6, gate_sigmoid=True, scale=0.0)):
        check(d, run(d, **how), str(how), **how)


def test_rows_in_one_call_are_rows_in_many():
    """Where rows are many another launch shape may serve them; sums have their own order then, and agree after rounding."""
    d = inputs(17, 2100, 512)
    whole = run(d, eps=1e-6)
    for first in (0, 1, 2099):
        part = {k: v[first:first + 1] if v is not None and v.ndim == 2 else v for k, v in d.items()}
        for a, b in zip(run(part, eps=1e-6), whole):
            assert np.array_equal(a[0], b[first])


def test_rows_beyond_32_bit_offsets():
    rows, width, stride = 3, 256, 1 << 30
    d = inputs(19, rows, width)
    x = torch.empty(2 * stride + width, dtype=torch.int16, device="cuda")
    for i in range(rows):
        x[i * stride:i * stride + width] = dev(d["x"][i])
    out, res = torch.zeros((rows, width), dtype=torch.int16, device="cuda"), dev(d["residual"])
    kmq.block_norm(x, stride, rows, width, out, width, x, stride, residual=res, residual_stride=width, pre_gain=dev(d["pre_gain"]), eps=1e-6)
    torch.cuda.synchronize()
    normed = np.stack([host(x[i * stride:i * stride + width]) for i in range(rows)])
    d["post_gain"] = None
    check(d, (host(out), normed), eps=1e-6)
