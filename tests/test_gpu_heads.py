"""Head norms and rotation (kmq_qk_norm_rope) on the GPU: bit for bit the oracle's 64-bit result rounded to fp32 and then to bf16."""
import numpy as np
import pytest
import torch

from oracle import kv as okv
from paper_2602_15563_amd import kmq
from tests.kv_util import NAN16, dev, host, patterns

pytestmark = pytest.mark.gpu


def inv_freq(rot, theta=10000.0):
    return (theta ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)


def run(seed, rows, nq, nk, D, rot, interleaved, norm, gains, pad=0, in_place=False, positions=None, x=None, eps=1e-5):
    g = np.random.default_rng(seed)
    print(f"heads seed={seed} rows={rows} q={nq} k={nk} D={D} rot={rot} interleaved={interleaved} norm={norm} gains={gains} pad={pad}", flush=True)
    heads, stride = nq + nk, (nq + nk) * D + pad
    x = patterns(g.standard_normal((rows, heads, D)) * 2.0 ** g.integers(-6, 7, (rows, heads, 1))) if x is None else x
    pos = g.integers(0, 200000, rows).astype(np.int32) if positions is None else np.asarray(positions, dtype=np.int32)
    gq, gk = patterns(1 + 0.3 * g.standard_normal(D)), patterns(1 + 0.3 * g.standard_normal(D))
    freq = inv_freq(rot)
    xd = torch.full((rows, stride), NAN16, dtype=torch.int16, device="cuda")
    xd[:, :heads * D] = dev(x.reshape(rows, heads * D))
    if in_place:
        q, qs, k, ks = xd, stride, xd[:, nq * D:], stride
    else:
        qs, ks = nq * D + pad, nk * D + pad
        q = torch.full((rows, max(qs, 8)), NAN16, dtype=torch.int16, device="cuda")
        k = torch.full((rows, max(ks, 8)), NAN16, dtype=torch.int16, device="cuda")
    kmq.qk_norm_rope(xd, stride, q, qs, k, ks, rows, nq, nk, D, positions=dev(pos) if rot else None, inv_freq=dev(freq) if rot else None,
                     rotary_dim=rot, interleaved=interleaved, rmsnorm=norm, q_gain=dev(gq) if gains else None, k_gain=dev(gk) if gains else None, eps=eps)
    torch.cuda.synchronize()
    for first, count, gain, out in ((0, nq, gq, q), (nq, nk, gk, k)):
        want = okv.round_bf16(okv.turn(x[:, first:first + count], pos, freq, rot, interleaved, norm, gain if gains else None, eps))
        got = host(out)[:, :count * D].reshape(rows, count, D)
        assert np.array_equal(got, want), f"{int((got != want).sum())} of {got.size} differ"
    if pad and not in_place:
        assert (host(q)[:, nq * D:] == NAN16).all() and (host(k)[:, nk * D:] == NAN16).all()
    if in_place and pad:
        assert (host(xd)[:, heads * D:] == NAN16).all()


@pytest.mark.parametrize("D,rot", [(8, 0), (16, 16), (40, 32), (64, 64), (64, 32), (80, 80), (96, 48), (128, 128), (128, 16), (200, 192), (256, 256), (512, 512)])
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("norm,gains", [(False, False), (True, False), (True, True)])
def test_sizes_of_heads(D, rot, interleaved, norm, gains):
    run(D + rot, 5, 3, 2, D, rot, interleaved, norm, gains, pad=8)


@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 0), (0, 1), (32, 8), (24, 24), (17, 5), (71, 1)])
@pytest.mark.parametrize("rows", (1, 3, 1030))
def test_numbers_of_heads_and_rows(nq, nk, rows):
    run(nq * 100 + nk, rows, nq, nk, 64 if rows > 100 else 128, 64, rows % 2 == 0, True, True)


@pytest.mark.parametrize("rows", (4, 1024))
@pytest.mark.parametrize("interleaved", (False, True))
def test_in_place(rows, interleaved):
    run(7, rows, 6, 2, 128, 128, interleaved, True, True, pad=24, in_place=True)


def test_far_and_negative_positions():
    run(8, 8, 2, 1, 128, 128, False, False, False, positions=[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 24, 1000003, 131071])


def test_rows_of_zeros_and_of_large_and_small_values():
    x = np.zeros((4, 2, 64), dtype=np.uint16)
    x[1] = 0x7F00                                              # 1.7e38: squares beyond 32 bits
    x[2] = 0x0001                                              # the smallest positive value
    x[3, :, ::2] = 0x0090
    run(9, 4, 1, 1, 64, 64, False, True, True, x=x)


def test_a_nan_or_an_infinity_stays_in_its_head():
    g = np.random.default_rng(10)
    x = patterns(g.standard_normal((2, 4, 64)))
    x[0, 1, 5], x[1, 2, 9] = 0x7F80, 0x7FC1
    xd, q = dev(x.reshape(2, 256)), torch.zeros((2, 256), dtype=torch.int16, device="cuda")
    freq, pos = inv_freq(64), np.array([3, 4], dtype=np.int32)
    kmq.qk_norm_rope(xd, 256, q, 256, None, 0, 2, 4, 0, 64, positions=dev(pos), inv_freq=dev(freq), rotary_dim=64, rmsnorm=True, eps=1e-5)
    torch.cuda.synchronize()
    got = okv.bf16_value(host(q)).reshape(2, 4, 64)
    want = okv.round_bf16(okv.turn(x, pos, freq, 64, False, True, None, 1e-5)).reshape(2, 4, 64)
    for r in range(2):
        for h in range(4):
            if (r, h) in ((0, 1), (1, 2)):
                assert np.isnan(got[r, h]).any()
            else:
                assert np.array_equal(host(q).reshape(2, 4, 64)[r, h], want[r, h])


def test_no_rows():
    x = torch.full((1, 128), NAN16, dtype=torch.int16, device="cuda")
    kmq.qk_norm_rope(x, 128, x, 128, None, 0, 0, 2, 0, 64, rmsnorm=True)
    torch.cuda.synchronize()
    assert (host(x) == NAN16).all()


@pytest.mark.parametrize("interleaved", (False, True))
def test_an_infinity_without_a_norm_reaches_its_partner_and_no_further(interleaved):
    x = patterns(np.random.default_rng(11).standard_normal((1, 2, 128)))
    x[0, 0, 100], x[0, 1, 4] = 0x7F80, 0xFF80                     # behind the rotated elements, and among them
    freq, pos = inv_freq(64), np.array([5], dtype=np.int32)
    xd, q = dev(x.reshape(1, 256)), torch.zeros((1, 256), dtype=torch.int16, device="cuda")
    kmq.qk_norm_rope(xd, 256, q, 256, None, 0, 1, 2, 0, 128, positions=dev(pos), inv_freq=dev(freq), rotary_dim=64, interleaved=interleaved)
    torch.cuda.synchronize()
    want = okv.round_bf16(okv.turn(x, pos, freq, 64, interleaved)).reshape(1, 256)
    assert np.array_equal(okv.bf16_value(host(q)), okv.bf16_value(want), equal_nan=True)
