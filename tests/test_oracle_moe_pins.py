"""The oracle of the norms and of the mixture of experts, held to values worked out by hand."""
import numpy as np

from oracle import moe
from oracle.kv import round_bf16


def patterns(x):
    return round_bf16(np.asarray(x, dtype=np.float64))


def test_block_norm():
    x = patterns([[3, 4] * 4])                                                     # mean square 12.5
    out, normed = moe.block_norm(x)
    np.testing.assert_allclose(out, [[3, 4] * 4])
    np.testing.assert_allclose(normed, np.array([[3, 4] * 4]) / np.sqrt(12.5), rtol=1e-15)
    out, normed = moe.block_norm(x, residual=patterns([[8] * 8]), gate=patterns([0.5] * 8), post_gain=patterns([2.0] * 8), pre_gain=patterns([4.0] * 8),
                                 scale=10.0, residual_scale=0.25, eps=12.5, post_norm=True)
    s = 2 + 10 * 0.5 * 2 * np.array([3, 4] * 4) / 5                                # 8, 10: mean square 82
    np.testing.assert_allclose(out[0], s, rtol=1e-15)
    np.testing.assert_allclose(normed[0], 4 * s / np.sqrt(82 + 12.5), rtol=1e-15)
    out, _ = moe.block_norm(x, gate=patterns([[0] * 8]), gate_sigmoid=True)
    np.testing.assert_allclose(out[0], [1.5, 2] * 4)


def test_route():
    w = np.zeros((4, 8), dtype=np.uint16)
    w[:, 0] = patterns([0, np.log(2), 1, 0])
    x = np.zeros((1, 8), dtype=np.uint16)
    ids, gates = moe.route(x, w, 3)                                                # all alike: the lowest indices
    assert ids.tolist() == [[0, 1, 2]]
    np.testing.assert_allclose(gates, [[1 / 3] * 3])
    x[0, 0] = 0x3F80
    ids, gates = moe.route(x, w, 2, normalise=False, scale=2.0)
    e = np.exp([0, float(np.float32(0.69140625)), 1, 0])
    assert ids.tolist() == [[2, 1]]
    np.testing.assert_allclose(gates[0], 2 * e[[2, 1]] / e.sum(), rtol=1e-15)
    ids, gates = moe.route(x, w, 1, sigmoid=True, bias=[0.5, 0, 0, 0])              # 1, 0.666, 0.731, 0.5
    assert ids.tolist() == [[0]] and gates.tolist() == [[1.0]]
    ids, _ = moe.route(x, w, 2, sigmoid=True, bias=[0.2, 0, 0, 0], groups=2, top_groups=1)   # 0.7 + 0.666 against 0.731 + 0.5
    assert ids.tolist() == [[0, 1]]
    w[1, 0] = 0x7FC0
    ids, _ = moe.route(x, w, 4, sigmoid=True)
    assert ids.tolist() == [[2, 0, 3, 1]]                                          # the NaN last


def test_experts():
    idx = np.array([[0] * 64 + [1] * 64])
    m = moe.matrix(idx, patterns([-1, 2]), patterns([[0.5, 3]]))
    assert m.tolist() == [[-0.5] * 64 + [6.0] * 64]
    up, down = np.array([[1.0, 0], [0, 2]]), np.array([[1.0, 1], [1, -1]])
    matrices = {0: (np.eye(2), up, down), 5: (np.zeros((2, 2)), up, down)}
    x = patterns([[1, 2]])
    y, pairs = moe.experts(x, np.array([[0, 5, -1, 0]]), np.array([[0.25, 9, 9, 0.75]]), matrices, residual=patterns([[10, 20]]))
    h = np.array([1 / (1 + np.exp(-1)), 2 / (1 + np.exp(-2)) * 4])
    np.testing.assert_allclose(y, [[10 + h.sum(), 20 + h[0] - h[1]]], rtol=1e-15)
    assert [(p["expert"], p["weight"]) for p in pairs] == [(0, 1.0), (5, 9.0)]
