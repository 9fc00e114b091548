"""Every instance of the experts' row kernel, in rows long enough for all that it does with them: the steady loop, in which a wave asks for
a super-block while it multiplies another, a second piece of the columns, the loop in that piece (tests/moe_launches.py)."""
import numpy as np
import pytest
import torch

from paper_2602_15563_amd import kmq
from tests.moe_launches import CASES
from tests.moe_util import Experts, check_experts, patterns, run_experts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,rows,top_k,experts,hidden,width", CASES)
def test_instance(bits, rows, top_k, experts, hidden, width):
    """Many experts are three.  One of them all tokens have, so that it takes as many turns as there are."""
    g = np.random.default_rng(hidden + 3 * width + rows + bits)
    e = Experts(hidden % 1009 + width, min(experts, 3), hidden, width, bits)
    of = np.arange(experts) % e.experts
    pick = torch.from_numpy(of).cuda()
    w = kmq.MoeWeights(*(t[pick].contiguous() for t in e.on_device().tensors), experts, hidden, width, bits)
    ids, gates = np.argsort(g.random((rows, experts)), axis=1)[:, :top_k].astype(np.int32), g.uniform(0.05, 0.6, (rows, top_k)).astype(np.float32)
    ids[:, -1][(ids[:, :-1] != experts - 1).all(1)] = experts - 1
    x, res = patterns(g.standard_normal((rows, hidden))), patterns(g.standard_normal((rows, hidden)))
    got = run_experts(w, x, ids, gates)
    check_experts(e, got, x, of[ids].astype(np.int32), gates, None, "", range(0, rows, -(-rows // 8)))
    assert np.array_equal(run_experts(w, x, ids, gates), got), "repeats are the same bits"
    check_experts(e, run_experts(w, x, ids, gates, res), x, of[ids].astype(np.int32), gates, res, "residual", range(0, rows, -(-rows // 3)))
