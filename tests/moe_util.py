"""Experts on the host (oracle) and on the device (library), for the tests of the mixture of experts."""
import numpy as np
import torch

from oracle import moe as omoe
from oracle.kv import bf16_value, round_bf16
from paper_2602_15563_amd import kmq, synth
from paper_2602_15563_amd.tolerance import moe_bound

NAN16 = 0x7FC1


def patterns(x):
    return round_bf16(np.asarray(x, dtype=np.float64))


def dev(a):
    a = np.ascontiguousarray(a)
    view = {np.dtype(np.uint16): np.int16, np.dtype(np.uint32): np.int32}.get(a.dtype, a.dtype)
    return torch.from_numpy(a.view(view)).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint16)


def rows_on_device(x, stride=None, behind=0):
    """Rows of patterns with NaN between their ends and the stride, and in `behind` rows after the last."""
    rows, width = x.shape
    t = torch.full((rows + behind, stride or width), NAN16, dtype=torch.int16, device="cuda")
    if rows:
        t[:rows, :width] = dev(x)
    return t


class Experts:
    """`experts` experts of hidden x width at `bits` bits, random indices, each with codebooks and scales of its own.  The scales of an
    expert in `poison` are all NaN."""

    def __init__(self, seed, experts, hidden, width, bits, poison=()):
        self.experts, self.hidden, self.width, self.bits = experts, hidden, width, bits
        self.shapes = ((width, hidden), (width, hidden), (hidden, width))
        make = lambda f: [[f(3 * e + m, n, k) for e in range(experts)] for m, (n, k) in enumerate(self.shapes)]  # noqa: E731
        self.idx = make(lambda i, n, k: synth.make_indices(seed, i, n, k, bits))
        self.books = make(lambda i, n, k: synth.make_shared_codebook(seed, i, bits))
        self.scales = make(lambda i, n, k: synth.make_scales(seed, i, n, k))
        for e in poison:
            for m in range(3):
                self.scales[m][e] = np.full_like(self.scales[m][e], NAN16)

    def matrices(self, chosen):
        return {e: tuple(omoe.matrix(self.idx[m][e], self.books[m][e], self.scales[m][e]) for m in range(3)) for e in chosen}

    def on_device(self):
        words = [np.stack([kmq.repack(kmq.pack(i, self.bits), i.shape[1], self.bits, kmq.LAYOUT_TILED) for i in self.idx[m]]) for m in range(3)]
        return kmq.MoeWeights(*(dev(w) for w in words), *(dev(np.stack([b.reshape(-1) for b in self.books[m]])) for m in range(3)),
                              *(dev(np.stack(self.scales[m])) for m in range(3)), self.experts, self.hidden, self.width, self.bits)


def run_experts(weights, x, ids, gates, residual=None, x_stride=None, y_stride=None, behind=1):
    """Output patterns; the buffer starts as NaN, and what is no output stays so."""
    rows, hidden = x.shape
    top_k = ids.shape[1]
    xd = rows_on_device(x, x_stride, behind)
    y = torch.full((rows + behind, y_stride or hidden), NAN16, dtype=torch.int16, device="cuda")
    rd = rows_on_device(residual) if residual is not None else None
    need = kmq.moe_experts_workspace_bytes(weights, rows, top_k)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None      # NaNs: what is read is written first
    kmq.moe_experts(weights, xd, x_stride or hidden, rows, dev(ids), dev(gates), top_k, y, y_stride or hidden, residual=rd,
                    residual_stride=hidden if residual is not None else 0, workspace=ws)
    torch.cuda.synchronize()
    got = host(y)
    assert (got[rows:] == NAN16).all() and (got[:, hidden:] == NAN16).all(), "something behind the output was written"
    return got[:rows, :hidden]


def check_experts(experts, got, x, ids, gates, residual=None, label="", rows=None):
    """Every output (of the rows given) within the bound."""
    mine = np.arange(len(x)) if rows is None else np.asarray(rows)
    chosen = sorted(set(int(i) for i in ids[mine].reshape(-1)) & set(range(experts.experts)))
    matrices = experts.matrices(chosen or [0])
    res = residual[mine] if residual is not None else None
    ids_mine = np.where((ids[mine] >= 0) & (ids[mine] < experts.experts), ids[mine], -1)
    want, pairs = omoe.experts(x[mine], ids_mine, gates[mine], matrices, res)
    most = moe_bound(want, pairs, matrices, experts.hidden, experts.width, np.abs(bf16_value(res)) if res is not None else np.zeros_like(want))
    value = bf16_value(got[mine])
    assert not np.isnan(value).any(), f"{label}: NaN"
    off = np.abs(value - want)
    assert (off <= most).all(), f"{label}: {int((off > most).sum())} outputs off, worst {np.max(off / np.maximum(most, 1e-30)):.2f} of the bound"
    # that is a worst case over thousands of roundings.  Independent ones: those to bf16, of h and of y, are 2^-8 of themselves at most and
    # 2^-8 / sqrt(3) spread evenly, 0.82 * 2^-8 of the output together; those to 32 bits do not count beside them
    size, error = np.sqrt((want ** 2).mean()), np.sqrt((off ** 2).mean())
    assert error <= 2.0 ** -8 * size, f"{label}: error {error / size:.4f} of the outputs"
