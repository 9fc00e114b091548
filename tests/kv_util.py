"""A cache and a batch over it, on the host (oracle) and on the device (library), for the tests of heads, cache and attention."""
import numpy as np
import torch

from oracle import kv as okv
from paper_2602_15563_amd import kmq
from paper_2602_15563_amd.tolerance import attention_bound, attention_lse_bound

NAN16 = 0x7FC1


def patterns(x):
    return okv.round_bf16(np.asarray(x, dtype=np.float64))


def dev(a):
    a = np.ascontiguousarray(a)
    view = {np.dtype(np.uint16): np.int16, np.dtype(np.uint32): np.int32}.get(a.dtype, a.dtype)
    return torch.from_numpy(a.view(view)).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint16)


def codebooks(g):
    """Two ascending codebooks in [-1, 1]."""
    c = np.sort(np.linspace(-1, 1, 16) + g.uniform(-0.05, 0.05, (2, 16)), axis=1).clip(-1, 1)
    return patterns(c)


class Case:
    """news: rows of every sequence; lengths: cached tokens of every one (the rows among them).  Pages of all sequences are mixed;
    `behind` rows belong to no sequence.  The cache starts with random bytes and finite scales (other tokens' values)."""

    def __init__(self, seed, news, lengths, page_size, kv_heads, head_dim, behind=0, spare=1, width=None, starts=True):
        g = self.g = np.random.default_rng(seed)
        self.news, self.lengths = list(news), list(lengths)
        self.kv_heads, self.D, self.page_size = kv_heads, head_dim, page_size
        used = [max(0, -(-m // page_size)) for m in lengths]
        self.width = width or max(1, max(used))
        used = [min(u, self.width) for u in used]
        self.num_pages = sum(used) + spare
        order = g.permutation(self.num_pages).astype(np.int32)
        self.table = np.full((len(used), self.width), -1, dtype=np.int32)
        at = 0
        for i, u in enumerate(used):
            self.table[i, :u] = order[at:at + u]
            at += u
        self.starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.rows = int(self.starts[-1]) + behind
        self.has_starts = starts
        assert starts or (set(news) == {1} and not behind)
        self.books = codebooks(g)
        fill = g.integers(0, 256, self.num_pages * kv_heads * (page_size // 16) * 17 * head_dim, dtype=np.uint8)
        tiles = fill.reshape(-1, 17 * head_dim)
        tiles[:, 16 * head_dim:] = patterns(g.uniform(0.5, 3.0, (tiles.shape[0], head_dim // 2))).view(np.uint8)
        self.pages = okv.Pages(self.num_pages, page_size, kv_heads, head_dim, fill=fill)

    def to_device(self):
        self.pages_d = dev(self.pages.bytes)
        self.cache = kmq.KvCache(self.pages_d, dev(self.books), self.num_pages, self.page_size, self.kv_heads, self.D)
        self.batch = kmq.KvBatch(dev(self.table), dev(np.array(self.lengths, dtype=np.int32)), dev(self.starts) if self.has_starts else None, self.rows)
        return self

    def position(self, row):
        """(sequence, position) of a row; (-1, 0) behind the last."""
        for b, n in enumerate(self.news):
            if self.starts[b] <= row < self.starts[b + 1]:
                return b, self.lengths[b] - n + row - self.starts[b]
        return -1, 0

    def places(self):
        """(row, page, token) of every row that has a place in the cache."""
        for row in range(self.rows):
            b, p = self.position(row)
            at = okv.place(self.table[b], self.page_size, self.num_pages, p) if b >= 0 else None
            if at:
                yield row, at[0], at[1]

    def check_pages(self):
        """The device's pages are the oracle's, byte for byte."""
        got = self.pages_d.cpu().numpy()
        assert np.array_equal(got, self.pages.bytes), f"{int((got != self.pages.bytes).sum())} bytes of the pages differ"


def run_attention(c, q, q_heads, scale, causal=True, window=0, out=None, stride=None, workspace=None, lse=True):
    """Attention of q (rows, heads, D; patterns) on the device: output patterns and lse, both of them first filled with NaN."""
    q_heads, D = q.shape[1], q.shape[2]
    row = q_heads * D
    stride = stride or row
    qd = torch.full((c.rows, stride), NAN16, dtype=torch.int16, device="cuda")
    qd[:, :row] = dev(q.reshape(c.rows, row))
    out = torch.full((c.rows, stride), NAN16, dtype=torch.int16, device="cuda")
    lse_d = torch.full((c.rows, q_heads), float("nan"), dtype=torch.float32, device="cuda") if lse else None
    need = kmq.kv_attention_workspace_bytes(c.cache, c.batch, q_heads)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None       # NaNs: a part that is read is written first
    kmq.kv_attention(c.cache, c.batch, qd, stride, out, stride, q_heads, scale, causal=causal, window=window, lse=lse_d, workspace=ws)
    torch.cuda.synchronize()
    got = host(out)
    assert (got[:, row:] == NAN16).all(), "the output's rows end before their stride"
    return got[:, :row].reshape(c.rows, q_heads, D), lse_d.cpu().numpy() if lse else None


def check_attention(c, q, scale, causal=True, window=0, rows=None, label="", **more):
    """Runs it and compares every row (or those given) with the oracle; rows behind the last sequence are untouched."""
    got, lse = run_attention(c, q, q.shape[1], scale, causal, window, **more)
    value = okv.bf16_value(got)
    for b, n in enumerate(c.news):
        if not n:
            continue
        k, v, there = okv.sequence(c.pages, c.table[b], c.lengths[b], c.books)
        mine = slice(c.starts[b], c.starts[b + 1])
        out, want, spread, size = okv.attention(q[mine], k, v, there, c.lengths[b], scale, causal, window)
        tokens = max(1, len(there))
        off, most = np.abs(value[mine] - out), attention_bound(out, spread, size, tokens, c.D)
        assert not np.isnan(value[mine]).any(), f"{label}: NaN in sequence {b}"
        assert (off <= most).all(), f"{label}: sequence {b}: {int((off > most).sum())} outputs off, worst {np.max(off / np.maximum(most, 1e-30)):.2f} of the bound"
        if lse is not None:
            empty = np.isneginf(want)
            assert np.array_equal(np.isneginf(lse[mine]), empty), f"{label}: sequence {b}: rows that see nothing"
            far = np.abs(lse[mine].astype(np.float64) - want)[~empty] - attention_lse_bound(size, tokens, c.D)[~empty]
            assert (far <= 0).all(), f"{label}: sequence {b}: log-sum-exp off by {far.max():.2e} more than the bound"
            assert (value[mine][empty] == 0).all()
    end = c.starts[-1]
    assert (got[end:] == NAN16).all(), f"{label}: rows behind the last sequence were written"
    if lse is not None:
        assert np.isnan(lse[end:]).all()
    return got, lse
