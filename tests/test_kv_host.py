"""Heads, cache and attention on the host: sizes, and every argument error reported before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2602_15563_amd import kmq

NULL, SHAPE, ALIGN, WORKSPACE = 1, 3, 4, 6
lib = kmq.raw()
A = 1 << 20                   # an address that is never looked at: every call here is refused, or has no rows


def cache(pages=A, books=A, num=4, page=32, heads=2, D=64):
    return kmq._CacheStruct(pages, books, num, page, heads, D)


def batch(table=A, lengths=A, starts=A, rows=0, sequences=2, width=3):
    return kmq._BatchStruct(table, lengths, starts, rows, sequences, width)


def turn(positions=A, freq=A, gq=A, gk=A, eps=1e-5, norm=1, rot=64, inter=0):
    return kmq._TurnStruct(positions, freq, gq, gk, eps, norm, rot, inter)


def ref(s):
    return ctypes.addressof(s) if s is not None else None


def heads(x=A, xs=256, rows=0, nq=2, nk=2, D=64, t=turn(), q=A, qs=128, k=A, ks=128):
    return lib.kmq_qk_norm_rope(x, xs, rows, nq, nk, D, ref(t), q, qs, k, ks, None)


def write(c=cache(), b=batch(), k=A, ks=128, v=A, vs=128, f=lib.kmq_kv_write):
    return f(ref(c), ref(b), k, ks, v, vs, None)


def read(**a):
    return write(f=lib.kmq_kv_read, **a)


def append(c=cache(), b=batch(), x=A, xs=512, nq=4, t=turn(positions=None), q=A, qs=256):
    return lib.kmq_kv_append(ref(c), ref(b), x, xs, nq, ref(t), q, qs, None)


def attend(c=cache(), b=batch(), q=A, qs=256, nq=4, scale=1.0, causal=1, window=0, out=A, os=256, lse=A, ws=None, n=0):
    return lib.kmq_kv_attention(ref(c), ref(b), q, qs, nq, scale, causal, window, out, os, lse, ws, n, None)


def test_page_bytes():
    assert kmq.kv_page_bytes(32, 1, 64) == 32 * 64 * 17 // 16
    assert kmq.kv_page_bytes(1056, 24, 256) == 1056 * 24 * 256 * 17 // 16
    assert kmq.kv_page_bytes(1 << 30, 4096, 256) == (1 << 30) * 4096 * 272
    for bad in ((0, 1, 64), (16, 1, 64), (48, 1, 64), (33, 1, 64), (-32, 1, 64), (32, 0, 64), (32, 4097, 64), (32, 1, 96), (32, 1, 0), ((1 << 30) + 32, 1, 64)):
        assert kmq.kv_page_bytes(*bad) == -1


def test_calls_without_rows_succeed():
    assert heads() == 0 and write() == 0 and read() == 0 and append() == 0 and attend() == 0
    assert heads(nq=0, q=None) == 0 and heads(nk=0, k=None) == 0
    assert heads(t=turn(positions=None, freq=None, rot=0)) == 0 and heads(t=turn(gq=None, gk=None)) == 0
    assert heads(t=turn(eps=-1.0, norm=0, gq=A + 2)) == 0
    assert attend(lse=None) == 0


@pytest.mark.parametrize("call", (write, read, append, attend))
def test_cache_and_batch(call):
    assert call(c=None) == NULL and call(b=None) == NULL
    assert call(c=cache(pages=None)) == NULL and call(c=cache(books=None)) == NULL
    assert call(b=batch(table=None)) == NULL and call(b=batch(lengths=None)) == NULL
    for bad in (dict(num=0), dict(num=1 << 31), dict(page=16), dict(page=40), dict(page=0), dict(heads=0), dict(heads=5000), dict(D=96), dict(D=32)):
        assert call(c=cache(**bad)) == SHAPE, bad
    for bad in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(sequences=0), dict(sequences=-1), dict(sequences=(1 << 20) + 1), dict(width=0), dict(width=1 << 26),
                dict(starts=None, rows=1), dict(starts=None, rows=3)):
        assert call(b=batch(**bad)) == SHAPE, bad
    assert call(c=cache(pages=A + 8)) == ALIGN and call(c=cache(books=A + 2)) == ALIGN
    for bad in (dict(table=A + 2), dict(lengths=A + 1), dict(starts=A + 2)):
        assert call(b=batch(**bad)) == ALIGN, bad


def test_heads():
    for bad in (dict(x=None), dict(t=None), dict(q=None), dict(k=None), dict(t=turn(positions=None)), dict(t=turn(freq=None))):
        assert heads(**bad) == NULL, bad
    for bad in (dict(rows=-1), dict(rows=1 << 25), dict(nq=-1), dict(nk=-1), dict(nq=0, nk=0), dict(nq=5000), dict(D=0), dict(D=4), dict(D=60), dict(D=520),
                dict(xs=248), dict(xs=260), dict(qs=120), dict(ks=129), dict(xs=-256), dict(t=turn(norm=2)), dict(t=turn(inter=2)), dict(t=turn(eps=-1e-9)),
                dict(t=turn(eps=float("nan"))), dict(t=turn(rot=-16)), dict(t=turn(rot=8)), dict(t=turn(rot=80)), dict(t=turn(rot=40))):
        assert heads(**bad) == SHAPE, bad
    for bad in (dict(x=A + 8), dict(q=A + 2), dict(k=A + 4), dict(t=turn(gq=A + 8)), dict(t=turn(gk=A + 2)), dict(t=turn(freq=A + 2)), dict(t=turn(positions=A + 1))):
        assert heads(**bad) == ALIGN, bad


@pytest.mark.parametrize("call", (write, read))
def test_write_and_read(call):
    assert call(k=None) == NULL and call(v=None) == NULL
    for bad in (dict(ks=120), dict(vs=132), dict(ks=0), dict(vs=1 << 32)):
        assert call(**bad) == SHAPE, bad
    assert call(k=A + 8) == ALIGN and call(v=A + 2) == ALIGN


def test_append():
    for bad in (dict(x=None), dict(q=None), dict(t=None), dict(t=turn(freq=None))):
        assert append(**bad) == NULL, bad
    for bad in (dict(nq=0), dict(nq=-4), dict(nq=5000), dict(xs=504), dict(qs=248), dict(t=turn(rot=128)), dict(t=turn(norm=3))):
        assert append(**bad) == SHAPE, bad
    for bad in (dict(x=A + 2), dict(q=A + 8), dict(t=turn(gk=A + 8))):
        assert append(**bad) == ALIGN, bad


def test_attention():
    assert attend(q=None) == NULL and attend(out=None) == NULL
    for bad in (dict(nq=0), dict(nq=3), dict(nq=-2), dict(nq=8192), dict(qs=248), dict(os=260), dict(scale=float("inf")), dict(scale=float("nan")), dict(causal=2),
                dict(window=-1), dict(nq=2048, qs=1 << 17, os=1 << 17, b=batch(rows=1 << 20))):
        assert attend(**bad) == SHAPE, bad
    for bad in (dict(q=A + 8), dict(out=A + 2), dict(lse=A + 2)):
        assert attend(**bad) == ALIGN, bad
    wide = dict(c=cache(heads=4096), nq=4096, qs=1 << 18, os=1 << 18)                # more workgroups than a launch takes
    assert attend(b=batch(rows=1 << 18, sequences=1 << 18, starts=None), **wide) == SHAPE
    assert attend(b=batch(rows=1024, sequences=1 << 20), **wide) == SHAPE
    assert lib.kmq_kv_attention_workspace_bytes(ref(cache(heads=4096)), ref(batch(rows=1024, sequences=1 << 20)), 4096) == 0
    long = batch(rows=1, sequences=1, width=4096)
    need = lib.kmq_kv_attention_workspace_bytes(ref(cache()), ref(long), 4)
    assert need > 0
    assert attend(b=long) == WORKSPACE and attend(b=long, ws=A, n=need - 1) == WORKSPACE and attend(b=long, ws=A + 4, n=need) == ALIGN


def test_workspace_and_name():
    """Both go by the structures' numbers alone, and both take the arguments that the call takes."""
    assert lib.kmq_kv_attention_workspace_bytes(ref(cache()), ref(batch(rows=2, sequences=2, width=1)), 4) == 0
    assert lib.kmq_kv_attention_workspace_bytes(None, None, 4) == 0 and lib.kmq_kv_attention_workspace_bytes(ref(cache()), ref(batch()), 3) == 0
    assert lib.kmq_kernel_name_kv_attention(ref(cache()), ref(batch(rows=2)), 4).startswith(b"kv_attention")
    assert lib.kmq_kernel_name_kv_attention(ref(cache(D=32)), ref(batch(rows=2)), 4) == b"invalid"
    assert lib.kmq_kernel_name_kv_attention(ref(cache()), ref(batch(rows=2)), 5) == b"invalid"


def test_the_binding_checks_what_it_wraps():
    pages, books = torch.zeros(4 * kmq.kv_page_bytes(32, 1, 64), dtype=torch.uint8), torch.zeros((2, 16), dtype=torch.bfloat16)
    kmq.KvCache(pages, books, 4, 32, 1, 64)
    for bad in ((pages, books, 5, 32, 1, 64), (pages, books[:1], 4, 32, 1, 64), (pages, books, 0, 32, 1, 64), (pages, books, 4, 32, 1, 65), (pages[::2], books, 2, 32, 1, 64)):
        with pytest.raises(kmq.KmqError):
            kmq.KvCache(*bad)
    table, lengths, starts = (torch.zeros(s, dtype=torch.int32) for s in ((2, 3), 2, 3))
    kmq.KvBatch(table, lengths, starts, 7)
    assert kmq.KvBatch(table, lengths).rows == 2
    for bad in ((table, lengths, starts), (table.long(), lengths, starts, 7), (table, lengths[:1], starts, 7), (table, lengths, lengths, 7),
                (table.float(), lengths, starts, 7), (table.t(), starts, None)):
        with pytest.raises(kmq.KmqError):
            kmq.KvBatch(*bad)
