"""Norms around a block, router and experts on the host: sizes, and every argument error reported before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2602_15563_amd import kmq

NULL, BITS, SHAPE, ALIGN, WORKSPACE, LAYOUT = 1, 2, 3, 4, 6, 7
lib = kmq.raw()
A = 1 << 20                   # an address that is never looked at: every call here is refused, or has no rows
INF, NAN = float("inf"), float("nan")


def ref(s):
    return ctypes.addressof(s) if s is not None else None


def join(residual=A, gate=A, post=A, pre=A, rs=64, gs=64, scale=1.0, r_scale=1.0, eps=1e-5, norm=1, sigmoid=0):
    return kmq._JoinStruct(residual, gate, post, pre, rs, gs, scale, r_scale, eps, norm, sigmoid)


def norm(x=A, xs=64, rows=0, width=64, j=join(), out=A, os=64, normed=A, ns=64):
    return lib.kmq_block_norm(x, xs, rows, width, ref(j), out, os, normed, ns, None)


def router(w=A, bias=A, width=64, experts=16, top_k=2, groups=4, top_groups=2, sigmoid=0, normalise=1, scale=1.0):
    return kmq._RouterStruct(w, bias, width, experts, top_k, groups, top_groups, sigmoid, normalise, scale)


def route(x=A, xs=64, rows=0, r=router(), ids=A, gates=A, ws=None, n=0):
    return lib.kmq_moe_route(x, xs, rows, ref(r), ids, gates, ws, n, None)


def matrix(words=A, books=A, scales=A):
    return kmq._MatrixStruct(words, books, scales)


def weights(gate=matrix(), up=matrix(), down=matrix(), hidden=512, width=1024, experts=8, bits=4):
    return kmq._WeightsStruct(gate, up, down, hidden, width, experts, bits)


def experts(w=weights(), x=A, xs=512, rows=0, ids=A, gates=A, top_k=2, res=A, rs=512, y=A, ys=512, ws=None, n=0):
    return lib.kmq_moe_experts(ref(w), x, xs, rows, ids, gates, top_k, res, rs, y, ys, ws, n, None)


def experts_workspace(w, rows, top_k):
    return lib.kmq_moe_experts_workspace_bytes(ref(w), rows, top_k)


def test_calls_without_rows_succeed():
    assert norm() == 0 and route() == 0 and experts() == 0
    assert norm(out=None) == 0 and norm(normed=None) == 0 and norm(j=join(residual=None, gate=None, post=None, pre=None)) == 0
    assert norm(j=join(residual=None, rs=3, gate=None, gs=5)) == 0 and norm(j=join(gs=0)) == 0
    assert route(r=router(bias=None, groups=1, top_groups=1)) == 0 and experts(res=None, rs=1) == 0
    assert norm(width=32768, xs=32768, os=32768, ns=32768, j=join(rs=32768, gs=0)) == 0
    assert route(r=router(experts=1024, groups=64, top_groups=1, top_k=16)) == 0


def test_norm():
    for bad in (dict(x=None), dict(j=None), dict(out=None, normed=None)):
        assert norm(**bad) == NULL, bad
    for bad in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(width=0), dict(width=60), dict(width=-8), dict(width=32776, xs=1 << 16, os=1 << 16, ns=1 << 16), dict(xs=56),
                dict(xs=65), dict(xs=1 << 32), dict(os=56), dict(ns=68), dict(j=join(rs=56)), dict(j=join(gs=56)), dict(j=join(gs=-64)), dict(j=join(gs=4)),
                dict(j=join(scale=INF)), dict(j=join(scale=NAN)), dict(j=join(r_scale=-INF)), dict(j=join(eps=-1e-9)), dict(j=join(eps=NAN)), dict(j=join(norm=2)),
                dict(j=join(sigmoid=-1))):
        assert norm(**bad) == SHAPE, bad
    for bad in (dict(x=A + 8), dict(out=A + 2), dict(normed=A + 8), dict(j=join(residual=A + 4)), dict(j=join(gate=A + 8)), dict(j=join(post=A + 2)), dict(j=join(pre=A + 8))):
        assert norm(**bad) == ALIGN, bad


def test_route():
    for bad in (dict(x=None), dict(r=None), dict(ids=None), dict(gates=None), dict(r=router(w=None))):
        assert route(**bad) == NULL, bad
    for bad in (dict(rows=-1), dict(rows=(1 << 20) + 1), dict(rows=1 << 20, r=router(experts=512)), dict(xs=56), dict(xs=66), dict(r=router(width=0)),
                dict(r=router(width=60)), dict(xs=1 << 17, r=router(width=65544)), dict(r=router(experts=0)), dict(r=router(experts=1028)), dict(r=router(experts=18)),
                dict(r=router(groups=0)), dict(r=router(experts=65, groups=65)), dict(r=router(top_groups=0)), dict(r=router(top_groups=5)), dict(r=router(top_k=0)),
                dict(r=router(top_k=9)), dict(r=router(experts=64, top_k=17)), dict(r=router(sigmoid=2)), dict(r=router(normalise=2)), dict(r=router(scale=NAN)),
                dict(r=router(scale=INF))):
        assert route(**bad) == SHAPE, bad
    for bad in (dict(x=A + 8), dict(ids=A + 2), dict(gates=A + 1), dict(r=router(w=A + 8)), dict(r=router(bias=A + 2))):
        assert route(**bad) == ALIGN, bad
    need = lib.kmq_moe_route_workspace_bytes(3, 16, 64)
    assert need > 0 and need % (3 * 16 * 8) == 0
    assert route(rows=3) == WORKSPACE and route(rows=3, ws=A, n=need - 1) == WORKSPACE and route(rows=3, ws=A + 8, n=need) == ALIGN
    for bad in ((-1, 16, 64), (3, 0, 64), (3, 1025, 64), (3, 16, 60), (3, 16, 0), (1 << 20, 512, 64), (0, 16, 64)):
        assert lib.kmq_moe_route_workspace_bytes(*bad) == 0


def test_experts():
    for bad in (dict(w=None), dict(x=None), dict(ids=None), dict(gates=None), dict(y=None), *(dict(w=weights(**{m: matrix(**{f: None})})) for m in ("gate", "up", "down")
                for f in ("words", "books", "scales"))):
        assert experts(**bad) == NULL, bad
    for bits in (0, 5, 8, -1):
        assert experts(w=weights(bits=bits)) == BITS
    for bad in (dict(rows=-1), dict(rows=129), dict(top_k=0), dict(top_k=17), dict(w=weights(hidden=0)), dict(w=weights(width=-128)), dict(w=weights(width=65664)),
                dict(w=weights(experts=0)), dict(w=weights(experts=1025)), dict(xs=504), dict(xs=516), dict(xs=(1 << 22) + 8), dict(rs=504), dict(ys=508)):
        assert experts(**bad) == SHAPE, bad
    for bits, unit in ((1, 512), (2, 256), (3, 128), (4, 128)):
        fits = dict(xs=3 * unit, rs=3 * unit, ys=3 * unit)
        assert experts(w=weights(bits=bits, hidden=3 * unit, width=unit), **fits) == 0
        assert experts(w=weights(bits=bits, hidden=3 * unit - 64, width=unit), **fits) == LAYOUT and experts(w=weights(bits=bits, hidden=unit, width=unit // 2), **fits) == LAYOUT
    for bad in (dict(x=A + 8), dict(res=A + 2), dict(y=A + 8), dict(ids=A + 2), dict(gates=A + 1), dict(w=weights(gate=matrix(words=A + 8))),
                dict(w=weights(up=matrix(books=A + 2))), dict(w=weights(down=matrix(scales=A + 8)))):
        assert experts(**bad) == ALIGN, bad
    need = experts_workspace(weights(), 3, 2)
    assert need >= 3 * 2 * 1024 * 2
    assert experts(rows=3) == WORKSPACE and experts(rows=3, ws=A, n=need - 1) == WORKSPACE and experts(rows=3, ws=A + 8, n=need) == ALIGN
    for bad in ((None, 3, 2), (weights(bits=8), 3, 2), (weights(hidden=100), 3, 2), (weights(), 129, 2), (weights(), 3, 17), (weights(), 0, 2)):
        assert experts_workspace(*bad) == 0


def test_the_binding_checks_what_it_wraps():
    E, H, W, b = 3, 128, 256, 4
    words = lambda n, k: torch.zeros((E, kmq.tiled_words(n, k, b, 1)), dtype=torch.int32)  # noqa: E731
    scales = lambda n, k: torch.zeros((E, n, k // 64), dtype=torch.bfloat16)  # noqa: E731
    books = torch.zeros((E, 16), dtype=torch.bfloat16)
    good = [words(W, H), words(W, H), words(H, W), books, books, books, scales(W, H), scales(W, H), scales(H, W)]
    kmq.MoeWeights(*good, E, H, W, b)
    for i in range(9):
        bad = list(good)
        bad[i] = good[i][:2]
        with pytest.raises(kmq.KmqError):
            kmq.MoeWeights(*bad, E, H, W, b)
        bad[i] = torch.cat([good[i]] * 2)[::2]
        with pytest.raises(kmq.KmqError):
            kmq.MoeWeights(*bad, E, H, W, b)
    for sizes in ((0, H, W, b), (E, H, 100, b), (E, H, W, 2), (E, H, W, 5), (E, 64, W, b)):
        with pytest.raises(kmq.KmqError):
            kmq.MoeWeights(*good, *sizes)


def test_norms_of_more_elements_than_a_launch_has_threads_for():
    assert norm(rows=1 << 24, width=1032, xs=1032, os=1032, ns=1032, j=join(rs=1032, gs=0)) == SHAPE
    assert norm(rows=(1 << 19) + 1, width=32768, xs=32768, os=32768, ns=32768, j=join(rs=32768, gs=0)) == SHAPE


@pytest.mark.parametrize("ids, gates", ((torch.int64, torch.float32), (torch.float32, torch.float32), (torch.int32, torch.bfloat16), (torch.int32, torch.int32)))
def test_choices_of_another_type(ids, gates):
    choice = torch.zeros(2, 2, dtype=ids), torch.zeros(2, 2, dtype=gates)
    x = torch.zeros(2, 512, dtype=torch.bfloat16)
    with pytest.raises(kmq.KmqError) as e:
        kmq.moe_route(x, 512, 2, torch.zeros(16, 512, dtype=torch.bfloat16), 16, 512, *choice, 2)
    assert e.value.status == SHAPE
    w = kmq.MoeWeights.__new__(kmq.MoeWeights)
    w._struct = weights()
    w._at = ref(w._struct)
    with pytest.raises(kmq.KmqError) as e:
        kmq.moe_experts(w, x, 512, 2, *choice, 2, x, 512)
    assert e.value.status == SHAPE
