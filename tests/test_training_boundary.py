"""The training operators' C entry points reject bad arguments on the host, before any CUDA call."""
import ctypes

import pytest

import paper_2406_17918_b200 as gs

i32, i64, f32, sz, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p
WS = 0x100000


@pytest.fixture(scope="module")
def L():
    lib = ctypes.CDLL(gs.library_path())
    lib.gs_last_error.restype = ctypes.c_char_p
    lib.gs_kernel_launches.restype = ctypes.c_int64
    return lib


def _lookup(L, table=0x1000, tt=0, rows=10, dim=8, ld=8, ids=0x2000, n=4, out=0x4000, ot=0, old=8):
    return L.gs_embedding_lookup(vp(table), tt, i64(rows), i32(dim), i64(ld), vp(ids), None, i32(n), f32(1), vp(out), ot, i64(old), None)


def test_embedding_lookup(L):
    assert _lookup(L, n=0) == 0                              # nothing to do, nothing launched
    assert _lookup(L, tt=7) == 1 and _lookup(L, ot=-1) == 1
    assert _lookup(L, rows=0) == 1 and _lookup(L, rows=1 << 31) == 1
    assert _lookup(L, dim=0) == 1 and _lookup(L, n=-1) == 1
    assert _lookup(L, table=0) == 1 and _lookup(L, ids=0) == 1 and _lookup(L, out=0) == 1
    assert _lookup(L, ld=7) == 1 and b"pitch" in L.gs_last_error()
    assert _lookup(L, old=7) == 1
    assert _lookup(L, table=0x1002) == 2 and _lookup(L, ids=0x2001) == 2 and _lookup(L, out=0x4001, ot=1) == 2


def _grad(L, dout=0x1000, dt=0, dld=8, ids=0x2000, n=4, rows=10, dim=8, out=0x4000, ot=0, old=8, ws=WS, wsb=1 << 30):
    return L.gs_embedding_backward(vp(dout), dt, i64(dld), vp(ids), None, i32(n), i64(rows), i32(dim), f32(1), vp(out), ot, i64(old), vp(ws), sz(wsb), None)


def test_embedding_gradient(L):
    need = sz()
    assert L.gs_embedding_workspace_bytes(i32(1000), i64(50), i32(16), ctypes.byref(need)) == 0 and need.value > 1000 * 16
    assert L.gs_embedding_workspace_bytes(i32(-1), i64(50), i32(16), ctypes.byref(need)) == 1
    assert L.gs_embedding_workspace_bytes(i32(5), i64(50), i32(16), None) == 1
    assert _grad(L, dt=3) == 1 and _grad(L, n=-1) == 1 and _grad(L, n=1 << 30) == 1 and _grad(L, rows=0) == 1
    assert _grad(L, dout=0) == 1 and _grad(L, ids=0) == 1 and _grad(L, out=0) == 1
    assert _grad(L, dld=7) == 1 and _grad(L, old=4) == 1 and _grad(L, dld=1 << 31) == 1
    assert _grad(L, ws=0) == 1 and _grad(L, ws=WS + 16) == 2 and _grad(L, wsb=64) == 4
    assert L.gs_embedding_backward_sparse(vp(0x1000), 0, i64(8), vp(0x2000), None, i32(4), i64(10), i32(8), f32(1), None, vp(0x3000), vp(0x4000), 0,
                                          i64(8), vp(WS), sz(1 << 30), None) == 1


class Block(ctypes.Structure):
    _fields_ = [("max_dst", i32), ("max_src", i32), ("max_edges", i32), ("n", vp * 3), ("indptr", vp), ("indices", vp)]


class Heads(ctypes.Structure):
    _fields_ = [("data", vp), ("row", i64), ("head", i64)]


def _block(dst=4, src=9, edges=12, counts=(None, None, None), indptr=0x1000, indices=0x2000):
    b = Block(dst, src, edges, (vp * 3)(*counts), indptr, indices)
    return ctypes.byref(b)


def _attend(L, block=None, max_row=0, t=0, hq=4, hk=2, d=8, q=(0x10000, 32, 8), k=(0x20000, 16, 8), lse=0x3000, ws=WS, wsb=1 << 30):
    h = lambda x: ctypes.byref(Heads(*x))  # noqa: E731
    return L.gs_block_attention_forward(_block() if block is None else block, i32(max_row), t, i32(hq), i32(hk), i32(d), f32(1), h(q), h(k), h(k), h(q),
                                        vp(lse), vp(ws), sz(wsb), None)


def test_block_attention(L):
    need = sz()
    assert L.gs_block_attention_workspace_bytes(i32(4), i32(12), i32(4), i32(8), ctypes.byref(need)) == 0 and need.value > 0
    assert L.gs_block_attention_workspace_bytes(i32(4), i32(12), i32(4), i32(257), ctypes.byref(need)) == 1
    assert _attend(L, block=_block(dst=0)) == 0
    assert _attend(L, block=ctypes.cast(None, ctypes.POINTER(Block))) == 1
    assert _attend(L, block=_block(dst=-1)) == 1 and _attend(L, block=_block(indptr=None)) == 1 and _attend(L, block=_block(indices=None)) == 1
    assert _attend(L, block=_block(counts=(0x9000, None, None))) == 1       # device counts: all or none
    assert _attend(L, block=_block(indices=0x2002)) == 2
    assert _attend(L, max_row=-1) == 1 and _attend(L, t=2) == 1
    assert _attend(L, hq=0) == 1 and _attend(L, hk=3) == 1 and _attend(L, hq=256, hk=1) == 1 and _attend(L, d=0) == 1 and _attend(L, d=300) == 1
    assert _attend(L, q=(0, 32, 8)) == 1 and _attend(L, q=(0x10000, 7, 8)) == 1 and _attend(L, k=(0x20000, 16, 4)) == 1
    assert _attend(L, q=(0x10002, 32, 8)) == 2 and _attend(L, lse=0) == 1 and _attend(L, lse=0x3002) == 2
    assert _attend(L, ws=0) == 1 and _attend(L, ws=WS + 4) == 2 and _attend(L, wsb=100) == 4
    rev = lambda p, d, e, w=1 << 30: L.gs_block_reverse(_block(), vp(p), vp(d), vp(e), vp(WS), sz(w), None)  # noqa: E731
    assert rev(0, 0x2000, 0x3000) == 1 and rev(0x1000, 0, 0x3000) == 1 and rev(0x1000, 0x2000, 0) == 1
    assert rev(0x1001, 0x2000, 0x3000) == 2 and rev(0x1000, 0x2000, 0x3000, 8) == 4


def _xent(L, h=0x10000, hld=16, w=0x20000, wld=16, t=1, rows=4, vocab=9, dim=16, y=0x3000, loss=0x4000, lse=0x5000, ws=WS, wsb=1 << 30):
    return L.gs_xent_forward(vp(h), i64(hld), vp(w), i64(wld), t, i32(rows), i64(vocab), i32(dim), f32(1), vp(y), vp(loss), vp(lse), vp(ws), sz(wsb), None)


def test_cross_entropy(L):
    need = sz()
    assert L.gs_xent_workspace_bytes(i32(4), i64(9), i32(16), 1, ctypes.byref(need)) == 0 and need.value > 0
    assert L.gs_xent_workspace_bytes(i32(4), i64(0), i32(16), 1, ctypes.byref(need)) == 1
    assert L.gs_xent_workspace_bytes(i32(4), i64((1 << 31) - 100), i32(16), 1, ctypes.byref(need)) == 1
    assert _xent(L, rows=0, ws=0) == 0
    assert _xent(L, t=5) == 1 and _xent(L, rows=-1) == 1 and _xent(L, vocab=0) == 1 and _xent(L, dim=0) == 1 and _xent(L, dim=5000) == 1
    assert _xent(L, h=0) == 1 and _xent(L, w=0) == 1 and _xent(L, y=0) == 1 and _xent(L, loss=0) == 1 and _xent(L, lse=0) == 1
    assert _xent(L, hld=15) == 1 and _xent(L, wld=8) == 1
    assert _xent(L, h=0x10001) == 2 and _xent(L, y=0x3002) == 2 and _xent(L, loss=0x4002) == 2
    assert _xent(L, ws=0) == 1 and _xent(L, ws=WS + 8) == 2 and _xent(L, wsb=8) == 4
    back = lambda **k: L.gs_xent_backward(vp(0x10000), i64(16), vp(0x20000), i64(16), 1, i32(4), i64(9), i32(16), f32(1), vp(0x3000), vp(k.get("lse", 0x5000)),  # noqa: E731
                                          vp(k.get("dl", 0x6000)), vp(k.get("dh", 0x7000)), i64(k.get("dhld", 16)), vp(k.get("dw", 0x8000)), i64(k.get("dwld", 16)),
                                          k.get("gt", 1), vp(WS), sz(1 << 30), None)
    for bad, status in ((dict(lse=0), 1), (dict(dl=0), 1), (dict(dh=0), 1), (dict(dw=0), 1), (dict(dhld=8), 1), (dict(dwld=8), 1), (dict(gt=9), 1),
                        (dict(dh=0x7001), 2), (dict(dl=0x6002), 2)):
        assert back(**bad) == status, bad


def test_nothing_was_launched(L):
    assert L.gs_kernel_launches() == 0
