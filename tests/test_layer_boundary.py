"""The C entry points around an attention layer reject bad arguments on the host, before any CUDA call."""
import ctypes

import pytest
import torch

import paper_2406_17918_b200 as gs

i32, i64, f32, sz, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p
WS = 0x100000


@pytest.fixture(scope="module")
def L():
    lib = ctypes.CDLL(gs.library_path())
    lib.gs_last_error.restype = ctypes.c_char_p
    lib.gs_kernel_launches.restype = ctypes.c_int64
    return lib


class Heads(ctypes.Structure):
    _fields_ = [("data", vp), ("row", i64), ("head", i64)]


class Coded(ctypes.Structure):
    _fields_ = [("codes", vp), ("scales", vp), ("rows", i64), ("row_stride", i64), ("scale_stride", i64), ("heads", i32), ("head_dim", i32), ("block", i32)]


class Block(ctypes.Structure):
    _fields_ = [("max_dst", i32), ("max_src", i32), ("max_edges", i32), ("n", vp * 3), ("indptr", vp), ("indices", vp)]


class Grad(ctypes.Structure):
    _fields_ = [("grad", vp), ("out", vp), ("elems", i64), ("rows", vp), ("row_elems", i64), ("dtype", i32)]


def _coded(codes=0x10000, scales=0x20001, rows=100, row_stride=64, scale_stride=4, heads=4, head_dim=16, block=16):
    return Coded(codes, scales, rows, row_stride, scale_stride, heads, head_dim, block)


def _norm(L, x=0x1000, xld=8, r=0x2000, rld=8, t=0, w=0x3000, wt=0, n=4, d=8, eps=1e-6, h=0x4000, hld=8, out=0x5000, old=8, count=None):
    return L.gs_rms_norm_forward(vp(x), i64(xld), vp(r), i64(rld), t, vp(w), wt, vp(count), i32(n), i32(d), f32(eps), vp(h), i64(hld), vp(out), i64(old), None)


def test_norm(L):
    need = sz()
    assert L.gs_rms_norm_workspace_bytes(i32(10), i32(64), ctypes.byref(need)) == 0 and need.value >= 64 * 4
    assert L.gs_rms_norm_workspace_bytes(i32(-1), i32(64), ctypes.byref(need)) == 1 and L.gs_rms_norm_workspace_bytes(i32(1), i32(8193), ctypes.byref(need)) == 1
    assert L.gs_rms_norm_workspace_bytes(i32(1), i32(8), None) == 1
    assert _norm(L, n=0, x=0, out=0) == 0
    assert _norm(L, t=2) == 1 and _norm(L, wt=5) == 1 and _norm(L, n=-1) == 1 and _norm(L, d=0) == 1 and _norm(L, d=8193, xld=9000) == 1
    assert _norm(L, eps=-1.0) == 1 and _norm(L, eps=float("nan")) == 1
    assert _norm(L, x=0) == 1 and _norm(L, out=0) == 1
    assert _norm(L, xld=7) == 1 and _norm(L, rld=7) == 1 and _norm(L, hld=7) == 1 and _norm(L, old=7) == 1 and b"pitch" in L.gs_last_error()
    assert _norm(L, x=0x1002) == 2 and _norm(L, t=1, r=0x2001) == 2 and _norm(L, w=0x3002) == 2 and _norm(L, count=0x9001) == 2 and _norm(L, out=0x5001, t=1) == 2


def test_norm_in_eight_bits(L):
    def call(out, n=4, d=64, x=0x1000):
        return L.gs_rms_norm_coded(vp(x), i64(d), None, i64(0), 0, None, 0, None, i32(n), i32(d), f32(0), None, i64(0), None if out is None else ctypes.byref(out), None)

    assert call(_coded(block=1), n=0) == 0
    assert call(None) == 1 and call(_coded(block=16)) == 1 and call(_coded(block=1), d=60) == 1 and call(_coded(block=1, rows=3)) == 1
    assert call(_coded(block=1, codes=0)) == 1 and call(_coded(block=1, codes=0x10008)) == 2 and call(_coded(block=1), x=0) == 1


def test_norm_gradient(L):
    def call(h=0x1000, dy=0x2000, dh=0x3000, dx=0x4000, dw=0x5000, n=4, d=8, ld=8, ws=WS, wsb=1 << 20, w=0x6000, wt=0):
        return L.gs_rms_norm_backward(vp(h), i64(ld), vp(dy), i64(ld), vp(dh), i64(ld), 0, vp(w), wt, None, i32(n), i32(d), f32(1e-6), vp(dx), i64(ld), vp(dw),
                                      vp(ws), sz(wsb), None)

    assert call(h=0) == 1 and call(dy=0) == 1 and call(dx=0) == 1 and call(ld=4) == 1 and call(wt=3) == 1 and call(w=0, wt=3) == 1
    assert call(dx=0x4002) == 2 and call(dw=0x5001) == 2 and call(ws=0) == 1 and call(ws=WS + 8) == 2 and call(wsb=8) == 4
    assert call(n=0, dw=0, ws=0) == 0


def test_stores(L):
    def write(c, t=0, rows=(0x30000, 64, 16), ids=0x4000, first=0, n=4, claims=0x5000, count=None):
        return L.gs_coded_write(ctypes.byref(c), t, ctypes.byref(Heads(*rows)), vp(ids), i64(first), vp(count), i32(n), vp(claims), None)

    def read(c, t=1, out=(0x30000, 64, 16), ids=0x4000, first=0, n=4):
        return L.gs_coded_read(ctypes.byref(c), vp(ids), i64(first), None, i32(n), t, ctypes.byref(Heads(*out)), None)

    assert write(_coded(), n=0) == 0 and read(_coded(), n=0) == 0 and write(_coded(rows=0, codes=0, scales=0)) == 0
    for call in (write, read):
        for bad in (dict(rows=-1), dict(rows=1 << 31), dict(heads=0), dict(head_dim=0), dict(head_dim=(1 << 16) + 1), dict(block=0), dict(block=3), dict(block=128),
                    dict(codes=0), dict(scales=0), dict(row_stride=48), dict(row_stride=72), dict(scale_stride=3), dict(head_dim=17)):
            assert call(_coded(**bad)) == 1, bad
        assert call(_coded(codes=0x10008)) == 2
        assert call(_coded(), t=2) == 1 and call(_coded(), n=-1) == 1 and call(_coded(), ids=0x4002) == 2
        assert call(_coded(), ids=0, first=-1) == 1 and call(_coded(), ids=0, first=97) == 1 and b"range" in L.gs_last_error()
    assert write(_coded(), rows=(0, 64, 16)) == 1 and write(_coded(), rows=(0x30000, 15, 16)) == 1 and write(_coded(), rows=(0x30002, 64, 16)) == 2
    assert write(_coded(), claims=0) == 1 and write(_coded(), claims=0x5002) == 2 and write(_coded(), count=0x6001) == 2
    assert read(_coded(), out=(0, 64, 16)) == 1 and read(_coded(), out=(0x30001, 64, 16)) == 2


def test_attention_over_a_store(L):
    def call(k=None, v=None, dst=4, src=9, edges=12, rows=None, max_row=0, t=0, hq=4, d=16, q=(0x10000, 64, 16), lse=0x3000, ws=WS, wsb=1 << 30, indptr=0x1000):
        b = Block(dst, src, edges, (vp * 3)(None, None, None), indptr, 0x2000)
        k, v = k or _coded(heads=2), v or _coded(heads=2)
        return L.gs_coded_attention_forward(ctypes.byref(b), vp(rows), i32(max_row), t, i32(hq), i32(d), f32(1), ctypes.byref(Heads(*q)), ctypes.byref(k), ctypes.byref(v),
                                            ctypes.byref(Heads(*q)), vp(lse), vp(ws), sz(wsb), None)

    need = sz()
    assert L.gs_coded_attention_workspace_bytes(i32(12), i32(4), i32(16), ctypes.byref(need)) == 0 and need.value > 0
    for bad in ((-1, 4, 16), (1 << 30, 4, 16), (1, 0, 16), (1, 129, 16), (1, 4, 0), (1, 4, 257)):
        assert L.gs_coded_attention_workspace_bytes(*(i32(x) for x in bad), ctypes.byref(need)) == 1
    assert L.gs_coded_attention_workspace_bytes(i32(1), i32(1), i32(1), None) == 1
    assert call(dst=0) == 0
    assert call(dst=-1) == 1 and call(indptr=None) == 1 and call(max_row=-1) == 1 and call(t=2) == 1 and call(d=0) == 1 and call(d=257) == 1
    assert call(hq=0) == 1 and call(hq=3) == 1 and call(hq=130) == 1 and call(d=8) == 1
    assert call(src=101) == 1 and b"sources" in L.gs_last_error()
    assert call(v=_coded(heads=2, rows=99)) == 1 and call(v=_coded(heads=2, block=8)) == 1 and call(v=_coded(heads=4)) == 1 and call(k=_coded(heads=2, block=5)) == 1
    assert call(q=(0, 64, 16)) == 1 and call(q=(0x10001, 64, 16)) == 2 and call(lse=0) == 1 and call(lse=0x3002) == 2 and call(rows=0x5002) == 2
    assert call(ws=0) == 1 and call(ws=WS + 16) == 2 and call(wsb=64) == 4


def test_gradients(L):
    def clip(grads, max_norm=1.0, ws=WS, wsb=1 << 20, norm=0x9000, n=None):
        a = (Grad * max(1, len(grads)))(*[Grad(*g) for g in grads])
        return L.gs_grad_clip(a, i32(len(grads) if n is None else n), f32(max_norm), vp(norm), vp(ws), sz(wsb), None)

    need = sz()
    assert L.gs_grad_workspace_bytes(i32(3), ctypes.byref(need)) == 0 and need.value > 0
    assert L.gs_grad_workspace_bytes(i32(-1), ctypes.byref(need)) == 1 and L.gs_grad_workspace_bytes(i32(65537), ctypes.byref(need)) == 1
    assert L.gs_grad_norm(None, i32(1), vp(0x9000), vp(WS), sz(1 << 20), None) == 1
    assert L.gs_grad_norm(None, i32(0), None, vp(WS), sz(1 << 20), None) == 1
    ok = (0x10000, 0x10000, 100, None, 0, 0)
    assert clip([ok], n=-1) == 1 and clip([ok], max_norm=-0.5) == 1 and clip([ok], max_norm=float("nan")) == 1 and clip([ok], norm=0x9002) == 2
    for bad, status in (((0, 0x10000, 100, None, 0, 0), 1), ((0x10000, 0, 100, None, 0, 0), 1), ((0x10000, 0x10000, -1, None, 0, 0), 1), ((0x10000, 0x10000, 4, None, 0, 7), 1),
                        ((0x10000, 0x10000, 100, 0x8000, 0, 0), 1), ((0x10000, 0x10000, 100, 0x8000, 101, 0), 1), ((0x10000, 0x10000, 100, 0x8001, 10, 0), 2),
                        ((0x10002, 0x10002, 100, None, 0, 0), 2), ((0x10000, 0x10010, 100, None, 0, 0), 1)):
        assert clip([bad]) == status, bad
    assert clip([ok, ok]) == 1 and b"overlap" in L.gs_last_error()
    assert clip([ok, (0x20000, 0x10004, 10, None, 0, 0)]) == 1 and clip([(0x30000, 0x10000, 100, None, 0, 0), (0x10000, 0x40000, 100, None, 0, 0)]) == 1
    assert clip([ok], ws=0) == 1 and clip([ok], ws=WS + 4) == 2 and clip([ok], wsb=16) == 4


def test_binding_refuses_on_the_cpu():
    x, w, ws = torch.ones(4, 8), torch.ones(8), torch.empty(1 << 20, dtype=torch.uint8)
    for call in (lambda: gs.gs_rms_norm_forward(x, w), lambda: gs.gs_rms_norm_backward(x, x, ws), lambda: gs.gs_grad_norm([x], ws), lambda: gs.gs_grad_clip([x], 1.0, ws),
                 lambda: gs.CodedRows(torch.zeros(4, 2, 16, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 16)):
        with pytest.raises((TypeError, ValueError)):
            call()


def test_nothing_was_launched(L):
    assert L.gs_kernel_launches() == 0
