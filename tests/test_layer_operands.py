"""Operands around an attention layer whose memory overlaps, or whose sizes no kernel counts to: refused on the host, before any CUDA call."""
import ctypes

import pytest

import paper_2406_17918_b200 as gs

i32, i64, f32, sz, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p
X, R, H, O = 0x10000, 0x20000, 0x40000, 0x50000
N, D = 4, 8                                                   # f32: rows of 32 bytes


@pytest.fixture(scope="module")
def L():
    lib = ctypes.CDLL(gs.library_path())
    lib.gs_last_error.restype = ctypes.c_char_p
    lib.gs_kernel_launches.restype = ctypes.c_int64
    return lib


def _forward(L, x=(X, D), r=(R, D), h=(H, D), o=(O, D), n=N):
    status = L.gs_rms_norm_forward(vp(x[0]), i64(x[1]), vp(r[0]), i64(r[1]), 0, None, 0, None, i32(n), i32(D), f32(1e-6), vp(h[0]), i64(h[1]), vp(o[0]), i64(o[1]), None)
    assert status == 1 and b"overlap" in L.gs_last_error()


def test_results_of_the_norm(L):
    _forward(L, h=(O, D))                                     # h would be written and then overwritten
    _forward(L, h=(X, D), o=(X, D))
    _forward(L, h=(O + 4, D))
    _forward(L, h=(O + 32, D))                                # a row further
    _forward(L, h=(O + 3 * 32, D))                            # its first row is the other's last
    _forward(L, h=(O, 20), o=(O + 7 * 4, 20))                 # columns 0 to 7 and 7 to 14 of rows of 20
    _forward(L, h=(O, 20), o=(O + 13 * 4, 20))                # columns 13 to 20: the next row's first
    _forward(L, h=(O, 16), o=(O + 8 * 4, 20))                 # two pitches in one range


def test_results_across_operands_of_the_norm(L):
    _forward(L, o=(X + 4, D))
    _forward(L, o=(X, D + 1))                                 # the array of x, at another pitch
    _forward(L, h=(R + 32, D))
    _forward(L, h=(R, 12))
    _forward(L, x=(X, 16), o=(X + 28, 16))


def test_gradient_across_operands(L):
    def call(dx, ld=D, h=(X, D), dy=(R, D), dh=(H, D)):
        status = L.gs_rms_norm_backward(vp(h[0]), i64(h[1]), vp(dy[0]), i64(dy[1]), vp(dh[0]), i64(dh[1]), 0, None, 0, None, i32(N), i32(D), f32(1e-6), vp(dx), i64(ld),
                                        None, vp(0x100000), sz(1 << 20), None)
        assert status == 1 and b"overlap" in L.gs_last_error()

    for array in (X, R, H):
        call(array + 4)
        call(array + 32)
        call(array, ld=D + 4)


class Coded(ctypes.Structure):
    _fields_ = [("codes", vp), ("scales", vp), ("rows", i64), ("row_stride", i64), ("scale_stride", i64), ("heads", i32), ("head_dim", i32), ("block", i32)]


class Heads(ctypes.Structure):
    _fields_ = [("data", vp), ("row", i64), ("head", i64)]


def test_norm_in_eight_bits(L):
    c = Coded(0x90000, 0xA0000, N, 16, 1, 1, D, 1)
    assert L.gs_rms_norm_coded(vp(X), i64(D), vp(R), i64(D), 0, None, 0, None, i32(N), i32(D), f32(1e-6), vp(X + 4), i64(D), ctypes.byref(c), None) == 1
    assert b"overlap" in L.gs_last_error()


@pytest.mark.parametrize("heads,dim", [(1 << 16, 1 << 16), (1 << 16, 32769), (1 << 14, 1 << 16), (1 << 16, 16369)])
def test_rows_in_eight_bits_of_2_30_bytes(L, heads, dim):
    """A lane counts a row's pieces in 32 bits."""
    c = Coded(0x90000, 0xA0000, 1, 0, 0, heads, dim, 1)
    a = Heads(0x100000, 0, dim)
    assert L.gs_coded_read(ctypes.byref(c), None, i64(0), None, i32(0), 1, ctypes.byref(a), None) == 1 and b"2^30" in L.gs_last_error()
    assert L.gs_coded_write(ctypes.byref(c), 1, ctypes.byref(a), None, i64(0), None, i32(0), None, None) == 1 and b"2^30" in L.gs_last_error()


def test_nothing_was_launched(L):
    assert L.gs_kernel_launches() == 0
