"""Attention over 8-bit rows for bf16 heads that share a key head by fours, where rows go to one kernel or the other by their number and
length, and chunks of long rows always to the tensor cores: on both sides of every border, long rows among the short ones.  Definition and bounds
are those of the attention's other tests."""
import pytest
import torch

import paper_2406_17918_b200 as gs
from test_gpu_coded_attention import B, _block, _check, _gen, _reference, _store, _values, _ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,d,block", [(4, 1, 8, 1), (8, 2, 16, 16), (8, 1, 24, 4), (4, 1, 32, 16), (4, 1, 33, 2), (8, 2, 64, 16), (4, 1, 100, 16), (4, 1, 128, 8), (4, 1, 130, 1),
                                           (8, 2, 256, 16)])
@pytest.mark.parametrize("edges", [2, 4, 6, 9, 11, 19, 21])
@pytest.mark.parametrize("longs", [False, True])
def test_rows_of_either_kernel(hq, hk, d, block, edges, longs):
    g = _gen(d * 100 + edges)
    n = 2600 if d > 128 else 5000                             # more than two rounds of the warps that are resident
    lengths = [max(0, edges - 2 + i % 5) for i in range(n)]
    if longs:
        lengths[3], lengths[n // 2], lengths[n - 1] = 700, 65, 3000
    indptr, idx = _block(lengths, 403, g, masked=0.1)
    store = _store(403, 2 * hk, d, block, g)
    q = torch.randn(n, hq, d, generator=g, device="cuda").to(B)
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :hk], both[:, hk:], d ** -0.5, B)
    for max_row in (0, max(lengths)):
        out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, hk), store.heads(hk, 2 * hk), _ws(n, idx.numel(), hq, d), max_row=max_row)
        _check("out", out, want["out"])
        _check("lse", lse, want["lse"])


@pytest.mark.parametrize("cap", [1, 7])
@pytest.mark.parametrize("d,edges", [(16, 5), (64, 3), (64, 12), (256, 4)])
def test_any_grid(cap, d, edges):
    g = _gen(cap)
    lengths = [edges] * 3000 + [900, 0, 70]
    indptr, idx = _block(lengths, 300, g, masked=0.1)
    store = _store(300, 4, d, 16, g)
    q = torch.randn(len(lengths), 8, d, generator=g, device="cuda").to(B)
    args = (indptr, idx, q, store.heads(0, 2), store.heads(2, 4))
    out, lse = gs.gs_coded_attention_forward(*args, _ws(len(lengths), idx.numel(), 8, d))
    gs.gs_debug_set_grid_cap(cap)
    try:
        again, alse = gs.gs_coded_attention_forward(*args, _ws(len(lengths), idx.numel(), 8, d))
    finally:
        gs.gs_debug_set_grid_cap(0)
    assert torch.equal(out, again) and torch.equal(lse, alse)
