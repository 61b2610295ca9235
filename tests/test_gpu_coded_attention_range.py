"""Attention over 8-bit rows where the results hang on little: edges beside a sink without a value, columns that the heavy edges leave at
zero, scores from columns far below a query's largest, keys and queries whose sizes cancel.  Definition, bounds and helpers are those of
the attention's other tests; every bound is relative to what the element itself sums up, so none is met by leaving small things out."""
import pytest
import torch

import paper_2406_17918_b200 as gs
from test_gpu_coded_attention import B, F, _block, _check, _gen, _reference, _values, _ws

pytestmark = pytest.mark.gpu


def _compare(indptr, idx, q, store, hk, tiny=None):
    """tiny: for results smaller than the helpers' least slack, a power of two that they are compared in units of.  Below 2^-126 numbers of
    either type have steps of one size, 2^-133 (bf16: 7 bits below 2^-126) and 2^-149 (f32: 23 bits): the rounding of such a result is off by half
    of that, 2^-134 and 2^-150, and not by half a step relative to itself, which is all that the helpers' bound holds."""
    n, hq, d = q.shape
    out, lse = gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, hk), store.heads(hk, 2 * hk), _ws(n, idx.numel(), hq, d))
    both = _values(store)
    want = _reference(indptr, idx, q, both[:, :hk], both[:, hk:], d ** -0.5, q.dtype)
    if tiny is not None:
        ref, slack = want["out"]
        want["out"] = ref / tiny, (slack + (2.0 ** -134 if q.dtype == B else 2.0 ** -150)) / tiny
    _check("out", out if tiny is None else out.double() / tiny, want["out"])
    _check("lse", lse, want["lse"])
    return out


SHAPES = [(F, 4, 32), (B, 1, 32), (B, 4, 16), (B, 4, 32), (B, 4, 33), (B, 4, 64), (B, 8, 128), (B, 4, 256)]


@pytest.mark.parametrize("t,hq,d", SHAPES)
@pytest.mark.parametrize("nats", [10, 25, 40, 60, 66, 70, 75, 80])
def test_sink_without_a_value(t, hq, d, nats):
    """Node 0 takes nearly all weight and its value row is zero: the results are what is left, of weights about e^-nats."""
    g = _gen(nats * 1000 + d + hq)
    x = torch.randn(200, 2, d, generator=g, device="cuda")
    x[:, 0] *= 0.3                                            # scores within a few nats of one another: none leaves the range of 32 bits
    x[:, 1] *= 2.0 ** 60
    x[:, 0, 0] = 0.0
    x[0, 0] = 0.0
    x[0, 0, 0] = 1.0                                          # column 0 of a query meets the sink's key alone
    x[0, 1] = 0.0
    store = gs.gs_coded_rows(200, 2, d, 16)
    gs.gs_coded_write(store, x)
    indptr, idx = _block([20, 1, 40, 700, 7], 199, g)
    idx += 1
    idx[3], idx[21 + 30], idx[61 + 500], idx[-1] = 0, 0, 0, 0    # in the first tile, in a later one, in a chunk, at a row's end
    q = torch.randn(5, hq, d, generator=g, device="cuda")
    q[:, :, 0] = nats * d ** 0.5
    out = _compare(indptr, idx, q.to(t), store, 1)
    assert (out[[0, 2, 3, 4]] != 0).all()


@pytest.mark.parametrize("t,hq,d", SHAPES)
@pytest.mark.parametrize("high,low", [(100, -60), (60, -100), (20, -20)])
def test_zero_rows_of_large_scales(t, hq, d, high, low):
    """The heaviest edges' value rows are zero, in blocks whose scale other rows have made large: what counts has a scale far below."""
    g = _gen(high - low + d)
    x = torch.randn(64, 2, d, generator=g, device="cuda").clamp(-4, 4)
    x[:, 0] *= 0.5
    x[:, 1] *= 2.0 ** low
    x[32:48, 1] = 0.0
    x[47, 1] = 2.0 ** high                                    # in the block of nodes 32 to 47; no edge names it
    x[32:47, 0] = 0.0
    x[32:47, 0, 0] = 1.0
    store = gs.gs_coded_rows(64, 2, d, 16)
    gs.gs_coded_write(store, x)
    indptr = torch.tensor([0, 20, 42, 82, 85, 85 + 300], dtype=torch.int32, device="cuda")
    idx = torch.randint(0, 32, (385,), generator=g, device="cuda", dtype=torch.int32)
    idx[0], idx[41], idx[60], idx[83], idx[85 + 17], idx[85 + 280] = 32, 33, 40, 46, 35, 32
    q = torch.randn(5, hq, d, generator=g, device="cuda")
    q[:, :, 0] = 20 * d ** 0.5
    out = _compare(indptr, idx, q.to(t), store, 1, tiny=2.0 ** (low - 60))
    assert (out != 0).flatten(1).any(1).all()


@pytest.mark.parametrize("t,hq,d", SHAPES)
def test_columns_that_the_heavy_edges_leave_at_zero(t, hq, d):
    """Edges whose weights fall by 6 nats each; the values of all but the last few are zero in every other column."""
    g = _gen(d + hq)
    x = torch.zeros(14, 2, d, device="cuda")
    x[:, 0, 0] = -torch.arange(14, device="cuda").float()
    x[:, 1, ::2] = torch.randn(14, (d + 1) // 2, generator=g, device="cuda")
    x[11:, 1] = torch.randn(3, d, generator=g, device="cuda")
    store = gs.gs_coded_rows(14, 2, d, 1)
    gs.gs_coded_write(store, x)
    indptr = torch.tensor([0, 12, 24, 38, 41], dtype=torch.int32, device="cuda")
    idx = torch.cat([torch.arange(12), torch.arange(11, -1, -1), torch.randperm(14), torch.tensor([13, 0, 12])]).int().cuda()
    q = torch.zeros(4, hq, d, device="cuda")
    q[:, :, 0] = 6 * d ** 0.5
    out = _compare(indptr, idx, q.to(t), store, 1)
    assert (out[[0, 1, 2, 3]] != 0).all()


@pytest.mark.parametrize("t,hq,d", SHAPES)
@pytest.mark.parametrize("apart", [20, 40, 60])
def test_queries_whose_columns_are_far_apart(t, hq, d, apart):
    """The largest columns of a query meet keys of zero: the scores come from columns 2^-apart of them."""
    g = _gen(apart + d)
    x = torch.randn(60, 2, d, generator=g, device="cuda")
    x[:, 0, :3] = 0.0
    x[:, 0] *= 2.0 ** (apart // 2)
    store = gs.gs_coded_rows(60, 2, d, 4)
    gs.gs_coded_write(store, x)
    indptr, idx = _block([20, 300, 16, 1], 60, g)
    q = torch.randn(4, hq, d, generator=g, device="cuda") * 2.0 ** -(apart // 2)
    q[:, :, :3] *= 2.0 ** apart
    q[2] = torch.randn(hq, d, generator=g, device="cuda") * 2.0 ** -(apart // 2)      # an ordinary row beside them
    _compare(indptr, idx, q.to(t), store, 1)


@pytest.mark.parametrize("t,hq,d", SHAPES)
@pytest.mark.parametrize("power", [-115, -100, 100, 110])
def test_keys_and_queries_of_opposite_sizes(t, hq, d, power):
    """Keys of 2^power and queries of 2^-power: scores of ordinary size."""
    g = _gen(power + d)
    x = torch.randn(60, 2, d, generator=g, device="cuda").clamp(-4, 4)
    x[:, 0] *= 2.0 ** power
    store = gs.gs_coded_rows(60, 2, d, 4)
    gs.gs_coded_write(store, x)
    indptr, idx = _block([20, 300, 16, 1], 60, g)
    q = torch.randn(4, hq, d, generator=g, device="cuda") * 2.0 ** -power
    _compare(indptr, idx, q.to(t), store, 1)


@pytest.mark.parametrize("t,hq,d", SHAPES)
@pytest.mark.parametrize("std", [8, 32, 200])
def test_scores_far_apart(t, hq, d, std):
    """Weights of every size in one row, many of them out of the range of 32 bits; values with columns of zeros."""
    g = _gen(std + d)
    x = torch.randn(300, 2, d, generator=g, device="cuda")
    x[torch.rand(300, generator=g, device="cuda") < 0.5, 1, ::3] = 0.0
    x[:, 1, d // 2] = 0.0
    store = gs.gs_coded_rows(300, 2, d, 16)
    gs.gs_coded_write(store, x)
    indptr, idx = _block([20] * 60 + [700, 1, 0, 64, 33], 300, g, masked=0.1)
    q = torch.randn(65, hq, d, generator=g, device="cuda") * std
    _compare(indptr, idx, q.to(t), store, 1)
