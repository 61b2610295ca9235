"""Attention over 8-bit rows: what blocks and stores that other code has made may hold without results or memory beyond theirs being touched."""
import pytest
import torch

import paper_2406_17918_b200 as gs
from test_gpu_coded_attention import B, F, _gen, _store, _ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,hq", [(F, 1), (B, 4)])
def test_rows_that_ask_for_more_chunks_than_32_bits_count(t, hq):
    """131,372 rows that each name all of 2^24 edges ask for more than 2^32 chunks of at most 512.  The lists have 2^18 + 1 places, so nine
    rows are on them and no place is handed out twice; the others stay as they were."""
    g = _gen(1)
    edges, n = 1 << 24, 131072 + 300
    store = _store(50, 2, 8, 1, g)
    idx = torch.randint(0, 50, (edges,), generator=g, device="cuda", dtype=torch.int32)
    indptr = torch.tensor([0, edges], dtype=torch.int32, device="cuda").repeat(n + 1)[:2 * n + 1]        # every other row is empty
    q = torch.randn(1, hq, 8, generator=g, device="cuda").to(t).expand(2 * n, hq, 8).contiguous()
    out = torch.full((2 * n, hq, 8), 5.0, dtype=t, device="cuda")
    need = gs.gs_coded_attention_workspace_bytes(2 * n, edges, hq, 8)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    gs.gs_coded_attention_forward(indptr, idx, q, store.heads(0, 1), store.heads(1, 2), ws[:need], out=out)
    assert (ws[need:] == 77).all() and (out[1::2] == 0).all()
    listed = out[::2][(out[::2] != 5).flatten(1).any(1)]
    one, _ = gs.gs_coded_attention_forward(indptr[:2], idx, q[:1], store.heads(0, 1), store.heads(1, 2), _ws(1, edges, hq, 8))
    assert len(listed) == 9 and int((listed == one).flatten(1).all(1).sum()) == 8       # the ninth has one place for its many chunks


@pytest.mark.parametrize("t,hq", [(F, 1), (F, 2), (F, 4), (B, 1), (B, 2), (B, 4)])
@pytest.mark.parametrize("d", [1, 7, 8, 24, 33, 100, 130, 250])
def test_bytes_behind_the_columns_have_no_part(t, hq, d):
    """A store that other code has filled may hold anything between head_dim and the pitch, NaN codes among it."""
    g = _gen(d)
    store = _store(50, 4, d, 4, g)
    lengths = [0, 300, 5, 20, 17]
    indptr = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    idx = torch.randint(0, 50, (sum(lengths),), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randn(5, 2 * hq, d, generator=g, device="cuda").to(t)
    args = (indptr, idx, q, store.heads(0, 2), store.heads(2, 4), _ws(5, idx.numel(), 2 * hq, d))
    out, lse = gs.gs_coded_attention_forward(*args)
    store.codes.view(torch.uint8)[:, :, d:] = 0x7F
    again, alse = gs.gs_coded_attention_forward(*args)
    assert torch.isfinite(out).all() and torch.equal(out, again) and torch.equal(lse, alse)
