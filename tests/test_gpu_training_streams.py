"""Calls on a stream that is not the current one, with outputs that the call allocates: their memory must not be something
that queued work of the current stream is still going to write to."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _cases():
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    ids = torch.randint(0, 500, (3000,), generator=g, device="cuda", dtype=torch.int32)
    table, dout = rand(500, 32), rand(3000, 32)
    ews = torch.empty(gs.gs_embedding_workspace_bytes(3000, 500, 32), dtype=torch.uint8, device="cuda")
    indptr = torch.arange(0, 3001, 6, dtype=torch.int32, device="cuda")
    q, k, v, do = rand(500, 4, 16), rand(500, 4, 16), rand(500, 4, 16), rand(500, 4, 16)
    aws = torch.empty(gs.gs_block_attention_workspace_bytes(500, 500, 3000, 4, 4, 16), dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, ids, q, k, v, aws)
    rev = gs.gs_block_reverse(indptr, ids, 500, aws)
    y, dl = ids[:200].contiguous(), rand(200)
    h = rand(200, 32)
    xws = torch.empty(gs.gs_xent_workspace_bytes(200, 500, 32, torch.float32), dtype=torch.uint8, device="cuda")
    xlse = gs.gs_xent_forward(h, table, y, xws)[1]
    return {
        "lookup": lambda s: [gs.gs_embedding_lookup(table, ids, stream=s)],
        "gradient": lambda s: [gs.gs_embedding_backward(dout, ids, 500, ews, stream=s)],
        "touched": lambda s: gs.gs_embedding_backward_sparse(dout, ids, 500, ews, stream=s),
        "forward": lambda s: gs.gs_block_attention_forward(indptr, ids, q, k, v, aws, stream=s),
        "reverse": lambda s: gs.gs_block_reverse(indptr, ids, 500, aws, stream=s),
        "backward": lambda s: gs.gs_block_attention_backward(indptr, ids, rev, q, k, v, out, lse, do, aws, stream=s),
        "loss": lambda s: gs.gs_xent_forward(h, table, y, xws, stream=s),
        "loss gradients": lambda s: gs.gs_xent_backward(h, table, y, xlse, dl, xws, stream=s),
    }


@pytest.mark.parametrize("name", ["lookup", "gradient", "touched", "forward", "reverse", "backward", "loss", "loss gradients"])
def test_outputs_belong_to_the_call_s_stream(name):
    call = _cases()[name]
    side = torch.cuda.Stream()
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    call(side)                                                # the side stream's first use
    torch.cuda.synchronize()
    # memory of the current stream, of the outputs' sizes, that queued work is going to write to after its owner is gone
    torch.cuda._sleep(100_000_000)                            # some 50 ms
    old = [torch.empty_like(t) for t in want for _ in range(8)]
    for t in old:
        t.fill_(77)
    del old, t
    got = call(side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b), name
