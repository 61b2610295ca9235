"""Operands that the training operators' binding turns down before anything is launched: workspaces, device scalars and
statistics that are on the host, of another type, or not there."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def calls():
    """Every call as a function of the operand in question."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    ids = torch.randint(0, 9, (12,), generator=g, device="cuda", dtype=torch.int32)
    table, dout = rand(9, 8), rand(12, 8)
    ews = torch.empty(gs.gs_embedding_workspace_bytes(12, 9, 8), dtype=torch.uint8, device="cuda")
    indptr = torch.tensor([0, 4, 7, 12], dtype=torch.int32, device="cuda")
    q, k = rand(3, 2, 8), rand(9, 2, 8)
    aws = torch.empty(gs.gs_block_attention_workspace_bytes(3, 9, 12, 2, 2, 8), dtype=torch.uint8, device="cuda")
    out, lse = gs.gs_block_attention_forward(indptr, ids, q, k, k, aws)
    rev = gs.gs_block_reverse(indptr, ids, 9, aws)
    h, y, dl = rand(12, 8), ids, rand(12)
    xws = torch.empty(gs.gs_xent_workspace_bytes(12, 9, 8, torch.float32), dtype=torch.uint8, device="cuda")
    xlse = gs.gs_xent_forward(h, table, y, xws)[1]
    workspace = {
        "gradient": (ews, lambda w: gs.gs_embedding_backward(dout, ids, 9, w)),
        "touched": (ews, lambda w: gs.gs_embedding_backward_sparse(dout, ids, 9, w)),
        "forward": (aws, lambda w: gs.gs_block_attention_forward(indptr, ids, q, k, k, w)),
        "reverse": (aws, lambda w: gs.gs_block_reverse(indptr, ids, 9, w)),
        "backward": (aws, lambda w: gs.gs_block_attention_backward(indptr, ids, rev, q, k, k, out, lse, q, w)),
        "loss": (xws, lambda w: gs.gs_xent_forward(h, table, y, w)),
        "loss gradients": (xws, lambda w: gs.gs_xent_backward(h, table, y, xlse, dl, w)),
    }
    three = lambda c: (c, torch.tensor(9, dtype=torch.int32, device="cuda"), torch.tensor(12, dtype=torch.int32, device="cuda"))  # noqa: E731
    scalar = {
        "lookup": (12, lambda c: gs.gs_embedding_lookup(table, ids, count=c)),
        "gradient": (12, lambda c: gs.gs_embedding_backward(dout, ids, 9, ews, count=c)),
        "touched": (12, lambda c: gs.gs_embedding_backward_sparse(dout, ids, 9, ews, count=c)),
        "rows": (0, lambda c: gs.gs_embedding_backward_sparse(dout, ids, 9, ews, num_rows=c)),
        "forward": (3, lambda c: gs.gs_block_attention_forward(indptr, ids, q, k, k, aws, counts=three(c))),
        "reverse": (3, lambda c: gs.gs_block_reverse(indptr, ids, 9, aws, counts=three(c))),
        "backward": (3, lambda c: gs.gs_block_attention_backward(indptr, ids, rev, q, k, k, out, lse, q, aws, counts=three(c))),
    }
    return workspace, scalar, lambda l: gs.gs_block_attention_forward(indptr, ids, q, k, k, aws, lse=l)


@pytest.mark.parametrize("name", ["gradient", "touched", "forward", "reverse", "backward", "loss", "loss gradients"])
def test_workspace(calls, name):
    good, call = calls[0][name]
    launched = gs.gs_kernel_launches()
    for bad in (good.cpu(), torch.empty(good.numel(), dtype=torch.float32, device="cuda"), torch.empty(2 * good.numel(), dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(TypeError, match="workspace"):
            call(bad)
    assert gs.gs_kernel_launches() == launched
    call(good)


@pytest.mark.parametrize("name", ["lookup", "gradient", "touched", "rows", "forward", "reverse", "backward"])
def test_device_scalars(calls, name):
    value, call = calls[1][name]
    launched = gs.gs_kernel_launches()
    for bad in (torch.tensor(value, dtype=torch.int32), torch.tensor(value, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")):
        with pytest.raises(TypeError, match="int32 CUDA"):
            call(bad)
    assert gs.gs_kernel_launches() == launched
    for good in (torch.tensor(value, dtype=torch.int32, device="cuda"), torch.tensor([value], dtype=torch.int32, device="cuda")):
        call(good)
    torch.cuda.synchronize()


def test_statistics_on_the_host(calls):
    with pytest.raises(TypeError, match="lse"):
        calls[2](torch.empty(3, 2))
    calls[2](torch.empty(3, 2, device="cuda"))
