"""A table of 2^29 rows: one block multiplies a tile of hidden rows with four million tiles of the table, for longer than any
single wait of the kernel may take (2.4 s; the limit is 4e9 clocks)."""
import pytest
import torch

import paper_2406_17918_b200 as gs

pytestmark = pytest.mark.gpu


def test_a_row_of_tiles_may_take_longer_than_a_wait():
    n, v, d = 148 * 128, 1 << 29, 8                    # a row of tiles per SM: each finished by one block
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    w = torch.zeros(v, d, dtype=torch.bfloat16, device="cuda")
    y = (torch.arange(n, device="cuda") * (v // n)).int()
    lse = torch.full((n,), float(torch.tensor(float(v)).log()), device="cuda")          # all logits are zero
    ws = torch.empty(gs.gs_xent_workspace_bytes(n, v, d), dtype=torch.uint8, device="cuda")
    dh = torch.full((n, d), 5.0, dtype=torch.bfloat16, device="cuda")
    dh, dw = gs.gs_xent_backward(h, w, y, lse, torch.ones(n, device="cuda"), ws, dhidden=dh)
    gs.gs_train_status()
    assert (dh == 0).all()
    # a label's row: the negative hidden row, beside 18,943 times 2^-29 of others
    assert (dw[y.long()].float() + h.float()).abs().max() <= 2.0 ** -7 * h.float().abs().max()
    other = dw[y.long() + 1].float().abs().max()
    assert other <= 1e-4
