"""The binding of the row operators reports what the library refuses, also where an argument that it takes the sizes from is missing.  No GPU needed:
everything is refused on the host."""
import pytest
import torch

import paper_2508_16769_amd as P


@pytest.mark.parametrize("given", ["X_out", "Y", "x8", "y8", "nothing"])
def test_backward_without_incoming_gradients(given):
    n, D = 4, 40
    x, st = torch.zeros(n, D), torch.ones(n)
    ck = P.alloc_act8(n, D, device="cpu")
    ws = torch.zeros(P.dr_block_bwd_workspace_bytes(n, D) + 256, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:]
    kw = {given: ck} if given.endswith("8") else {}
    with pytest.raises(P.DrError) as e:
        P.dr_block_bwd(None, None, x if given == "X_out" else None, x if given == "Y" else None, None, stats_after=st, stats_before=st,
                       dX=torch.zeros(n, D), workspace=ws, stream=0, **kw)
    assert e.value.code == P.DR_ERR_INVALID_ARG
    assert given == "nothing" or "neither dX_out nor dN" in str(e.value)
