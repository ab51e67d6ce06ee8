"""Sums over the rows of the block's backward pass lose no more for being long: a lane adds up sixteen rows in fp32, everything beyond that is
added in 64 bits.

The numbers are the worst for a running sum in fp32: 1 + 2^-17 - 2^-22 added to 128 or more is rounded to 1, so that a lane that walks 300 rows by itself
is off by 75 * 2^-24 of its sum.  Every term is exact here, so what is allowed is 16 additions, the rounding of a workgroup's sum and that of
the result: 18 * 2^-24."""
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
C = 1 + 2.0 ** -17 - 2.0 ** -22
# rows that all workgroups together walk at a time: 512 workgroups of 256 lanes of four columns, 768 of any width
CASES = [(128, 300 * 4096 + 5), (1024, 300 * 512 + 1), (77, 300 * 6144 + 3), (1023, 300 * 768 + 2), (3, 300 * 49152 + 31)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("D,n", CASES)
def test_sums_over_rows(D, n, bits):
    say(f"long sums n={n} D={D} bits={bits}")
    c = torch.full((n, D), C, device="cuda")
    one = torch.ones(n, D, device="cuda")
    r = torch.ones(n, device="cuda")
    ck = P.alloc_act8(n, D)
    P.dr_act8_pack(one, ck)
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    s = torch.full((5, D), float("nan"), device="cuda")
    x, x8 = (None, ck) if bits == 8 else (one, None)
    P.dr_block_bwd(c, None, None, x, None, y8=x8, stats_after=r, dw_after=s[0], db_after=s[1], dscale=s[2], workspace=ws)
    P.dr_block_bwd(None, c, x, None, None, x8=x8, stats_before=r, dw_before=s[3], db_before=s[4], workspace=ws)
    off = (s.double() - n * C).abs() / (n * C)
    assert (off <= 18 * U).all(), float(off.max()) / U
