"""The residual block where a workgroup walks several blocks of rows: rows loaded a block ahead, scale bytes of later blocks, sums that meet in LDS
by turns, sums over rows from block to block, a ragged end -- for every shape of rows over lanes, from tensors, checkpoints and both."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
import test_gpu_block as tb
from gpu_util import dev, say
from oracle import block as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# (D, rows of a workgroup's block, workgroups): rows of whole quads in 8 .. 256 lanes, rows of any width in 4 .. 256 lanes of one to four columns
TILES = [(32, 32, 512), (64, 16, 512), (128, 8, 512), (256, 4, 512), (512, 2, 512), (1000, 1, 512),
         (3, 64, 768), (7, 32, 768), (13, 16, 768), (31, 8, 768), (50, 8, 768), (77, 8, 768), (99, 8, 768), (150, 4, 768), (250, 4, 768),
         (301, 2, 768), (501, 2, 768), (601, 1, 768), (1023, 1, 768)]
GATES = ("none", "row", "full")
CASES = []
for _i, (_D, _R, _wgs) in enumerate(TILES):
    _n = 3 * _R * _wgs + _R // 2 + 5               # three blocks for every workgroup, a fourth for some, the last one ragged
    CASES += [(_D, _n, ("rms", "layer")[_i % 2], GATES[_i % 3], "32"), (_D, _n, ("layer", "rms")[_i % 2], GATES[(_i + 1) % 3], "8"),
              (_D, _n, ("rms", "layer")[_i % 2], "full", "mixed")]


@pytest.mark.parametrize("D,n,norm,gate,bits", CASES)
def test_several_blocks_of_rows(D, n, norm, gate, bits):
    say(f"block trips n={n} D={D} {norm} gate={gate} bits={bits}")
    rng = np.random.default_rng(D + n)
    a = tb._inputs(rng, n, D, gate)
    o, ck = tb._forward(a, norm, 1e-5, 32 if bits == "32" else 8)
    tb._check_forward(a, norm, 1e-5, o, ck)
    if bits == "mixed":
        ck = {k: ck[k] for k in (("x8",), ("y8", "g8"), ("x8", "y8"))[D % 3]}
    dX_out, dN = (0.1 * rng.standard_normal((2, n, D))).astype(np.float32)
    g = tb._backward(a, norm, dX_out, dN, o, ck)
    val = lambda name, t: ob.act8_values(ck[name][0].cpu().numpy(), ck[name][1].cpu().numpy()) if name in ck else t    # noqa: E731
    want = ob.block_bwd(dX_out, dN, val("x8", o["X_out"].cpu().numpy()), tb._pair(o["stats_before"], norm), val("y8", a["Y"]),
                        tb._pair(o["stats_after"], norm), val("g8", a["G"]), norm == "layer", a["w_after"], a["b_after"], a["scale"], a["w_before"])
    assert set(g) == {k for k in want if k != "abs"}
    for name, t in g.items():
        # terms as exact as any entry; their sums add sixteen rows in fp32 and round twice beyond that
        tb._close(t, want[name], want["abs"][name], tb.BWD + (18 * U if name.startswith(("dw", "db", "ds")) else 0), name)


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("D,n", [(128, (1 << 18) + 13), (64, (1 << 19) + 7), (96, 350_003)])
def test_ten_tensors_at_once(D, n, norm):
    """A gate per element and three checkpoints of 2^25 elements and more: half as many workgroups, a hundred blocks of rows each."""
    assert n * D >= 1 << 25
    say(f"block ten tensors n={n} D={D} {norm}")
    rng = np.random.default_rng(D)
    gen = torch.Generator(device="cuda").manual_seed(D)
    full = {k: torch.randn(n, D, generator=gen, device="cuda") for k in "XYG"}
    params = {k: v for k, v in tb._inputs(rng, 1, D, "none").items() if k not in "XYG"}
    X_out, N = torch.full((n, D), float("nan"), device="cuda"), torch.full((n, D), float("nan"), device="cuda")
    st = dict(stats_after=tb._stats_room(n, norm), stats_before=tb._stats_room(n, norm))
    ck = {k: P.alloc_act8(n, D) for k in ("x8", "y8", "g8")}
    P.dr_block_fwd(full["X"], full["Y"], full["G"], X_out, N, norm=tb.NORMS[norm], eps=1e-5, **{k: dev(v) for k, v in params.items()}, **st, **ck)
    # whole eights of rows, from every block that a workgroup walks, and the last rows
    eights = np.unique(np.concatenate((rng.integers(0, n // 8, 1000), np.arange(0, n // 8, 2048 // 8 + 1), [n // 8 - 1])))
    rows = np.concatenate(((8 * eights[:, None] + np.arange(8)).ravel(), np.arange(n // 8 * 8, n)))
    at = torch.from_numpy(rows).cuda()
    a = dict({k: t[at].cpu().numpy() for k, t in full.items()}, **params)
    groups = -(-D // 32)
    blocks = torch.from_numpy(np.concatenate((eights, [n // 8]))).cuda()
    cks = {k: (q[at], s.view(-1, groups * 8)[blocks].reshape(-1)) for k, (q, s) in ck.items()}
    tb._check_forward(a, norm, 1e-5, dict(X_out=X_out[at], N=N[at], **{k: s[at] for k, s in st.items()}), cks)
    assert not torch.isnan(X_out).any() and not torch.isnan(N).any()
