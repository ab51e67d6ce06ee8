"""Weight gradients from checkpoints over so many rows that every workgroup adds its running sums up several times on the way, for every shape of
tile; and gradients at the small end of the fp32 range.

The long ones are exact: rows hold 1, 2 and 3, gradients are multiples of 2^-9 below 8 in magnitude (12 bits, which takes two of the three bf16 parts).  A
wavefront's sum of 1 280 rows is at most 1280 * 3 * 4095 < 2^24 of these units whatever the order, so nothing is rounded before the sums in 64 bits,
and those are rounded once."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev, say

pytestmark = pytest.mark.gpu

CHUNKS, WGS = 40, 256                              # chunks of 32 rows a workgroup (16 between two flushes), workgroups of a launch


def _cases():
    def tile(D, F):                                # (width of a tile of dW, rows of a chunk)
        td = 32 if D <= 32 else 64 if D <= 64 else 96 if D <= 96 and F > 64 else 128
        tf = 32 if F <= 32 else 64 if F <= 64 else 96 if td == 128 and F <= 96 else 128
        return td, tf, {(32, 32): 128, (32, 64): 64, (64, 32): 64, (64, 64): 64}.get((td, tf), 32)
    out = []
    for D, F in ((32, 32), (32, 64), (32, 128), (64, 32), (64, 64), (64, 128), (96, 96), (128, 32), (128, 64), (128, 96), (128, 128), (96, 200),
                 (300, 257), (77, 33)):
        td, tf, rows = tile(D, F)
        tiles = -(-D // td) * -(-F // tf)
        out.append((D, F, CHUNKS * rows * (WGS // tiles) - 13))
    return out


@pytest.mark.parametrize("sign", ["both", "plus"])
@pytest.mark.parametrize("D,F,n", _cases())
def test_sums_of_many_chunks(D, F, n, sign):
    say(f"wgrad many chunks n={n} D={D} F={F} {sign}")
    g = torch.Generator(device="cuda").manual_seed(D + F)
    x = torch.randint(1, 4, (n, D), generator=g, device="cuda").float()
    dZ = torch.randint(-4095 if sign == "both" else 0, 4096, (n, F), generator=g, device="cuda").float() * 2.0 ** -9
    ck = P.alloc_act8(n, D)
    P.dr_act8_pack(x, ck)
    v = torch.empty(n, D, device="cuda")
    P.dr_act8_unpack(ck, v)
    assert torch.equal(v, x)
    dW = torch.full((D, F), float("nan"), device="cuda")
    ws = torch.full((P.dr_act8_wgrad_workspace_bytes(n, D, F),), 255, dtype=torch.uint8, device="cuda")
    P.dr_act8_wgrad(ck, dZ, dW, ws)
    want = torch.zeros(D, F, dtype=torch.float64, device="cuda")
    for r in range(0, n, 1 << 17):
        want += torch.mm(x[r:r + (1 << 17)].double().t().contiguous(), dZ[r:r + (1 << 17)].double())
    assert torch.equal(dW, want.float()), float((dW.double() - want).abs().max())
    base = dW * 0.5
    twice = base.clone()
    P.dr_act8_wgrad(ck, dZ, twice, ws, True)
    assert torch.equal(twice, (want + base.double()).float())


@pytest.mark.parametrize("D,F", [(128, 128), (96, 40)])
def test_gradients_of_the_smallest_numbers(D, F):
    """Denormal gradients, and normal ones whose second and third parts are denormals.  Each part takes what bf16 holds of what the ones before it left;
    the steps of bf16 end at 2^-133, where those of fp32 go on to 2^-149: less than 2^-133 of a gradient is left out, whatever its size."""
    rng = np.random.default_rng(3)
    n = 100
    x = (rng.integers(1, 100, (n, D)) * 2.0 ** 60).astype(np.float32)
    ck = P.alloc_act8(n, D)
    P.dr_act8_pack(dev(x), ck)
    v = torch.empty(n, D, device="cuda")
    P.dr_act8_unpack(ck, v)
    for e in (-118, -124, -127, -132):
        dZ = (rng.uniform(1, 2, (n, F)) * rng.choice((-1, 1), (n, F)) * 2.0 ** e).astype(np.float32)
        dW = torch.full((D, F), float("nan"), device="cuda")
        ws = torch.empty(P.dr_act8_wgrad_workspace_bytes(n, D, F), dtype=torch.uint8, device="cuda")
        P.dr_act8_wgrad(ck, dev(dZ), dW, ws)
        A, B = v.cpu().numpy().astype(np.float64), dZ.astype(np.float64)
        err = np.abs(dW.cpu().numpy().astype(np.float64) - A.T @ B)
        bound = n * 2.0 ** -23 * (np.abs(A).T @ np.abs(B)) + 2.0 ** -133 * np.abs(A).sum(0)[:, None]
        assert np.all(err <= bound), (e, float((err / bound).max()))
