"""Weight gradients of a layer from checkpoints that hold what a forward pass may leave in them: groups that are not finite, and both ends of the scales."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev, random_csr, say

pytestmark = pytest.mark.gpu


def _pass(layer, dY, W, saved):
    D = layer.D
    dX = torch.empty(layer.Nc, D, device="cuda"), torch.empty(layer.Nn, D, device="cuda")
    dW = {n: torch.full((D, D), float("nan"), device="cuda") for n in P.WEIGHT_NAMES}
    layer.heteroconv_bwd_act8(*dY, W, saved, *dX, dW)
    return dX, dW


@pytest.mark.parametrize("mode", [P.DR_OVERLAP_ON, P.DR_OVERLAP_OFF])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_groups_of_all_kinds(D, mode):
    say(f"act8 layer extremes D={D}")
    rng = np.random.default_rng(D)
    Nc, Nn = 901, 640
    rel = [P.Csr(m, n, *(dev(a) for a in random_csr(rng, m, n, 4, dup=True))) for m, n in ((Nc, Nc), (Nn, Nc), (Nc, Nn))]
    layer = P.HeteroConv(*rel, D, 16, 16)
    layer.heteroconv_set_overlap(mode)
    f = lambda *s: dev(rng.standard_normal(s).astype(np.float32))                  # noqa: E731
    W = {n: f(D, D) for n in P.WEIGHT_NAMES}
    X, dY, saved = (f(Nc, D), f(Nn, D)), (f(Nc, D), f(Nn, D)), layer.alloc_saved8()
    layer.heteroconv_fwd_act8(*X, W, torch.empty(Nc, D, device="cuda"), torch.empty(Nn, D, device="cuda"), saved)
    dX0, want = _pass(layer, dY, W, saved)
    messages = {"H_near": "neigh_near", "H_pinned": "pinned", "H_pins": "neigh_pins"}
    last = D // 32 - 1
    for h, name in messages.items():
        # one group of one row not finite: its 32 rows of one weight gradient, and nothing else
        q, s = saved[h]
        keep = q.clone(), s.clone()
        row = len(q) - 2
        s.view(-1, D // 32, 8)[row // 8, last, row % 8] = 255
        q[row, 32 * last:] = 0
        dX, dW = _pass(layer, dY, W, saved)
        assert all(torch.equal(a, b) for a, b in zip(dX, dX0))
        assert torch.isnan(dW[name][32 * last:]).all()
        assert torch.equal(dW[name][:32 * last], want[name][:32 * last])
        assert all(torch.equal(dW[n], want[n]) for n in P.WEIGHT_NAMES if n != name)
        q.copy_(keep[0])
        s.copy_(keep[1])
    # the largest and the smallest scales there are: sums of one row each, exact but for their roundings
    mask = saved["mask"].float()
    for byte, by in ((248, 2.0 ** -100), (1, 2.0 ** 100)):
        g = tuple(t * by for t in dY)
        for h, name in messages.items():
            q, s = saved[h]
            s.fill_(byte)
            q.zero_()
            q[5] = torch.arange(D, device="cuda").sub(D // 2).clamp(-127, 127).to(torch.int8)
        _, dW = _pass(layer, g, W, saved)
        v = saved["H_near"][0][5].double() * 2.0 ** (byte - 127)
        for name, row in (("neigh_near", g[0][5] * mask[5]), ("pinned", g[0][5] * (1 - mask[5])), ("neigh_pins", g[1][5])):
            exact = v[:, None] * row.double()[None]
            # a product is exact to 2^-24 and rounded once more; the other rows add zeros
            assert ((dW[name].double() - exact).abs() <= 2.0 ** -22 * exact.abs()).all(), (byte, name)
    layer.heteroconv_destroy()
