"""Gates far open and far shut: the gate's own gradient, in which sigmoid(G) and 1 - sigmoid(G) both are factors, is as exact relative to itself
at any G; the forward pass is off by no more than a denormal where the sigmoid itself is one."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev, say
from oracle import block as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# roundings on the way to an entry, as everywhere in the block's tests: two norms with two means each, the exponential (2 ulp), the sigmoid
# and its complement (a reciprocal and a product each), and some twenty products
FWD, BWD = 64 * U, 128 * U
# below the least normal number a factor is off by as much as that number: 2^-126 of the other factors, each rounded once or twice
TINY = 2.0 ** -125
GATES = np.array([0, 1e-3, 1, 3, 5, 8, 9, 10, 11, 12, 14, 16, 16.5, 17, 18, 20, 25, 30, 45, 60, 80, 86, 87.5, 88.5, 92, 100, 103, 104, 120, 200,
                  1e4, 3e38], np.float32)


def _saved(rng, n, D):
    f = lambda *s: rng.standard_normal(s).astype(np.float32)                      # noqa: E731
    G = np.concatenate((GATES, -GATES))
    return dict(Y=f(n, D), d=f(n, D), wa=1 + f(D) / 5, ba=f(D) / 5, sc=(0.5 + f(D) / 5).astype(np.float32), G=G)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gate", ["row", "full"])
@pytest.mark.parametrize("D", [1, 20, 64, 77, 300])
def test_gradient_of_open_and_shut_gates(D, gate, bits):
    say(f"gates D={D} {gate} bits={bits}")
    rng = np.random.default_rng(D)
    n = 2 * len(GATES)
    a = _saved(rng, n, D)
    if gate == "row" or D == 1:
        G = a["G"][:, None].copy()
    else:                                          # (in 8 bits, gates of one size share a scale)
        G = np.resize(a["G"], (n, D)).copy() if bits == 32 else np.repeat(a["G"][:, None], D, axis=1)
    norm, eps = P.DR_ROWNORM_RMS, 1e-5
    y, g = dev(a["Y"]), dev(G)
    r = dev((1 / np.sqrt((a["Y"].astype(np.float64) ** 2).mean(1) + eps)).astype(np.float32))
    ck, val = {}, dict(Y=a["Y"], G=G)
    if bits == 8:
        for name, t in (("y8", y),) + ((("g8", g),) if G.shape[1] == D else ()):
            ck[name] = P.alloc_act8(n, D)
            P.dr_act8_pack(t, ck[name])
            val[name[0].upper()] = ob.act8_values(ck[name][0].cpu().numpy(), ck[name][1].cpu().numpy())
    dG, dX, dY = torch.full(G.shape, float("nan"), device="cuda"), torch.empty(n, D, device="cuda"), torch.empty(n, D, device="cuda")
    sums = torch.empty(3, D, device="cuda")
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    P.dr_block_bwd(dev(a["d"]), None, None, None if bits == 8 else y, None if "g8" in ck else g, norm=norm, eps=eps, w_after=dev(a["wa"]),
                   b_after=dev(a["ba"]), scale=dev(a["sc"]), stats_after=r, **ck, dX=dX, dY=dY, dG=dG, dw_after=sums[0], db_after=sums[1],
                   dscale=sums[2], workspace=ws)
    # the formula, in 64 bits: sigmoid(-G) is 1 - sigmoid(G)
    d, sc, wa, ba = (a[k].astype(np.float64) for k in ("d", "sc", "wa", "ba"))
    G64 = np.asarray(val["G"], dtype=np.float64)
    with np.errstate(over="ignore"):
        both = 1 / (1 + np.exp(-G64)) * (1 / (1 + np.exp(G64)))
    yh = np.asarray(val["Y"], dtype=np.float64) * r.cpu().numpy().astype(np.float64)[:, None]
    term, mag = d * sc * (yh * wa + ba), np.abs(d * sc) * (np.abs(yh * wa) + np.abs(ba))
    if G.shape[1] == 1:
        term, mag = term.sum(1, keepdims=True), mag.sum(1, keepdims=True)
    err = np.abs(dG.cpu().numpy().astype(np.float64) - term * both)
    bad = ~(err <= BWD * mag * both + TINY * (1 + mag))
    assert not bad.any(), (G[bad][:8], float((err / (mag * both + TINY * (1 + mag))).max() / U))
    assert torch.isfinite(dX).all() and torch.isfinite(dY).all() and torch.isfinite(sums).all()


def test_forward_of_open_and_shut_gates():
    rng = np.random.default_rng(1)
    for D in (64, 77):
        n = 2 * len(GATES)
        a = _saved(rng, n, D)
        G = np.resize(a["G"], (n, D)).copy()
        X_out = torch.full((n, D), float("nan"), device="cuda")
        P.dr_block_fwd(torch.zeros(n, D, device="cuda"), dev(a["Y"]), dev(G), X_out, None, w_after=dev(a["wa"]), b_after=dev(a["ba"]),
                       scale=dev(a["sc"]))
        with np.errstate(over="ignore"):
            want = ob.block_fwd(np.zeros((n, D)), a["Y"], G, w_after=a["wa"], b_after=a["ba"], scale=a["sc"])
        err = np.abs(X_out.cpu().numpy().astype(np.float64) - want["X_out"])
        assert np.all(err <= FWD * want["abs"]["X_out"] + TINY * 64)               # |scale * u| is far below 64 here


def test_infinite_gates_and_not_a_numbers():
    D, n = 64, 3
    y = torch.ones(n, D, device="cuda")
    g = torch.zeros(n, D, device="cuda")
    g[0], g[1], g[2] = float("inf"), float("-inf"), float("nan")
    dG, r = torch.empty(n, D, device="cuda"), torch.ones(n, device="cuda")
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    P.dr_block_bwd(y, None, None, y, g, stats_after=r, dG=dG, workspace=ws)
    assert not dG[:2].any() and torch.isnan(dG[2]).all()
