"""Rows of one value under a layer norm: their deviation is zero, the norm is zero and its reciprocal deviation is as large as eps lets it be,
whatever the value -- also where the value times that is past the fp32 range, in widths that leave some of a row's lanes without a column."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev
from oracle import block as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 2.0 ** -100                                  # r = 2^50
VALUE = 2.0 ** 90                                  # times r: 2^140
BWD = 128 * U
LAYER = P.DR_ROWNORM_LAYER


def _exact_mean(D):
    """The mean of D equal numbers comes out as that number: their sum is exact, and the product with the rounded 1 / D is it again."""
    return np.float32(D) * (np.float32(1) / np.float32(D)) == np.float32(1)


WIDTHS = [D for D in (1, 2, 3, 5, 9, 20, 33, 36, 65, 77, 90, 96, 99, 100, 132, 200, 260, 300, 500, 516, 600, 1000, 1023) if _exact_mean(D)]


def test_widths_hold_both_kinds():
    assert sum(D % 4 == 0 for D in WIDTHS) >= 4 and sum(D % 4 != 0 for D in WIDTHS) >= 6


@pytest.mark.parametrize("D", WIDTHS)
def test_forward(D):
    rng = np.random.default_rng(D)
    n = 19
    Y = rng.standard_normal((n, D)).astype(np.float32)
    X = rng.standard_normal((n, D)).astype(np.float32)
    Y[3], Y[8], X[12] = VALUE, -VALUE, VALUE
    Y[12] = 0
    b, sc = rng.standard_normal((2, D)).astype(np.float32)
    t = dict(norm=LAYER, eps=EPS)
    X_out, N = torch.full((n, D), float("nan"), device="cuda"), torch.full((n, D), float("nan"), device="cuda")
    x8, y8 = P.alloc_act8(n, D), P.alloc_act8(n, D)
    stats = torch.empty(2, n, 2, device="cuda")
    zero = torch.zeros(D, device="cuda")
    # (row 12 stays the constant that X is: what is added to it is far below its last bit)
    P.dr_block_fwd(dev(X), dev(Y), None, X_out, N, b_after=dev(b), scale=dev(sc), w_before=None, b_before=zero, stats_after=stats[0],
                   stats_before=stats[1], x8=x8, y8=y8, **t)
    got = X_out.cpu().numpy()
    assert np.isfinite(got).all()
    for i in (3, 8):
        want = X[i].astype(np.float64) + sc.astype(np.float64) * b
        assert np.all(np.abs(got[i] - want) <= 2 * U * (np.abs(X[i]) + np.abs(sc * b)))
    assert (got[12] == X[12]).all()
    # the norm of what comes out is the norm of a row by itself, and the checkpoints are those of the rows
    alone = torch.full((n, D), float("nan"), device="cuda")
    P.dr_block_fwd(X_out, None, None, None, alone, b_before=zero, **t)
    assert torch.isfinite(N).all() and torch.equal(N, alone)
    assert not N[12].any() and (stats[0, [3, 8], 1] == 2.0 ** 50).all() and (stats[1, 12, 1] == 2.0 ** 50).all()
    for ck, m in ((x8, got), (y8, Y)):
        q, s = ob.act8_pack(m)
        assert np.array_equal(ck[0].cpu().numpy(), q) and np.array_equal(ck[1].cpu().numpy(), s)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gate", [0, 1])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(D, gate, bits):
    """The gradient of such a row has only the mean's projection: g - mean(g), times r."""
    rng = np.random.default_rng(D)
    n = 11
    dN, dX_out = rng.standard_normal((2, n, D)).astype(np.float32)
    X, Y = np.full((n, D), VALUE, np.float32), np.full((n, D), -VALUE, np.float32)
    r = 2.0 ** 50
    st = [dev(np.repeat(np.array([[v, r]], np.float32), n, 0)) for v in (VALUE, -VALUE)]
    w, sc = (1 + rng.standard_normal((2, D)) / 5).astype(np.float32)
    G = rng.standard_normal((n, 1)).astype(np.float32) if gate else None
    b = rng.standard_normal(D).astype(np.float32)
    kw = dict(norm=LAYER, eps=EPS, b_after=dev(b), scale=dev(sc), w_before=dev(w), stats_before=st[0], stats_after=st[1])
    if bits == 8:
        for name, m in (("x8", X), ("y8", Y)):
            kw[name] = P.alloc_act8(n, D)
            P.dr_act8_pack(dev(m), kw[name])
    out = {k: torch.full((n, D), float("nan"), device="cuda") for k in ("dX", "dY")}
    if gate:
        out["dG"] = torch.full((n, 1), float("nan"), device="cuda")
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    P.dr_block_bwd(dev(dX_out), dev(dN), None if bits == 8 else dev(X), None if bits == 8 else dev(Y), None if G is None else dev(G), **kw, **out,
                   workspace=ws)
    mean = lambda x: x.mean(1, keepdims=True)                                     # noqa: E731
    g = dN.astype(np.float64) * w
    d, ad = dX_out + r * (g - mean(g)), np.abs(dX_out) + r * (np.abs(g) + mean(np.abs(g)))
    s = 1 / (1 + np.exp(-G.astype(np.float64))) if gate else np.ones((n, 1))
    du, adu = d * sc * s, ad * np.abs(sc) * s
    want = dict(dX=(d, ad), dY=(r * (du - mean(du)), r * (adu + mean(adu))))
    if gate:
        want["dG"] = ((du * b * (1 - s)).sum(1, keepdims=True), (adu * np.abs(b) * (1 - s)).sum(1, keepdims=True))
    for k, (v, mag) in want.items():
        err = np.abs(out[k].cpu().numpy().astype(np.float64) - v)
        assert np.all(err <= BWD * mag), (k, float(np.nanmax(err / mag)) / U, bool(torch.isnan(out[k]).any()))
