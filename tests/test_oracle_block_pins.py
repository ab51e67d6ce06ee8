"""Pins of the row operators' oracle: its gradients against differences of its forward and against torch's autograd of the
formulas, its 8-bit codes against their definition.  No GPU needed."""
import numpy as np
import pytest
import torch

from oracle import block as ob


def _inputs(rng, n, D, gate):
    f = rng.standard_normal
    cols = {"none": 0, "row": 1, "full": D}[gate]
    return dict(X=f((n, D)), Y=2 * f((n, D)) + 0.3, G=f((n, cols)) if cols else None, w_after=1 + 0.2 * f(D), b_after=0.1 * f(D),
                scale=0.5 + 0.2 * f(D), w_before=1 + 0.2 * f(D), b_before=0.1 * f(D))


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", ["none", "row", "full"])
def test_gradients_against_autograd_and_differences(layer, gate):
    rng = np.random.default_rng(3)
    n, D, eps = 5, 7, 1e-3
    a = _inputs(rng, n, D, gate)
    dX_out, dN = rng.standard_normal((n, D)), rng.standard_normal((n, D))
    fwd = ob.block_fwd(layer=layer, eps=eps, **a)
    got = ob.block_bwd(dX_out, dN, fwd["X_out"], (fwd["m_before"], fwd["r_before"]), a["Y"], (fwd["m_after"], fwd["r_after"]), a["G"],
                       layer, a["w_after"], a["b_after"], a["scale"], a["w_before"])
    names = dict(X="dX", Y="dY", G="dG", w_after="dw_after", b_after="db_after", scale="dscale", w_before="dw_before", b_before="db_before")
    t = {k: None if v is None else torch.tensor(v, dtype=torch.float64, requires_grad=True) for k, v in a.items()}

    def norm(x):
        m = x.mean(1, keepdim=True) if layer else 0.0
        return (x - m) / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + eps)
    g = 1.0 if t["G"] is None else torch.sigmoid(t["G"])
    xo = t["X"] + t["scale"] * g * (norm(t["Y"]) * t["w_after"] + t["b_after"])
    N = norm(xo) * t["w_before"] + t["b_before"]
    assert np.allclose(xo.detach().numpy(), fwd["X_out"], rtol=1e-12) and np.allclose(N.detach().numpy(), fwd["N"], rtol=1e-11)
    (torch.tensor(dX_out) * xo).sum().add((torch.tensor(dN) * N).sum()).backward()
    for k, name in names.items():
        if a[k] is not None:
            assert np.allclose(got[name], t[k].grad.numpy(), rtol=1e-9, atol=1e-11), name
            assert np.all(got["abs"][name] >= np.abs(got[name]) * (1 - 1e-12)), name
    # central differences along a random direction of every input: h^2 times a third derivative of order one, and 1e-16 / h
    h = 1e-5
    for k, name in names.items():
        if a[k] is None:
            continue
        v = rng.standard_normal(a[k].shape)
        val = []
        for sign in (1, -1):
            o = ob.block_fwd(layer=layer, eps=eps, **{**a, k: a[k] + sign * h * v})
            val.append((dX_out * o["X_out"]).sum() + (dN * o["N"]).sum())
        assert abs((val[0] - val[1]) / (2 * h) - (got[name] * v).sum()) < 1e-6, name


def test_codes_by_definition():
    x = np.zeros((6, 70), np.float32)
    x[0, :3] = (127.0, 126.5, -125.5)                         # scale 2^0: ties go to even
    x[1, 0] = 127.5                                           # one step up
    x[1, 1] = 3.0
    x[2, 0] = np.nextafter(np.float32(127.5), np.float32(0))
    x[3, 40] = np.inf
    x[3, 0] = 1.0
    x[4, 69] = np.finfo(np.float32).max
    x[5, 0] = 2.0 ** -140
    q, s = ob.act8_pack(x)
    b = s.reshape(1, 3, 8)[0]
    assert list(q[0, :3]) == [127, 126, -126] and b[0, 0] == 127
    assert q[1, 0] == 64 and b[0, 1] == 128 and q[1, 1] == 2   # 63.75 -> 64; 1.5 -> 2
    assert q[2, 0] == 127 and b[0, 2] == 127
    assert b[1, 3] == 255 and not q[3, 32:64].any() and b[0, 3] == 121 and q[3, 0] == 64
    assert b[2, 4] == 248 and q[4, 69] == 127
    assert b[0, 5] == 1 and q[5, 0] == 0
    assert not b[:, 6:].any()
    v = ob.act8_values(q, s)
    assert np.isnan(v[3, 32:64]).all() and np.isfinite(np.delete(v, 3, 0)).all()
    fin = np.delete(v, 3, 0)[:4], np.delete(x, 3, 0)[:4].astype(np.float64)
    assert np.all(np.abs(fin[0] - fin[1])[:3] <= np.abs(fin[1][:3]).max(axis=1, keepdims=True) / 127.5)
