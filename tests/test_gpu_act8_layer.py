"""The layer with its messages kept in 8 bits, and residual blocks and checkpoints around layers as a model uses them."""
import numpy as np
import pytest
import torch

import oracle
import paper_2508_16769_amd as P
from gpu_util import dev, random_csr, say
from oracle import block as ob

pytestmark = pytest.mark.gpu

WIDTHS = [(32, 4, 20, 32), (64, 16, 16, 16), (64, 40, 8, 64), (96, 33, 12, 33), (128, 32, 32, 32), (128, 70, 128, 16)]


def _layer(rng, Nc, Nn, D, ks, deg=4):
    rel = [P.Csr(m, n, *(dev(a) for a in random_csr(rng, m, n, deg, dup=True))) for m, n in ((Nc, Nc), (Nn, Nc), (Nc, Nn))]
    return P.HeteroConv(*rel, D, per_relation=ks)


def _tensors(rng, Nc, Nn, D):
    f = lambda *s: dev(rng.standard_normal(s).astype(np.float32))                  # noqa: E731
    return dict(X=(f(Nc, D), f(Nn, D)), dY=(f(Nc, D), f(Nn, D)), W={n: f(D, D) for n in P.WEIGHT_NAMES})


def _nan(*s):
    return torch.full(s, float("nan"), device="cuda")


def _run(layer, t, eight, saved=None, stream=None):
    Nc, Nn, D = layer.Nc, layer.Nn, layer.D
    Y, dX, dW = (_nan(Nc, D), _nan(Nn, D)), (_nan(Nc, D), _nan(Nn, D)), {n: _nan(D, D) for n in P.WEIGHT_NAMES}
    if saved is None:
        saved = layer.alloc_saved8() if eight else layer.alloc_saved()
    (layer.heteroconv_fwd_act8 if eight else layer.heteroconv_fwd)(*t["X"], t["W"], *Y, saved, stream=stream)
    (layer.heteroconv_bwd_act8 if eight else layer.heteroconv_bwd)(*t["dY"], t["W"], saved, *dX, dW, stream=stream)
    return dict(Y=Y, dX=dX, dW=dW, saved=saved)


def _check(a, b, t, layer):
    """b from checkpoints against a: everything but the messages and the weight gradients bit for bit, those by definition."""
    assert all(torch.equal(x, y) for x, y in zip(a["Y"] + a["dX"], b["Y"] + b["dX"]))
    for n, s in a["saved"].items():
        if not n.startswith("H_"):
            assert torch.equal(s, b["saved"][n]), n
    val = {}
    for n in ("H_near", "H_pins", "H_pinned"):
        q, s = ob.act8_pack(a["saved"][n].cpu().numpy())
        assert np.array_equal(b["saved"][n][0].cpu().numpy(), q) and np.array_equal(b["saved"][n][1].cpu().numpy(), s), n
        val[n] = ob.act8_values(q, s)

    def kept(vals, idx, n):
        s = a["saved"]
        vals, idx = (vals, idx) if vals in s else (vals.rsplit("_", 1)[0], idx.rsplit("_", 1)[0])
        m = np.zeros((n, layer.D))
        np.put_along_axis(m, s[idx].cpu().numpy().view(np.uint16).astype(np.int64), s[vals].cpu().numpy().astype(np.float64), axis=1)
        return m
    val["cell"], val["net"] = kept("vals_cell", "idx_cell", layer.Nc), kept("vals_net_self", "idx_net_self", layer.Nn)
    mask = a["saved"]["mask"].cpu().numpy().astype(np.float64)
    dYc, dYn = (x.cpu().numpy().astype(np.float64) for x in t["dY"])
    for name, A, B in (("neigh_near", val["H_near"], dYc * mask), ("pinned", val["H_pinned"], dYc * (1 - mask)), ("neigh_pins", val["H_pins"], dYn),
                       ("self_near", val["cell"], dYc * mask), ("self_pins", val["net"], dYn)):
        got, want, l1 = b["dW"][name].cpu().numpy().astype(np.float64), A.T @ B, np.abs(A).T @ np.abs(B)
        # n products, each exact to 2^-24, in sums of which every addition rounds by at most 2^-24 of its result.  (That goes for the self
        # terms too: how many workgroups share their rows, and with it the order of their sums, depends on what a launch holds.)
        assert np.all(np.abs(got - want) <= max(len(A), 4) * 2.0 ** -23 * l1), name


@pytest.mark.parametrize("rows", [1, 31, 33, 64, 65, 129, 700])
@pytest.mark.parametrize("D,k_near,k_pins,k_pinned", WIDTHS)
def test_layer_at_tile_edges(D, k_near, k_pins, k_pinned, rows):
    say(f"act8 layer rows={rows} D={D}")
    rng = np.random.default_rng(100 * D + rows)
    Nc, Nn = rows, max(1, rows - 1)
    layer = _layer(rng, Nc, Nn, D, (k_near, k_pins, k_pinned))
    t = _tensors(rng, Nc, Nn, D)
    _check(_run(layer, t, False), _run(layer, t, True), t, layer)
    layer.heteroconv_destroy()


@pytest.mark.parametrize("mode", [P.DR_OVERLAP_ON, P.DR_OVERLAP_OFF])
def test_schedules_and_kernel_times(mode):
    rng = np.random.default_rng(5)
    Nc, Nn, D = 20_000, 12_000, 64
    layer = _layer(rng, Nc, Nn, D, (16, 16, 16), 8)
    layer.heteroconv_set_overlap(mode)
    t = _tensors(rng, Nc, Nn, D)
    a, b = _run(layer, t, False), _run(layer, t, True)
    _check(a, b, t, layer)
    layer.heteroconv_profile(True)
    layer.heteroconv_kernel_times()
    c = _run(layer, t, True)
    times = layer.heteroconv_kernel_times()
    assert times["wgrad.cell"][1] == 1 and times["wgrad.pins"][1] == 1
    _check(a, c, t, layer)
    layer.heteroconv_destroy()


def test_placed_cells_on_staged_tiles():
    """`near` in the order of a placement: its transposed DR-SpMM runs on staged tiles, beside nothing of the checkpoints."""
    rng = np.random.default_rng(9)
    Nc, Nn, D = 50_000, 3_000, 64
    near = ((np.arange(Nc)[:, None] + np.array([-4, -3, -2, -1, 1, 2, 3, 4])) % Nc).astype(np.int32).ravel()
    rel = [P.Csr(Nc, Nc, dev(8 * np.arange(Nc + 1, dtype=np.int32)), dev(near), dev(np.full(8 * Nc, 0.125, np.float32)))]
    rel += [P.Csr(m, n, *(dev(a) for a in random_csr(rng, m, n, 3, dup=True))) for m, n in ((Nn, Nc), (Nc, Nn))]
    layer = P.HeteroConv(*rel, D, 16, 16)
    assert layer.heteroconv_set_cell_order(dev(np.arange(Nc, dtype=np.int32)))
    t = _tensors(rng, Nc, Nn, D)
    _check(_run(layer, t, False), _run(layer, t, True), t, layer)
    layer.heteroconv_destroy()


def test_passes_on_alternating_streams():
    """The messages of a forward pass lie in the context's scratch: passes on several streams follow one another by themselves."""
    rng = np.random.default_rng(6)
    Nc, Nn, D = 30_000, 20_000, 64
    layer = _layer(rng, Nc, Nn, D, (16, 16, 16), 8)
    ts = [_tensors(rng, Nc, Nn, D) for _ in range(4)]
    want = [_run(layer, t, True) for t in ts]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), None, torch.cuda.Stream()]
    saved = [layer.alloc_saved8() for _ in ts]
    torch.cuda.synchronize()
    got = [_run(layer, t, True, s, side[i % 3]) for i, (t, s) in enumerate(zip(ts, saved))]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a["Y"] + a["dX"], b["Y"] + b["dX"]))
        assert all(torch.equal(a["dW"][n], b["dW"][n]) for n in P.WEIGHT_NAMES)
        assert all(torch.equal(a["saved"][n][0], b["saved"][n][0]) for n in ("H_near", "H_pins", "H_pinned"))
    layer.heteroconv_destroy()


def test_captured_layer():
    rng = np.random.default_rng(7)
    Nc, Nn, D = 3000, 2000, 64
    layer = _layer(rng, Nc, Nn, D, (16, 16, 16))
    t = _tensors(rng, Nc, Nn, D)
    saved = layer.alloc_saved8()
    Y, dX, dW = (_nan(Nc, D), _nan(Nn, D)), (_nan(Nc, D), _nan(Nn, D)), {n: _nan(D, D) for n in P.WEIGHT_NAMES}

    def step():
        layer.heteroconv_fwd_act8(*t["X"], t["W"], *Y, saved)
        layer.heteroconv_bwd_act8(*t["dY"], t["W"], saved, *dX, dW)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        for x in t["X"] + t["dY"]:
            x.copy_(dev(rng.standard_normal(x.shape).astype(np.float32)))
        step()
        torch.cuda.synchronize()
        outs = (*Y, *dX, *dW.values(), saved["H_near"][0], saved["H_pins"][1])
        want = [x.clone() for x in outs]
        for x in (*Y, *dX, *dW.values()):
            x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, outs)), i
    layer.heteroconv_destroy()


def test_refusals():
    rng = np.random.default_rng(8)
    layer = _layer(rng, 40, 30, 64, (16, 16, 16))
    t = _tensors(rng, 40, 30, 64)
    for n in ("H_near", "H_pins", "H_pinned", "vals_cell", "mask"):
        saved = layer.alloc_saved8()
        saved[n] = None
        with pytest.raises(P.DrError) as e:
            _run(layer, t, True, saved)
        assert e.value.code == P.DR_ERR_INVALID_ARG
        layer.heteroconv_fwd_act8(*t["X"], t["W"], _nan(40, 64), _nan(30, 64), layer.alloc_saved8())
        with pytest.raises(P.DrError):
            layer.heteroconv_bwd_act8(*t["dY"], t["W"], saved, _nan(40, 64), _nan(30, 64), {m: _nan(64, 64) for m in P.WEIGHT_NAMES})
    layer.heteroconv_destroy()


# ---- layers with blocks around them ---------------------------------------------------------------------------------
NORM, EPS, L = P.DR_ROWNORM_RMS, 1e-5, 3


class _Stack:
    """norm -> layer -> block -> layer -> block ... on cells and nets: what a user of the entry points writes."""

    def __init__(self, rng, Nc, Nn, D, k, eight):
        self.layer = [_layer(np.random.default_rng(50), Nc, Nn, D, (k, k, k)) for _ in range(L)]
        self.n, self.D, self.eight = (Nc, Nn), D, eight
        v = lambda at, by: dev((at + by * rng.standard_normal(D)).astype(np.float32))      # noqa: E731
        self.W = [{n: dev((rng.standard_normal((D, D)) / np.sqrt(D)).astype(np.float32)) for n in P.WEIGHT_NAMES} for _ in range(L)]
        self.after = [[dict(w_after=v(1, .2), scale=v(.5, .1)) for _ in range(2)] for _ in range(L)]
        self.before = [[dict(w_before=v(1, .2)) for _ in range(2)] for _ in range(L)]

    def forward(self, X):
        D = self.D
        self.tape = []
        x, xs8, st0, N = list(X), [], [], []
        for q in range(2):                                        # the norm in front of the first layer
            N.append(_nan(self.n[q], D))
            st0.append(_nan(self.n[q]))
            xs8.append(P.alloc_act8(self.n[q], D) if self.eight else None)
            P.dr_block_fwd(x[q], None, None, None, N[q], norm=NORM, eps=EPS, stats_before=st0[q], x8=xs8[q], **self.before[0][q])
        self.first = dict(x=list(x), x8=xs8, stats=st0)
        for i in range(L):
            saved = self.layer[i].alloc_saved8() if self.eight else self.layer[i].alloc_saved()
            Y = [_nan(n, D) for n in self.n]
            (self.layer[i].heteroconv_fwd_act8 if self.eight else self.layer[i].heteroconv_fwd)(*N, self.W[i], *Y, saved)
            rec = dict(N=N, Y=Y, saved=saved, q=[])
            out, N2 = [], []
            for q in range(2):
                last = i == L - 1
                xo, n2 = _nan(self.n[q], D), None if last else _nan(self.n[q], D)
                s = dict(stats_after=_nan(self.n[q]), stats_before=None if last else _nan(self.n[q]))
                if self.eight:
                    s["y8"] = P.alloc_act8(self.n[q], D)
                    if not last:
                        s["x8"] = P.alloc_act8(self.n[q], D)
                P.dr_block_fwd(x[q], Y[q], None, xo, n2, norm=NORM, eps=EPS, **self.after[i][q], **({} if last else self.before[i + 1][q]), **s)
                rec["q"].append(dict(s, x_out=xo))
                out.append(xo)
                N2.append(n2)
            self.tape.append(rec)
            x, N = out, N2
        return x

    def backward(self, dX):
        """gradients of the inputs and of every parameter"""
        D, grads = self.D, dict(W=[None] * L, after=[[None, None] for _ in range(L)], before=[[None, None] for _ in range(L)])
        d, dN = list(dX), [None, None]
        for i in reversed(range(L)):
            rec, last = self.tape[i], i == L - 1
            dY, dx = [], []
            for q in range(2):
                r, s = rec["q"][q], torch.zeros(3, D, device="cuda")
                ws = torch.empty(P.dr_block_bwd_workspace_bytes(self.n[q], D), dtype=torch.uint8, device="cuda")
                dY.append(_nan(self.n[q], D))
                dx.append(_nan(self.n[q], D))
                e = self.eight
                P.dr_block_bwd(d[q], dN[q], None if e or last else r["x_out"], None if e else rec["Y"][q], None, norm=NORM, eps=EPS,
                               **self.after[i][q], **({} if last else self.before[i + 1][q]), stats_after=r["stats_after"],
                               stats_before=r["stats_before"], x8=r.get("x8"), y8=r.get("y8"), dX=dx[q], dY=dY[q], dw_after=s[0],
                               dscale=s[1], dw_before=None if last else s[2], workspace=ws)
                grads["after"][i][q] = dict(w_after=s[0], scale=s[1])
                if not last:
                    grads["before"][i + 1][q] = dict(w_before=s[2])
            dN = [_nan(n, D) for n in self.n]
            grads["W"][i] = {n: _nan(D, D) for n in P.WEIGHT_NAMES}
            (self.layer[i].heteroconv_bwd_act8 if self.eight else self.layer[i].heteroconv_bwd)(*dY, self.W[i], rec["saved"], *dN, grads["W"][i])
            d = dx
        out = []
        for q in range(2):
            s = torch.zeros(D, device="cuda")
            ws = torch.empty(P.dr_block_bwd_workspace_bytes(self.n[q], D), dtype=torch.uint8, device="cuda")
            out.append(_nan(self.n[q], D))
            P.dr_block_bwd(d[q], dN[q], None if self.eight else self.first["x"][q], None, None, norm=NORM, eps=EPS, **self.before[0][q],
                           stats_before=self.first["stats"][q], x8=self.first["x8"][q], dX=out[q], dw_before=s, workspace=ws)
            grads["before"][0][q] = dict(w_before=s)
        return out, grads


def _autograd(st, X, dX):
    """The same in fp64 with torch's autograd on the CPU, selections and merge masks held to those of the GPU's pass."""
    c = lambda t: t.detach().cpu().double().requires_grad_(True)                           # noqa: E731
    D = st.D
    W = [{n: c(w) for n, w in Wl.items()} for Wl in st.W]
    after = [[{k: c(v) for k, v in a.items()} for a in row] for row in st.after]
    before = [[{k: c(v) for k, v in a.items()} for a in row] for row in st.before]
    x0 = [c(x) for x in X]
    x = list(x0)

    def dense(A):
        rp, ci, v = (t.cpu().numpy() for t in (A.rowptr, A.colidx, A.vals))
        M = np.zeros((A.n_rows, A.n_cols))
        np.add.at(M, (np.repeat(np.arange(A.n_rows), np.diff(rp)), ci), v.astype(np.float64))
        return torch.from_numpy(M)

    def norm(t):
        return t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)
    N = [norm(x[q]) * before[0][q]["w_before"] for q in range(2)]
    for i in range(L):
        rec, s = st.tape[i], st.tape[i]["saved"]
        A = [dense(a) for a in st.layer[i]._keep]

        def kept(t, idx):
            m = torch.zeros(t.shape, dtype=torch.float64)
            m.scatter_(1, torch.from_numpy(idx.cpu().numpy().view(np.uint16).astype(np.int64)), 1.0)
            return t * m
        fc, fn = kept(N[0], s["idx_cell"]), kept(N[1], s["idx_net"])
        near = fc @ W[i]["self_near"] + (A[0] @ fc) @ W[i]["neigh_near"]
        pinned = (A[2] @ fn) @ W[i]["pinned"]
        m = s["mask"].cpu().double()
        Y = [near * m + pinned * (1 - m), fn @ W[i]["self_pins"] + (A[1] @ fc) @ W[i]["neigh_pins"]]
        x = [x[q] + after[i][q]["scale"] * norm(Y[q]) * after[i][q]["w_after"] for q in range(2)]
        if i < L - 1:
            N = [norm(x[q]) * before[i + 1][q]["w_before"] for q in range(2)]
    sum((x[q] * dX[q].cpu().double()).sum() for q in range(2)).backward()
    return x, x0, W, after, before


def _stack_pairs(dx, g, x0, W, after, before):
    pairs = [(f"X{q}", dx[q], x0[q].grad) for q in range(2)]
    for i in range(L):
        pairs += [(f"{n}{i}", g["W"][i][n], W[i][n].grad) for n in P.WEIGHT_NAMES]
        for q in range(2):
            pairs += [(f"{n}{i}{q}", g["after"][i][q][n], after[i][q][n].grad) for n in ("w_after", "scale")]
            pairs.append((f"w_before{i}{q}", g["before"][i][q]["w_before"], before[i][q]["w_before"].grad))
    return pairs


@pytest.mark.parametrize("eight", [False, True])
def test_stack_of_layers_and_blocks(eight):
    """Gradients through three layers with blocks around them.  In fp32: relative 2-norm, a few hundred roundings of 2^-24 on the way to any
    entry, amplified by no more than the six norms and three layers between (their gradients have norms of order one): 1e-4.  From checkpoints: a
    value of a group is off by at most a 127.5th of the group's largest, at most its 2-norm; a uniform error of that width has 1/sqrt(3) of it
    as its own root mean square, and a group of 32 normal values has a largest of some 2.2 root mean squares, so that an operand of a
    gradient is 2.2 / 127.5 / sqrt(3) = 1 % off.  Every gradient goes through at most 2 L + 1 = 7 operands: 7 % (the errors add up at worst)."""
    rng = np.random.default_rng(11)
    Nc, Nn, D, k = 500, 300, 64, 16
    st = _Stack(rng, Nc, Nn, D, k, eight)
    X = [dev(rng.standard_normal((n, D)).astype(np.float32)) for n in (Nc, Nn)]
    dX = [dev(rng.standard_normal((n, D)).astype(np.float32)) for n in (Nc, Nn)]
    out = st.forward(X)
    dx, g = st.backward(dX)
    x, x0, W, after, before = _autograd(st, X, dX)
    for q in range(2):
        assert (out[q].cpu().double() - x[q]).norm() <= 1e-4 * x[q].norm()
    for name, got, want in _stack_pairs(dx, g, x0, W, after, before):
        off = float((got.cpu().double() - want).norm() / want.norm())
        assert off <= (0.07 if eight else 1e-4), (name, off)
    for l in st.layer:
        l.heteroconv_destroy()


def test_stack_against_differences():
    """A directional derivative of the whole stack by central differences, on the GPU's own forward in fp32: along a direction of the last
    layer's scale, in which the output is linear, so that only roundings of the two outputs count."""
    rng = np.random.default_rng(12)
    Nc, Nn, D, k = 400, 250, 64, 16
    st = _Stack(rng, Nc, Nn, D, k, False)
    X = [dev(rng.standard_normal((n, D)).astype(np.float32)) for n in (Nc, Nn)]
    dX = [dev(rng.standard_normal((n, D)).astype(np.float32)) for n in (Nc, Nn)]
    st.forward(X)
    _, g = st.backward(dX)
    want = sum(float(g["after"][L - 1][q]["scale"].double().sum()) for q in range(2))
    base = [a["scale"].clone() for a in st.after[L - 1]]
    val, mag = [], 0.0
    for sign in (1, -1):
        for q in range(2):
            st.after[L - 1][q]["scale"] = base[q] + sign * 0.25
        o = st.forward(X)
        val.append(sum(float((o[q].double() * dX[q].double()).sum()) for q in range(2)))
        mag += sum(float((o[q].double() * dX[q].double()).abs().sum()) for q in range(2))
    # every output is off by some 16 * 2^-24 of itself at most, over a step of 0.5
    assert abs((val[0] - val[1]) / 0.5 - want) <= 16 * 2.0 ** -24 * mag / 0.5
    for l in st.layer:
        l.heteroconv_destroy()
