"""The residual block around a layer (norm behind it, gate, residual scale, residual sum, norm in front of the next layer), forward and
backward, from fp32 tensors and from 8-bit checkpoints, against the fp64 oracle."""
import itertools

import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev, say
from oracle import block as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# roundings on the way to an entry.  A row's mean: at most 16 additions in a lane and 6 between lanes, a division, a square root, a
# reciprocal; the forward passes two norms.  Backward: two norms with two means each, the sigmoid, and some twenty products.
FWD, BWD = 64 * U, 128 * U
NORMS = {"rms": P.DR_ROWNORM_RMS, "layer": P.DR_ROWNORM_LAYER}
PARAMS = ("w_after", "b_after", "scale", "w_before", "b_before")


def _inputs(rng, n, D, gate, params=True):
    f = lambda *s: rng.standard_normal(s).astype(np.float32)                      # noqa: E731
    size = np.exp(0.5 * rng.standard_normal((2, n, 1))).astype(np.float32)
    size[:, rng.random(n) < 0.05] = 0
    cols = {"none": 0, "row": 1, "full": D}[gate]
    a = dict(X=f(n, D) * size[0], Y=f(n, D) * size[1], G=3 * f(n, cols) if cols else None)
    for name, at, by in (("w_after", 1, .2), ("b_after", 0, .1), ("scale", .5, .2), ("w_before", 1, .2), ("b_before", 0, .1)):
        a[name] = (at + by * f(D)).astype(np.float32) if params else None
    return a


def _dev(a):
    return None if a is None else dev(a)


def _stats_room(n, norm):
    return torch.full((n,) if norm == "rms" else (n, 2), float("nan"), device="cuda")


def _pair(stats, norm):
    s = stats.cpu().numpy().astype(np.float64)
    return (np.zeros((len(s), 1)), s[:, None]) if norm == "rms" else (s[:, :1], s[:, 1:])


def _close(got, want, mag, k, what):
    got = got.cpu().numpy().astype(np.float64).reshape(want.shape)
    err = np.abs(got - want)
    bad = ~(err <= k * mag + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(err / np.maximum(mag, 1e-300)) / U))


def _forward(a, norm, eps, bits):
    n, D = a["X"].shape
    o = dict(X_out=torch.full((n, D), float("nan"), device="cuda"), N=torch.full((n, D), float("nan"), device="cuda"),
             stats_after=_stats_room(n, norm), stats_before=_stats_room(n, norm))
    ck = {}
    if bits == 8:
        for name in ("x8", "y8") + (("g8",) if a["G"] is not None and a["G"].shape[1] == D else ()):
            ck[name] = P.alloc_act8(n, D)
    P.dr_block_fwd(_dev(a["X"]), _dev(a["Y"]), _dev(a["G"]), o["X_out"], o["N"], norm=NORMS[norm], eps=eps,
                   stats_after=o["stats_after"], stats_before=o["stats_before"], **{p: _dev(a[p]) for p in PARAMS}, **ck)
    return o, ck


def _check_forward(a, norm, eps, o, ck):
    want = ob.block_fwd(layer=norm == "layer", eps=eps, **a)
    _close(o["X_out"], want["X_out"], want["abs"]["X_out"], FWD, "X_out")
    _close(o["N"], want["N"], want["abs"]["N"], FWD, "N")
    for which in ("after", "before"):
        m, r = _pair(o["stats_" + which], norm)
        assert np.all(np.abs(m - want["m_" + which]) <= FWD * want["abs"]["m_" + which])
        assert np.all(np.abs(r - want["r_" + which]) <= FWD * want["abs"]["r_" + which])
    # checkpoints are those of the fp32 tensors
    for name, t in (("x8", o["X_out"].cpu().numpy()), ("y8", a["Y"]), ("g8", a["G"])):
        if name in ck:
            q, s = ob.act8_pack(t)
            assert np.array_equal(ck[name][0].cpu().numpy(), q) and np.array_equal(ck[name][1].cpu().numpy(), s), name


def _backward(a, norm, dX_out, dN, o, ck, want_all=True):
    n, D = (dX_out if dX_out is not None else dN).shape
    g = dict(dX=torch.full((n, D), float("nan"), device="cuda"))
    if a["Y"] is not None:
        g["dY"] = torch.full((n, D), float("nan"), device="cuda")
        for name in ("dw_after", "db_after", "dscale"):
            g[name] = torch.full((D,), float("nan"), device="cuda")
        if a["G"] is not None:
            g["dG"] = torch.full(a["G"].shape, float("nan"), device="cuda")
    for name in ("dw_before", "db_before"):
        g[name] = torch.full((D,), float("nan"), device="cuda")
    ws = torch.full((P.dr_block_bwd_workspace_bytes(n, D),), 255, dtype=torch.uint8, device="cuda")
    P.dr_block_bwd(_dev(dX_out), _dev(dN), None if "x8" in ck else o["X_out"], None if "y8" in ck else _dev(a["Y"]),
                   None if "g8" in ck else _dev(a["G"]), norm=NORMS[norm], w_after=_dev(a["w_after"]), b_after=_dev(a["b_after"]),
                   scale=_dev(a["scale"]), w_before=_dev(a["w_before"]), b_before=_dev(a["b_before"]), stats_after=o["stats_after"],
                   stats_before=o["stats_before"], **ck, **g, workspace=ws)
    return g


def _check_backward(a, norm, dX_out, dN, o, ck, g):
    val = lambda name, t: ob.act8_values(ck[name][0].cpu().numpy(), ck[name][1].cpu().numpy()) if name in ck else t    # noqa: E731
    n = (dX_out if dX_out is not None else dN).shape[0]
    want = ob.block_bwd(dX_out, dN, None if dN is None else val("x8", o["X_out"].cpu().numpy()),
                        None if dN is None else _pair(o["stats_before"], norm), None if a["Y"] is None else val("y8", a["Y"]),
                        None if a["Y"] is None else _pair(o["stats_after"], norm), val("g8", a["G"]), norm == "layer", a["w_after"],
                        a["b_after"], a["scale"], a["w_before"])
    for name, t in g.items():
        if name not in want:                                   # sums of a part that is left out
            assert not t.any(), name
            continue
        sums = name.startswith(("dw", "db", "ds"))
        # a lane adds up the rows that it walks, one after the other
        _close(t, want[name], want["abs"][name], BWD + (n * U if sums else 0), name)


@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 32, 33, 48, 64, 77, 96, 99, 128, 129, 200, 256, 257, 512, 516, 600, 1000, 1023, 1024])
def test_widths(D):
    rng = np.random.default_rng(D)
    for n, (norm, gate, bits) in zip(itertools.cycle((1, 5, 8, 33, 130, 701)), itertools.product(NORMS, ("none", "row", "full"), (32, 8))):
        say(f"block n={n} D={D} {norm} gate={gate} bits={bits}")
        a = _inputs(rng, n, D, gate)
        o, ck = _forward(a, norm, 1e-5, bits)
        _check_forward(a, norm, 1e-5, o, ck)
        dX_out, dN = (0.1 * rng.standard_normal((2, n, D))).astype(np.float32)
        g = _backward(a, norm, dX_out, dN, o, ck)
        _check_backward(a, norm, dX_out, dN, o, ck, g)


@pytest.mark.parametrize("D", [20, 64, 99, 300, 1000])
def test_some_from_tensors_some_from_checkpoints(D):
    rng = np.random.default_rng(D + 1)
    n, norm = 90, "layer"
    a = _inputs(rng, n, D, "full")
    o, ck = _forward(a, norm, 1e-5, 8)
    dX_out, dN = (0.1 * rng.standard_normal((2, n, D))).astype(np.float32)
    for names in (("x8",), ("y8",), ("g8",), ("x8", "y8"), ("x8", "g8"), ("y8", "g8")):
        some = {k: ck[k] for k in names}
        _check_backward(a, norm, dX_out, dN, o, some, _backward(a, norm, dX_out, dN, o, some))


@pytest.mark.parametrize("norm", list(NORMS))
@pytest.mark.parametrize("D", [64, 77])
def test_parts_left_out(norm, D):
    """Only the norm in front, only the part behind the layer, no parameters, one incoming gradient."""
    rng = np.random.default_rng(7)
    n, eps = 300, 1e-3
    a = _inputs(rng, n, D, "full", params=False)
    dX_out, dN = (0.1 * rng.standard_normal((2, n, D))).astype(np.float32)
    o, ck = _forward(a, norm, eps, 32)
    _check_forward(a, norm, eps, o, ck)
    for x, y in ((dX_out, dN), (None, dN), (dX_out, None)):
        _check_backward(a, norm, x, y, o, ck, _backward(a, norm, x, y, o, ck))
    # behind the layer only
    only = torch.full((n, D), float("nan"), device="cuda")
    st = _stats_room(n, norm)
    P.dr_block_fwd(_dev(a["X"]), _dev(a["Y"]), _dev(a["G"]), only, None, norm=NORMS[norm], eps=eps, stats_after=st)
    assert torch.equal(only, o["X_out"]) and torch.equal(st, o["stats_after"])
    # in front only, with the checkpoint of its input
    front = dict(a, Y=None, G=None)
    N, st, x8 = torch.full((n, D), float("nan"), device="cuda"), _stats_room(n, norm), P.alloc_act8(n, D)
    P.dr_block_fwd(_dev(a["X"]), None, None, None, N, norm=NORMS[norm], eps=eps, stats_before=st, x8=x8)
    want = ob.block_fwd(a["X"], layer=norm == "layer", eps=eps)
    _close(N, want["N"], want["abs"]["N"], FWD, "N")
    q, s = ob.act8_pack(a["X"])
    assert np.array_equal(x8[0].cpu().numpy(), q) and np.array_equal(x8[1].cpu().numpy(), s)
    oo = dict(X_out=_dev(a["X"]), stats_before=st, stats_after=None)
    for x, y in ((dX_out, dN), (None, dN)):
        for c in ({}, {"x8": x8}):
            _check_backward(front, norm, x, y, oo, c, _backward(front, norm, x, y, oo, c))


def test_no_rows():
    D = 40
    e = torch.empty(0, D, device="cuda")
    P.dr_block_fwd(e, e, None, e, e, stats_after=e, stats_before=e)
    sums = torch.full((5, D), float("nan"), device="cuda")
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(0, D), dtype=torch.uint8, device="cuda")
    P.dr_block_bwd(e, e, e, e, None, stats_after=e, stats_before=e, dX=e, dY=e, dw_after=sums[0], db_after=sums[1], dscale=sums[2],
                   dw_before=sums[3], db_before=sums[4], workspace=ws)
    assert not sums.any()


@pytest.mark.parametrize("D", [64, 77, 1000])
def test_results_in_place_of_inputs(D):
    rng = np.random.default_rng(D)
    n, norm = 500, "layer"
    a = _inputs(rng, n, D, "full")
    kw = {p: _dev(a[p]) for p in PARAMS}
    o, _ = _forward(a, norm, 1e-5, 32)
    dX_out, dN = (0.1 * rng.standard_normal((2, n, D))).astype(np.float32)
    g = _backward(a, norm, dX_out, dN, o, {})
    for to in (("X", "Y"), ("Y", "X"), ("G", "X"), ("X", "G")):
        t = {k: _dev(a[k]) for k in "XYG"}
        P.dr_block_fwd(t["X"], t["Y"], t["G"], t[to[0]], t[to[1]], norm=NORMS[norm], eps=1e-5, **kw)
        assert torch.equal(t[to[0]], o["X_out"]) and torch.equal(t[to[1]], o["N"]), to
    for to in (("dX_out", "dN"), ("Y", "X"), ("G", "Y"), ("X", "G"), ("dN", "dX_out")):
        t = dict(X=o["X_out"].clone(), Y=_dev(a["Y"]), G=_dev(a["G"]), dX_out=dev(dX_out), dN=dev(dN))
        ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
        dG = torch.empty(n, D, device="cuda")
        P.dr_block_bwd(t["dX_out"], t["dN"], t["X"], t["Y"], t["G"], norm=NORMS[norm], **kw, stats_after=o["stats_after"],
                       stats_before=o["stats_before"], dX=t[to[0]], dY=t[to[1]], dG=dG, workspace=ws)
        assert torch.equal(t[to[0]], g["dX"]) and torch.equal(t[to[1]], g["dY"]) and torch.equal(dG, g["dG"]), to


def test_wild_rows_stay_by_themselves():
    """Infinities, not-a-numbers and saturated gates: other rows are what they are without them."""
    rng = np.random.default_rng(9)
    n, D, norm = 200, 96, "rms"
    a = _inputs(rng, n, D, "full")
    clean, _ = _forward(a, norm, 1e-5, 8)
    a["X"][3, 5], a["Y"][50, 7], a["Y"][90] = np.inf, np.nan, 3e38
    a["G"][120], a["G"][121] = 200.0, -200.0
    o, ck = _forward(a, norm, 1e-5, 8)
    rest = np.delete(np.arange(n), [3, 50, 90, 120, 121])
    assert torch.equal(o["N"][rest], clean["N"][rest]) and torch.equal(o["X_out"][rest], clean["X_out"][rest])
    assert torch.isnan(o["X_out"][50]).all() and torch.isfinite(o["N"][120:122]).all()
    assert torch.equal(o["X_out"][121], dev(a["X"])[121])      # a closed gate
    g = _backward(a, norm, *(0.1 * rng.standard_normal((2, n, D))).astype(np.float32), o, {})
    assert torch.isfinite(g["dX"][rest]).all() and torch.isfinite(g["dY"][rest]).all() and torch.isfinite(g["dG"][rest]).all()
    assert not g["dG"][120:122].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_nothing_of_a_norm_that_is_left_out_counts(bits):
    """Without dN the rows and statistics of the norm in front are not part of the gradient, whatever they hold."""
    rng = np.random.default_rng(10)
    n, D, norm = 50, 64, "layer"
    a = _inputs(rng, n, D, "none")
    o, ck = _forward(a, norm, 1e-5, bits)
    dX_out = (0.1 * rng.standard_normal((n, D))).astype(np.float32)
    want = _backward(a, norm, dX_out, None, o, ck)
    o["X_out"].fill_(float("inf"))
    o["stats_before"].fill_(float("nan"))
    if bits == 8:
        ck["x8"][1].fill_(255)
    got = _backward(a, norm, dX_out, None, o, ck)
    for k in ("dX", "dY", "dw_after", "db_after", "dscale", "dw_before", "db_before"):
        assert torch.equal(got[k], want[k]), k
    assert torch.equal(got["dX"], dev(dX_out)) and not got["dw_before"].any()


def test_rows_at_any_alignment():
    rng = np.random.default_rng(11)
    n, D, norm = 60, 64, "layer"
    a = _inputs(rng, n, D, "full")
    o, _ = _forward(a, norm, 1e-5, 32)

    def off(x):
        room = torch.zeros(x.numel() + 1, device="cuda")
        room[1:] = x.reshape(-1)
        return room[1:].view(x.shape)
    X_out, N = off(o["X_out"] * 0), off(o["N"] * 0)
    y8 = P.alloc_act8(n, D)
    P.dr_block_fwd(off(dev(a["X"])), off(dev(a["Y"])), off(dev(a["G"])), X_out, N, norm=NORMS[norm], eps=1e-5, y8=y8,
                   **{p: off(_dev(a[p])) for p in PARAMS})
    want = ob.block_fwd(layer=True, eps=1e-5, **a)
    _close(X_out, want["X_out"], want["abs"]["X_out"], FWD, "X_out")
    _close(N, want["N"], want["abs"]["N"], FWD, "N")
    assert np.array_equal(y8[0].cpu().numpy(), ob.act8_pack(a["Y"])[0])


def test_offsets_past_32_bits():
    """More than 2^31 elements a tensor; only the last rows are not zero."""
    n, D, norm = 2_150_000, 1024, "rms"
    rng = np.random.default_rng(13)
    k = 9
    a = _inputs(rng, k, D, "none")
    big = {}
    for name in "XY":
        big[name] = torch.zeros(n, D, device="cuda")
        big[name][-k:] = dev(a[name])
    o = dict(stats_after=_stats_room(n, norm), stats_before=_stats_room(n, norm))
    kw = {p: _dev(a[p]) for p in PARAMS}
    y8 = P.alloc_act8(n, D)
    P.dr_block_fwd(big["X"], big["Y"], None, big["X"], big["Y"], y8=y8, **o, **kw)        # in place
    small, _ = _forward(a, norm, 1e-5, 32)
    assert torch.equal(big["X"][-k:], small["X_out"]) and torch.equal(big["Y"][-k:], small["N"])
    dX_out = torch.zeros(n, D, device="cuda")
    d = (0.1 * rng.standard_normal((k, D))).astype(np.float32)
    dX_out[-k:] = dev(d)
    sums = torch.full((3, D), float("nan"), device="cuda")
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    P.dr_block_bwd(dX_out, None, None, None, None, y8=y8, stats_after=o["stats_after"], dX=dX_out, dY=big["Y"], dw_after=sums[0],
                   db_after=sums[1], dscale=sums[2], workspace=ws, **kw)
    q, s = ob.act8_pack(a["Y"])
    want = ob.block_bwd(d, None, Y=ob.act8_values(q, s), stats_after=_pair(o["stats_after"][-k:], norm), w_after=a["w_after"],
                        b_after=a["b_after"], scale=a["scale"])
    _close(big["Y"][-k:], want["dY"], want["abs"]["dY"], BWD, "dY")
    for i, name in enumerate(("dw_after", "db_after", "dscale")):
        _close(sums[i], want[name], want["abs"][name], BWD + k * U, name)
    assert not big["Y"][:-k].any() and not dX_out[:-k].any()


def test_captured_with_checkpoints_and_weight_gradients():
    """Forward, backward from checkpoints and a weight gradient as one graph, replayed on new inputs between eager passes."""
    rng = np.random.default_rng(17)
    n, D, norm = 3000, 64, "rms"
    a = {k: _dev(v) for k, v in _inputs(rng, n, D, "full").items()}
    kw = {p: a[p] for p in PARAMS}
    d = dev((0.1 * rng.standard_normal((n, D))).astype(np.float32))
    ck = {k: P.alloc_act8(n, D) for k in ("x8", "y8", "g8")}
    st = dict(stats_after=_stats_room(n, norm), stats_before=_stats_room(n, norm))
    bufs = {k: torch.empty(n, D, device="cuda") for k in ("X_out", "N", "dX", "dY", "dG", "back")}
    sums, dW = torch.empty(5, D, device="cuda"), torch.empty(D, D, device="cuda")
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(P.dr_act8_wgrad_workspace_bytes(n, D, D), dtype=torch.uint8, device="cuda")

    def step():
        P.dr_block_fwd(a["X"], a["Y"], a["G"], bufs["X_out"], bufs["N"], **kw, **ck, **st)
        P.dr_block_bwd(d, d, None, None, None, **kw, **ck, **st, dX=bufs["dX"], dY=bufs["dY"], dG=bufs["dG"], dw_after=sums[0],
                       db_after=sums[1], dscale=sums[2], dw_before=sums[3], db_before=sums[4], workspace=ws)
        P.dr_act8_unpack(ck["y8"], bufs["back"])
        P.dr_act8_wgrad(ck["x8"], bufs["dY"], dW, ws2)
    step()                                                     # first calls ask the runtime about the device
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        for k in "XYG":
            a[k].copy_(dev(rng.standard_normal((n, D)).astype(np.float32)))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (*bufs.values(), sums, dW)]
        for t in (*bufs.values(), sums, dW):
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (*bufs.values(), sums, dW))), i


def test_on_a_stream_of_its_own():
    """Inputs that a side stream is still writing: the calls follow on that stream."""
    rng = np.random.default_rng(19)
    n, D = 20_000, 128
    a = _inputs(rng, n, D, "none")
    o, _ = _forward(a, "rms", 1e-5, 32)
    kw = {p: _dev(a[p]) for p in PARAMS}
    x, y = dev(a["X"]), dev(a["Y"])
    s = torch.cuda.Stream()
    big = torch.randn(6000, 6000, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(4):
            big = big @ big * 1e-4
        X, Y = torch.zeros_like(x), torch.zeros_like(y)
        X.copy_(x)
        Y.copy_(y)
        X_out, N = torch.empty_like(X), torch.empty_like(X)
        P.dr_block_fwd(X, Y, None, X_out, N, **kw)
        ck = P.alloc_act8(n, D)
        P.dr_act8_pack(X_out, ck)
    s.synchronize()
    assert torch.equal(X_out, o["X_out"]) and torch.equal(N, o["N"])
    assert np.array_equal(ck[0].cpu().numpy(), ob.act8_pack(o["X_out"].cpu().numpy())[0])
