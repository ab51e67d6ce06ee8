"""Cases for the row-block and 8-bit checkpoint operators, with their plain forms.

A case is a dict of plain values.  ``kind`` says which operator a pass goes through:

* ``ckpt``       a matrix of activations to an 8-bit checkpoint and back (dr_act8_pack, dr_act8_unpack)
* ``block_fwd``  X_out = X + scale * sigmoid(G) * norm(Y), N = norm(X_out) (dr_block_fwd); with ``bits`` = 8 also the checkpoints
                 of X_out, Y and G, read back as the values they stand for
* ``block_bwd``  its gradients (dr_block_bwd), from fp32 tensors (``bits`` = 32) or from checkpoints (8)
* ``wgrad``      dW = A^T dZ with A held as an 8-bit checkpoint (dr_act8_wgrad)

``norm`` is "rms" or "layer", ``gate`` "none", "row" (one gate per row) or "full" (one per element).
A checkpoint has one power-of-two scale per 32 columns of a row; the scales of eight consecutive rows lie side by side.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
GROUP = 32
# elements of the largest matrix: 1.2 million cells of width 128
MOST = 1_200_000 * 128


# ----------------------------------------------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the messages of a freshly cut corner of a design: launches are all there is
        dict(name="ckpt_tiny", kind="ckpt", n=2048, D=64),
        # a block of odd size, a width that no vector load divides
        dict(name="ckpt_odd", kind="ckpt", n=20011, D=77),
        # all cells of a whole design
        dict(name="ckpt_design", kind="ckpt", n=1_200_000, D=128),
        # a residual block on a corner of a design, nothing gated, tensors kept in 32 bits
        dict(name="block_fwd_tiny", kind="block_fwd", n=2048, D=64, norm="rms", gate="none", bits=32),
        # odd rows and columns, a gate per cell
        dict(name="block_fwd_odd", kind="block_fwd", n=30011, D=99, norm="layer", gate="row", bits=32),
        # half a million cells with a gate per element, checkpoints written on the way
        dict(name="block_fwd_ckpt", kind="block_fwd", n=500_000, D=128, norm="rms", gate="full", bits=8),
        # gradients on a corner of a design, from checkpoints
        dict(name="block_bwd_tiny", kind="block_bwd", n=2048, D=64, norm="rms", gate="none", bits=8),
        # wide rows of a read-out, everything in 32 bits
        dict(name="block_bwd_wide", kind="block_bwd", n=20000, D=1000, norm="layer", gate="full", bits=32),
        # all cells of a whole design, from checkpoints
        dict(name="block_bwd_design", kind="block_bwd", n=1_200_000, D=128, norm="rms", gate="row", bits=8),
        # weight gradient of a projection on a corner of a design
        dict(name="wgrad_tiny", kind="wgrad", n=2048, D=64, F=64),
        # a ragged block projected to a wider read-out
        dict(name="wgrad_ragged", kind="wgrad", n=60013, D=96, F=200),
        # all cells of a whole design
        dict(name="wgrad_design", kind="wgrad", n=1_200_000, D=128, F=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    """Half of the widths are a layer's or a multiple of it, half are any."""
    return rng.choice((32, 64, 96, 128, 256, 512)) if rng.random() < 0.5 else _log(rng, 1, 1024)


def draw(rng):
    kind = rng.choice(("ckpt", "block_fwd", "block_bwd", "wgrad"))
    D = _width(rng)
    if kind == "wgrad":
        F = _width(rng)
        most = min(1_200_000, 1_200_000 * 128 * 128 // (D * F), MOST * 5 // (D + 4 * F))
        return dict(kind=kind, n=_log(rng, 1, most), D=D, F=F)
    n = _log(rng, 1, min(1_200_000, MOST // D))
    if kind == "ckpt":
        return dict(kind=kind, n=n, D=D)
    gate = rng.choice(("none", "row", "full"))
    if gate == "full":
        n = max(1, n // 2)
    return dict(kind=kind, n=n, D=D, norm=rng.choice(("rms", "layer")), gate=gate, bits=rng.choice((8, 32)))


# ----------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------
def _rows(g, n, D):
    """Embeddings: rows of different size, one in fifty all zeros (cells without edges have no messages)."""
    x = torch.randn(n, D, generator=g, device="cuda")
    size = torch.exp(0.5 * torch.randn(n, 1, generator=g, device="cuda"))
    size[torch.rand(n, 1, generator=g, device="cuda") < 0.02] = 0
    return x * size


def _checkpoint_room(n, D):
    """q [n, D] and the scale bytes [ceil(n / 8), groups, 8] of a checkpoint."""
    return (torch.empty(n, D, dtype=torch.int8, device="cuda"),
            torch.empty(-(-n // 8) * -(-D // GROUP) * 8, dtype=torch.uint8, device="cuda"))


def _groups(x):
    n, D = x.shape
    G = -(-D // GROUP)
    v = x.new_zeros(n, G * GROUP)
    v[:, :D] = x
    return v.view(n, G, GROUP)


def _codes(x):
    """Codes [n, G, 32] (32-bit floats) and scale bytes [n, G] of the checkpoint of x."""
    v = _groups(x)
    top = v.abs().amax(-1)
    byte = (((top.view(torch.int32) + 0x10000) >> 23) - 6).clamp(min=1)          # 2^(byte - 127) * 127.5 > top
    q = torch.round(v * ((254 - byte) << 23).view(torch.float32).unsqueeze(-1))
    bad = ~torch.isfinite(top)
    return torch.where(bad.unsqueeze(-1), torch.zeros_like(q), q), torch.where(bad, torch.full_like(byte, 255), byte)


def _power(byte):
    """2^(byte - 127); not-a-number for 255."""
    f = (byte << 23).view(torch.float32)
    return torch.where(byte == 255, torch.full_like(f, math.nan), f)


def _checkpoint(x):
    n, D = x.shape
    q, byte = _codes(x)
    G = byte.shape[1]
    b = byte.new_zeros(-(-n // 8) * 8, G)
    b[:n] = byte
    scale = b.view(-1, 8, G).transpose(1, 2).contiguous().to(torch.uint8).view(-1)
    return q.view(n, -1)[:, :D].to(torch.int8).contiguous(), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, D, kind = case["n"], case["D"], case["kind"]
    f32 = dict(dtype=torch.float32, device="cuda")
    st = {"case": case}
    if kind == "ckpt":
        st.update(X=_rows(g, n, D), room=_checkpoint_room(n, D), out=torch.empty(n, D, **f32))
        return st
    if kind == "wgrad":
        st.update(A=_checkpoint(_rows(g, n, D)), dZ=0.1 * _rows(g, n, case["F"]), dW=torch.empty(D, case["F"], **f32))
        return st

    def vec(at, by):
        return at + by * torch.randn(D, generator=g, device="cuda")

    gate_cols = {"none": 0, "row": 1, "full": D}[case["gate"]]
    stat = (n,) if case["norm"] == "rms" else (n, 2)
    st.update(w_after=vec(1.0, 0.2), b_after=vec(0.0, 0.1), scale=vec(0.5, 0.2), w_before=vec(1.0, 0.2), b_before=vec(0.0, 0.1))
    G = torch.randn(n, gate_cols, generator=g, device="cuda") if gate_cols else None
    X, Y = _rows(g, n, D), _rows(g, n, D)
    if kind == "block_fwd":
        st.update(X=X, Y=Y, G=G, X_out=torch.empty(n, D, **f32), N=torch.empty(n, D, **f32),
                  stats_after=torch.empty(stat, **f32), stats_before=torch.empty(stat, **f32))
        if case["bits"] == 8:
            for name in ("x", "y") + (("g",) if gate_cols == D else ()):
                st["room_" + name], st["values_" + name] = _checkpoint_room(n, D), torch.empty(n, D, **f32)
        return st
    # what the forward pass left: X_out is X here, the statistics are those of the rows themselves
    st.update(dX_out=0.1 * torch.randn(n, D, generator=g, device="cuda"), dN=0.1 * torch.randn(n, D, generator=g, device="cuda"),
              stats_after=_stats(Y, case["norm"]), stats_before=_stats(X, case["norm"]),
              dX=torch.empty(n, D, **f32), dY=torch.empty(n, D, **f32), dG=torch.empty(n, gate_cols, **f32) if gate_cols else None,
              sums=torch.empty(5, D, **f32))
    if case["bits"] == 8:
        st.update(x8=_checkpoint(X), y8=_checkpoint(Y), g8=_checkpoint(G) if gate_cols == D else None,
                  X=None, Y=None, G=None if gate_cols == D else G)
    else:
        st.update(X=X, Y=Y, G=G, x8=None, y8=None, g8=None)
    return st


def _stats(x, norm):
    if norm == "rms":
        return 1 / torch.sqrt((x * x).mean(1) + EPS)
    m = x.mean(1)
    return torch.stack((m, 1 / torch.sqrt(((x - m[:, None]) ** 2).mean(1) + EPS)), 1)


# ----------------------------------------------------------------------------------------------------------------
# passes
# ----------------------------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if own:
        return _own(st, case)
    return {"ckpt": _plain_ckpt, "block_fwd": _plain_fwd, "block_bwd": _plain_bwd, "wgrad": _plain_wgrad}[case["kind"]](st, case)


def _own(st, case):
    import paper_2508_16769_amd as P
    kind, n, D = case["kind"], case["n"], case["D"]
    if kind == "ckpt":
        P.dr_act8_pack(st["X"], st["room"])
        P.dr_act8_unpack(st["room"], st["out"])
        return st["out"]
    if kind == "wgrad":
        ws = torch.empty(P.dr_act8_wgrad_workspace_bytes(n, D, case["F"]), dtype=torch.uint8, device="cuda")
        P.dr_act8_wgrad(st["A"], st["dZ"], st["dW"], ws)
        return st["dW"]
    block = dict(norm=P.DR_ROWNORM_RMS if case["norm"] == "rms" else P.DR_ROWNORM_LAYER, eps=EPS, w_after=st["w_after"],
                 b_after=st["b_after"], scale=st["scale"], w_before=st["w_before"], b_before=st["b_before"],
                 stats_after=st["stats_after"], stats_before=st["stats_before"])
    if kind == "block_fwd":
        P.dr_block_fwd(st["X"], st["Y"], st["G"], st["X_out"], st["N"], x8=st.get("room_x"), y8=st.get("room_y"),
                       g8=st.get("room_g"), **block)
        out = {k: st[k] for k in ("X_out", "N", "stats_after", "stats_before")}
        for name in "xyg":
            if "room_" + name in st:
                P.dr_act8_unpack(st["room_" + name], st["values_" + name])
                out[name + "8"] = st["values_" + name].to(torch.bfloat16)          # exactly what the codes stand for
        return out
    ws = torch.empty(P.dr_block_bwd_workspace_bytes(n, D), dtype=torch.uint8, device="cuda")
    s = st["sums"]
    P.dr_block_bwd(st["dX_out"], st["dN"], st["X"], st["Y"], st["G"], x8=st["x8"], y8=st["y8"], g8=st["g8"], dX=st["dX"],
                   dY=st["dY"], dG=st["dG"], dw_after=s[0], db_after=s[1], dscale=s[2], dw_before=s[3], db_before=s[4],
                   workspace=ws, **block)
    return {"dX": st["dX"], "dY": st["dY"], "dG": st["dG"], "sums": s}


def _values(ckpt):
    """What a checkpoint stands for, in 32 bits (exact)."""
    q, scale = ckpt
    n, D = q.shape
    G = -(-D // GROUP)
    f = _power(scale.view(-1, G, 8).transpose(1, 2).reshape(-1, G)[:n].to(torch.int32))
    return (_groups(q.to(torch.float32)) * f.unsqueeze(-1)).view(n, -1)[:, :D]


def _rounded(x):
    """x as its checkpoint holds it."""
    q, byte = _codes(x)
    return (q * _power(byte).unsqueeze(-1)).view(x.shape[0], -1)[:, :x.shape[1]]


def _plain_ckpt(st, case):
    return _rounded(st["X"]).contiguous()


def _plain_wgrad(st, case):
    # sums of 2048 rows in 32 bits, those of the blocks in 64
    A, dZ, block = _values(st["A"]), st["dZ"], 2048
    n, whole = case["n"], case["n"] // block * block
    s = (A[whole:].t() @ dZ[whole:]).double()
    if whole:
        s = s + torch.bmm(A[:whole].reshape(-1, block, case["D"]).transpose(1, 2).contiguous(),
                          dZ[:whole].reshape(-1, block, case["F"])).sum(0, dtype=torch.float64)
    return s.float()


def _hat(x, stats, norm):
    return x * stats[:, None] if norm == "rms" else (x - stats[:, :1]) * stats[:, 1:]


def _plain_fwd(st, case):
    sa = _stats(st["Y"], case["norm"])
    u = _hat(st["Y"], sa, case["norm"]) * st["w_after"] + st["b_after"]
    if st["G"] is not None:
        u = u / (1 + torch.exp(-st["G"]))
    X_out = st["X"] + st["scale"] * u
    sb = _stats(X_out, case["norm"])
    out = {"X_out": X_out, "N": _hat(X_out, sb, case["norm"]) * st["w_before"] + st["b_before"], "stats_after": sa, "stats_before": sb}
    if case["bits"] == 8:
        out["x8"], out["y8"] = _rounded(X_out).to(torch.bfloat16), _rounded(st["Y"]).to(torch.bfloat16)
        if case["gate"] == "full":
            out["g8"] = _rounded(st["G"]).to(torch.bfloat16)
    return out


def _norm_back(g, hat, stats, norm):
    r = stats[:, None] if norm == "rms" else stats[:, 1:]
    d = g - hat * (g * hat).mean(1, keepdim=True)
    return r * (d if norm == "rms" else d - g.mean(1, keepdim=True))


def _plain_bwd(st, case):
    norm = case["norm"]
    X = st["X"] if st["x8"] is None else _values(st["x8"])
    Y = st["Y"] if st["y8"] is None else _values(st["y8"])
    G = st["G"] if st["g8"] is None else _values(st["g8"])
    xh, yh = _hat(X, st["stats_before"], norm), _hat(Y, st["stats_after"], norm)
    d = st["dX_out"] + _norm_back(st["dN"] * st["w_before"], xh, st["stats_before"], norm)
    u = yh * st["w_after"] + st["b_after"]
    t = d * st["scale"]
    dG = None
    if G is None:
        du, gated = t, d * u
    else:
        sig = 1 / (1 + torch.exp(-G))
        du, gated = t * sig, d * sig * u
        dG = t * u * sig * (1 - sig)
        if case["gate"] == "row":
            dG = dG.sum(1, keepdim=True)
    dY = _norm_back(du * st["w_after"], yh, st["stats_after"], norm)
    sums = [v.sum(0, dtype=torch.float64).float() for v in (du * yh, du, gated, st["dN"] * xh, st["dN"])]
    return {"dX": d, "dY": dY, "dG": dG, "sums": torch.stack(sums)}


# ----------------------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# ----------------------------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e in 64 bits, exactly (pow() is off by an ulp here and there)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _held(x):
    """The checkpoint of x: per 32 columns the least power of two 2^s, s >= -126, with max|x| < 127.5 * 2^s; x to the nearest
    multiple of it, ties to even."""
    out = []
    for c in range(0, x.shape[1], GROUP):
        v = x[:, c:c + GROUP].double()
        top = v.abs().max(dim=1, keepdim=True).values
        step = torch.full_like(top, 2.0 ** -126)
        m, e = torch.frexp(top / 127.5)                                            # top = m * 2^e * 127.5, 0.5 <= m < 1: s = e
        big = (top > 0) & (e > -126)
        step = torch.where(big, _two_to(e), step)
        step = torch.where(big & (top >= 127.5 * step), 2 * step, step)
        step = torch.where(big & (top < 127.5 * step / 2), step / 2, step)
        step = torch.where(torch.isfinite(top), step, torch.full_like(step, math.nan))
        out.append(torch.round(v / step) * step)
    return torch.cat(out, 1)


def _standing_for(ckpt):
    q, scale = ckpt
    n, D = q.shape
    row, col = torch.arange(n, device=q.device)[:, None], torch.arange(D, device=q.device)[None] // GROUP
    b = scale[((row // 8) * -(-D // GROUP) + col) * 8 + row % 8].to(torch.int64)
    return torch.where(b == 255, math.nan, q.double() * _two_to(b - 127))


def _moments(x, norm):
    m = torch.zeros_like(x[:, :1]) if norm == "rms" else x.mean(1, keepdim=True)
    return m, ((x - m).square().mean(1, keepdim=True) + EPS).rsqrt()


def exact(case, seed):
    st = prepare(case, seed)
    kind, norm = case["kind"], case.get("norm")
    if kind == "ckpt":
        return _held(st["X"])
    if kind == "wgrad":
        out = torch.zeros(case["D"], case["F"], dtype=torch.float64, device="cuda")
        A = _standing_for(st["A"])
        for r in range(0, case["n"], 1 << 17):
            out += torch.mm(A[r:r + (1 << 17)].t(), st["dZ"][r:r + (1 << 17)].double())
        return out
    wa, ba, sc, wb, bb = (st[k].double() for k in ("w_after", "b_after", "scale", "w_before", "b_before"))

    def told(m, r):
        return r[:, 0] if norm == "rms" else torch.cat((m, r), 1)

    if kind == "block_fwd":
        Y = st["Y"].double()
        m, r = _moments(Y, norm)
        sig = 1.0 if st["G"] is None else torch.sigmoid(st["G"].double())
        X_out = st["X"].double() + sc * sig * ((Y - m) * r * wa + ba)
        m2, r2 = _moments(X_out, norm)
        out = {"X_out": X_out, "N": (X_out - m2) * r2 * wb + bb, "stats_after": told(m, r), "stats_before": told(m2, r2)}
        if case["bits"] == 8:
            out["x8"], out["y8"] = _held(X_out), _held(Y)
            if case["gate"] == "full":
                out["g8"] = _held(st["G"])
        return out

    def given(name, ckpt):
        return st[name].double() if st[ckpt] is None else _standing_for(st[ckpt])

    def kept(stats):
        s = stats.double()
        return (0.0, s[:, None]) if norm == "rms" else (s[:, :1], s[:, 1:])

    def through(g, xh, r):
        """Gradient of the row's input: r * (g less its projections on the row of ones (layer) and on xh), both over D entries."""
        D = case["D"]
        along = torch.linalg.vecdot(g, xh, dim=1)[:, None] / D
        return r * (g - along * xh - (0.0 if norm == "rms" else g.sum(1, keepdim=True) / D))

    (m1, r1), (m2, r2) = kept(st["stats_before"]), kept(st["stats_after"])
    xh, yh = (given("X", "x8") - m1) * r1, (given("Y", "y8") - m2) * r2
    dN = st["dN"].double()
    d = st["dX_out"].double() + through(wb * dN, xh, r1)
    gate = torch.ones_like(d[:, :1]) if case["gate"] == "none" else torch.sigmoid(given("G", "g8"))
    u = wa * yh + ba
    dG = d * sc * u * gate * (1 - gate)
    if case["gate"] != "full":
        dG = dG.sum(1, keepdim=True) if case["gate"] == "row" else None
    sums = torch.stack([(d * sc * gate * yh).sum(0), (d * sc * gate).sum(0), (d * gate * u).sum(0), (dN * xh).sum(0), dN.sum(0)])
    return {"dX": d, "dY": through(d * sc * gate * wa, yh, r2), "dG": dG, "sums": sums}


# ----------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------------------------
def work(case):
    n, D, kind = case["n"], case["D"], case["kind"]
    e, held = n * D, n * D + n * -(-D // GROUP)
    if kind == "ckpt":
        return {"bytes": 8 * e + 2 * held, "flops": 4 * e}
    if kind == "wgrad":
        return {"bytes": held + 4 * n * case["F"] + 4 * D * case["F"], "flops": 2 * e * case["F"]}
    gate = {"none": 0, "row": 4 * n, "full": 4 * e}[case["gate"]]
    stats = 2 * n * (4 if case["norm"] == "rms" else 8)
    tensors = 3 if case["gate"] == "full" else 2
    if kind == "block_fwd":
        back = tensors * (2 * held + 2 * e) if case["bits"] == 8 else 0             # written, read back, given as two bytes a value
        return {"bytes": 16 * e + gate + stats + 20 * D + back, "flops": 20 * e}
    read = tensors * held + (gate if case["gate"] == "row" else 0) if case["bits"] == 8 else 8 * e + gate
    return {"bytes": 16 * e + read + gate + stats + 40 * D, "flops": 40 * e}
