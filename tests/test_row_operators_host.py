"""What the row operators (8-bit checkpoints, residual block) refuse, on the host: nothing is launched, no GPU needed."""
import ctypes

import pytest

import paper_2508_16769_amd as P
from paper_2508_16769_amd.binding import dr_act8, dr_block, dr_block_grads, dr_block_saved

A, ODD, BIG = 4096, 4098, 1 << 24                 # addresses that nothing reads; room enough for any workspace


def ref(x):
    return ctypes.byref(x)


def ck(q=A, scale=A):
    return dr_act8(q, scale)


def test_sizes_of_scales_and_workspaces():
    assert P.DR_ACT8_GROUP == 32
    assert [P.dr_act8_scale_bytes(n, D) for n, D in ((0, 5), (1, 1), (8, 32), (9, 33), (9, 64))] == [0, 8, 8, 32, 32]
    assert P.dr_act8_scale_bytes(-1, 5) == 0 and P.dr_act8_scale_bytes(5, 0) == 0
    assert P.dr_block_bwd_workspace_bytes(0, 7) >= 1 and P.dr_block_bwd_workspace_bytes(-1, 7) == 0
    assert P.dr_act8_wgrad_workspace_bytes(0, 3, 5) >= 1 and P.dr_act8_wgrad_workspace_bytes(4, 0, 5) == 0
    # bounded however many rows there are: partial sums of as many workgroups as the chip has room for
    assert P.dr_block_bwd_workspace_bytes(1 << 30, 1024) <= 64 << 20
    assert P.dr_act8_wgrad_workspace_bytes(1 << 30, 1024, 1024) <= 2 << 30


@pytest.mark.parametrize("name", ["dr_act8_pack", "dr_act8_unpack"])
def test_checkpoint_refusals(name):
    lib = P.load()

    def call(x=A, n=4, D=8, c=None, null=False):
        c = ck() if c is None else c
        p = None if null else ref(c)
        return lib.dr_act8_pack(x, n, D, p, None) if name == "dr_act8_pack" else lib.dr_act8_unpack(p, n, D, x, None)
    for kw in (dict(x=None), dict(x=ODD), dict(n=-1), dict(n=1 << 31), dict(D=0), dict(null=True), dict(c=ck(q=None)), dict(c=ck(scale=None)),
               dict(c=ck(scale=A + 4))):
        assert call(**kw) == P.DR_ERR_INVALID_ARG, kw
        assert name in P.dr_last_error()
    assert call(D=1025) == P.DR_ERR_UNSUPPORTED
    assert call(n=0, x=None, null=True) == P.DR_OK


def test_weight_gradient_refusals():
    lib = P.load()

    def call(c=None, null=False, n=4, D=8, dZ=A, F=8, dW=A, ws=A, wsb=BIG):
        c = ck() if c is None else c
        return lib.dr_act8_wgrad(None if null else ref(c), n, D, dZ, F, dW, 0, ws, wsb, None)
    for kw in (dict(null=True), dict(c=ck(q=None)), dict(c=ck(scale=A + 2)), dict(n=-1), dict(n=1 << 31), dict(D=0), dict(F=0), dict(dZ=None),
               dict(dZ=ODD), dict(dW=None), dict(dW=ODD), dict(ws=None), dict(ws=A + 64)):
        assert call(**kw) == P.DR_ERR_INVALID_ARG, kw
    assert call(D=1025) == P.DR_ERR_UNSUPPORTED and call(F=1025) == P.DR_ERR_UNSUPPORTED
    assert call(wsb=P.dr_act8_wgrad_workspace_bytes(4, 8, 8) - 1) == P.DR_ERR_WORKSPACE


def block(norm=0, gate=0, eps=1e-5, w=A):
    return dr_block(norm, gate, eps, w, A, A, A, A)


def saved(sa=A, sb=A, x=None, y=None, g=None):
    return dr_block_saved(sa, sb, x or dr_act8(), y or dr_act8(), g or dr_act8())


def test_block_forward_refusals():
    lib = P.load()

    def call(b=None, n=4, D=8, X=A, Y=A, G=None, Xo=A + 16, N=A + 32, s=None, null=False):
        b = block() if b is None else b
        s = saved() if s is None else s
        return lib.dr_block_fwd(None if null else ref(b), n, D, X, Y, G, Xo, N, ref(s), None)
    bad = (dict(null=True), dict(b=block(norm=2)), dict(b=block(eps=0.0)), dict(b=block(eps=-1.0)), dict(b=block(eps=1e-40)), dict(b=block(eps=float("inf"))), dict(b=block(eps=float("nan"))),
           dict(b=block(gate=3), G=A), dict(b=block(gate=8)), dict(b=block(gate=0), G=A), dict(b=block(w=ODD)), dict(n=-1), dict(n=1 << 31),
           dict(D=0), dict(X=None), dict(X=ODD), dict(Y=ODD), dict(N=ODD), dict(Xo=None), dict(Y=None), dict(Y=None, Xo=None, N=None),
           dict(Xo=A + 32), dict(N=None), dict(Y=None, Xo=None), dict(Y=None, Xo=None, s=saved(sa=None, y=ck())),
           dict(b=block(gate=1), G=A, s=saved(g=ck())), dict(s=saved(x=ck(scale=None))), dict(s=saved(y=ck(scale=A + 1))),
           dict(s=saved(sa=ODD)))
    for kw in bad:
        assert call(**kw) == P.DR_ERR_INVALID_ARG, kw
        assert "dr_block_fwd" in P.dr_last_error()
    assert call(D=2000) == P.DR_ERR_UNSUPPORTED
    assert call(n=0, X=None, Y=None) == P.DR_OK


def test_block_backward_refusals():
    lib = P.load()

    def call(b=None, n=4, D=8, dXo=A, dN=A, Xo=A, Y=A, G=None, s=None, g=None, ws=A, wsb=BIG, null=False, no_grads=False):
        b = block() if b is None else b
        s = saved() if s is None else s
        g = dr_block_grads(A, A + 16, None, A, A, A, A, A) if g is None else g
        return lib.dr_block_bwd(None if null else ref(b), n, D, dXo, dN, Xo, Y, G, ref(s), None if no_grads else ref(g), ws, wsb, None)
    only_front = dr_block_grads(A, None, None, None, None, None, A, A)
    bad = (dict(null=True), dict(no_grads=True), dict(n=-1), dict(D=0), dict(dXo=None, dN=None), dict(Xo=None), dict(s=saved(x=ck())),
           dict(s=saved(y=ck())), dict(b=block(gate=8), G=A, s=saved(g=ck())), dict(s=saved(sa=None)), dict(s=saved(sb=None)),
           dict(b=block(gate=1)), dict(G=A), dict(b=block(gate=1), s=saved(g=ck())), dict(Y=None), dict(Y=None, G=A, b=block(gate=1), g=only_front),
           dict(g=dr_block_grads(A, A, None, A, A, A, A, A)), dict(b=block(gate=8), G=A, g=dr_block_grads(A, A + 16, A, A, A, A, A, A)),
           dict(b=block(gate=8), G=A, g=dr_block_grads(A, A + 16, A + 16, A, A, A, A, A)), dict(g=dr_block_grads(A, A + 16, A, A, A, A, A, A)), dict(dXo=ODD),
           dict(g=dr_block_grads(A, A + 16, None, ODD, A, A, A, A)), dict(ws=None), dict(ws=A + 16))
    for kw in bad:
        assert call(**kw) == P.DR_ERR_INVALID_ARG, kw
        assert "dr_block_bwd" in P.dr_last_error()
    assert call(D=1025) == P.DR_ERR_UNSUPPORTED
    assert call(wsb=P.dr_block_bwd_workspace_bytes(4, 8) - 1) == P.DR_ERR_WORKSPACE
