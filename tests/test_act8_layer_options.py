"""A layer's backward pass from checkpoints with the options that a stacked model sets: weight gradients alone, and several graphs at once.  The
options are not part of the C interface; the passes are called through the library's own symbol."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from paper_2508_16769_amd import binding as B

SYMBOL = "_ZN3drc19heteroconv_backwardEPKNS_8LayerBwdEiPK21dr_heteroconv_weightsP12ihipStream_tNS_15BackwardOptionsE"


class Options(ctypes.Structure):
    _fields_ = [("gate_inputs", ctypes.c_bool), ("skip_dx", ctypes.c_bool), ("dy_net_zero", ctypes.c_bool), ("saved8", ctypes.c_void_p)]


class LayerBwd(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("c", "dY_cell", "dY_net", "S", "dX_cell", "dX_net", "self_near", "neigh_near", "self_pins",
                                               "neigh_pins", "pinned")]


def _backward():
    f = getattr(P.load(), SYMBOL)
    f.argtypes = [ctypes.POINTER(LayerBwd), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, Options]
    f.restype = ctypes.c_int
    return f


def test_checkpoints_of_several_graphs_are_refused():
    saved8 = B.dr_heteroconv_saved8()
    opt = Options(False, False, False, ctypes.addressof(saved8))
    assert _backward()((LayerBwd * 2)(), 2, None, None, opt) == P.DR_ERR_INVALID_ARG
    assert "checkpoints" in P.dr_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [P.DR_OVERLAP_ON, P.DR_OVERLAP_OFF])
@pytest.mark.parametrize("D,Nc,Nn", [(64, 700, 500), (128, 5000, 3000)])
def test_weight_gradients_alone_are_those_of_the_checkpoints(D, Nc, Nn, mode):
    from gpu_util import dev, random_csr
    rng = np.random.default_rng(D)
    rel = [P.Csr(m, n, *(dev(a) for a in random_csr(rng, m, n, 4, dup=True))) for m, n in ((Nc, Nc), (Nn, Nc), (Nc, Nn))]
    layer = P.HeteroConv(*rel, D, 16, 16)
    layer.heteroconv_set_overlap(mode)
    f = lambda *s: dev(rng.standard_normal(s).astype(np.float32))                  # noqa: E731
    W = {n: f(D, D) for n in P.WEIGHT_NAMES}
    X, dY, saved = (f(Nc, D), f(Nn, D)), (f(Nc, D), f(Nn, D)), layer.alloc_saved8()
    layer.heteroconv_fwd_act8(*X, W, torch.empty(Nc, D, device="cuda"), torch.empty(Nn, D, device="cuda"), saved)
    dX = torch.empty(Nc, D, device="cuda"), torch.empty(Nn, D, device="cuda")
    want, got = ({n: torch.full((D, D), float("nan"), device="cuda") for n in P.WEIGHT_NAMES} for _ in range(2))
    layer.heteroconv_bwd_act8(*dY, W, saved, *dX, want)
    # what a pass of the same context with fp32 messages is given, its messages anywhere but where the checkpoints' were
    fp32 = {**layer.alloc_saved(), **{n: t for n, t in saved.items() if not n.startswith("H_")}}
    for n in ("H_near", "H_pins", "H_pinned"):
        fp32[n].fill_(float("nan"))
    s8, s32, w = layer._saved8(saved), layer._saved(fp32), layer._weights(W)
    g = LayerBwd(layer._ctx.value, dY[0].data_ptr(), dY[1].data_ptr(), ctypes.addressof(s32), None, None,
                 *(got[n].data_ptr() for n in P.WEIGHT_NAMES))
    opt = Options(False, True, False, ctypes.addressof(s8))
    rc = _backward()(ctypes.byref(g), 1, ctypes.addressof(w), torch.cuda.current_stream().cuda_stream, opt)
    assert rc == P.DR_OK, P.dr_last_error()
    torch.cuda.synchronize()
    # the same products, each exact to 2^-24, in sums of which every addition rounds by at most 2^-24 of its result, in two orders; the terms of
    # an entry weigh no more than the norms of its two columns multiplied
    for n, A, q in (("self_near", X[0], 0), ("neigh_near", "H_near", 0), ("self_pins", X[1], 1), ("neigh_pins", "H_pins", 1), ("pinned", "H_pinned", 0)):
        if isinstance(A, str):
            v = torch.empty(dY[q].shape, device="cuda")
            P.dr_act8_unpack(saved[A], v)
            A = v
        weigh = A.double().norm(dim=0)[:, None] * dY[q].double().norm(dim=0)[None]
        assert ((want[n].double() - got[n].double()).abs() <= 2 * len(A) * 2.0 ** -23 * weigh).all(), n
    layer.heteroconv_destroy()
