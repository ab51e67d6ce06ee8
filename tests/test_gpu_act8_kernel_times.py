"""Kernel times of the layer with its messages in 8 bits: every launch of a pass is among them, packing too."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev, random_csr

pytestmark = pytest.mark.gpu

FORWARD = ("dr_topk.cell", "dr_topk.net", "dr_spmm_fwd.near", "dr_spmm_fwd.pins", "dr_spmm_fwd.pinned", "proj.cell+merge", "proj.pins")


def test_forward_launches():
    rng = np.random.default_rng(0)
    Nc, Nn, D = 3000, 2000, 64
    rel = [P.Csr(m, n, *(dev(a) for a in random_csr(rng, m, n, 4, dup=True))) for m, n in ((Nc, Nc), (Nn, Nc), (Nc, Nn))]
    layer = P.HeteroConv(*rel, D, 16, 16)
    f = lambda *s: dev(rng.standard_normal(s).astype(np.float32))                  # noqa: E731
    X, W = (f(Nc, D), f(Nn, D)), {n: f(D, D) for n in P.WEIGHT_NAMES}
    Y = torch.empty(Nc, D, device="cuda"), torch.empty(Nn, D, device="cuda")
    plain, eight = layer.alloc_saved(), layer.alloc_saved8()
    layer.heteroconv_profile(True)
    for passes in (1, 3):
        layer.heteroconv_kernel_times()
        for _ in range(passes):
            layer.heteroconv_fwd_act8(*X, W, *Y, eight)
        t = layer.heteroconv_kernel_times()
        assert {n for n, (_, launches) in t.items() if launches} == {*FORWARD, "dr_act8_pack.messages"}
        assert all(t[n][1] == passes and t[n][0] > 0 for n in (*FORWARD, "dr_act8_pack.messages"))
    layer.heteroconv_fwd(*X, W, *Y, plain)
    t = layer.heteroconv_kernel_times()
    assert {n for n, (_, launches) in t.items() if launches} == set(FORWARD)
    layer.heteroconv_destroy()
