"""What may lie where: outputs take the place of tensors of their own shape; a gate of one column is no room for a tensor of D, nor the other way
round.  Refused on the host: nothing is launched, no GPU needed."""
import ctypes

import paper_2508_16769_amd as P
from paper_2508_16769_amd.binding import dr_block, dr_block_grads, dr_block_saved

A = [4096 * (i + 1) for i in range(16)]           # addresses that nothing reads
ref = ctypes.byref


def block(gate):
    return dr_block(P.DR_ROWNORM_RMS, gate, 1e-5, None, None, None, None, None)


def test_forward():
    lib = P.load()

    def call(gate, G, X_out, N, n=4, D=8):
        return lib.dr_block_fwd(ref(block(gate)), n, D, A[0], A[1], G, X_out, N, None, None)
    for X_out, N in ((A[2], A[4]), (A[3], A[2])):
        assert call(1, A[2], X_out, N) == P.DR_ERR_INVALID_ARG
        assert "one column" in P.dr_last_error()
    assert call(1, A[2], A[2], A[3], n=0) == P.DR_OK


def test_backward():
    lib = P.load()
    dXo, dN, Xo, Y, G, stats, ws = A[:7]
    saved = dr_block_saved(stats, stats)

    def call(gate, dX, dY, dG, D=8):
        g = dr_block_grads(dX, dY, dG)
        return lib.dr_block_bwd(ref(block(gate)), 4, D, dXo, dN, Xo, Y, G, ref(saved), ref(g), ws, 1 << 24, None)
    for dX, dY, dG in ((G, A[8], None), (A[8], G, None), (None, None, dXo), (None, None, dN), (None, None, Xo), (None, None, Y)):
        assert call(1, dX, dY, dG) == P.DR_ERR_INVALID_ARG, (dX, dY, dG)
        assert "one column" in P.dr_last_error()
