"""8-bit activation checkpoints: codes and scales bit for bit against the fp64 oracle, and weight gradients from them."""
import numpy as np
import pytest
import torch

import paper_2508_16769_amd as P
from gpu_util import dev, say
from oracle import block as ob

pytestmark = pytest.mark.gpu

WIDTHS = [1, 3, 4, 8, 13, 16, 31, 32, 33, 36, 64, 77, 96, 100, 128, 130, 256, 260, 500, 512, 1000, 1021, 1024]


def _matrix(rng, n, D):
    """Rows of very different size, zeros, values at code and scale borders, and both ends of the fp32 range."""
    x = rng.standard_normal((n, D)).astype(np.float32) * np.exp(3 * rng.standard_normal((n, 1))).astype(np.float32)
    x[rng.random((n, D)) < 0.1] = 0
    special = [0.0, -0.0, 127.5, -127.5, np.nextafter(np.float32(127.5), np.float32(0)), 63.75, 0.5, 1.5, 2.0 ** -126, -(2.0 ** -127), 2.0 ** -149,
               np.finfo(np.float32).max, -np.finfo(np.float32).max, 2.0 ** 127 * 1.99, 1e-38]
    for i in range(n // 3):
        x[i, rng.integers(0, D)] = special[i % len(special)]
    if n > 4:
        x[n // 2] = 0
        x[n - 2] *= np.float32(2.0 ** -130)
    return x


def _pack(x):
    n, D = x.shape
    q, scale = P.alloc_act8(n, D)
    q.fill_(85)
    scale.fill_(77)
    P.dr_act8_pack(dev(x), (q, scale))
    return q, scale


@pytest.mark.parametrize("D", WIDTHS)
def test_codes_and_values(D):
    rng = np.random.default_rng(D)
    for n in (1, 2, 7, 8, 9, 65, 700):
        say(f"act8 n={n} D={D}")
        x = _matrix(rng, n, D)
        q, scale = _pack(x)
        want_q, want_s = ob.act8_pack(x)
        assert np.array_equal(q.cpu().numpy(), want_q), (n, D)
        assert np.array_equal(scale.cpu().numpy(), want_s), (n, D)
        out = torch.full((n, D), -3.0, device="cuda")
        P.dr_act8_unpack((q, scale), out)
        v = out.cpu().numpy()
        assert np.array_equal(v.astype(np.float64), ob.act8_values(want_q, want_s)), (n, D)
        assert np.array_equal(v, torch.from_numpy(v).to(torch.bfloat16).float().numpy())        # exact in bf16
        # packing what a checkpoint stands for gives the same values again
        q2, s2 = _pack(v)
        P.dr_act8_unpack((q2, s2), out)
        assert np.array_equal(out.cpu().numpy(), v)


def test_groups_that_are_not_finite():
    x = np.ones((20, 100), np.float32)
    for i, bad in enumerate((np.inf, -np.inf, np.nan, -np.nan)):
        x[4 * i, 30 * i] = bad
    q, scale = _pack(x)
    out = torch.empty(20, 100, device="cuda")
    P.dr_act8_unpack((q, scale), out)
    v = out.cpu().numpy()
    for i in range(4):
        g = 30 * i // 32
        assert np.isnan(v[4 * i, 32 * g:32 * g + 32]).all()
        assert (np.delete(v[4 * i], np.s_[32 * g:32 * g + 32]) == 1).all()
    assert (np.delete(v, [0, 4, 8, 12], axis=0) == 1).all()
    assert not q.cpu().numpy()[0, :32].any()


def test_rows_at_any_alignment():
    """Rows in the middle of a larger buffer, four bytes off every wider alignment."""
    rng = np.random.default_rng(0)
    for D in (32, 64, 128, 512):
        x = _matrix(rng, 50, D)
        room = torch.zeros(50 * D + 1, device="cuda")
        room[1:] = dev(x).view(-1)
        qroom = torch.zeros(50 * D + 3, dtype=torch.int8, device="cuda")
        q, scale = qroom[3:].view(50, D), P.alloc_act8(50, D)[1]
        P.dr_act8_pack(room[1:].view(50, D), (q, scale))
        want_q, want_s = ob.act8_pack(x)
        assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(scale.cpu().numpy(), want_s)
        out = torch.zeros(50 * D + 1, device="cuda")
        P.dr_act8_unpack((q, scale), out[1:].view(50, D))
        assert np.array_equal(out[1:].cpu().numpy().reshape(50, D), ob.act8_values(want_q, want_s)) and out[0] == 0


def test_offsets_past_32_bits():
    n, D = 2_200_000, 1024                       # 2.25e9 elements: more than 2^31 codes, 9 GB of fp32
    x = torch.zeros(n, D, device="cuda")
    rng = np.random.default_rng(5)
    tail = _matrix(rng, 11, D)
    x[-11:] = dev(tail)
    ck = P.alloc_act8(n, D)
    ck[0].fill_(1)
    P.dr_act8_pack(x, ck)
    first = (n - 11) // 8 * 8
    want_q, want_s = ob.act8_pack(np.concatenate((np.zeros((n - 11 - first, D), np.float32), tail)))
    assert np.array_equal(ck[0][first:].cpu().numpy(), want_q)
    assert np.array_equal(ck[1][first // 8 * 256:].cpu().numpy(), want_s)
    assert not ck[0][:-11].any()
    x.fill_(7.0)
    P.dr_act8_unpack(ck, x)
    assert np.array_equal(x[first:].cpu().numpy(), ob.act8_values(want_q, want_s).astype(np.float32))
    assert not x[:-11].any()


# ---- weight gradients ----------------------------------------------------------------------------------------------
def _wgrad(q, scale, dZ, dW=None, accumulate=False):
    n, D = q.shape
    F = dZ.shape[1]
    out = torch.full((D, F), float("nan"), device="cuda") if dW is None else dW
    ws = torch.full((P.dr_act8_wgrad_workspace_bytes(n, D, F),), 255, dtype=torch.uint8, device="cuda")
    P.dr_act8_wgrad((q, scale), dZ, out, ws, accumulate)
    return out


def _check(got, q, scale, dZ, base=None):
    """n products, each exact to 2^-24, in sums of which every addition rounds by at most 2^-24 of its result."""
    A, B = ob.act8_values(q.cpu().numpy(), scale.cpu().numpy()), dZ.cpu().numpy().astype(np.float64)
    want, l1 = A.T @ B, np.abs(A).T @ np.abs(B)
    if base is not None:
        want, l1 = want + base, l1 + np.abs(base)
    n = max(A.shape[0], 4)
    err = np.abs(got.cpu().numpy().astype(np.float64) - want)
    assert np.all(err <= n * 2.0 ** -23 * l1), float((err / np.maximum(l1, 1e-300)).max())
    # roundings do not all fall to one side: the sums as a whole are off by what sqrt(n) of them make, with a factor of 8
    if A.shape[0] >= 64 and base is None:
        assert np.linalg.norm(err) <= 8 * 2.0 ** -24 * np.sqrt(A.shape[0]) * np.linalg.norm(np.sqrt(np.square(A).T @ np.square(B)))


@pytest.mark.parametrize("D,F", [(1, 1), (3, 5), (16, 16), (31, 33), (32, 32), (64, 64), (64, 1), (1, 64), (77, 100), (96, 200), (128, 128),
                                 (128, 130), (129, 127), (260, 36), (300, 257), (1024, 1), (1000, 1024)])
def test_weight_gradients(D, F):
    rng = np.random.default_rng(D * 2000 + F)
    for n in (1, 7, 31, 32, 33, 64, 129, 1000, 5003):
        if n * D * F > 600e6:
            continue
        say(f"wgrad n={n} D={D} F={F}")
        x = (rng.standard_normal((n, D)) * np.exp(rng.standard_normal((n, 1)))).astype(np.float32)
        dZ = dev((0.1 * rng.standard_normal((n, F)) * np.exp(rng.standard_normal((n, 1)))).astype(np.float32))
        q, scale = _pack(x)
        got = _wgrad(q, scale, dZ)
        _check(got, q, scale, dZ)
        base = got.cpu().numpy().astype(np.float64) * 0.5
        again = _wgrad(q, scale, dZ, dev(base.astype(np.float32)), True)
        _check(again, q, scale, dZ, base.astype(np.float32).astype(np.float64))
        assert torch.equal(_wgrad(q, scale, dZ), got)                            # reproducible


def test_weight_gradients_of_no_rows():
    ck = P.alloc_act8(0, 40)
    dZ = torch.empty(0, 24, device="cuda")
    assert torch.equal(_wgrad(*ck, dZ), torch.zeros(40, 24, device="cuda"))
    base = torch.randn(40, 24, device="cuda")
    assert torch.equal(_wgrad(*ck, dZ, base.clone(), True), base)


def test_padding_bytes_are_not_read():
    """Scale bytes of the rows behind the last one may hold anything."""
    rng = np.random.default_rng(1)
    for n in (3, 41, 1001):
        q, scale = _pack(rng.standard_normal((n, 128)).astype(np.float32))
        dZ = dev(rng.standard_normal((n, 128)).astype(np.float32))
        want = _wgrad(q, scale, dZ)
        scale.view(-1, 4, 8)[-1, :, n % 8:] = 255
        assert torch.equal(_wgrad(q, scale, dZ), want)
        out = torch.empty(n, 128, device="cuda")
        P.dr_act8_unpack((q, scale), out)
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("D,F", [(96, 40), (128, 128)])
def test_weight_gradients_of_extreme_values(D, F):
    """Infinities and not-a-numbers stay in the entries they belong to; values at the ends of the fp32 range are exact."""
    rng = np.random.default_rng(2)
    n = 100
    x = rng.integers(1, 9, (n, D)).astype(np.float32)
    dZ = rng.standard_normal((n, F)).astype(np.float32)
    dZ[17, 3], dZ[40, 7], dZ[63, 11] = np.inf, -np.inf, np.nan
    x[80, 2] = np.nan                                          # columns 0 .. 31 of dW's rows
    q, scale = _pack(x)
    got = _wgrad(q, scale, dev(dZ)).cpu().numpy()
    assert np.isnan(got[:32]).all()
    assert (got[32:, 3] == np.inf).all() and (got[32:, 7] == -np.inf).all() and np.isnan(got[32:, 11]).all()
    rest = [c for c in range(F) if c not in (3, 7, 11)]
    A = ob.act8_values(q.cpu().numpy(), scale.cpu().numpy())[:, 32:]
    want, l1 = A.T @ dZ[:, rest].astype(np.float64), np.abs(A).T @ np.abs(dZ[:, rest]).astype(np.float64)
    assert np.all(np.abs(got[32:, rest] - want) <= n * 2.0 ** -23 * l1)
    # one row each: the largest and the smallest normal numbers
    for a, b in ((2.0 ** 100, 2.0 ** 27), (2.0 ** -60, 2.0 ** -60), (1.0, np.finfo(np.float32).max), (2.0 ** -126, 2.0 ** 120)):
        x = np.zeros((5, D), np.float32)
        x[2] = a
        z = np.zeros((5, F), np.float32)
        z[2] = b
        got = _wgrad(*_pack(x), dev(z)).cpu().numpy()
        assert (got == np.float32(np.float64(a) * b)).all(), (a, b, got[0, 0])


def test_long_sums():
    """As many rows as a design has cells: sums stay as exact as their partial sums allow."""
    n, D, F = 300_000, 64, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dZ = torch.randn(n, D, generator=g, device="cuda"), torch.randn(n, F, generator=g, device="cuda") + 0.5
    ck = P.alloc_act8(n, D)
    P.dr_act8_pack(x + 0.5, ck)
    got = _wgrad(*ck, dZ)
    v = torch.empty(n, D, device="cuda")
    P.dr_act8_unpack(ck, v)
    want = v.double().t() @ dZ.double()
    # sums of 0.25 per row on average: a workgroup's running sum rounds by 2^-24 of itself per chunk, far below 2^-20 of the whole
    assert ((got.double() - want).abs() <= 2.0 ** -20 * want.abs().max()).all()
