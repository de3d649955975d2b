"""albireo_matmul_w4 against the product in 64 bits.

Where the rows are small integers and the scales powers of two, every partial sum in any order is exact in
fp32 (below 2^24 of the smallest unit), so those results are compared bit for bit.  For real-valued inputs
the error of an fp32 sum in any order is at most (number of dependent additions) * 2^-24 * sum of the
magnitudes.  A weight reaches the sums as a value of magnitude at most 31 scales (its 4 bits and an offset of
16) with the offset taken off again, at most 24 + 8 more for zero points other than 8; the dependent
additions are at most K (one column after another).  Their errors are independent, so the bound taken is the
square root of K times 4 instead of K.
"""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _weights(rng, N, K, G, zeros, exact, scale_dtype, pad=0):
    import torch

    import paper_2606_01927_amd as alb

    q = rng.integers(0, 16, size=(N, K), dtype=np.uint8)
    packed = q[:, 0::2] | (q[:, 1::2] << 4)
    s = 2.0 ** rng.integers(-2, 1, size=(N, K // G)) if exact else rng.uniform(0.002, 0.02, size=(N, K // G))
    st = torch.from_numpy(s).to(scale_dtype)
    z = rng.integers(0, 16, size=(N, K // G), dtype=np.uint8) if zeros else None

    def place(a, dt):  # rows of a longer stride, from an odd address
        a = torch.as_tensor(a)
        if not pad:
            return a.to("cuda")
        buf = torch.zeros(pad + a.shape[0] * (a.shape[1] + pad), dtype=dt, device="cuda")
        v = buf[pad:].as_strided(a.shape, (a.shape[1] + pad, 1))
        v.copy_(a)
        return v

    w = alb.W4Weight(place(packed, torch.uint8), place(st, scale_dtype), place(z, torch.uint8) if zeros else None)
    dense = (q.astype(np.float64) - (np.repeat(z, G, 1) if zeros else 8.0)) * np.repeat(st.double().numpy(), G, 1)
    return w, dense, np.repeat(st.double().numpy(), G, 1)


def _rows_in(rng, B, K, i8, exact):
    import torch

    if i8:
        x = rng.integers(-12, 13, size=(B, K)) if exact else rng.integers(-127, 128, size=(B, K))
        sc = np.ones(B) if exact else rng.uniform(0.01, 0.05, B)
        return torch.from_numpy(x.astype(np.int8)).cuda(), torch.from_numpy(sc.astype(np.float32)).cuda()
    x = rng.integers(-8, 9, size=(B, K)).astype(np.float32) if exact else rng.normal(0, 1, (B, K)).astype(np.float32)
    return torch.from_numpy(x).to(torch.bfloat16).cuda(), None


def _dense_x(x, sc):
    d = x.double().cpu().numpy()
    return d if sc is None else d * sc.double().cpu().numpy()[:, None]


SHAPES = [(1, 1, 32, 32), (1, 17, 64, 32), (3, 16, 128, 128), (1, 1000, 512, 128), (2, 63, 96, 32), (15, 129, 160, 32),
          (16, 64, 256, 64), (17, 65, 320, 64), (31, 200, 640, 128), (33, 257, 1024, 128), (64, 128, 512, 64),
          (65, 130, 384, 128), (100, 1001, 256, 128), (128, 333, 2048, 128), (129, 48, 128, 32), (257, 100, 256, 64),
          (1, 5000, 2080, 32), (5, 3, 4096, 128), (300, 513, 1152, 128)]


@pytest.mark.parametrize("B,N,K,G", SHAPES)
@pytest.mark.parametrize("i8", [False, True])
def test_exact_products(B, N, K, G, i8):
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(B * 7919 + N * 31 + K + i8)
    for zeros, sdt in ((False, torch.bfloat16), (True, torch.float32), (True, torch.bfloat16), (False, torch.float32)):
        w, dense, _ = _weights(rng, N, K, G, zeros, True, sdt)
        x, sc = _rows_in(rng, B, K, i8, True)
        want = _dense_x(x, sc) @ dense.T
        got = alb.matmul_w4(x, w, x_scale=sc)
        assert got.shape == (B, N) and got.dtype == torch.float32
        assert np.array_equal(got.double().cpu().numpy(), want), (zeros, sdt)
        gb = alb.matmul_w4(x, w, x_scale=sc, out_dtype=torch.bfloat16)
        assert torch.equal(gb, torch.from_numpy(want).to(torch.bfloat16).cuda()) or \
            torch.equal(gb, torch.from_numpy(want).float().to(torch.bfloat16).cuda())


@pytest.mark.parametrize("B,N,K,G", [(1, 777, 4096, 128), (8, 500, 1024, 32), (40, 300, 2048, 64), (200, 260, 8192, 128)])
@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("zeros", [False, True])
def test_real_values(B, N, K, G, i8, zeros):
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(B + N + K + i8)
    w, dense, s = _weights(rng, N, K, G, zeros, False, torch.bfloat16)
    x, sc = _rows_in(rng, B, K, i8, False)
    xd = _dense_x(x, sc)
    want = xd @ dense.T
    mag = 64.0 * np.abs(xd) @ s.T if not i8 else np.abs(xd) @ np.abs(dense).T
    tol = 4 * np.sqrt(K) * 2.0 ** -24 * mag
    got = alb.matmul_w4(x, w, x_scale=sc).double().cpu().numpy()
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    gb = alb.matmul_w4(x, w, x_scale=sc, out_dtype=torch.bfloat16).double().cpu().numpy()
    assert (np.abs(gb - want) <= tol * 1.01 + 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("B,N,K", [(3, 70, 256), (20, 33, 128), (70, 65, 640)])
def test_strides_alignment_and_guards(B, N, K, i8):
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(K + i8)
    w, dense, _ = _weights(rng, N, K, 32, True, True, torch.bfloat16, pad=3)
    x, sc = _rows_in(rng, B, K, i8, True)
    xb = torch.zeros(5 + B * (K + 7), dtype=x.dtype, device="cuda")
    xv = xb[5:].as_strided((B, K), (K + 7, 1))
    xv.copy_(x)
    for dt in (torch.float32, torch.bfloat16):
        buf = torch.full((9 + B * (N + 5) + 64,), 3.0, dtype=dt, device="cuda")
        out = buf[9:].as_strided((B, N), (N + 5, 1))
        assert alb.matmul_w4(xv, w, x_scale=sc, out=out) is out
        want = torch.from_numpy(_dense_x(x, sc) @ dense.T).to(dt)
        assert torch.equal(out.cpu(), want)
        out.fill_(3.0)
        assert (buf == 3.0).all()


def test_non_finite_rows_stay_apart():
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(5)
    w, dense, _ = _weights(rng, 100, 256, 128, False, True, torch.float32)
    x, _ = _rows_in(rng, 6, 256, False, True)
    x[1, 7] = float("nan")
    x[4, 200] = float("inf")
    got = alb.matmul_w4(x, w).double().cpu().numpy()
    want = x.double().cpu().numpy() @ dense.T
    for b in (0, 2, 3, 5):
        assert np.array_equal(got[b], want[b])
    for b in (1, 4):
        assert not np.isfinite(got[b][dense[:, 7 if b == 1 else 200] != 0]).any()
    xi, sc = _rows_in(rng, 3, 256, True, True)
    sc[1] = float("nan")
    got = alb.matmul_w4(xi, w, x_scale=sc)
    assert torch.isnan(got[1]).all() and torch.isfinite(got[0]).all() and torch.isfinite(got[2]).all()


def test_rows_past_32_bit_offsets():
    """A weight row range that starts past 2^31 bytes of its array: a long stride between the rows."""
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(11)
    N, K, G = 40, 256, 128
    w, dense, _ = _weights(rng, N, K, G, False, True, torch.bfloat16)
    stride = 1 << 27  # 40 rows over 5 GiB
    buf = torch.empty(N * stride, dtype=torch.uint8, device="cuda")
    far = buf.as_strided((N, K // 2), (stride, 1))
    far.copy_(w.q)
    for i8 in (False, True):
        x, sc = _rows_in(rng, 4, K, i8, True)
        got = alb.matmul_w4(x, alb.W4Weight(far, w.scales), x_scale=sc)
        assert np.array_equal(got.double().cpu().numpy(), _dense_x(x, sc) @ dense.T)


def test_repeatable_on_another_stream_and_empty():
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(12)
    w, _, _ = _weights(rng, 3000, 1024, 128, True, False, torch.bfloat16)
    for B in (1, 20, 150):
        for i8 in (False, True):
            x, sc = _rows_in(rng, B, 1024, i8, False)
            a = alb.matmul_w4(x, w, x_scale=sc)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                b = alb.matmul_w4(x, w, x_scale=sc)
            s.synchronize()
            assert torch.equal(a, b)
    assert alb.matmul_w4(torch.empty((0, 1024), dtype=torch.bfloat16, device="cuda"), w).shape == (0, 3000)


@pytest.mark.parametrize("K", [384, 512, 640, 896, 1152])
@pytest.mark.parametrize("B,N", [(64, 9001), (66, 49300)])
def test_groups_that_end_inside_a_load_of_scales(B, N, K):
    """8-bit rows and groups of 128 in weights wide enough for whole rounds of workgroups: 3 to 9 groups a row."""
    import torch

    import paper_2606_01927_amd as alb

    rng = np.random.default_rng(B + N + K)
    for zeros, sdt, pad in ((False, torch.bfloat16, 0), (True, torch.float32, 1), (True, torch.bfloat16, 0), (False, torch.float32, 1)):
        w, dense, _ = _weights(rng, N, K, 128, zeros, True, sdt, pad if sdt == torch.float32 else 0)
        x, sc = _rows_in(rng, B, K, True, True)
        got = alb.matmul_w4(x, w, x_scale=sc).double().cpu().numpy()
        assert np.array_equal(got, _dense_x(x, sc) @ dense.T), (zeros, sdt, pad)
