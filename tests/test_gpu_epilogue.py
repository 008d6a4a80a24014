"""The BF16 product with bias, activation and residual in its epilogue, the layer's gradients from a copy in 8 bits, and a
feed-forward block that uses the operators together.

Tolerances: the accumulator is within 1e-4 * T of the exact sum, T = sum |a||b| (see test_gpu_bf16.py); through an activation with slope at
most L between z and its neighbours that is 1e-4 * T * L; fast exponentials 64 * 2^-24; a rounding to bf16 2^-8."""
import numpy as np
import pytest
import torch

import around_ref as R
from paper_2509_25149_b200 import binding as B

pytestmark = pytest.mark.gpu
U, BF16 = 2.0 ** -24, 2.0 ** -8


def ints(shape, seed, lo, hi):
    return torch.randint(lo, hi + 1, shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def normal(shape, seed, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


# few rows (up to 32: one to eight shares of k, short last blocks and steps); one CTA pair, few tiles with shared contractions, 128- and
# 256-wide tiles, several rounds, 512-wide tiles (rows off 32 bytes)
SHAPES = [(1, 8, 8), (1, 136, 264), (3, 520, 72), (8, 256, 2048), (9, 72, 520), (16, 2048, 4104), (17, 264, 16384), (31, 40, 40),
          (32, 1048, 2056), (2, 20480, 264), (33, 1048, 2056), (40, 8, 8), (300, 24, 40), (40, 264, 128), (129, 1000, 200), (257, 520, 1088), (300, 2056, 64),
          (1000, 2504, 136), (2049, 2304, 72), (2305, 2600, 1032)]
SHAPES += [(1, 40, 33000), (13, 72, 33000), (21, 40, 33000), (4, 7144, 4104)]  # few rows, long contractions
# up to 128 rows: every width of tile with and without shares of k, short last tiles and k-blocks, one CTA and a full chip
SHAPES += [(3, 10248, 4104), (12, 5128, 4104), (16, 2056, 10248), (20, 2568, 2056), (32, 1000, 5320), (33, 8, 1024), (50, 19208, 72), (57, 1160, 1096),
           (64, 264, 16392), (64, 5000, 1032), (65, 392, 4104), (100, 2600, 4360), (128, 5128, 4104), (128, 8, 8200)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("keep", [None, "bf16", "8"])
@pytest.mark.parametrize("residual", [False, True])
def test_whole_numbers_are_exact(shape, keep, residual):
    """Sums of products of small whole numbers are exact, so every element of z, of its copy and of D is known to the bit."""
    M, N, K = shape
    a, b = ints((M, K), 1, -1, 1), ints((N, K), 2, -1, 1)
    if K > 64:
        a[:, 64:] *= (ints((M, K - 64), 7, 0, 7) == 0).to(a.dtype)  # (few enough that z stays small)
    bias, res = ints((N,), 3, -20, 20).float(), ints((M, N), 4, -60, 60)
    z64 = R.f64(a) @ R.f64(b).T + R.f64(bias)
    for act in ("none", "relu2"):
        A, a_ok = R.guarded(M, K, torch.bfloat16, K + 8, a.cuda())
        Bm, b_ok = R.guarded(N, K, torch.bfloat16, K + 16, b.cuda())
        D, d_ok = R.guarded(M, N, torch.bfloat16, N + 24)
        rd, r_ok = R.guarded(M, N, torch.bfloat16, N + 8, res.cuda()) if residual else (None, lambda: True)
        z, z_ok = R.guarded_copy(M, N) if keep == "8" else R.guarded(M, N, torch.bfloat16, N + 8) if keep else (None, lambda: True)
        B.nvfp4_gemm_bf16_epilogue(A, Bm, D, bias.cuda(), R.ACTS[act], rd, z)
        B.nvfp4_device_status()
        want = R.act64(z64, act) + (R.f64(res) if residual else 0)
        assert np.array_equal(R.f64(D), torch.from_numpy(want).to(torch.bfloat16).double().numpy()), act
        if keep == "8":
            codes, scales = R.copy8(z64)
            assert np.array_equal(z.scales.cpu().numpy(), scales)
            got = z.codes.cpu().numpy()
            assert np.array_equal(np.where(got == 128, 0, got), np.where(codes == 128, 0, codes))  # (the sign of a zero aside)
        elif keep:
            assert np.array_equal(R.f64(z), torch.from_numpy(z64).to(torch.bfloat16).double().numpy())
        assert a_ok() and b_ok() and d_ok() and r_ok() and z_ok()


def check(M, N, K, act, residual, keep, bias=True, std=1.0):
    a, b = normal((M, K), 11), normal((N, K), 12, std / K ** 0.5)
    bv, res = normal((N,), 13, 0.5, torch.float32) if bias else None, normal((M, N), 14) if residual else None
    D = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    z = B.alloc_tensor(M, N, format=B.FORMAT_MXFP8) if keep == "8" else torch.empty_like(D) if keep else None
    B.nvfp4_gemm_bf16_epilogue(a.cuda(), b.cuda(), D, bv.cuda() if bias else None, R.ACTS[act], res.cuda() if residual else None, z)
    B.nvfp4_device_status()
    z64 = R.f64(a) @ R.f64(b).T + (R.f64(bv) if bias else 0)
    off = 1e-4 * (np.abs(R.f64(a)) @ np.abs(R.f64(b)).T) + 2 * U * np.abs(z64)
    slope = 2 * np.abs(z64) + off if act == "relu2" else 1.2
    want = R.act64(z64, act)
    tol = off * slope + (8 * U if act in ("none", "relu2") else 64 * U) * np.abs(want)
    if residual:
        want = want + R.f64(res)
    R.assert_within(R.f64(D), want, tol + BF16 * (np.abs(want) + tol) + 1e-38, "D")
    if keep == "bf16":
        R.assert_within(R.f64(z), z64, off + BF16 * (np.abs(z64) + off), "z")
    if keep == "8":
        got = R.decode8(z.codes.cpu().numpy(), z.scales.cpu().numpy())
        top = np.repeat(np.abs(np.pad(np.abs(z64) + off, ((0, 0), (0, -N % 32))).reshape(M, -1, 32)).max(2), 32, axis=1)[:, :N]
        R.assert_within(got, z64, off + np.maximum(2.0 ** -4 * (np.abs(z64) + off), 2.0 ** -10 * top / 224), "z8")


@pytest.mark.parametrize("shape", [(1, 1024, 4096), (5, 264, 5120), (12, 5128, 1032), (32, 136, 8200), (264, 512, 4096), (1000, 2000, 3000), (1040, 3664, 904), (4096, 1024, 256)])
@pytest.mark.parametrize("act", sorted(R.ACTS))
def test_random_data(shape, act):
    check(*shape, act, True, "bf16")
    check(*shape, act, False, "8")
    check(*shape, act, True, None, bias=False, std=3.0)


@pytest.mark.parametrize("shape", [(10, 2568, 8200), (30, 2056, 2568), (48, 1032, 4104), (64, 520, 2056), (90, 392, 8200), (120, 2056, 4104)])
@pytest.mark.parametrize("act", sorted(R.ACTS))
def test_random_data_of_some_tens_of_rows(shape, act):
    check(*shape, act, True, "bf16")
    check(*shape, act, False, "8")
    check(*shape, act, True, None, bias=False, std=3.0)


def test_more_tiles_than_share_a_contraction():
    check(66, 19080, 4104, "silu", True, "bf16")


def test_residual_in_place():
    """D may be the residual: each element is read by the thread that writes it."""
    for M, N, K in [(5, 520, 264), (20, 2568, 2056), (40, 1032, 1096), (60, 19208, 72), (128, 2056, 4104), (300, 520, 264)]:
        a, b, res = ints((M, K), 21, -1, 1), ints((N, K), 22, -1, 1), ints((M, N), 23, -60, 60)
        D = res.cuda()
        B.nvfp4_gemm_bf16_epilogue(a.cuda(), b.cuda(), D, residual=D)
        B.nvfp4_device_status()
        want = R.f64(a) @ R.f64(b).T + R.f64(res)
        assert np.array_equal(R.f64(D), torch.from_numpy(want).to(torch.bfloat16).double().numpy()), (M, N, K)


@pytest.mark.parametrize("tile", [512, 640, 642, 644])
@pytest.mark.parametrize("keep", [None, "bf16", "8"])
def test_every_tile(tile, keep):
    B.nvfp4_set_gemm_tile_n(tile)
    try:
        check(300, 776, 1032, "gelu", True, keep)
    finally:
        B.nvfp4_set_gemm_tile_n(0)


def test_outputs_of_more_than_two_to_the_31_elements():
    M, N, K = 131080, 16392, 8
    a, b = ints((M, K), 61, -2, 2), ints((N, K), 62, -2, 2)
    res = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    rows = [0, 4, M // 2, M - 129, M - 1]
    res[rows] = 3
    z8 = B.alloc_tensor(M, N, format=B.FORMAT_MXFP8)
    B.nvfp4_gemm_bf16_epilogue(a.cuda(), b.cuda(), res, None, B.ACT_RELU2, res, z8)
    B.nvfp4_device_status()
    for r in rows:
        z = R.f64(a[r:r + 1]) @ R.f64(b).T
        want = torch.from_numpy(np.maximum(z, 0) ** 2 + 3).to(torch.bfloat16).double().numpy()
        assert np.array_equal(R.f64(res[r:r + 1]), want)
        assert np.array_equal(R.decode8(z8.codes[r:r + 1].cpu().numpy(), z8.scales[r:r + 1].cpu().numpy()), R.decode8(*R.copy8(z)))


def test_agrees_with_the_plain_product_bit_for_bit():
    for M, N, K in [(512, 1024, 1024), (2048, 2048, 512), (264, 512, 4096)]:
        a, b = normal((M, K), 21).cuda(), normal((N, K), 22).cuda()
        D, E = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        B.nvfp4_gemm_bf16(a, b, D)
        B.nvfp4_gemm_bf16_epilogue(a, b, E)
        assert torch.equal(D, E)


def test_residual_in_place_on_another_stream_in_a_graph():
    M, N, K = 520, 1032, 264
    a, b, bias, res = normal((M, K), 31).cuda(), normal((N, K), 32).cuda(), normal((N,), 33, 1.0, torch.float32).cuda(), normal((M, N), 34).cuda()
    want = torch.empty_like(res)
    B.nvfp4_gemm_bf16_epilogue(a, b, want, bias, B.ACT_SILU, res)
    D = res.clone()
    B.nvfp4_gemm_bf16_epilogue(a, b, D, bias, B.ACT_SILU, D)
    assert torch.equal(D, want)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        B.nvfp4_gemm_bf16_epilogue(a, b, D, bias, B.ACT_SILU, res)
    for _ in range(3):
        D.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(D, want)


# ---------------------------------------------------------------------------------- gradients of a layer from a copy ----
def exact_tolerance(T, contraction):
    """A tensor-core addition cuts off less than a unit in the last place of its sum, 2^-23 of it, and up to 64 of them (16 products each) make
    a share: 2^-17 T.  The shares are added rounded to nearest, 2^-24 each."""
    return (2.0 ** -17 + (contraction // 1024 + 2) * U) * T


@pytest.mark.parametrize("shape", [(8, 128, 136), (264, 520, 1048), (1000, 512, 2056), (520, 264, 264), (4104, 1032, 1544), (2056, 2600, 2312)])
def test_layer_gradients_from_a_copy(shape):
    M, N, K = shape
    dy, w, x = normal((M, N), 41, 1e-2).cuda(), normal((N, K), 42, 0.05).cuda(), normal((M, K), 43)
    x8 = R.copy_on_gpu(R.f64(x))
    dx, dw0 = torch.empty((M, K), dtype=torch.bfloat16, device="cuda"), normal((N, K), 44, 1.0, torch.float32).cuda()
    ws = torch.empty(B.nvfp4_linear_bf16_bwd8_workspace_bytes(M, K), dtype=torch.uint8, device="cuda")
    x64 = R.decode8(*R.copy8(R.f64(x)))
    T = np.abs(R.f64(dy)).T @ np.abs(x64)
    for accumulate in (False, True):
        dw = dw0.clone()
        B.nvfp4_linear_bf16_bwd8(dy, x8, w, dx, dw, ws, accumulate)
        B.nvfp4_device_status()
        want = R.f64(dy).T @ x64 + (R.f64(dw0) if accumulate else 0)
        R.assert_within(R.f64(dw), want, exact_tolerance(T, M) + 2 * U * np.abs(want), "dW")
        again = dw0.clone()
        B.nvfp4_linear_bf16_bwd8(dy, x8, w, dx, again, ws, accumulate)
        assert torch.equal(again, dw)
    want = R.f64(dy) @ R.f64(w)
    R.assert_within(R.f64(dx), want, 1e-4 * (np.abs(R.f64(dy)) @ np.abs(R.f64(w))) + BF16 * np.abs(want), "dX")
    only = torch.empty_like(dx)
    B.nvfp4_linear_bf16_bwd8(dy, None, w, only, None)
    R.assert_within(R.f64(only), want, 1e-4 * (np.abs(R.f64(dy)) @ np.abs(R.f64(w))) + BF16 * np.abs(want), "dX alone")
    only = torch.empty_like(dw0)
    B.nvfp4_linear_bf16_bwd8(dy, x8, None, None, only, ws)
    R.assert_within(R.f64(only), R.f64(dy).T @ x64, exact_tolerance(T, M) + U * T, "dW alone")


def test_long_contractions_of_one_sign():
    """Where every addition to an accumulator is cut off in the same direction the error would grow with the tokens:
    3.1e-5 of the sum in the mean for these."""
    M, N, K = 16384, 264, 520
    dy, x = normal((M, N), 45, 1e-2).abs().cuda(), normal((M, K), 46).abs()
    x8 = B.alloc_tensor(M, K, format=B.FORMAT_MXFP8)
    B.nvfp4_quantize(x.cuda(), B.quant_opts(), x8)
    x64 = R.decode8(x8.codes.cpu().numpy(), x8.scales.cpu().numpy())
    ws = torch.empty(B.nvfp4_linear_bf16_bwd8_workspace_bytes(M, K), dtype=torch.uint8, device="cuda")
    T = R.f64(dy).T @ x64
    for tile in (0, 642, 644):
        B.nvfp4_set_gemm_tile_n(tile)
        try:
            dw = torch.empty((N, K), device="cuda")
            B.nvfp4_linear_bf16_bwd8(dy, x8, None, None, dw, ws)
            B.nvfp4_device_status()
        finally:
            B.nvfp4_set_gemm_tile_n(0)
        R.assert_within(R.f64(dw), T, exact_tolerance(T, M), f"dW {tile}")


# ---------------------------------------------------------------------------------------------------------- together ----
def test_feed_forward_block_and_its_gradients():
    """norm -> up-projection with bias and squared ReLU -> down-projection with bias and residual, everything that the backward pass needs
    kept in 8 bits; gradients against torch's of the exact block in 64 bits, and against differences of it."""
    M, H, F = 264, 256, 520
    x, r = normal((M, H), 51), normal((M, H), 52, 2.0)
    gain = normal((H,), 53, 0.2, torch.float32) + 1
    w1, b1 = normal((F, H), 54, H ** -0.5), normal((F,), 55, 0.1, torch.float32)
    w2, b2 = normal((H, F), 56, F ** -0.5), normal((H,), 57, 0.1, torch.float32)
    dout = normal((M, H), 58)
    new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
    c = lambda t: t.cuda()
    h, y, rstd = new(M, H), new(M, H), new(M, dtype=torch.float32)
    y8, h8, z8 = B.alloc_tensor(M, H, format=B.FORMAT_MXFP8), B.alloc_tensor(M, H, format=B.FORMAT_MXFP8), B.alloc_tensor(M, F, format=B.FORMAT_MXFP8)
    a, out = new(M, F), new(M, H)
    B.nvfp4_rmsnorm_fwd(c(x), c(gain), 1e-5, y, rstd, residual=c(r), h=h, y8=y8, h8=h8)
    B.nvfp4_gemm_bf16_epilogue(y, c(w1), a, c(b1), B.ACT_RELU2, z=z8)
    B.nvfp4_gemm_bf16_epilogue(a, c(w2), out, c(b2), residual=h)

    g = c(dout)
    da, dz, a2, dy, dh = new(M, F), new(M, F), new(M, F), new(M, H), new(M, H)
    db1, db2, dgain = new(F, dtype=torch.float32), new(H, dtype=torch.float32), new(H, dtype=torch.float32)
    dw1, dw2 = new(F, H, dtype=torch.float32), new(H, F, dtype=torch.float32)
    ws = torch.empty(max(B.nvfp4_act_bwd_workspace_bytes(M, F), B.nvfp4_rmsnorm_bwd_workspace_bytes(M, H),
                         B.nvfp4_linear_bf16_bwd8_workspace_bytes(M, H)), dtype=torch.uint8, device="cuda")
    B.nvfp4_act_bwd(g, None, B.ACT_NONE, dbias=db2, workspace=ws)
    B.nvfp4_linear_bf16_bwd(g, None, c(w2), F, da, None)
    B.nvfp4_act_bwd(da, z8, B.ACT_RELU2, dz, a2, db1, workspace=ws)
    B.nvfp4_linear_bf16_bwd(g, a2, None, F, None, dw2)
    B.nvfp4_linear_bf16_bwd8(dz, y8, c(w1), dy, dw1, ws)
    B.nvfp4_rmsnorm_bwd(dy, h8, c(gain), rstd, dh, dgain, ws, residual_grad=g)
    B.nvfp4_device_status()

    leaf = lambda t: t.double().requires_grad_()
    X, G, W1, B1, W2, B2 = leaf(x.double() + r.double()), leaf(gain), leaf(w1), leaf(b1), leaf(w2), leaf(b2)
    Y = X * torch.rsqrt(X.square().mean(1, keepdim=True) + 1e-5) * G
    Z = Y @ W1.t() + B1
    O = Z.clamp_min(0).square() @ W2.t() + B2 + X
    rel = lambda got, want: np.linalg.norm(R.f64(got) - R.f64(want)) / np.linalg.norm(R.f64(want))
    assert rel(out, O) < 2 ** -7
    O.backward(dout.double())
    # Mean-square error of a copy: an element is off by at most half a step, 2^-4 of itself, uniformly: 2^-4 / sqrt(3) = 3.6 % or less.  A
    # gradient has at most three such factors (z8, y8 or h8, and z8 again through dz), and bf16 roundings of 2^-8 / sqrt(3): below 8 %.
    for got, want, name in ((db2, B2.grad, "db2"), (dw2, W2.grad, "dw2"), (db1, B1.grad, "db1"), (dw1, W1.grad, "dw1"),
                            (dgain, G.grad, "dgain"), (dh, X.grad, "dh")):
        assert rel(got, want) < 0.08, name
    # and against differences of the block along the gradient's direction, in 64 bits
    with torch.no_grad():
        v = W1.grad / W1.grad.norm()
        f = lambda t: (((Y @ (W1 + t * v).t() + B1).clamp_min(0).square() @ W2.t() + B2 + X) * dout.double()).sum()
        along = float((f(1e-5) - f(-1e-5)) / 2e-5)
    assert abs((R.f64(dw1) * R.f64(v)).sum() - along) <= 0.08 * abs(along)
