"""Norm, copies in 8 bits and the activation's gradient against 64-bit references.

Tolerances, with u = 2^-24 (a binary32 rounding) and 2^-8 for a rounding to bf16:
  - a sum of squares or products over a row goes through at most 80 additions in a lane, 5 in a warp and 16 between warps: its relative
    error (absolute, against the sum of magnitudes) is below 128 u = 2^-17, a root's half of that;
  - a column's sum goes through the rows of a lane (rows / 148 or 128 at most), up to 16 groups or warps and 256 partial sums in
    eight shares: below (rows / 64 + 96) u of the sum of magnitudes;
  - fast exponentials and quotients are off by a few u times the size of the exponent: 64 u for the arguments here (below 40).
"""
import numpy as np
import pytest
import torch

import around_ref as R
from paper_2509_25149_b200 import binding as B

pytestmark = pytest.mark.gpu
U, BF16 = 2.0 ** -24, 2.0 ** -8


def normal(shape, seed, std=1.0, dtype=torch.bfloat16, far=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * std
    if far:
        x = torch.where(torch.rand(shape, generator=g) < 0.01, x * far, x)
    return x.to(dtype)


SHAPES = [(1, 8), (1, 5120), (2, 24), (3, 40), (7, 520), (37, 1048), (129, 2056), (5, 5120), (3, 10248), (2, 20480), (2, 20488), (3, 41000),
          (1500, 64)]


# ---------------------------------------------------------------------------------------------- copies in 8 bits ----
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_copy_is_the_format_bit_for_bit(shape, dtype):
    rows, cols = shape
    x = normal(shape, 1, 3.0, dtype, far=300.0)
    x[:, :8] = torch.tensor([0.0, -0.0, 2.0 ** -130, -1e-30, 448.0, 1e30, -3e38, 1.75], dtype=dtype)
    if cols > 40:
        x[:, 32:40] = 0
    src, src_ok = R.guarded(rows, cols, dtype, cols + 24, x.cuda())
    q, q_ok = R.guarded_copy(rows, cols)
    B.nvfp4_quantize(src, B.quant_opts(), q)
    codes, scales = R.copy8(R.f64(x))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    out, out_ok = R.guarded(rows, cols, torch.bfloat16, cols + 8)
    B.nvfp4_dequantize_bf16(q, out)
    want = R.decode8(codes, scales)
    assert np.array_equal(R.f64(out), torch.from_numpy(want).to(torch.bfloat16).double().numpy())
    assert np.array_equal(R.f64(B.nvfp4_dequantize(q)), want)
    assert src_ok() and q_ok() and out_ok()
    # half a step of E4M3, or half the smallest step where the element is that far below its block's maximum
    E = R.scale_exponent(np.abs(np.pad(R.f64(x), ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)).max(2))
    tol = np.maximum(2.0 ** -4 * np.abs(R.f64(x)), np.repeat(2.0 ** -10 * 2.0 ** E.astype(float), 32, axis=1)[:, :cols])
    R.assert_within(want, R.f64(x), tol, "copy")


def test_every_code_and_every_border_of_a_scale():
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)
    codes[codes % 128 == 127] = 0  # (the two codes that are no numbers)
    scales = torch.arange(256, dtype=torch.uint8).clamp_max(247).view(256, 1).repeat(1, 8).contiguous()
    q = B.alloc_tensor(256, 256, format=B.FORMAT_MXFP8)
    q.codes.copy_(codes)
    q.scales.copy_(scales)
    with np.errstate(over="ignore"):  # (the output is binary32: 320 * 2^120 and more are beyond it)
        want = R.decode8(codes.numpy(), scales.numpy()).astype(np.float32)
    assert np.array_equal(B.nvfp4_dequantize(q).cpu().numpy(), want)
    # maxima next to 448 * 2^E, in binary32
    exps = torch.arange(-126, 118).double()
    top = torch.stack([448 * 2 ** exps, 448 * 2 ** exps * (1 + 2.0 ** -23), 448 * 2 ** exps * (1 - 2.0 ** -24)]).reshape(-1, 1).float()
    x = torch.cat([top, top * 0.3, -top * 0.01, torch.zeros(top.shape[0], 5)], 1)
    q = B.alloc_tensor(x.shape[0], 8, format=B.FORMAT_MXFP8)
    B.nvfp4_quantize(x.cuda(), B.quant_opts(), q)
    codes, scales = R.copy8(x.double().numpy())
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)


def test_copy_of_more_than_two_to_the_31_elements():
    rows, cols = 131080, 16392  # 2.15e9 elements: offsets beyond 31 bits, short last blocks
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-1] = normal((cols,), 3).cuda()
    x[rows // 2] = normal((cols,), 4).cuda()
    q = B.alloc_tensor(rows, cols, format=B.FORMAT_MXFP8)
    B.nvfp4_quantize(x, B.quant_opts(), q)
    back = B.nvfp4_dequantize_bf16(q)
    for r in (0, rows // 2, rows - 1):
        codes, scales = R.copy8(R.f64(x[r:r + 1]))
        assert np.array_equal(q.codes[r].cpu().numpy(), codes[0]) and np.array_equal(q.scales[r].cpu().numpy(), scales[0])
        assert np.array_equal(R.f64(back[r]), R.decode8(codes, scales)[0])


# ---------------------------------------------------------------------------------------------------------- norm ----
def norm64(x, res, gain, eps):
    h = R.f64(x)
    if res is not None:
        h = (h + R.f64(res)).astype(np.float32).astype(np.float64)
    r = 1 / np.sqrt((h * h).mean(1) + eps)
    return h, r, h * r[:, None] * (R.f64(gain) if gain is not None else 1.0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("res", [None, torch.bfloat16, torch.float32])
def test_norm_forward(shape, res):
    rows, cols = shape
    x, gain = normal(shape, 11, 1.0, far=50.0), normal((cols,), 12, 0.5, torch.float32) + 1
    r = normal(shape, 13, 2.0, res) if res is not None else None
    if rows > 1:
        x[1] = 0
        if r is not None:
            r[1] = 0
    eps = 1e-5
    xd, x_ok = R.guarded(rows, cols, torch.bfloat16, cols + 8, x.cuda())
    rd, r_ok = R.guarded(rows, cols, res, cols + 16, r.cuda()) if res is not None else (None, lambda: True)
    h, h_ok = R.guarded(rows, cols, res, cols + 8) if res is not None else (None, lambda: True)
    y, y_ok = R.guarded(rows, cols, torch.bfloat16, cols + 32)
    rstd = torch.empty(rows, device="cuda")
    (y8, y8_ok), (h8, h8_ok) = R.guarded_copy(rows, cols), R.guarded_copy(rows, cols)
    B.nvfp4_rmsnorm_fwd(xd, gain.cuda(), eps, y, rstd, residual=rd, h=h, y8=y8, h8=h8)
    h64, r64, y64 = norm64(x, r, gain, eps)
    R.assert_within(R.f64(rstd), r64, r64 * 2.0 ** -17, "rstd")
    off = 2.0 ** -17 + 4 * U
    R.assert_within(R.f64(y), y64, np.abs(y64) * (BF16 + off) + 1e-38, "y")
    codes, scales = R.copy8(h64)
    assert np.array_equal(h8.codes.cpu().numpy(), codes) and np.array_equal(h8.scales.cpu().numpy(), scales)
    if h is not None:
        assert np.array_equal(R.f64(h), torch.from_numpy(h64).float().to(res).double().numpy())
    got = R.decode8(y8.codes.cpu().numpy(), y8.scales.cpu().numpy())
    top = np.repeat(np.abs(np.pad(y64, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)).max(2), 32, axis=1)[:, :cols]
    # half a step of the element, or of the smallest normal number: 2^-10 * 2^E with 2^E <= amax / 224
    R.assert_within(got, y64, np.maximum(2.0 ** -4 * np.abs(y64), 2.0 ** -10 * top / 224) * (1 + 2 * off) + off * np.abs(y64) + 1e-38, "y8")
    assert all(ok() for ok in (x_ok, r_ok, h_ok, y_ok, y8_ok, h8_ok))


def test_norm_in_place_and_with_single_outputs():
    rows, cols = 70, 1544
    x, r, gain = normal((rows, cols), 21).cuda(), normal((rows, cols), 22, 2.0).cuda(), normal((cols,), 23, 1.0, torch.float32).cuda()
    y, h, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    y8, h8 = (B.alloc_tensor(rows, cols, format=B.FORMAT_MXFP8) for _ in range(2))
    B.nvfp4_rmsnorm_fwd(x, gain, 1e-6, y, rstd, residual=r, h=h, y8=y8, h8=h8)
    x2, r2 = x.clone(), r.clone()
    B.nvfp4_rmsnorm_fwd(x2, gain, 1e-6, x2, residual=r2, h=r2)
    assert torch.equal(x2, y) and torch.equal(r2, h)
    one = lambda **k: B.nvfp4_rmsnorm_fwd(x, gain, 1e-6, residual=r, **k)
    for out, want in ((torch.empty_like(y), y), (torch.empty_like(h), h), (torch.empty_like(rstd), rstd)):
        one(**{"y" if want is y else "h" if want is h else "rstd": out})
        assert torch.equal(out, want)
    for name, want in (("y8", y8), ("h8", h8)):
        q = B.alloc_tensor(rows, cols, format=B.FORMAT_MXFP8)
        one(**{name: q})
        assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    # long rows in place: the second sweep reads what the first one read
    x, r = normal((3, 30000), 24).cuda(), normal((3, 30000), 25, 1.0, torch.float32).cuda()
    y, h = torch.empty_like(x), torch.empty_like(r)
    B.nvfp4_rmsnorm_fwd(x, None, 1e-6, y, residual=r, h=h)
    B.nvfp4_rmsnorm_fwd(x, None, 1e-6, x, residual=r, h=r)
    assert torch.equal(x, y) and torch.equal(r, h)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kept", ["bf16", "fp32", "8"])
@pytest.mark.parametrize("grad", [None, torch.bfloat16, torch.float32])
def test_norm_gradient(shape, kept, grad):
    rows, cols = shape
    dy, gain = normal(shape, 31, 1e-3), normal((cols,), 32, 0.5, torch.float32) + 1
    h = normal(shape, 33, 2.0, torch.float32 if kept == "fp32" else torch.bfloat16, far=30.0)
    if kept == "8":
        hd = R.copy_on_gpu(R.f64(h))
        h64, h_ok = R.decode8(*R.copy8(R.f64(h))), lambda: True
    else:
        hd, h_ok = R.guarded(rows, cols, h.dtype, cols + 8, h.cuda())
        h64 = R.f64(h)
    rstd = torch.from_numpy(1 / np.sqrt((h64 ** 2).mean(1) + 1e-5)).float()
    out_type = grad or torch.float32
    rg = normal(shape, 34, 1e-3, grad) if grad is not None else None
    dyd, dy_ok = R.guarded(rows, cols, torch.bfloat16, cols + 16, dy.cuda())
    rgd, rg_ok = R.guarded(rows, cols, grad, cols + 8, rg.cuda()) if grad is not None else (None, lambda: True)
    dh, dh_ok = R.guarded(rows, cols, out_type, cols + 24)
    start = normal((cols,), 35, 1.0, torch.float32)
    dgain = start.cuda()
    ws = torch.empty(B.nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_rmsnorm_bwd(dyd, hd, gain.cuda(), rstd.cuda(), dh, dgain, ws, residual_grad=rgd, accumulate_dgain=True)
    r, d64 = R.f64(rstd)[:, None], R.f64(dy)
    n, g = h64 * r, d64 * R.f64(gain)
    c = (g * n).mean(1, keepdims=True)
    want = r * (g - n * c)
    tol = r * (8 * U * (np.abs(g) + np.abs(n * c)) + np.abs(n) * 2.0 ** -17 * np.abs(g * n).mean(1, keepdims=True))
    if rg is not None:
        want = want + R.f64(rg)
    tol = tol + np.abs(want) * (BF16 if out_type == torch.bfloat16 else U) + 1e-40
    R.assert_within(R.f64(dh), want, tol, "dh")
    sums = (d64 * n).sum(0) + R.f64(start)
    tol = (rows / 64 + 96) * U * np.abs(d64 * n).sum(0) + 2 * U * np.abs(sums) + U * np.abs(R.f64(start))
    R.assert_within(R.f64(dgain), sums, tol, "dgain")
    assert h_ok() and dy_ok() and rg_ok() and dh_ok()
    # written instead of added; left out; and the same bits again
    again, dh2 = torch.full_like(dgain, float("nan")), torch.empty((rows, cols), dtype=out_type, device="cuda")
    B.nvfp4_rmsnorm_bwd(dyd, hd, gain.cuda(), rstd.cuda(), dh2, again, ws, residual_grad=rgd)
    assert torch.equal(dh2, dh)
    R.assert_within(R.f64(again), sums - R.f64(start), tol, "dgain written")
    B.nvfp4_rmsnorm_bwd(dyd, hd, gain.cuda(), rstd.cuda(), dh2.zero_(), None, ws if cols > 20480 else None, residual_grad=rgd)
    assert torch.equal(dh2, dh)


def test_norm_gradient_many_rows_and_in_place():
    rows, cols = 9001, 264
    dy, h, rg = normal((rows, cols), 41, 1e-3).cuda(), normal((rows, cols), 42).cuda(), normal((rows, cols), 43, 1e-3).cuda()
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-5).float()
    dgain, dh = torch.empty(cols, device="cuda"), torch.empty_like(dy)
    ws = torch.empty(B.nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_rmsnorm_bwd(dy, h, None, rstd, dh, dgain, ws, residual_grad=rg)
    n = R.f64(h) * R.f64(rstd)[:, None]
    R.assert_within(R.f64(dgain), (R.f64(dy) * n).sum(0), (rows / 64 + 96) * U * np.abs(R.f64(dy) * n).sum(0), "dgain")
    B.nvfp4_rmsnorm_bwd(dy, h, None, rstd, rg, None, None, residual_grad=rg)
    assert torch.equal(rg, dh)


def test_norm_gradient_agrees_with_differences():
    """Directional differences of the forward formula in 64 bits: the gradient is the formula's, not only this file's reading of it."""
    rows, cols = 4, 96
    h, gain, dy = normal((rows, cols), 51, 1.0, torch.float32), normal((cols,), 52, 1.0, torch.float32), normal((rows, cols), 53)
    eps = 1e-5
    f = lambda v, g: (R.f64(dy) * (v / np.sqrt((v * v).mean(1, keepdims=True) + eps) * g)).sum()
    rstd = torch.from_numpy(1 / np.sqrt((R.f64(h) ** 2).mean(1) + eps)).float().cuda()
    dh, dgain = torch.empty((rows, cols), device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_rmsnorm_bwd(dy.cuda(), h.cuda(), gain.cuda(), rstd, dh, dgain, ws)
    for seed in range(3):
        v, w, t = R.f64(normal((rows, cols), 60 + seed, 1.0, torch.float32)), R.f64(normal((cols,), 70 + seed, 1.0, torch.float32)), 1e-5
        along = (f(R.f64(h) + t * v, R.f64(gain)) - f(R.f64(h) - t * v, R.f64(gain))) / (2 * t)
        assert abs(along - (R.f64(dh) * v).sum()) <= 1e-5 * np.abs(R.f64(dh) * v).sum() + 1e-8
        along = (f(R.f64(h), R.f64(gain) + t * w) - f(R.f64(h), R.f64(gain) - t * w)) / (2 * t)
        assert abs(along - (R.f64(dgain) * w).sum()) <= 1e-5 * np.abs(R.f64(dgain) * w).sum() + 1e-8


# ------------------------------------------------------------------------------------------ gradient of an activation ----
@pytest.mark.parametrize("shape", [(1, 8), (2, 40), (31, 264), (33, 256), (129, 2056), (257, 1048), (1500, 64), (70, 5128)])
@pytest.mark.parametrize("act", sorted(R.ACTS))
@pytest.mark.parametrize("kept", ["bf16", "8"])
def test_gradient_of_an_activation(shape, act, kept):
    rows, cols = shape
    da, z = normal(shape, 81, 1e-3), normal(shape, 82, 3.0, far=4.0)
    if kept == "8":
        zd, z64, z_ok = R.copy_on_gpu(R.f64(z)), R.decode8(*R.copy8(R.f64(z))), lambda: True
    else:
        zd, z_ok = R.guarded(rows, cols, torch.bfloat16, cols + 8, z.cuda())
        z64 = R.f64(z)
    dad, da_ok = R.guarded(rows, cols, torch.bfloat16, cols + 16, da.cuda())
    (dz, dz_ok), (a, a_ok) = R.guarded(rows, cols, torch.bfloat16, cols + 8), R.guarded(rows, cols, torch.bfloat16, cols + 24)
    start = normal((cols,), 83, 1e-2, torch.float32)
    dbias = start.cuda()
    ws = torch.empty(B.nvfp4_act_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_act_bwd(dad, zd, R.ACTS[act], dz, a, dbias, True, ws)
    d64 = R.f64(da)
    want, value = d64 * R.slope64(z64, act), R.act64(z64, act)
    fast = 0.0 if act in ("none", "relu2") else 64 * U
    # the slope is a sum of terms up to 1 + |z s(1 - s) u'|, below 3 in magnitude; s carries the fast functions' error
    off = np.abs(d64) * 3 * (fast + 8 * U) + 4 * U * np.abs(want)
    R.assert_within(R.f64(dz), want, BF16 * np.abs(want) + off * (1 + BF16) + 1e-40, "dz")
    # z / (1 + e): the fast quotient is zero where its denominator is above 2^126, and the true one is then below |z| 2^-126
    R.assert_within(R.f64(a), value, (BF16 + fast + 8 * U) * np.abs(value) + (1 + np.abs(z64)) * 2.0 ** -126, "a")
    sums = want.sum(0) + R.f64(start)
    tol = off.sum(0) + (rows / 64 + 96) * U * np.abs(want).sum(0) + 2 * U * np.abs(sums) + U * np.abs(R.f64(start))
    R.assert_within(R.f64(dbias), sums, tol, "dbias")
    assert z_ok() and da_ok() and dz_ok() and a_ok()
    # each output alone, in place, and the sums written instead of added
    only = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    B.nvfp4_act_bwd(dad, zd, R.ACTS[act], only)
    assert torch.equal(only, dz)
    B.nvfp4_act_bwd(dad, zd, R.ACTS[act], a=only)
    assert torch.equal(only, a)
    alone = torch.full_like(dbias, float("nan"))
    B.nvfp4_act_bwd(dad, zd, R.ACTS[act], dbias=alone, workspace=ws)
    R.assert_within(R.f64(alone), want.sum(0), tol, "dbias alone")
    inplace = da.cuda()
    if kept == "bf16":
        zc = z.cuda()
        B.nvfp4_act_bwd(inplace, zc, R.ACTS[act], inplace, zc)
        assert torch.equal(zc, a)
    else:
        B.nvfp4_act_bwd(inplace, zd, R.ACTS[act], inplace)
    assert torch.equal(inplace, dz)


def test_bias_gradient_without_an_activation():
    rows, cols = 3001, 520
    da = normal((rows, cols), 91).cuda()
    dbias = torch.empty(cols, device="cuda")
    ws = torch.empty(B.nvfp4_act_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_act_bwd(da, None, B.ACT_NONE, dbias=dbias, workspace=ws)
    R.assert_within(R.f64(dbias), R.f64(da).sum(0), (rows / 64 + 96) * U * np.abs(R.f64(da)).sum(0), "dbias")


def test_far_arguments_of_the_activations():
    z = torch.tensor([[0.0, -0.0, 1e-38, -1e-38, 90.0, -90.0, 1000.0, -1000.0, 3e4, -3e4, 12.0, -12.0, 6.0, -6.0, 1.0, -1.0]], dtype=torch.bfloat16)
    da = torch.ones_like(z)
    for act in ("silu", "gelu", "relu2"):
        dz, a = torch.empty_like(z).cuda(), torch.empty_like(z).cuda()
        B.nvfp4_act_bwd(da.cuda(), z.cuda(), R.ACTS[act], dz, a)
        with np.errstate(over="ignore", invalid="ignore"):
            want, value = R.slope64(R.f64(z), act), R.act64(R.f64(z), act)
        # (the exponent's size is up to 90 where the result is not zero: 256 u; results below 2^-126 may be zero)
        R.assert_within(R.f64(dz), want, (BF16 + 256 * U) * np.abs(want) + 8 * U, act)
        R.assert_within(R.f64(a), value, (BF16 + 256 * U) * np.abs(value) + 2.0 ** -110, act)


def test_more_than_two_to_the_31_elements():
    rows, cols = 131080, 16392
    at = [0, 5, rows // 2, rows - 1]
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[at] = normal((len(at), cols), 95).cuda()
    x8 = B.alloc_tensor(rows, cols, format=B.FORMAT_MXFP8)
    B.nvfp4_quantize(x, B.quant_opts(), x8)
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    B.nvfp4_rmsnorm_fwd(x, None, 1e-5, y, rstd)
    h64, r64, y64 = norm64(x[at].cpu(), None, None, 1e-5)
    R.assert_within(R.f64(y[at]), y64, np.abs(y64) * (BF16 + 2.0 ** -16) + 1e-38, "y")
    # its gradient from the copy, with y for dy (rows of zeros leave rows of zeros)
    dgain, ws = torch.empty(cols, device="cuda"), torch.empty(B.nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    dh = x  # (x has served)
    B.nvfp4_rmsnorm_bwd(y, x8, None, rstd, dh, dgain, ws)
    r, n = R.f64(rstd[at])[:, None], R.decode8(x8.codes[at].cpu().numpy(), x8.scales[at].cpu().numpy()) * R.f64(rstd[at])[:, None]
    g = R.f64(y[at])
    c = (g * n).mean(1, keepdims=True)
    want = r * (g - n * c)
    tol = r * (8 * U * (np.abs(g) + np.abs(n * c)) + np.abs(n) * 2.0 ** -17 * np.abs(g * n).mean(1, keepdims=True)) + np.abs(want) * BF16 + 1e-40
    R.assert_within(R.f64(dh[at]), want, tol, "dh")
    R.assert_within(R.f64(dgain), (g * n).sum(0), 128 * U * np.abs(g * n).sum(0) + 1e-40, "dgain")
    assert not dh[1].any()
    dbias, ws = torch.empty(cols, device="cuda"), torch.empty(B.nvfp4_act_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_act_bwd(y, x8, B.ACT_RELU2, dh, dbias=dbias, workspace=ws)
    z = R.decode8(x8.codes[at].cpu().numpy(), x8.scales[at].cpu().numpy())
    want = g * 2 * np.maximum(z, 0)
    R.assert_within(R.f64(dh[at]), want, np.abs(want) * (BF16 + 4 * U), "dz")
    R.assert_within(R.f64(dbias), want.sum(0), 128 * U * np.abs(want).sum(0), "dbias")


# --------------------------------------------------------------------------------------------- streams and graphs ----
def test_captured_on_another_stream_beside_each_other():
    """Two captured graphs with workspaces of their own, replayed on two streams at once, give the bits of direct calls."""
    def make(seed):
        rows, cols = 700, 2056
        s = {"dy": normal((rows, cols), seed, 1e-3).cuda(), "x": normal((rows, cols), seed + 1).cuda(),
             "r": normal((rows, cols), seed + 2).cuda(), "gain": normal((cols,), seed + 3, 1.0, torch.float32).cuda()}
        s["y"], s["h"], s["dh"], s["dz"] = (torch.empty_like(s["x"]) for _ in range(4))
        s["rstd"], s["dgain"], s["dbias"] = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        s["h8"] = B.alloc_tensor(rows, cols, format=B.FORMAT_MXFP8)
        s["ws"] = torch.empty(B.nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        s["ws2"] = torch.empty(B.nvfp4_act_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")

        def step():
            B.nvfp4_rmsnorm_fwd(s["x"], s["gain"], 1e-5, s["y"], s["rstd"], residual=s["r"], h=s["h"], h8=s["h8"])
            B.nvfp4_act_bwd(s["dy"], s["y"], B.ACT_SILU, s["dz"], dbias=s["dbias"], workspace=s["ws2"])
            B.nvfp4_rmsnorm_bwd(s["dz"], s["h8"], s["gain"], s["rstd"], s["dh"], s["dgain"], s["ws"], residual_grad=s["dy"])
        return s, step

    both = [make(100), make(200)]
    names = ("y", "h", "rstd", "dz", "dbias", "dh", "dgain")
    want = []
    for s, step in both:
        step()
        torch.cuda.synchronize()
        want.append([s[n].clone() for n in names])
    graphs, streams = [], [torch.cuda.Stream() for _ in both]
    for (s, step), stream in zip(both, streams):
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        graphs.append(graph)
    for s, _ in both:
        for n in names:
            s[n].fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (s, _), ref in zip(both, want):
        for n, r in zip(names, ref):
            assert torch.equal(s[n], r), n
