"""Where the operators around the linear layers have little room: long contractions whose codes must not show how the tensor cores add,
finite arguments whose squares are beyond binary32, and roundings that are promised one by one."""
import numpy as np
import pytest
import torch

import around_ref as R
from paper_2509_25149_b200 import binding as B

pytestmark = pytest.mark.gpu
U, BF16 = 2.0 ** -24, 2.0 ** -8


def one_sign(shape, seed):
    """Uniform in [1, 2): products with sixteen bits, sums that binary32 cannot hold."""
    return (torch.rand(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") + 1).to(torch.bfloat16)


# M, N, tile: few rows with one and two shares of k (few_rows_kernel), then the pair kernels in every tile
LONG = [(1, 7144, 0), (8, 7144, 0), (12, 7144, 0), (16, 4104, 0), (32, 7144, 0), (64, 264, 0), (128, 264, 0), (300, 264, 0), (300, 264, 512),
        (300, 264, 640), (300, 264, 642), (300, 264, 644)]


@pytest.mark.parametrize("M,N,tile", LONG)
def test_codes_of_long_contractions_of_one_sign(M, N, tile):
    """Kept in 8 bits, z is a sum of sums of 1024 products: an addition on the tensor cores cuts off less than a unit in the last place of
    its sum, 2^-23 of it, and 64 of them (16 products each) make a share, 2^-17 of the sum of magnitudes T; shares are added rounded to
    nearest, 2^-24 each (65536 / 1024 of them, and two to four parts).  A bias of minus the sum lays this error open: what is left of z is
    the error, and D and the codes have it to their own relative precision.  Left in one accumulator the sum is off by some 3e-5 T."""
    K = 65536
    a, b = one_sign((1, K), 101), one_sign((N, K), 102)
    dots = torch.cat([p.double() @ a[0].double() for p in b.split(1024)])  # (exact but for additions in 64 bits)
    bias = -dots.float()
    z64 = R.f64(dots) + R.f64(bias)
    D = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    z = B.alloc_tensor(M, N, format=B.FORMAT_MXFP8)
    B.nvfp4_set_gemm_tile_n(tile)
    try:
        B.nvfp4_gemm_bf16_epilogue(a.expand(M, K).contiguous(), b, D, bias, z=z)
        B.nvfp4_device_status()
    finally:
        B.nvfp4_set_gemm_tile_n(0)
    T = R.f64(dots)
    off = (2.0 ** -17 + (K // 1024 + 4) * U) * T
    R.assert_within(R.f64(D), z64 + np.zeros((M, 1)), off + BF16 * (np.abs(z64) + off) + np.zeros((M, 1)), "D")
    got = R.decode8(z.codes.cpu().numpy(), z.scales.cpu().numpy())
    # (an element's own half step, or half the smallest step of its block, 2^-10 of the scale, which is at most a 224th of the maximum)
    top = np.repeat(np.pad(np.abs(z64) + off, (0, -N % 32)).reshape(-1, 32).max(1), 32)[:N]
    R.assert_within(got, z64 + np.zeros((M, 1)), off + np.maximum(2.0 ** -4 * (np.abs(z64) + off), 2.0 ** -10 * top / 224) + np.zeros((M, 1)), "z8")


def test_slope_of_finite_arguments_is_finite():
    """Squares of these are beyond binary32; the slope is 1 or 0 (squared ReLU: twice the argument)."""
    far = [8.0, 50.0, 100.0, 101.0, 1e4, 1.8e19, 1.9e19, 1e20, 3e38]
    z = torch.tensor([[s * v for v in far for s in (1, -1)] * 4], dtype=torch.bfloat16)
    da = torch.full_like(z, 0.75)
    for act in sorted(R.ACTS):
        for kept in (z.cuda(), R.copy_on_gpu(R.f64(z))):
            z64 = R.f64(z) if isinstance(kept, torch.Tensor) else R.decode8(*R.copy8(R.f64(z)))
            dz, a, dbias = torch.empty_like(z).cuda(), torch.empty_like(z).cuda(), torch.empty(z.shape[1], device="cuda")
            ws = torch.empty(B.nvfp4_act_bwd_workspace_bytes(*z.shape), dtype=torch.uint8, device="cuda")
            B.nvfp4_act_bwd(da.cuda(), kept, R.ACTS[act], dz, a, dbias, workspace=ws)
            with np.errstate(over="ignore", invalid="ignore"):
                want, value = 0.75 * R.slope64(z64, act), R.act64(z64, act)
            ok = np.abs(want) < 2.0 ** 127  # (twice the largest argument is beyond bf16)
            # 256 u for the fast functions (see test_far_arguments_of_the_activations); results below 2^-126 may be zero
            for got in (dz, dbias.view(1, -1)):
                R.assert_within(R.f64(got)[ok], want[ok], ((BF16 + 256 * U) * np.abs(want) + 8 * U)[ok], act)
            ok = np.abs(value) < 2.0 ** 127
            R.assert_within(R.f64(a)[ok], value[ok], ((BF16 + 256 * U) * np.abs(value) + 2.0 ** -110)[ok], act)


@pytest.mark.parametrize("cols", [8, 40, 520, 1048, 2056, 5120, 10248, 20480, 30008])
@pytest.mark.parametrize("res", [None, torch.bfloat16, torch.float32])
def test_norm_of_rows_whose_squares_exceed_binary32(cols, res):
    """Finite rows: mean and root are in 64 bits, so the norm is too."""
    tops = [1.0, 3e17, 1.7e19, 1.9e19, 1e20, 1e30, 3e38]
    rows = len(tops)
    x = (torch.rand((rows, cols), generator=torch.Generator().manual_seed(cols)) * 2 - 1).double()
    x[:, cols // 2] = 1.0  # (the largest)
    x = x * torch.tensor(tops, dtype=torch.float64)[:, None]
    gain = torch.rand(cols, generator=torch.Generator().manual_seed(cols + 1)) + 0.5
    if res is None:
        x, r = x.to(torch.bfloat16), None
    else:
        x, r = (x / 2).to(torch.bfloat16), (x / 2).to(res)
    h = R.f64(x) if r is None else (R.f64(x) + R.f64(r)).astype(np.float32).astype(np.float64)
    r64 = 1 / np.sqrt((h * h).mean(1) + 1e-5)
    y64 = h * r64[:, None] * R.f64(gain)
    y, rstd = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"), torch.empty(rows, device="cuda")
    y8 = B.alloc_tensor(rows, cols, format=B.FORMAT_MXFP8)
    B.nvfp4_rmsnorm_fwd(x.cuda(), gain.cuda(), 1e-5, y, rstd, residual=r.cuda() if r is not None else None, y8=y8)
    # (rstd of the last rows is below 2^-126: multiples of 2^-149)
    R.assert_within(R.f64(rstd), r64, r64 * 2.0 ** -17 + 2.0 ** -150, "rstd")
    off = 2.0 ** -17 + 4 * U + 2.0 ** -150 / r64[:, None]
    R.assert_within(R.f64(y), y64, np.abs(y64) * (BF16 + off) + 1e-38, "y")
    got = R.decode8(y8.codes.cpu().numpy(), y8.scales.cpu().numpy())
    top = np.repeat(np.abs(np.pad(y64, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)).max(2), 32, axis=1)[:, :cols]
    R.assert_within(got, y64, np.maximum(2.0 ** -4 * np.abs(y64), 2.0 ** -10 * top / 224) * (1 + 2 * off) + off * np.abs(y64) + 1e-38, "y8")
    # the gradient from the kept h and this rstd: nothing in it is beyond binary32 either
    dy, kept = torch.rand((rows, cols), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16), x if r is None else torch.from_numpy(h).to(res)
    dh, dgain = torch.empty((rows, cols), device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.nvfp4_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.nvfp4_rmsnorm_bwd(dy.cuda(), kept.cuda(), gain.cuda(), rstd, dh, dgain, ws)
    k64, d64, s = R.f64(kept), R.f64(dy), R.f64(rstd)[:, None]
    n, g = k64 * s, d64 * R.f64(gain)
    c = (g * n).mean(1, keepdims=True)
    tol = s * (8 * U * (np.abs(g) + np.abs(n * c)) + np.abs(n) * 2.0 ** -17 * np.abs(g * n).mean(1, keepdims=True))
    R.assert_within(R.f64(dh), s * (g - n * c), tol + U * np.abs(s * (g - n * c)) + 1e-40, "dh")
    R.assert_within(R.f64(dgain), (d64 * n).sum(0), (rows / 64 + 96) * U * np.abs(d64 * n).sum(0), "dgain")


def test_layer_gradients_of_any_number_of_tokens():
    """1003 tokens in buffers of 1008 rows: zeros behind them in dY, anything that is a number in the copy."""
    M, rows, N, K = 1003, 1008, 264, 520
    dy, w = (torch.randint(-2, 3, s, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16) for i, s in enumerate(((rows, N), (N, K))))
    dy[M:] = 0
    x = torch.randint(-4, 5, (rows, K), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    x[M:] = 1000
    x8 = B.alloc_tensor(rows, K, format=B.FORMAT_MXFP8)
    B.nvfp4_quantize(x.cuda(), B.quant_opts(), x8)
    dx, dw = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda"), torch.empty((N, K), device="cuda")
    ws = torch.empty(B.nvfp4_linear_bf16_bwd8_workspace_bytes(rows, K), dtype=torch.uint8, device="cuda")
    B.nvfp4_linear_bf16_bwd8(dy.cuda(), x8, w.cuda(), dx, dw, ws)
    assert np.array_equal(R.f64(dw), R.f64(dy[:M]).T @ R.f64(x[:M]))
    assert np.array_equal(R.f64(dx[:M]), torch.from_numpy(R.f64(dy[:M]) @ R.f64(w)).to(torch.bfloat16).double().numpy())
    assert not dx[M:].any()
    with pytest.raises(RuntimeError, match="nvfp4_linear_bf16_bwd8"):
        short = B.NVFP4Tensor(x8.codes, x8.scales, None, M, K, B.SF_LINEAR, B.FORMAT_MXFP8)
        B.nvfp4_linear_bf16_bwd8(dy[:M].cuda(), short, w.cuda(), dx[:M], dw, ws)


# ------------------------------------------------------------------------------------- roundings of the norm, one by one ----
def whole_rows(rows, cols, seed):
    """Whole numbers whose sums of squares binary32 holds exactly, whatever the order (below 2^24)."""
    top = int((2.0 ** 24 / cols) ** 0.5 * 1.5) - 1  # (uniform in [-top, top]: a mean square of top^2 / 3)
    h = torch.randint(-min(top, 255), min(top, 255) + 1, (rows, cols), generator=torch.Generator().manual_seed(seed))
    h[h == 0] = 1
    assert int((h.long() ** 2).sum(1).max()) < 2 ** 24
    return h.to(torch.bfloat16)


@pytest.mark.parametrize("cols", [64, 1048, 5120, 20480, 41000])
def test_reciprocal_root_is_rounded_once(cols):
    """Where the sum of squares is exact, mean, root and reciprocal leave rstd at the binary32 number next to the true one: they are taken to
    2^-45 and better, so that only a root within that of a border between two numbers could go the other way."""
    h = whole_rows(512, cols, 7 + cols)
    rstd = torch.empty(512, device="cuda")
    B.nvfp4_rmsnorm_fwd(h.cuda(), None, 1e-5, rstd=rstd)
    h64 = R.f64(h)
    exact = 1 / np.sqrt((h64 * h64).mean(1) + float(np.float32(1e-5)))
    assert np.array_equal(rstd.cpu().numpy(), exact.astype(np.float32))


@pytest.mark.parametrize("cols", [1024, 5120, 20480, 40960])
def test_y_of_a_copy_is_rounded_once_before_it_is_coded(cols):
    """Gains that put y between 1.05 and 2.5 roundings of binary32 beside a border of two codes: with one rounding, by 2^-24 at most, each
    must come out on its side of the border."""
    rng = np.random.default_rng(cols)
    h = whole_rows(1, cols, 3 + cols)
    h64 = R.f64(h)[0]
    rstd = 1 / np.sqrt((h64 * h64).mean() + float(np.float32(1e-5)))
    borders = (R.GRID[8:118] + R.GRID[9:119]) / 2  # (of normal codes up to 240)
    want = rng.choice(borders, cols) * np.sign(h64)
    want[::32] = 300.0 * np.sign(h64[::32])  # (every block's maximum: a scale of one)
    gain = (want / (h64 * rstd) * (1 + rng.uniform(-4, 4, cols) * U)).astype(np.float32)
    y64 = h64 * rstd * gain.astype(np.float64)
    beside = np.abs(y64 / want - 1) / U
    tested = (beside > 1.05) & (beside < 2.5)
    tested[::32] = False
    assert tested.sum() > cols // 4
    y8 = B.alloc_tensor(1, cols, format=B.FORMAT_MXFP8)
    B.nvfp4_rmsnorm_fwd(h.cuda(), torch.from_numpy(gain).cuda(), 1e-5, y8=y8)
    codes, scales = R.copy8(y64[None])
    assert np.array_equal(y8.scales.cpu().numpy(), scales)
    got = y8.codes.cpu().numpy()[0]
    assert np.array_equal(got[tested], codes[0][tested]), int((got[tested] != codes[0][tested]).sum())


# ------------------------------------------------------------------------------------- layer gradients, in their bounds ----
@pytest.mark.parametrize("shape", [(8, 24, 40), (1000, 264, 136), (200, 520, 1048), (2056, 1032, 520)])
def test_layer_gradients_from_a_copy_stay_in_their_buffers(shape):
    """Whole numbers, so that both gradients are known to the bit; what lies around every buffer stays as it was."""
    M, N, K = shape
    dy, w = (torch.randint(-2, 3, s, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16) for i, s in enumerate(((M, N), (N, K))))
    x = torch.randint(-4, 5, (M, K), generator=torch.Generator().manual_seed(5)).double().numpy()
    dyd, dy_ok = R.guarded(M, N, torch.bfloat16, fill=dy.cuda())
    wd, w_ok = R.guarded(N, K, torch.bfloat16, fill=w.cuda())
    x8, x_ok = R.guarded_copy(M, K)
    codes, scales = R.copy8(x)
    x8.codes.copy_(torch.from_numpy(codes))
    x8.scales.copy_(torch.from_numpy(scales))
    dx, dx_ok = R.guarded(M, K, torch.bfloat16)
    dw, dw_ok = R.guarded(N, K, torch.float32, fill=torch.full((N, K), 3.0, device="cuda"))
    need = B.nvfp4_linear_bf16_bwd8_workspace_bytes(M, K)
    held = torch.full((need + 512,), 77, dtype=torch.uint8, device="cuda")
    at = -held.data_ptr() % 256
    for tile in (0, 512, 640, 642, 644):
        dw.fill_(3.0)
        dx.fill_(float("nan"))
        B.nvfp4_set_gemm_tile_n(tile)
        try:
            B.nvfp4_linear_bf16_bwd8(dyd, x8, wd, dx, dw, held[at:at + need], accumulate_dw=True)
            B.nvfp4_device_status()
        finally:
            B.nvfp4_set_gemm_tile_n(0)
        assert np.array_equal(R.f64(dw), R.f64(dy).T @ x + 3.0), tile
        assert np.array_equal(R.f64(dx), torch.from_numpy(R.f64(dy) @ R.f64(w)).to(torch.bfloat16).double().numpy()), tile
        assert all(ok() for ok in (dy_ok, w_ok, x_ok, dx_ok, dw_ok)), tile
        assert bool((held[:at] == 77).all()) and bool((held[at + need:] == 77).all()), tile


def steps_off(M, N, K, seed):
    """Codes of z = A B^T + bias that are not those of z in 64 bits: of the call's and of a copy of the product in binary32."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    a, b = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16) for s in ((M, K), (N, K)))
    bias = torch.randn(N, generator=g, device="cuda") * K ** 0.5
    z, D = B.alloc_tensor(M, N, format=B.FORMAT_MXFP8), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    B.nvfp4_gemm_bf16_epilogue(a, b, D, bias, z=z)
    B.nvfp4_device_status()
    exact = torch.cat([torch.addmm(bias.double(), p.double(), b.double().t()) for p in a.split(256)])
    blocks = exact.view(M, N // 32, 32)
    m, e = torch.frexp(blocks.abs().amax(2, keepdim=True))
    scale = torch.ldexp(torch.ones_like(m), torch.where(m <= 0.875, e - 9, e - 8))  # (448 = 0.875 * 2^9)
    v = blocks / scale
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v.abs().clamp_min(2.0 ** -6))[1] - 4)
    want = (torch.round(v / step) * step * scale).view(M, N)
    plain = B.alloc_tensor(M, N, format=B.FORMAT_MXFP8)
    torch.backends.cuda.matmul.allow_tf32 = False
    B.nvfp4_quantize(a.float() @ b.float().t() + bias, B.quant_opts(), plain)
    return (int((B.nvfp4_dequantize(q).double() != want).sum()) for q in (z, plain))


# rows, columns, contraction, draws: one, two, three and more shares of every length, each kernel
OFF = [(2048, 4096, K, 1) for K in (520, 776, 1024, 1096, 1536, 1608, 2048, 4096, 5120, 8200)]
OFF += [(32, 8192, 5120, 6), (32, 8192, 16384, 6), (16, 8192, 20480, 12), (8, 20480, 4096, 12), (8, 20480, 8200, 12), (1, 20480, 20480, 40)]
OFF += [(16, 8192, 4096, 16), (32, 8192, 4096, 12), (32, 5120, 20480, 12), (64, 8192, 4096, 8), (64, 5120, 20480, 8), (100, 8192, 4096, 6), (128, 5120, 16384, 6)]


@pytest.mark.parametrize("M,N,K,draws", OFF)
def test_codes_are_about_as_exact_as_those_of_binary32_sums(M, N, K, draws):
    """A code is a step off where the error of z carries it across a border, so their number goes with the error, and their error in the mean
    square with its root: 1.5 times that of binary32 sums is 2.25 times as many.  (Counts have deviations of their root: four of both.)"""
    mine = plain = 0
    for seed in range(draws):
        x, y = steps_off(M, N, K, 200 + seed)
        mine, plain = mine + x, plain + y
    assert mine <= 2.25 * plain + 4 * (mine + 2.25 ** 2 * plain) ** 0.5, (mine, plain)


def test_products_with_codes_beside_each_other():
    """Every kernel of the products that keep z in 8 bits, in two captured graphs that are replayed on two streams at once: the bits of direct calls."""
    shapes = [(8, 20480, 1032), (20, 5120, 5120), (64, 2568, 5120), (100, 5128, 4104), (300, 2056, 2568), (2048, 2304, 520)]

    def make(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
        calls = [(new(M, K), new(N, K), new(M, N), torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), B.alloc_tensor(M, N, format=B.FORMAT_MXFP8))
                 for M, N, K in shapes]

        def step():
            for a, b, res, D, z in calls:
                B.nvfp4_gemm_bf16_epilogue(a, b, D, None, B.ACT_SILU, res, z)
        return step, [t for _, _, _, D, z in calls for t in (D, z.codes, z.scales)]

    both, want = [make(300), make(400)], []
    for step, outs in both:
        step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    graphs, streams = [], [torch.cuda.Stream() for _ in both]
    for (step, outs), stream in zip(both, streams):
        for t in outs:
            t.fill_(77)
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(10):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    B.nvfp4_device_status()
    for (_, outs), ref in zip(both, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, ref))
