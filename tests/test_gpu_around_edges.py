"""Where the operators around the linear layers have little room: long contractions whose codes must not show how the tensor cores add."""
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
