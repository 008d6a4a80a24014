"""Refusals of the operators around the linear layers, on the CPU: every call is turned down before anything is launched."""
import ctypes

import pytest
import torch

from paper_2509_25149_b200 import binding as B

FAKE = 0x7F0000000000  # never dereferenced: validation fails first
NULL, SHAPE, ALIGN, ARG, WORKSPACE = 1, 2, 3, 4, 5


def copy(rows=64, cols=128, codes=FAKE, scales=FAKE, layout=B.SF_LINEAR, fmt=B.FORMAT_MXFP8):
    return B.CTensor(codes, scales, None, rows, cols, layout, fmt)


@pytest.fixture(autouse=True)
def nothing_is_launched():
    before = B.lib().nvfp4_launch_count()
    yield
    assert B.lib().nvfp4_launch_count() == before


def test_copies():
    L, o = B.lib(), B.quant_opts()
    q = lambda t, x=FAKE, rows=64, cols=128, ld=128, opts=o, col=None: L.nvfp4_quantize(x, rows, cols, ld, ctypes.byref(opts), t, col, None)
    assert q(copy(), x=None) == NULL and q(copy(codes=None)) == NULL and q(copy(scales=None)) == NULL
    assert q(copy(cols=124), cols=124) == SHAPE and q(copy(rows=63)) == SHAPE and q(copy(), ld=120) == SHAPE
    assert q(copy(rows=0), rows=0) == SHAPE and q(copy(rows=-1), rows=-1) == SHAPE
    assert q(copy(), ld=132) == ALIGN and q(copy(), x=FAKE + 8) == ALIGN and q(copy(codes=FAKE + 8)) == ALIGN
    assert q(copy(layout=B.SF_SWIZZLED)) == ARG and q(copy(), col=copy(128, 64)) == ARG
    for bad in (dict(block_rows=32), dict(rounding=B.ROUND_STOCHASTIC), dict(rht_rowwise=True), dict(rht_colwise=True),
                dict(flags=B.AMAX_PROVIDED), dict(flags=B.SR_INDEPENDENT_COPIES)):
        assert q(copy(), opts=B.quant_opts(**bad)) == ARG, bad
    # as the transposed copy of another call, and as an operand of the products, it is no format
    assert q(None, col=copy(128, 64)) == ARG
    assert L.nvfp4_quantize(FAKE, 128, 128, 128, ctypes.byref(o), copy(128, 128, fmt=0), copy(128, 128), None) == ARG
    a = B.CTensor(FAKE, FAKE, FAKE, 256, 256, B.SF_SWIZZLED, B.FORMAT_MXFP8)
    assert L.nvfp4_gemm(a, a, FAKE, 0, 256, 0, None) == ARG
    assert L.nvfp4_quant_error(FAKE, 256, 256, 256, a, FAKE, None) == ARG
    assert L.nvfp4_linear_fwd(FAKE, FAKE, 256, 256, 256, ctypes.byref(o), FAKE, None, a, None, 0, FAKE, 1 << 30, None) == ARG
    d = L.nvfp4_dequantize_bf16
    assert d(None, FAKE, 128, None) == NULL and d(copy(), None, 128, None) == NULL
    assert d(copy(), FAKE, 120, None) == SHAPE and d(copy(), FAKE, 132, None) == ALIGN and d(copy(), FAKE + 2, 128, None) == ALIGN
    assert d(copy(fmt=0), FAKE, 128, None) == ARG and d(copy(rows=0), FAKE, 128, None) == SHAPE
    assert L.nvfp4_dequantize(copy(), None, None) == NULL and L.nvfp4_dequantize(copy(), FAKE + 4, None) == ALIGN


def norm(x=FAKE, ldx=128, res=FAKE, ldr=128, res32=0, gain=FAKE, rows=64, cols=128, eps=1e-5, h=FAKE, ldh=128, y=FAKE, ldy=128, y8=None,
         h8=None, rstd=FAKE):
    return B.lib().nvfp4_rmsnorm_fwd(x, ldx, res, ldr, res32, gain, rows, cols, eps, h, ldh, y, ldy, y8, h8, rstd, None)


def test_norm():
    assert norm(x=None) == NULL and norm(h=None, y=None, rstd=None) == NULL
    assert norm(rows=0) == SHAPE and norm(cols=0) == SHAPE and norm(cols=124) == SHAPE and norm(rows=(1 << 30) + 1) == SHAPE
    for name in ("ldx", "ldr", "ldh", "ldy"):
        assert norm(**{name: 120}) == SHAPE and norm(**{name: 132}) == ALIGN
    for name in ("x", "res", "h", "y", "gain"):
        assert norm(**{name: FAKE + 8}) == ALIGN
    assert norm(rstd=FAKE + 2) == ALIGN
    assert norm(res32=1, ldr=130) == ALIGN and norm(res32=1, ldh=130) == ALIGN
    for eps in (0.0, -1e-5, float("nan"), float("inf")):
        assert norm(eps=eps) == ARG
    assert norm(res=None) == ARG  # h without a residual
    assert norm(y8=copy(64, 136)) == SHAPE and norm(h8=copy(63, 128)) == SHAPE and norm(y8=copy(fmt=1)) == ARG
    assert norm(y8=copy(codes=None)) == NULL and norm(h8=copy(scales=FAKE + 1)) == ALIGN


def norm_bwd(dy=FAKE, lddy=128, h=FAKE, ldh=128, h32=0, h8=None, gain=FAKE, rstd=FAKE, rows=64, cols=128, rg=FAKE, ldrg=128, dh=FAKE, lddh=128,
             dh32=0, dgain=FAKE, acc=0, ws=FAKE, nws=1 << 30):
    return B.lib().nvfp4_rmsnorm_bwd(dy, lddy, h, ldh, h32, h8, gain, rstd, rows, cols, rg, ldrg, dh, lddh, dh32, dgain, acc, ws, nws, None)


def test_norm_gradient():
    for name in ("dy", "h", "rstd", "dh"):
        assert norm_bwd(**{name: None}) == NULL, name
    assert norm_bwd(h8=copy()) == ARG
    assert norm_bwd(rows=0) == SHAPE and norm_bwd(cols=12) == SHAPE
    for name in ("lddy", "ldh", "ldrg", "lddh"):
        assert norm_bwd(**{name: 120}) == SHAPE and norm_bwd(**{name: 132}) == ALIGN, name
    for name in ("dy", "h", "rg", "dh", "gain"):
        assert norm_bwd(**{name: FAKE + 8}) == ALIGN, name
    assert norm_bwd(h=None, h8=copy(64, 64)) == SHAPE and norm_bwd(h=None, h8=copy(fmt=2)) == ARG
    need = B.nvfp4_rmsnorm_bwd_workspace_bytes(64, 128)
    assert need >= 64 // 16 * 128 * 4
    assert norm_bwd(ws=None) == WORKSPACE and norm_bwd(nws=need - 1) == WORKSPACE and norm_bwd(ws=FAKE + 16) == ALIGN
    # rows too long for registers need it without dgain as well
    wide = dict(cols=20488, lddy=20488, ldh=20488, ldrg=20488, lddh=20488, dgain=None)
    assert norm_bwd(ws=None, **wide) == WORKSPACE
    assert B.nvfp4_rmsnorm_bwd_workspace_bytes(0, 8) == 0


def product(A=FAKE, lda=64, Bm=FAKE, ldb=64, M=5, N=128, K=64, D=FAKE, ldd=128, e=True, bias=0, residual=0, ldr=128, z=0, ldz=128, z8=0, act=0,
            reserved=0):
    epilogue = B._EPILOGUE_FIELDS.pack(bias, residual, ldr, z, ldz, z8, act, reserved) if e else None
    return B.lib().nvfp4_gemm_bf16_epilogue(A, lda, Bm, ldb, M, N, K, epilogue, D, ldd, None)


def test_product_with_an_epilogue():
    assert product(A=None) == NULL and product(Bm=None) == NULL and product(D=None) == NULL and product(e=False) == NULL
    assert product(M=0) == SHAPE and product(N=124) == SHAPE and product(K=60) == SHAPE and product(N=0) == SHAPE and product(K=0) == SHAPE
    assert product(lda=56) == SHAPE and product(ldb=56) == SHAPE and product(ldd=120) == SHAPE
    assert product(residual=FAKE, ldr=120) == SHAPE and product(z=FAKE, ldz=120) == SHAPE
    for name in ("lda", "ldb", "ldd"):
        assert product(**{name: 132}) == ALIGN, name
    assert product(residual=FAKE, ldr=132) == ALIGN and product(z=FAKE, ldz=132) == ALIGN
    for name in ("A", "Bm", "D", "bias", "residual", "z"):
        assert product(**{name: FAKE + 8}) == ALIGN, name
    assert product(act=-1) == ARG and product(act=4) == ARG and product(reserved=1) == ARG
    held = [copy(5, 128), copy(5, 136), copy(5, 128, fmt=1), copy(5, 128, codes=FAKE + 8)]
    at = [ctypes.addressof(t) for t in held]
    assert product(z=FAKE, z8=at[0]) == ARG
    assert product(z8=at[1]) == SHAPE and product(z8=at[2]) == ARG and product(z8=at[3]) == ALIGN
    assert B._EPILOGUE_FIELDS.size == 56


def test_the_epilogue_struct_is_packed_as_a_c_compiler_lays_it_out(tmp_path):
    import os
    import subprocess
    import sys
    src = tmp_path / "layout.c"
    src.write_text("""#include "nvfp4.h"
#include <stdio.h>
#define AT(f) (int)offsetof(nvfp4_epilogue, f)
int main(void) { printf("%d %d %d %d %d %d %d %d %d", (int)sizeof(nvfp4_epilogue), AT(bias), AT(residual), AT(ldr), AT(z_bf16), AT(ldz), AT(z8),
                        AT(act), AT(reserved)); return 0; }
""")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    said = [int(v) for v in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()]
    packed = B._EPILOGUE_FIELDS.pack(1, 2, 3, 4, 5, 6, 7, 8)
    assert said[0] == len(packed)
    assert [int.from_bytes(packed[o:o + 4], sys.byteorder) for o in said[1:]] == [1, 2, 3, 4, 5, 6, 7, 8]


def act_bwd(da=FAKE, ldda=128, z=FAKE, ldz=128, z8=None, act=1, rows=64, cols=128, dz=FAKE, lddz=128, a=FAKE, lda=128, dbias=FAKE, acc=0, ws=FAKE,
            nws=1 << 30):
    return B.lib().nvfp4_act_bwd(da, ldda, z, ldz, z8, act, rows, cols, dz, lddz, a, lda, dbias, acc, ws, nws, None)


def test_gradient_of_an_activation():
    assert act_bwd(da=None) == NULL and act_bwd(z=None) == NULL and act_bwd(dz=None, a=None, dbias=None) == NULL
    assert act_bwd(z=None, act=0) == NULL  # act(z) is asked for
    assert act_bwd(z8=copy()) == ARG and act_bwd(act=4) == ARG and act_bwd(act=-1) == ARG
    assert act_bwd(rows=0) == SHAPE and act_bwd(cols=100) == SHAPE
    for name in ("ldda", "ldz", "lddz", "lda"):
        assert act_bwd(**{name: 120}) == SHAPE and act_bwd(**{name: 132}) == ALIGN, name
    for name in ("da", "z", "dz", "a"):
        assert act_bwd(**{name: FAKE + 8}) == ALIGN, name
    assert act_bwd(dbias=FAKE + 2) == ALIGN
    assert act_bwd(z=None, z8=copy(64, 136)) == SHAPE and act_bwd(z=None, z8=copy(fmt=0)) == ARG
    need = B.nvfp4_act_bwd_workspace_bytes(64, 128)
    assert need >= 128 * 4
    assert act_bwd(ws=None) == WORKSPACE and act_bwd(nws=need - 1) == WORKSPACE and act_bwd(ws=FAKE + 64) == ALIGN


def test_layer_gradients_from_a_copy():
    f = lambda dY=FAKE, X=copy(64, 128), W=FAKE, M=64, N=256, K=128, dX=FAKE, dW=FAKE, ws=FAKE, nws=1 << 30: B.lib().nvfp4_linear_bf16_bwd8(
        dY, X, W, M, N, K, dX, dW, 0, ws, nws, None)
    assert f(dY=None) == NULL and f(X=None) == NULL and f(W=None) == NULL and f(dX=None, dW=None) == NULL
    assert f(M=0) == SHAPE and f(M=60, X=copy(60, 128)) == SHAPE and f(N=252) == SHAPE and f(K=120) == SHAPE
    assert f(X=copy(64, 128, fmt=1)) == ARG and f(dX=FAKE + 2) == ALIGN and f(dW=FAKE + 8) == ALIGN
    need = B.nvfp4_linear_bf16_bwd8_workspace_bytes(64, 128)
    assert need >= 64 * 128 * 2
    assert f(ws=None) == WORKSPACE and f(nws=need - 1) == WORKSPACE and f(ws=FAKE + 128) == ALIGN


def test_python_calls_refuse_what_is_no_matrix_of_theirs():
    x = torch.zeros(4, 16, dtype=torch.bfloat16)  # not on a GPU (and where there is none, the current device cannot be asked for)
    with pytest.raises((AssertionError, RuntimeError)):
        B.nvfp4_rmsnorm_fwd(x, None, 1e-5, x)
    with pytest.raises((AssertionError, RuntimeError)):
        B.nvfp4_act_bwd(x, x, B.ACT_SILU, x)
    with pytest.raises((AssertionError, RuntimeError)):
        B.nvfp4_gemm_bf16_epilogue(x, x, torch.zeros(4, 4, dtype=torch.bfloat16))
