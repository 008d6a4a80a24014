"""Refusals of the operators at the ends of a training step, on the CPU: every call is turned down before anything is launched."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2509_25149_b200 import binding as B

FAKE = 0x7F0000000000  # never dereferenced: validation fails first
NULL, SHAPE, ALIGN, ARG, WORKSPACE = 1, 2, 3, 4, 5
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(autouse=True)
def nothing_is_launched():
    before = B.lib().nvfp4_launch_count()
    yield
    assert B.lib().nvfp4_launch_count() == before


def heads(x=FAKE, ldx=768, rows=64, hq=4, hk=2, dim=128, gq=FAKE, gk=FAKE, eps=1e-5, f=FAKE, rotary=128, near=0, pos=FAKE, wide=1, y=FAKE + 64, ldy=768):
    return B.lib().nvfp4_headnorm_fwd(x, ldx, rows, hq, hk, dim, gq, gk, eps, f, rotary, near, pos, wide, y, ldy, None)


def heads_bwd(dy=FAKE, lddy=768, x=FAKE + 64, ldx=768, rows=64, hq=4, hk=2, dim=128, gq=FAKE, gk=FAKE, eps=1e-5, f=FAKE, rotary=128, near=0, pos=FAKE, wide=1,
              dx=FAKE + 128, lddx=768, dgq=FAKE, dgk=FAKE, acc=0, ws=FAKE, nws=1 << 30):
    return B.lib().nvfp4_headnorm_bwd(dy, lddy, x, ldx, rows, hq, hk, dim, gq, gk, eps, f, rotary, near, pos, wide, dx, lddx, dgq, dgk, acc, ws, nws, None)


@pytest.mark.parametrize("call, out, ldo", [(heads, "y", "ldy"), (heads_bwd, "dx", "lddx")])
def test_heads(call, out, ldo):
    for name in ("x", out, "f"):
        assert call(**{name: None}) == NULL, name
    for bad in (dict(rows=0), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(hq=0, hk=0), dict(hq=-1), dict(hk=-1), dict(dim=0), dict(dim=124), dict(dim=264),
                dict(rotary=-16), dict(rotary=24), dict(rotary=144), dict(ldx=760), {ldo: 760}, dict(hq=1 << 30, hk=1 << 30), dict(hq=(1 << 31) - 1, hk=1)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(ldx=772), {ldo: 772}, dict(x=FAKE + 8), {out: FAKE + 8}, dict(gq=FAKE + 8), dict(gk=FAKE + 4), dict(f=FAKE + 2), dict(pos=FAKE + 4),
                dict(pos=FAKE + 2, wide=0)):
        assert call(**bad) == ALIGN, bad
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert call(eps=eps) == ARG
    assert call(**{"x": FAKE + 64, out: FAKE + 64, "ldx": 776}) == ARG  # in place with another distance of the rows


def test_heads_gradient():
    assert heads_bwd(dy=None) == NULL and heads_bwd(lddy=760) == SHAPE and heads_bwd(lddy=772) == ALIGN and heads_bwd(dy=FAKE + 8) == ALIGN
    assert heads_bwd(dgq=FAKE + 2) == ALIGN and heads_bwd(dgk=FAKE + 2) == ALIGN
    assert heads_bwd(dx=FAKE, lddy=776) == ARG
    need = B.nvfp4_headnorm_bwd_workspace_bytes(64, 4, 2, 128)
    assert need > 0 and heads_bwd(ws=None) == WORKSPACE and heads_bwd(nws=need - 1) == WORKSPACE and heads_bwd(ws=FAKE + 128) == ALIGN
    assert B.nvfp4_headnorm_bwd_workspace_bytes(0, 4, 2, 128) == 0 == B.nvfp4_headnorm_bwd_workspace_bytes(64, 4, 2, 12)


def embed(tokens=FAKE, wide=1, n=10, table=FAKE, t32=0, ldt=128, vocab=50, cols=128, scale=1.0, out=FAKE, o32=0, ldo=128):
    return B.lib().nvfp4_embedding_fwd(tokens, wide, n, table, t32, ldt, vocab, cols, scale, out, o32, ldo, None)


def embed_bwd(tokens=FAKE, wide=1, n=10, table=FAKE, t32=0, ldt=128, vocab=50, cols=128, scale=1.0, out=FAKE, o32=1, ldo=128, acc=0, ws=FAKE, nws=1 << 30):
    return B.lib().nvfp4_embedding_bwd(tokens, wide, n, out, 0, ldo, vocab, cols, scale, table, ldt, acc, ws, nws, None)


@pytest.mark.parametrize("call", [embed, embed_bwd])
def test_embedding(call):
    for name in ("tokens", "table", "out"):
        assert call(**{name: None}) == NULL
    for bad in (dict(n=0), dict(n=-1), dict(n=(1 << 30) + 1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(cols=0), dict(cols=124), dict(ldt=120), dict(ldo=120)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(tokens=FAKE + 4), dict(tokens=FAKE + 2, wide=0), dict(table=FAKE + 8), dict(out=FAKE + 8), dict(ldo=132), dict(ldt=130)):
        assert call(**bad) == ALIGN, bad
    for scale in (float("nan"), float("inf")):
        assert call(scale=scale) == ARG


def test_embedding_gradient():
    need = B.nvfp4_embedding_bwd_workspace_bytes(10, 50, 128)
    assert need > 0 and embed_bwd(ws=None) == WORKSPACE and embed_bwd(nws=need - 1) == WORKSPACE and embed_bwd(ws=FAKE + 16) == ALIGN
    assert B.nvfp4_embedding_bwd_workspace_bytes(0, 50, 128) == 0


def logprob(x=FAKE, f32=0, ld=128, rows=4, vocab=100, t=FAKE, wide=1, scale=1.0, lp=FAKE, lse=FAKE, stats=FAKE, ent=FAKE, top=5, ids=FAKE, tlp=FAKE):
    return B.lib().nvfp4_logprob_fwd(x, f32, ld, rows, vocab, t, wide, scale, lp, lse, stats, ent, top, ids, tlp, None)


def logprob_bwd(x=FAKE, f32=0, ld=128, rows=4, vocab=100, t=FAKE, wide=1, scale=1.0, stats=FAKE, ent=FAKE, dlp=FAKE, de=FAKE, dx=FAKE + 64, d32=0, lddl=128, dcols=104):
    return B.lib().nvfp4_logprob_bwd(x, f32, ld, rows, vocab, t, wide, scale, stats, ent, dlp, de, dx, d32, lddl, dcols, None)


@pytest.mark.parametrize("call", [logprob, logprob_bwd])
def test_logprob(call):
    assert call(x=None) == NULL and call(t=None) == NULL
    for bad in (dict(rows=0), dict(rows=(1 << 30) + 1), dict(vocab=0), dict(vocab=-1), dict(ld=96)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(ld=132), dict(x=FAKE + 8), dict(t=FAKE + 4), dict(t=FAKE + 2, wide=0), dict(stats=FAKE + 4), dict(ent=FAKE + 2), dict(f32=1, ld=130)):
        assert call(**bad) == ALIGN, bad
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e-38, 1e38):
        assert call(scale=scale) == ARG


def test_logprob_outputs():
    assert logprob(lp=None, lse=None, stats=None, ent=None, ids=None, tlp=None) == NULL
    for top in (0, -1, 33):
        assert logprob(top=top) == SHAPE and logprob(top=top, ids=None) == SHAPE
    assert logprob(top=8, vocab=7) == SHAPE
    for name in ("lp", "lse", "ids", "tlp"):
        assert logprob(**{name: FAKE + 2}) == ALIGN
    for name in ("stats", "dx"):
        assert logprob_bwd(**{name: None}) == NULL
    assert logprob_bwd(dlp=None, de=None) == NULL and logprob_bwd(ent=None) == NULL
    assert logprob_bwd(dcols=99) == SHAPE and logprob_bwd(lddl=96) == SHAPE and logprob_bwd(dcols=136) == SHAPE and logprob_bwd(lddl=132) == ALIGN
    assert logprob_bwd(dx=FAKE + 8) == ALIGN and logprob_bwd(dlp=FAKE + 2) == ALIGN and logprob_bwd(de=FAKE + 2) == ALIGN
    assert logprob_bwd(dx=FAKE, d32=1) == ARG and logprob_bwd(dx=FAKE, lddl=136) == ARG


def packed(*fields):
    return b"".join(B._GRAD_FIELDS.pack(*f) for f in fields)


def test_clipping():
    L = B.lib()
    good = (FAKE, FAKE, 10, 1, 1)
    norm = lambda g, n=1, total=FAKE, ws=FAKE, nws=1 << 30: L.nvfp4_grad_sq_norm(g, n, total, 0, ws, nws, None)
    clip = lambda g, n=1, total=FAKE, most=1.0, stats=FAKE: L.nvfp4_grad_clip(g, n, total, most, stats, None)
    for call in (norm, clip):
        assert call(None) == NULL and call(packed(good), total=None) == NULL and call(packed(good), n=0) == SHAPE and call(packed(good), n=-1) == SHAPE
        assert call(packed(good), total=FAKE + 4) == ALIGN
        assert call(packed(good, (FAKE, 0, -1, 1, 1)), n=2) == SHAPE and call(packed(good, (0, 0, 1, 1, 1)), n=2) == NULL
        assert call(packed((FAKE + 2, 0, 1, 1, 1))) == ALIGN and call(packed((FAKE + 1, 0, 1, 0, 1))) == ALIGN and call(packed((FAKE, 0, 1 << 41, 0, 1))) == SHAPE
    assert norm(packed(good), ws=None) == WORKSPACE and norm(packed(good), nws=B.nvfp4_grad_sq_norm_workspace_bytes() - 1) == WORKSPACE
    assert norm(packed(good), ws=FAKE + 8) == ALIGN
    for most in (0.0, -1.0, float("nan"), float("inf")):
        assert clip(packed(good), most=most) == ARG
    assert clip(packed(good), stats=FAKE + 2) == ALIGN
    assert clip(packed((FAKE, FAKE + 2, 1, 1, 1))) == ALIGN and clip(packed((FAKE, FAKE, 1, 1, 0))) == ARG


def test_the_bindings_check_their_tensors():
    cpu = torch.zeros(4, 64, dtype=torch.bfloat16)
    calls = (lambda: B.grad_list([cpu]), lambda: B.grad_list([]), lambda: B.grad_list([cpu], []))
    for call in calls:
        with pytest.raises(AssertionError):
            call()


def test_layout_of_the_list_matches_the_header(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "nvfp4.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu %d", sizeof(nvfp4_grad), offsetof(nvfp4_grad, out), '
                   'offsetof(nvfp4_grad, count), offsetof(nvfp4_grad, is_fp32), offsetof(nvfp4_grad, out_is_fp32), sizeof(void*), NVFP4_TOP_MAX); return 0; }\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    out = [int(v) for v in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    assert out == [B._GRAD_FIELDS.size, 8, 16, 24, 28, 8, 32]
