"""Refusals of the operators between the quantized layers at the C ABI: checked on the host before anything is launched, so they
need no GPU."""
import pytest

import paper_2411_11038_amd as ef

FAKE = 0x1000          # non-NULL, 256-byte aligned; never dereferenced because validation fails first
NULL, SHAPE, LAYOUT, WORKSPACE, DTYPE, ALIGN = -1, -2, -5, -6, -8, -9


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(ef.lib_path()):
        from paper_2411_11038_amd import build
        build.build()
    return ef.lib()


def test_checkpoints(L):
    assert [L.efqat_ckpt8_pitch(c) for c in (-1, 0, 1, 16, 17, 4096)] == [0, 0, 16, 16, 32, 4096]

    def save(x=FAKE, ld=8, dt=0, rows=2, cols=8, codes=FAKE, scales=FAKE):
        return L.efqat_ckpt8_save(x, ld, dt, rows, cols, codes, scales, None)

    def load(codes=FAKE, scales=FAKE, rows=2, cols=8, x=FAKE, ld=8, dt=0):
        return L.efqat_ckpt8_load(codes, scales, rows, cols, x, ld, dt, None)

    for f in (save, load):
        assert f(x=None) == f(codes=None) == f(scales=None) == NULL
        assert f(rows=0) == f(cols=0) == f(rows=-1) == f(ld=7) == f(rows=1 << 41) == f(cols=1 << 31, ld=1 << 40) == SHAPE
        assert f(dt=2) == DTYPE
        assert f(x=FAKE + 2) == f(x=FAKE + 1, dt=1) == f(codes=FAKE + 8) == f(scales=FAKE + 2) == ALIGN


def test_activation(L):
    def fwd(x=FAKE, ldx=8, up=None, ldu=0, dt=1, rows=2, cols=8, kind=0, y=FAKE, ldy=8, xc=None, xs=None, uc=None, us=None):
        return L.efqat_act_fwd(x, ldx, up, ldu, dt, rows, cols, kind, y, ldy, xc, xs, uc, us, None)

    def bwd(dy=FAKE, lddy=8, dt=1, rows=2, cols=8, kind=1, xc=FAKE, xs=FAKE, uc=None, us=None, dx=FAKE, lddx=8, dup=None, lddup=0):
        return L.efqat_act_bwd(dy, lddy, dt, rows, cols, kind, xc, xs, uc, us, dx, lddx, dup, lddup, None)

    assert fwd(x=None) == fwd(y=None) == fwd(xc=FAKE) == fwd(xs=FAKE) == fwd(up=FAKE, ldu=8, xc=FAKE, xs=FAKE) == NULL
    assert fwd(up=FAKE, ldu=8, xc=FAKE, xs=FAKE, uc=FAKE) == NULL
    assert fwd(rows=0) == fwd(ldx=7) == fwd(ldy=7) == fwd(up=FAKE, ldu=7) == SHAPE
    assert fwd(dt=3) == DTYPE and fwd(kind=2) == LAYOUT
    assert fwd(x=FAKE + 1) == fwd(y=FAKE + 1) == fwd(up=FAKE + 1, ldu=8) == fwd(xc=FAKE + 4, xs=FAKE) == fwd(xc=FAKE, xs=FAKE + 2) == ALIGN
    assert bwd(dy=None) == bwd(xc=None) == bwd(xs=None) == bwd(dx=None) == NULL
    assert bwd(uc=FAKE, us=FAKE, lddup=8) == bwd(uc=FAKE, dup=FAKE, lddup=8) == bwd(dup=FAKE, lddup=8) == NULL
    assert bwd(rows=0) == bwd(cols=0) == bwd(lddy=7) == bwd(lddx=7) == bwd(uc=FAKE, us=FAKE, dup=FAKE, lddup=7) == SHAPE
    assert bwd(dt=-1) == DTYPE and bwd(kind=-1) == LAYOUT
    assert bwd(dy=FAKE + 1) == bwd(dx=FAKE + 1) == bwd(xc=FAKE + 1) == bwd(xs=FAKE + 1) == ALIGN


def test_layer_norm(L):
    def fwd(x=FAKE, ldx=8, dt=0, rows=2, cols=8, w=FAKE, b=FAKE, eps=1e-5, y=FAKE, ldy=8, mean=FAKE, rstd=FAKE, xc=None, xs=None):
        return L.efqat_layer_norm_fwd(x, ldx, dt, rows, cols, w, b, eps, y, ldy, mean, rstd, xc, xs, None)

    assert fwd(x=None) == fwd(y=None) == fwd(xc=FAKE) == fwd(xs=FAKE) == NULL
    assert fwd(rows=0) == fwd(cols=0) == fwd(ldx=7) == fwd(ldy=7) == fwd(eps=-1.0) == fwd(eps=float("nan")) == SHAPE
    assert fwd(dt=5) == DTYPE
    assert fwd(x=FAKE + 2) == fwd(w=FAKE + 2) == fwd(b=FAKE + 1) == fwd(mean=FAKE + 2) == fwd(xc=FAKE + 8, xs=FAKE) == ALIGN
    need = L.efqat_layer_norm_bwd_workspace_bytes(4096, 768)
    assert need >= 2 * 2 * 768 * 4 and L.efqat_layer_norm_bwd_workspace_bytes(1, 768) >= 256
    assert L.efqat_layer_norm_bwd_workspace_bytes(0, 8) == L.efqat_layer_norm_bwd_workspace_bytes(8, -1) == 256

    def bwd(dy=FAKE, lddy=768, dt=0, x=FAKE, ldx=768, xc=None, xs=None, mean=FAKE, rstd=FAKE, w=FAKE, rows=4096, cols=768, dx=FAKE,
            lddx=768, dw=FAKE, db=FAKE, ws=FAKE, wsb=need):
        return L.efqat_layer_norm_bwd(dy, lddy, dt, x, ldx, xc, xs, mean, rstd, w, rows, cols, dx, lddx, dw, db, ws, wsb, None)

    assert bwd(dy=None) == bwd(dx=None) == bwd(mean=None) == bwd(rstd=None) == bwd(ws=None) == bwd(x=None) == bwd(x=None, xc=FAKE) == NULL
    assert bwd(rows=0) == bwd(cols=0) == bwd(lddy=767) == bwd(ldx=767) == bwd(lddx=767) == SHAPE
    assert bwd(dt=2) == DTYPE and bwd(wsb=need - 1) == WORKSPACE
    assert bwd(dy=FAKE + 2) == bwd(dw=FAKE + 2) == bwd(ws=FAKE + 128) == bwd(x=None, xc=FAKE + 8, xs=FAKE) == ALIGN


def test_cross_entropy(L):
    fneed, bneed = L.efqat_linear_xent_fwd_workspace_bytes(100, 64, 1000, 1), L.efqat_linear_xent_bwd_workspace_bytes(100, 64, 1000, 1)
    assert fneed > 100 * 64 * 2 and bneed > 100 * 1000 * 2
    assert L.efqat_linear_xent_fwd_workspace_bytes(0, 64, 10, 1) == L.efqat_linear_xent_bwd_workspace_bytes(1, 64, 10, 4) == 256

    def fwd(h=FAKE, ldh=64, w=FAKE, ldw=64, dt=1, T=100, D=64, V=1000, t=FAKE, red=1, loss=FAKE, lse=FAKE, n=None, ws=FAKE, wsb=fneed):
        return L.efqat_linear_xent_fwd(h, ldh, w, ldw, dt, T, D, V, t, -100, red, loss, lse, n, ws, wsb, None)

    def bwd(h=FAKE, ldh=64, w=FAKE, ldw=64, dt=1, T=100, D=64, V=1000, t=FAKE, red=1, lse=FAKE, dloss=None, dh=FAKE, lddh=64, dw=FAKE,
            lddw=64, ws=FAKE, wsb=bneed):
        return L.efqat_linear_xent_bwd(h, ldh, w, ldw, dt, T, D, V, t, -100, red, lse, dloss, dh, lddh, dw, lddw, ws, wsb, None)

    for f, need in ((fwd, fneed), (bwd, bneed)):
        assert f(h=None) == f(w=None) == f(t=None) == f(lse=None) == f(ws=None) == NULL
        assert f(T=0) == f(D=0) == f(V=0) == f(ldh=63) == f(ldw=63) == f(T=(1 << 30) + 1) == f(D=(1 << 20) + 1, ldh=1 << 21, ldw=1 << 21) == SHAPE
        assert f(dt=2) == DTYPE and f(red=3) == f(red=-1) == LAYOUT and f(wsb=need - 1) == WORKSPACE
        assert f(h=FAKE + 1) == f(t=FAKE + 4) == f(ws=FAKE + 8) == f(lse=FAKE + 2) == ALIGN
        assert f(w=FAKE + 2) == f(ldw=68) == ALIGN                       # whole stages of a bf16 row are read 16 bytes at a time
    assert fwd(loss=None) == NULL and fwd(loss=FAKE + 2) == fwd(n=FAKE + 2) == ALIGN
    assert bwd(dh=None, dw=None) == NULL and bwd(lddh=63) == bwd(lddw=63) == SHAPE and bwd(dloss=FAKE + 1) == bwd(dw=FAKE + 1) == ALIGN
