"""Refusals of the attention block's operators at the C ABI: checked on the host before anything is launched, so they need no GPU."""
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


def test_head_norm_rope(L):
    def fwd(q=FAKE, ldq=256, k=FAKE, ldk=128, dt=1, T=4, H=4, KV=2, D=64, norm=1, wq=FAKE, wk=FAKE, eps=1e-6, pos=FAKE, axes=1, axis=None,
            f=FAKE, n=32, nb=0, yq=FAKE, ldyq=256, yk=FAKE, ldyk=128):
        return L.efqat_head_norm_rope_fwd(q, ldq, k, ldk, dt, T, H, KV, D, norm, wq, wk, eps, pos, axes, axis, f, n, nb, yq, ldyq, yk, ldyk, None)

    need = L.efqat_head_norm_rope_bwd_workspace_bytes(4, 4, 2, 64)
    assert need >= 2 * 64 * 4 and need % 256 == 0
    assert L.efqat_head_norm_rope_bwd_workspace_bytes(0, 4, 2, 64) == L.efqat_head_norm_rope_bwd_workspace_bytes(4, 4, 2, 257) == 256
    assert L.efqat_head_norm_rope_bwd_workspace_bytes(1 << 20, 64, 8, 128) >= 2 * 128 * 4

    def bwd(q=FAKE, ldq=256, k=FAKE, ldk=128, dt=1, T=4, H=4, KV=2, D=64, norm=1, wq=FAKE, wk=FAKE, eps=1e-6, pos=FAKE, axes=1, axis=None,
            f=FAKE, n=32, nb=0, yq=FAKE, ldyq=256, yk=FAKE, ldyk=128, dyq=FAKE, lddyq=256, dyk=FAKE, lddyk=128, dwq=FAKE, dwk=FAKE, ws=FAKE,
            wsb=need):
        return L.efqat_head_norm_rope_bwd(dyq, lddyq, dyk, lddyk, q, ldq, k, ldk, dt, T, H, KV, D, norm, wq, wk, eps, pos, axes, axis, f, n, nb,
                                          yq, ldyq, yk, ldyk, dwq, dwk, ws, wsb, None)

    for g in (fwd, bwd):
        assert g(q=None) == g(yq=None) == g(k=None) == g(yk=None) == g(pos=None) == g(f=None) == g(axes=2) == NULL
        assert g(T=0) == g(H=0) == g(KV=-1) == g(D=0) == g(D=257, ldq=2000) == g(n=33) == g(n=-1) == g(axes=0) == g(axes=17, axis=FAKE) == SHAPE
        assert g(ldq=255) == g(ldk=127) == g(ldyq=255) == g(ldyk=127) == g(eps=-1.0) == g(eps=float("nan")) == g(T=(1 << 28) + 1) == SHAPE
        assert g(dt=2) == DTYPE and g(norm=2) == g(nb=-1) == LAYOUT
        assert g(q=FAKE + 1) == g(wq=FAKE + 2) == g(pos=FAKE + 2) == g(f=FAKE + 1) == g(yk=FAKE + 1) == g(dt=0, q=FAKE + 2) == ALIGN
    assert bwd(dyq=None) == bwd(dyk=None) == bwd(ws=None) == NULL and bwd(lddyq=255) == bwd(lddyk=127) == SHAPE
    assert bwd(wsb=need - 1) == WORKSPACE and bwd(ws=FAKE + 128) == bwd(dwq=FAKE + 2) == ALIGN and bwd(norm=0) == LAYOUT


def _attn(**kw):
    a = dict(q=FAKE, ldq=256, k=FAKE, ldk=128, v=FAKE, ldv=128, dt=1, Tq=12, Tk=12, n=2, qs=None, ks=None, H=4, KV=2, D=64, scale=0.125, causal=1,
             window=0, sinks=0)
    a.update(kw)
    return a


def test_attention(L):
    extra = dict(o=FAKE, ldo=256, lse=FAKE, do=FAKE, lddo=256, dq=FAKE, lddq=256, dk=FAKE, lddk=128, dv=FAKE, lddv=128, ws=FAKE)
    query = L.efqat_attention_bwd_workspace_bytes
    need = max(query(12, 12, 2, packed, 4, 2, 64, dt, 1, 0, 0) for packed in (0, 1) for dt in (0, 1))
    assert query(12, 12, 2, 0, 4, 2, 64, 1, 1, 0, 0) >= 12 * 4 * 4
    assert query(0, 12, 2, 0, 4, 2, 64, 1, 1, 0, 0) == query(12, 13, 2, 0, 4, 2, 64, 1, 1, 0, 0) == query(12, 12, 2, 0, 4, 3, 64, 1, 1, 0, 0) == 256
    least = query(12, 12, 2, 0, 4, 2, 64, 1, 1, 0, 0)

    def fwd(wsb=None, **kw):
        a = {**_attn(), **extra, **kw}
        return L.efqat_attention_fwd(*(a[x] for x in ("q ldq k ldk v ldv dt Tq Tk n qs ks H KV D scale causal window sinks o ldo lse".split())), None)

    def bwd(wsb=need, **kw):
        a = {**_attn(), **extra, **kw}
        return L.efqat_attention_bwd(*(a[x] for x in ("do lddo q ldq k ldk v ldv o ldo lse dt Tq Tk n qs ks H KV D scale causal window sinks dq lddq dk lddk "
                                                       "dv lddv ws".split())), wsb, None)

    for f in (fwd, bwd):
        assert f(q=None) == f(k=None) == f(v=None) == f(o=None) == f(qs=FAKE) == f(ks=FAKE) == NULL
        assert f(Tq=0) == f(Tk=0) == f(n=0) == f(Tq=13) == f(Tk=13) == f(H=3) == f(KV=0) == f(H=0) == SHAPE
        assert f(D=4) == f(D=60) == f(D=136, ldq=1000, ldk=1000, ldv=1000) == f(D=0) == SHAPE
        assert f(window=-1) == f(sinks=-1) == f(scale=0.0) == f(scale=-1.0) == f(scale=float("inf")) == f(scale=float("nan")) == SHAPE
        assert f(ldq=248) == f(ldk=120) == f(ldv=120) == f(ldo=248) == f(ldq=(1 << 24) + 8) == f(Tq=(1 << 28) + 2) == SHAPE
        assert f(dt=2) == DTYPE and f(causal=2) == LAYOUT
        assert f(q=FAKE + 8) == f(k=FAKE + 2) == f(ldq=260) == f(ldk=132) == f(ldv=129) == f(o=FAKE + 4) == f(lse=FAKE + 2) == ALIGN
        assert f(qs=FAKE + 2, ks=FAKE) == f(dt=0, ldq=258) == ALIGN
        assert f(Tq=1 << 28, Tk=1 << 28, n=1, H=16, KV=16, ldq=1024, ldk=1024, ldv=1024, ldo=1024, lddo=1024, lddq=1024, lddk=1024, lddv=1024, wsb=1 << 50) == SHAPE
    assert bwd(do=None) == bwd(lse=None) == bwd(dq=None) == bwd(dk=None) == bwd(dv=None) == bwd(ws=None) == NULL
    assert bwd(lddo=248) == bwd(lddq=248) == bwd(lddk=120) == bwd(lddv=120) == SHAPE and bwd(wsb=least - 1) == WORKSPACE
    assert bwd(ws=FAKE + 128) == bwd(do=FAKE + 8) == bwd(lddv=132) == ALIGN


def test_attention_backward_grids(L):
    """dk and dv of bf16 heads beyond 64 features take blocks of 512 lanes: no grid of 2^32 lanes and more is launched"""
    n, heads, cols = 1 << 20, 10, 1280
    blocks = (n // 128 + n - 1) * heads
    assert blocks * 256 < 2 ** 32 <= blocks * 512
    assert L.efqat_attention_bwd(FAKE, cols, FAKE, cols, FAKE, cols, FAKE, cols, FAKE, cols, FAKE, 1, n, n, n, FAKE, FAKE, heads, heads, 128, 0.1, 1, 0, 0,
                                 2 * FAKE, cols, 3 * FAKE, cols, 4 * FAKE, cols, FAKE, 1 << 50, None) == SHAPE


def test_attention_results_lie_apart(L):
    """the kernel of dk and dv reads q and do after dq was written, other blocks read keys and values"""
    at = {x: FAKE * (i + 2) for i, x in enumerate("q k v o do dq dk dv".split())}

    def call(fn, **kw):
        p = {**at, **kw}
        if fn == "fwd":
            return L.efqat_attention_fwd(p["q"], 256, p["k"], 256, p["v"], 256, 1, 8, 8, 1, None, None, 4, 4, 64, 0.1, 1, 0, 0, p["o"], 256, None, None)
        if fn == "decode":
            return L.efqat_attention_decode(p["q"], 256, p["k"], 256, 0, p["v"], 256, 0, 1, 1, 8, FAKE, 4, 4, 64, 0.1, 0, 0, p["o"], 256, FAKE, 1 << 20, None)
        return L.efqat_attention_bwd(p["do"], 256, p["q"], 256, p["k"], 256, p["v"], 256, p["o"], 256, FAKE, 1, 8, 8, 1, None, None, 4, 4, 64, 0.1, 1, 0, 0,
                                     p["dq"], 256, p["dk"], 256, p["dv"], 256, FAKE, 1 << 20, None)

    for fn in ("fwd", "decode"):
        assert [call(fn, o=at[x]) for x in "qkv"] == [LAYOUT] * 3
    for out in ("dq", "dk", "dv"):
        assert [call("bwd", **{out: at[x]}) for x in at if x != out] == [LAYOUT] * 7


def test_attention_decode(L):
    need = L.efqat_attention_decode_workspace_bytes(2, 4096, 4, 2, 64, 0, 0)
    assert need > 256 and L.efqat_attention_decode_workspace_bytes(2, 1, 4, 2, 64, 0, 0) == 256
    assert L.efqat_attention_decode_workspace_bytes(0, 1, 4, 2, 64, 0, 0) == L.efqat_attention_decode_workspace_bytes(1, 1 << 20, 4, 3, 64, 0, 0) == 256

    def f(q=FAKE, ldq=256, k=FAKE, ldk=128, sk=4096 * 128, v=FAKE, ldv=128, sv=4096 * 128, dt=1, n=2, cap=4096, lens=FAKE, H=4, KV=2, D=64, scale=0.1,
          window=0, sinks=0, o=FAKE, ldo=256, ws=FAKE, wsb=need):
        return L.efqat_attention_decode(q, ldq, k, ldk, sk, v, ldv, sv, dt, n, cap, lens, H, KV, D, scale, window, sinks, o, ldo, ws, wsb, None)

    assert f(q=None) == f(k=None) == f(v=None) == f(lens=None) == f(o=None) == f(ws=None) == NULL
    assert f(n=0) == f(cap=0) == f(H=5) == f(D=12) == f(scale=0.0) == f(window=-1) == f(ldo=248) == f(ldk=120) == f(sk=-8) == SHAPE
    assert f(sv=-128) == f(n=65536) == SHAPE and f(dt=7) == DTYPE and f(wsb=need - 1) == WORKSPACE
    assert f(lens=FAKE + 2) == f(k=FAKE + 8) == f(sk=4096 * 128 + 4) == f(ws=FAKE + 64) == f(ldv=132, sv=4096 * 132) == ALIGN


def test_dropout(L):
    def f(x=FAKE, ldx=9, res=None, ldr=0, dt=0, rows=2, cols=9, p=0.5, state=FAKE, y=FAKE, ldy=9):
        return L.efqat_dropout(x, ldx, res, ldr, dt, rows, cols, p, state, y, ldy, None)

    assert f(x=None) == f(y=None) == f(state=None) == NULL
    assert f(rows=0) == f(cols=0) == f(cols=1 << 31, ldx=1 << 40, ldy=1 << 40) == f(ldx=8) == f(ldy=8) == f(res=FAKE, ldr=8) == f(p=-0.1) == f(p=1.1) == f(p=float("nan")) == f(rows=(1 << 34) + 1) == SHAPE
    assert f(dt=2) == DTYPE and f(x=FAKE + 2) == f(state=FAKE + 4) == f(y=FAKE + 1, dt=1) == f(res=FAKE + 1, ldr=9) == ALIGN
