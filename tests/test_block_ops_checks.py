"""What the entry points around the linears refuse before anything is launched, on the host."""
import ctypes

import pytest
import torch

from paper_2510_27527_b200 import binding as b

L = b.lib
P, Q, R, S, T = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000  # aligned addresses that nothing looks at
OK, NULL, SHAPE, ALIGN, ENUM, WORKSPACE, LIMIT = 0, 1, 2, 3, 4, 5, 9


def _gemv(**change):
    a = dict(X=P, ldx=64, M=2, D=64, codes=Q, sf=R, gscale=S, N=40, K=64, gs=0, layout=1, keep=None, outl=None, n_out=0, wo=None, bias=None, Y=T, yt=0, ldy=40, ws=None, n=0)
    a.update(change)
    w = b.COperand(a["codes"], a["sf"], a["gscale"], a["N"], a["K"], a["gs"], a["layout"])
    return L.nvfp4_gemv(a["X"], a["ldx"], a["M"], a["D"], ctypes.byref(w), a["keep"], a["outl"], a["n_out"], a["wo"], a["bias"], a["Y"], a["yt"], a["ldy"], None, a["ws"], a["n"], None)


@pytest.mark.parametrize("change,status", [
    (dict(M=0), OK), (dict(N=0), OK), (dict(X=None), NULL), (dict(Y=None), NULL), (dict(codes=None), NULL), (dict(sf=None), NULL), (dict(gscale=None), NULL),
    (dict(gs=3), ENUM), (dict(layout=2), ENUM), (dict(layout=0), ENUM), (dict(yt=2), ENUM), (dict(M=-1), SHAPE), (dict(D=0, K=0), SHAPE), (dict(K=32), SHAPE), (dict(N=-1), SHAPE),
    (dict(M=3), WORKSPACE), (dict(M=3, ws=P, n=511), WORKSPACE), (dict(M=3, ws=P + 8, n=1 << 20), WORKSPACE), (dict(K=60, n_out=4), NULL), (dict(K=60, n_out=4, keep=P, outl=P), NULL), (dict(K=60, n_out=4, keep=P, outl=P, wo=P + 8), ALIGN),
    (dict(n_out=-1, K=65), SHAPE), (dict(X=P + 8), ALIGN), (dict(ldx=60), ALIGN), (dict(ldx=56), ALIGN), (dict(Y=T + 4), ALIGN), (dict(ldy=36), ALIGN), (dict(ldy=44), ALIGN),
    (dict(codes=Q + 8), ALIGN), (dict(gscale=S + 2), ALIGN), (dict(bias=P + 1), ALIGN), (dict(M=65535 * 32 + 1), LIMIT), (dict(D=(1 << 24) + 8, K=(1 << 24) + 8, ldx=(1 << 24) + 8), LIMIT)])
def test_gemv(change, status):
    assert _gemv(**change) == status
    assert [L.nvfp4_gemv_workspace_bytes(m, 64, 0) for m in (0, 1, 2)] == [0, 0, 0] and L.nvfp4_gemv_workspace_bytes(5, 64, 0) == 5 * 512 + 64
    assert L.nvfp4_gemv(P, 64, 2, 64, None, None, None, 0, None, None, T, 0, 40, None, None, 0, None) == NULL


def _ck(codes=P, scales=Q, R=4, K=40):
    return ctypes.byref(b.CCkpt8(codes, scales, R, K))


def test_checkpoints():
    assert [L.nvfp4_ckpt8_ld(k) for k in (1, 32, 33, 2816)] == [32, 32, 64, 2816]
    pack = lambda X=R, t=0, ld=40, r=4, k=40, out=_ck(): L.nvfp4_ckpt8_pack(X, t, ld, r, k, out, None)  # noqa: E731
    assert pack(out=None) == NULL and pack(X=None) == NULL and pack(out=_ck(codes=None)) == NULL and pack(out=_ck(scales=None)) == NULL
    assert pack(t=2) == ENUM and pack(t=-1) == ENUM and pack(r=-1) == SHAPE and pack(k=0) == SHAPE and pack(r=5) == SHAPE and pack(k=41) == SHAPE
    assert pack(X=R + 8) == ALIGN and pack(ld=36) == ALIGN and pack(ld=32) == ALIGN and pack(out=_ck(codes=P + 8)) == ALIGN
    assert pack(t=1, ld=42) == ALIGN  # 168 bytes a row
    assert pack(r=0, out=_ck(R=0), X=None) == OK
    big = (1 << 24) + 1
    assert pack(k=big, ld=big, out=_ck(K=big)) == LIMIT
    assert pack(r=1 << 33, k=1 << 10, ld=1 << 10, out=_ck(R=1 << 33, K=1 << 10)) == LIMIT
    unpack = lambda c=_ck(), X=R, t=0, ld=40: L.nvfp4_ckpt8_unpack(c, X, t, ld, None)  # noqa: E731
    assert unpack(c=None) == NULL and unpack(X=None) == NULL and unpack(t=3) == ENUM and unpack(ld=44) == ALIGN and unpack(c=_ck(K=0)) == SHAPE
    assert unpack(c=_ck(R=0), X=None) == OK


def test_swiglu():
    fwd = lambda G=P, ldg=40, U=Q, ldu=40, T=4, D=40, H=R, ldh=40, g8=None, u8=None: L.nvfp4_swiglu_fwd(G, ldg, U, ldu, T, D, H, ldh, g8, u8, None)  # noqa: E731
    assert fwd(G=None) == NULL and fwd(U=None) == NULL and fwd(H=None) == NULL and fwd(T=-1) == SHAPE and fwd(D=0) == SHAPE and fwd(g8=_ck()) == SHAPE and fwd(u8=_ck()) == SHAPE
    assert fwd(g8=_ck(), u8=_ck(K=48)) == SHAPE and fwd(ldg=36) == ALIGN and fwd(ldu=44) == ALIGN and fwd(ldh=32) == ALIGN and fwd(T=0) == OK
    bwd = lambda dH=P, G=Q, U=R, g8=None, u8=None, T=4, D=40, dG=S, dU=S + 0x1000, ldd=40: L.nvfp4_swiglu_bwd(dH, 40, G, 40, U, 40, g8, u8, T, D, dG, ldd, dU, 40, None)  # noqa: E731
    assert bwd(dH=None) == NULL and bwd(G=None) == NULL and bwd(U=None) == NULL and bwd(dG=None) == NULL and bwd(dU=None) == NULL
    assert bwd(g8=_ck()) == SHAPE and bwd(g8=_ck(R=5), u8=_ck()) == SHAPE and bwd(ldd=36) == ALIGN and bwd(T=0) == OK


def test_layernorm():
    def fwd(X=P, t=0, ld=40, T=4, D=40, gamma=Q, beta=None, pt=0, eps=1e-5, Y=R, ldy=40, stats=S, x8=None):
        return L.nvfp4_layernorm_fwd(X, t, ld, T, D, gamma, beta, pt, eps, Y, ldy, stats, x8, None)

    assert fwd(X=None) == NULL and fwd(gamma=None) == NULL and fwd(Y=None) == NULL and fwd(t=2) == ENUM and fwd(pt=-1) == ENUM
    assert fwd(T=-1) == SHAPE and fwd(D=0) == SHAPE and fwd(eps=-1e-9) == SHAPE and fwd(eps=float("nan")) == SHAPE and fwd(x8=_ck(R=3)) == SHAPE
    assert fwd(D=16385, ld=16392, ldy=16392) == LIMIT and fwd(T=1 << 31) == LIMIT and fwd(T=0) == OK
    assert fwd(X=P + 8) == ALIGN and fwd(ld=36) == ALIGN and fwd(ldy=44) == ALIGN and fwd(gamma=Q + 4) == ALIGN and fwd(beta=Q + 8) == ALIGN and fwd(stats=S + 4) == ALIGN

    need = L.nvfp4_layernorm_bwd_workspace_bytes(4, 40)
    assert 0 < need == L.nvfp4_layernorm_bwd_workspace_bytes(1, 40)

    def bwd(dY=P, X=Q, t=0, ld=40, x8=None, T=4, D=40, gamma=R, pt=0, stats=S, dX=P + 0x100, lddx=40, dg=P + 0x200, db=None, dt=0, ws=P + 0x400, n=need):
        return L.nvfp4_layernorm_bwd(dY, 40, X, t, ld, x8, T, D, gamma, pt, stats, dX, lddx, dg, db, dt, ws, n, None)

    assert bwd(dY=None) == NULL and bwd(X=None) == NULL and bwd(gamma=None) == NULL and bwd(stats=None) == NULL and bwd(dX=None) == NULL and bwd(dg=None) == NULL
    assert bwd(t=2) == ENUM and bwd(pt=2) == ENUM and bwd(dt=2) == ENUM and bwd(T=-1) == SHAPE and bwd(D=0) == SHAPE and bwd(x8=_ck(K=48)) == SHAPE
    assert bwd(D=16385) == LIMIT and bwd(ws=None) == WORKSPACE and bwd(n=need - 1) == WORKSPACE and bwd(ws=P + 8) == WORKSPACE
    assert bwd(ld=36) == ALIGN and bwd(lddx=44) == ALIGN and bwd(stats=S + 4) == ALIGN and bwd(gamma=R + 8) == ALIGN and bwd(dg=P + 1) == ALIGN and bwd(db=P + 0x201) == ALIGN


def test_the_binding_refuses_what_the_library_cannot_see():
    """Types, shapes, strides and devices of tensors: the library gets addresses."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    v = torch.ones(64, dtype=torch.bfloat16)
    w = b.Operand(torch.zeros(40 * 64, dtype=torch.uint8), torch.zeros(128 * 16, dtype=torch.uint8), torch.zeros(1), 40, 64, 0, 1)
    ck = b.alloc_ckpt8(4, 64, "cpu")
    on_cpu = [lambda: b.nvfp4_gemv(x, w, out=x), lambda: b.nvfp4_ckpt8_pack(x, ck), lambda: b.nvfp4_ckpt8_unpack(ck, out=x), lambda: b.nvfp4_swiglu_fwd(x, x, out=x),
              lambda: b.nvfp4_swiglu_bwd(x, b.SwigluSaved(4, 64, x, x)), lambda: b.nvfp4_layernorm_fwd(x, v, out=x),
              lambda: b.nvfp4_layernorm_bwd(x, b.LayerNormSaved(4, 64, 0, torch.zeros(4, 2), v, False, x))]
    for call in on_cpu:
        with pytest.raises(RuntimeError, match="CUDA device"):
            call()
    with pytest.raises(RuntimeError, match="Half"):
        b.nvfp4_layernorm_fwd(x.half(), v)
    with pytest.raises(RuntimeError, match="shape"):
        b.nvfp4_swiglu_fwd(x[0], x[0])
    with pytest.raises(RuntimeError, match="shape"):
        b.nvfp4_ckpt8_pack(x[0])
    meta = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="meta")  # noqa: E731
    with pytest.raises(RuntimeError, match="CUDA device"):
        b.nvfp4_gemv(meta(4, 64), w)
