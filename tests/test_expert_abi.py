"""Refusals of the projections with an epilogue and of the expert path, on the host: every call here
fails validation, or is empty, before anything would be launched (16 is a non-null, aligned
stand-in address that is never read)."""
import ctypes

import pytest
import torch

import paper_2609_15039_amd as sp

OK, ARG, SHAPE, DTYPE, ALIGN, UNSUP, WS = 0, -1, -2, -3, -4, -5, -7
P = 16
F32, BF16, TILED = sp.SPLITEE_F32, sp.SPLITEE_BF16, sp.SPLITEE_BF16_TILED
PF, PB, PX, PD = 0, 1, 2, 3
BIG = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return sp.load()


def epilogue(C=None, ldc=0, bias=None, bias_stride=0, residual=None, ldres=0, act=0, gated=0, out_type=F32):
    return sp.Epilogue(C, ldc, bias, bias_stride, residual, ldres, act, gated, out_type)


EPILOGUES = [(dict(act=5), ARG), (dict(act=-1), ARG), (dict(gated=2), ARG), (dict(gated=-1), ARG), (dict(out_type=TILED), DTYPE),
             (dict(out_type=7), DTYPE), (dict(C=P, ldc=12), SHAPE), (dict(C=P, ldc=16, gated=1), SHAPE), (dict(C=8, ldc=16), ALIGN),
             (dict(C=P, ldc=18), ALIGN), (dict(bias=18), ALIGN), (dict(bias=P, bias_stride=-1), SHAPE),
             (dict(residual=P, ldres=12), SHAPE), (dict(residual=24, ldres=16), ALIGN), (dict(residual=P, ldres=18), ALIGN),
             (dict(residual=P, ldres=20, out_type=BF16), ALIGN)]


def linear(lib, ep=None, A=P, prec=PB, lda=32, W=P, w_type=BF16, ldw=32, Y=P, ldy=16, M=4, N=16, K=32, ws=256, nbytes=1 << 40):
    ep = epilogue() if ep is None else ep
    return lib.splitee_linear_epilogue(A, prec, lda, W, w_type, ldw, ctypes.byref(ep) if ep else None, Y, ldy, M, N, K, ws, nbytes,
                                       None)


@pytest.mark.parametrize("kw,code", EPILOGUES)
def test_epilogue_validation(lib, kw, code):
    assert linear(lib, epilogue(**kw)) == code
    assert grouped(lib, epilogue(**kw)) == code


COMMON = [(dict(prec=PD), UNSUP), (dict(prec=9), UNSUP), (dict(ep=False), ARG), (dict(K=36, lda=40, ldw=40), SHAPE),
          (dict(lda=24), SHAPE), (dict(ldw=24), SHAPE), (dict(ldy=12), SHAPE), (dict(N=-1), SHAPE), (dict(K=-8), SHAPE),
          (dict(w_type=5), DTYPE), (dict(w_type=F32), UNSUP), (dict(w_type=TILED, prec=PF), UNSUP), (dict(A=None), ARG),
          (dict(W=None), ARG), (dict(Y=None), ARG), (dict(A=8), ALIGN), (dict(W=8), ALIGN), (dict(Y=8), ALIGN), (dict(lda=36), ALIGN),
          (dict(ldw=36), ALIGN), (dict(ldy=18), ALIGN), (dict(lda=BIG), UNSUP), (dict(ldw=BIG), UNSUP),
          (dict(w_type=TILED, K=BIG, lda=BIG), UNSUP), (dict(N=1 << 28, ldy=1 << 28), UNSUP), (dict(N=0), OK)]


@pytest.mark.parametrize("kw,code", COMMON + [(dict(M=-1), SHAPE), (dict(M=0), OK), (dict(ws=128), ALIGN)])
def test_linear_validation(lib, kw, code):
    assert linear(lib, **kw) == code


def test_linear_workspace(lib):
    need = 0
    for M in (1, 17, 64, 200):
        need = max(need, lib.splitee_epilogue_workspace_bytes(M, 2560, 9728, PB, 0))
        if need:
            assert linear(lib, M=M, N=2560, K=9728, lda=9728, ldw=9728, ldy=2560, ws=None, nbytes=0) == WS
            assert linear(lib, M=M, N=2560, K=9728, lda=9728, ldw=9728, ldy=2560, nbytes=need - 1) == WS
            break
    for bad in ((-1, 8, 8, PB, 0), (8, 8, 12, PB, 0), (8, 8, 8, PD, 0), (8, 8, 8, PB, 2), (0, 8, 8, PB, 0), (8, 0, 8, PB, 1)):
        assert lib.splitee_epilogue_workspace_bytes(*bad) == 0


def grouped(lib, ep=None, A=P, prec=PB, lda=32, a_rows=4, index=P, offsets=P, experts=2, W=P, w_type=BF16, ldw=32, w_stride=512,
            Y=P, ldy=16, rows=4, N=16, K=32):
    ep = epilogue() if ep is None else ep
    return lib.splitee_grouped_linear(A, prec, lda, a_rows, index, offsets, experts, W, w_type, ldw, w_stride,
                                      ctypes.byref(ep) if ep else None, Y, ldy, rows, N, K, None)


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(rows=-1), SHAPE), (dict(a_rows=-1), SHAPE), (dict(a_rows=0), SHAPE), (dict(index=None, a_rows=3), SHAPE),
    (dict(experts=-1), SHAPE), (dict(w_stride=-8), SHAPE), (dict(w_stride=516), ALIGN), (dict(offsets=None), ARG),
    (dict(a_rows=1 << 26), UNSUP), (dict(a_rows=1 << 25, prec=PF), UNSUP), (dict(offsets=18), ALIGN), (dict(index=18), ALIGN), (dict(rows=0), OK), (dict(experts=0), OK)])
def test_grouped_validation(lib, kw, code):
    assert grouped(lib, **kw) == code


def route(lib, logits=P, ldl=64, T=4, E=64, k=8, score=0, experts=P, weights=P, offsets=P, index=P, slot=P, ws=256, nbytes=1 << 40):
    return lib.splitee_route(logits, ldl, T, E, k, score, 1, experts, weights, offsets, index, slot, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(score=2), ARG), (dict(T=-1), SHAPE), (dict(E=0, k=0), SHAPE), (dict(k=0), SHAPE), (dict(k=65, E=64), SHAPE), (dict(ldl=63), SHAPE),
    (dict(E=1025, ldl=1025), UNSUP), (dict(k=65, E=100, ldl=100), UNSUP), (dict(T=1 << 28), UNSUP), (dict(ws=None), WS),
    (dict(nbytes=256), WS), (dict(ws=128), ALIGN), (dict(logits=None), ARG), (dict(experts=None), ARG), (dict(weights=None), ARG),
    (dict(offsets=None), ARG), (dict(index=None), ARG), (dict(slot=None), ARG), (dict(logits=18), ALIGN), (dict(slot=18), ALIGN),
    (dict(offsets=18), ALIGN)])
def test_route_validation(lib, kw, code):
    assert route(lib, **kw) == code


def test_route_workspace(lib):
    assert lib.splitee_route_workspace_bytes(4, 64, 8) > 0
    for bad in ((-1, 8, 2), (8, 8, 0), (8, 8, 9), (8, 1025, 8), (8, 100, 65), (1 << 28, 64, 8)):
        assert lib.splitee_route_workspace_bytes(*bad) == 0


def combine(lib, H=P, h_type=F32, ldh=16, h_rows=8, slot=P, weights=P, res=None, ldres=16, Y=P, out=F32, ldy=16, T=4, k=2, N=16):
    return lib.splitee_combine(H, h_type, ldh, h_rows, slot, weights, res, ldres, Y, out, ldy, T, k, N, None)


@pytest.mark.parametrize("kw,code", [
    (dict(h_type=TILED), DTYPE), (dict(out=9), DTYPE), (dict(T=-1), SHAPE), (dict(k=0), SHAPE), (dict(h_rows=-1), SHAPE),
    (dict(ldh=12), SHAPE), (dict(ldy=12), SHAPE), (dict(res=P, ldres=12), SHAPE), (dict(k=65), UNSUP),
    (dict(N=BIG, ldh=BIG, ldy=BIG), UNSUP), (dict(H=None), ARG), (dict(slot=None), ARG), (dict(weights=None), ARG), (dict(Y=None), ARG),
    (dict(H=8), ALIGN), (dict(ldh=18), ALIGN), (dict(Y=8), ALIGN), (dict(ldy=20, out=BF16), ALIGN), (dict(res=8), ALIGN),
    (dict(slot=18), ALIGN), (dict(weights=18), ALIGN), (dict(T=0), OK), (dict(N=0), OK)])
def test_combine_validation(lib, kw, code):
    assert combine(lib, **kw) == code


GB = 1 << 30


@pytest.mark.parametrize("call", [
    lambda lib: linear(lib, M=GB, N=1 << 20, K=8, ldy=1 << 20, nbytes=1 << 62),
    lambda lib: linear(lib, epilogue(act=1), prec=PF, M=1 << 22, N=1 << 20, K=8, ldy=1 << 20, nbytes=1 << 62),
    lambda lib: linear(lib, prec=PF, M=1 << 22, N=1 << 20, K=8, ldy=1 << 20, nbytes=1 << 62),
    lambda lib: grouped(lib, experts=GB, N=1 << 20, ldy=1 << 20),
    lambda lib: grouped(lib, prec=PX, experts=GB, N=1 << 20, ldy=1 << 20),
    lambda lib: grouped(lib, prec=PF, experts=GB, N=1 << 20, ldy=1 << 20),
    lambda lib: route(lib, T=(1 << 26) + 1, E=1, k=1, ldl=1),
    lambda lib: combine(lib, T=1 << 24)])
def test_more_than_a_launch_takes_is_refused(lib, call):
    """2^32 threads and more: refused before the launch, of which the device would say an error."""
    assert call(lib) == UNSUP


def test_binding_refuses_what_the_library_cannot_see():
    """Shapes and types of tensors, and tensors that are not on the device (none is here)."""
    A, W = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(16, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="A:"):
        sp.linear_epilogue(A.float(), sp.SPLITEE_PREC_BF16, W)
    with pytest.raises(ValueError, match="planes x rows x K"):
        sp.linear_epilogue(A, sp.SPLITEE_PREC_BF16X3, W)
    with pytest.raises(ValueError, match="planes are not"):
        sp.linear_epilogue(torch.zeros(3, 8, 32, dtype=torch.bfloat16)[:, :4], sp.SPLITEE_PREC_BF16X3, W)
    with pytest.raises(ValueError, match="columns"):
        sp.linear_epilogue(torch.zeros(32, 4, dtype=torch.bfloat16).t(), sp.SPLITEE_PREC_BF16, W)
    with pytest.raises(ValueError, match="W:"):
        sp.linear_epilogue(A, sp.SPLITEE_PREC_BF16, W[:, :24])
    with pytest.raises(ValueError, match="gated"):
        sp.linear_epilogue(A, sp.SPLITEE_PREC_BF16, W[:15], gated=True)
    with pytest.raises(ValueError, match="tiled"):
        sp.linear_epilogue(A, sp.SPLITEE_PREC_BF16, sp.TiledWeights(torch.zeros(2047, dtype=torch.bfloat16), 16, 32))
    with pytest.raises(ValueError, match="experts"):
        sp.grouped_linear(A, sp.SPLITEE_PREC_BF16, W, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="logits"):
        sp.route(A, 2)
    with pytest.raises(ValueError, match="slot"):
        sp.combine(A, torch.zeros(4, 2), torch.zeros(4, 2))


def ffn_arguments(**kw):
    a = dict(X=torch.zeros(6, 32), logits=torch.zeros(6, 4), k=2, W_gate_up=torch.zeros(4, 48, 32, dtype=torch.bfloat16),
             W_down=torch.zeros(4, 16, 24, dtype=torch.bfloat16))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,match", [
    (dict(X=torch.zeros(6, 32, dtype=torch.bfloat16)), "X:"), (dict(X=torch.zeros(2, 6, 32)), "X:"),
    (dict(X=torch.zeros(32, 6).t()), "X:"), (dict(logits=torch.zeros(5, 4)), "logits:"), (dict(logits=torch.zeros(6)), "logits:"),
    (dict(W_gate_up=torch.zeros(4, 48, 24, dtype=torch.bfloat16)), "W_gate_up:"),
    (dict(W_gate_up=torch.zeros(4, 42, 32, dtype=torch.bfloat16)), "W_gate_up:"),  # 21 outputs, whose rows are 24 apart
    (dict(W_gate_up=torch.zeros(4, 24, 32, dtype=torch.bfloat16)), "W_gate_up:"),
    (dict(residual=torch.zeros(5, 16)), "residual:"), (dict(residual=torch.zeros(6, 16, dtype=torch.bfloat16)), "residual:")])
def test_expert_ffn_refuses_before_anything_runs(kw, match):
    with pytest.raises(ValueError, match=match):
        sp.expert_ffn(**ffn_arguments(**kw))


@pytest.mark.parametrize("W", [torch.zeros(2, 32, 64), torch.zeros(32, 64, dtype=torch.bfloat16),
                               torch.zeros(2, 64, 32, dtype=torch.bfloat16).transpose(1, 2)])
def test_tile_experts_refuses(W):
    with pytest.raises(ValueError, match="W:"):
        sp.tile_experts(W)
