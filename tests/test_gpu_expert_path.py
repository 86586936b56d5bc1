"""The expert path as it is used: router, experts' gate and up, their down projections, weighted sum."""
import pytest
import torch

import paper_2609_15039_amd as sp
import workloads as WL

from tests import expert_ref as R
from tests.test_gpu_epilogue import BF16, DEV, F32, ints

pytestmark = pytest.mark.gpu


def pair_logits(T, E, k, seed):
    """k experts of each token at the same logit, the others masked: weights of exactly 1 / k for k a power of two."""
    g = torch.Generator().manual_seed(seed)
    L = torch.full((T, E), float("-inf"))
    for t in range(T):
        L[t, torch.randperm(E, generator=g)[:k]] = 0.5
    L[T // 2] = float("-inf")  # a padding token
    return L


@pytest.mark.parametrize("prec,layout", [("bf16x3", "rows"), ("bf16x3", "tiled"), ("f32", "f32"), ("f32", "rows")])
@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (9, 16, 4), (300, 8, 2), (2000, 4, 1)])
def test_integers_are_exact(T, E, k, prec, layout):
    """Every value on the way is an integer (halves and quarters at the end), so the path is exact."""
    K, N, D = 32, 64, 40
    X, L = ints((T, K), -1, 1, T), pair_logits(T, E, k, T)
    Wgu, Wd, res = ints((E, 2 * N, K), -1, 1, 2), ints((E, D, N), -1, 1, 3), ints((T, D), -9, 9, 4)
    H = torch.zeros((T, D), dtype=torch.float64)
    for t in range(T):
        for e in torch.nonzero(L[t] > -1).flatten().tolist():
            z = X[t].double() @ Wgu[e].double().T
            H[t] += (torch.relu(z[:N]) * z[N:]) @ Wd[e].double().T / k
    if layout == "f32":
        A, B = Wgu.to(DEV), Wd.to(DEV)
    else:
        A, B = Wgu.to(DEV, BF16), Wd.to(DEV, BF16)
        if layout == "tiled":
            A, B = sp.tile_experts(A), sp.tile_experts(B)
    Y = sp.expert_ffn(X.to(DEV), L.to(DEV), k, A, B, prec=sp.PRECS[prec], act="relu", residual=res.to(DEV))
    assert torch.equal(Y.cpu().double(), H + res.double())
    assert torch.equal(Y.cpu()[T // 2], res[T // 2])


@pytest.mark.parametrize("prec", ["bf16x3", "f32"])
@pytest.mark.parametrize("mech", ["gaussian", "laplace", "none"])
@pytest.mark.parametrize("T", [3, 130])
def test_masks_cancel(T, mech, prec):
    """Masked and unmasked at every stage: each stage against 64 bits on the inputs that it had, with the
    bound of its masked operand, and the path equal to its stages."""
    E, k, K, N, D = 8, 2, 256, 64, 128
    mech, gp, scale = sp.MECHS[mech], sp.PRECS[prec], 4.0
    X = torch.from_numpy(WL.gen_x(T, K, seed=T)).to(DEV)
    g = torch.Generator(device=DEV).manual_seed(T)
    L = torch.randn((T, E), generator=g, device=DEV)
    Wgu = (torch.randn((E, 2 * N, K), generator=g, device=DEV) * 0.06).to(BF16)
    Wd = (torch.randn((E, D, N), generator=g, device=DEV) * 0.1).to(BF16)
    res = torch.randn((T, D), generator=g, device=DEV)
    Y = sp.expert_ffn(X, L, k, Wgu, Wd, mech, scale, 1.0, seed=5, stream_id=9, row0=7, prec=gp, residual=res)

    r = sp.route(L, k)
    off = r.offsets.cpu()

    def stage(A, W, sid, first, index, **ep):
        rows, width = A.shape
        masked = mech != sp.SPLITEE_MECH_NONE
        eta = sp.noise(rows, width, mech, scale, 1.0, 5, sid, first) if masked else torch.zeros_like(A)
        C = sp.grouped_linear(sp.mask(torch.zeros_like(A), eta, gp), gp, W, r.offsets, row_index=index) if masked else None
        out = sp.grouped_linear(sp.mask(A, eta, gp), gp, W, r.offsets, row_index=index, C=C, **ep)
        a, e, ix = A.cpu().double(), eta.cpu().double(), None if index is None else index.cpu()
        P, S = R.grouped64(a, W.cpu().double(), off, ix)
        # the masked operand is rounded once (u of |x + eta|), the products sum |x + eta| |w| and |eta| |w|
        _, big = R.grouped64(a.abs() + 2 * e.abs(), W.cpu().double(), off, ix)
        want, bound = R.epilogue64(P, 2 * big, width + 2, None, None, ep.get("act", "none"), ep.get("gated", False), None, F32)
        assert ((out.cpu().double() - want).abs() <= bound).all()
        return out

    H = stage(X, Wgu, 9, 7, r.row_index, act="silu", gated=True)
    Z = stage(H, Wd, 10, 7 * k, None)
    assert torch.equal(Y, sp.combine(Z, r.slot, r.weights, residual=res))


def test_path_replays():
    """The whole path captured once and replayed on other tokens, which choose other experts."""
    T, E, k, K, N, D = 50, 16, 4, 128, 64, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    Wgu, Wd = torch.randn((E, 2 * N, K), generator=g, device=DEV).to(BF16), torch.randn((E, D, N), generator=g, device=DEV).to(BF16)
    X, L = torch.zeros((T, K), device=DEV), torch.zeros((T, E), device=DEV)

    def call():
        return sp.expert_ffn(X, L, k, Wgu, Wd, sp.SPLITEE_MECH_GAUSSIAN, 1.0, 1.0, seed=3, stream_id=2)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = call()
    for _ in range(3):
        X.copy_(torch.randn((T, K), generator=g, device=DEV))
        L.copy_(torch.randn((T, E), generator=g, device=DEV))
        L[3] = float("-inf")
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone()
        assert torch.equal(got, call()) and (got[3] == 0).all()


def test_no_tokens():
    Y = sp.expert_ffn(torch.empty((0, 32), device=DEV), torch.empty((0, 4), device=DEV), 2,
                      torch.zeros((4, 64, 32), dtype=BF16, device=DEV), torch.zeros((4, 16, 32), dtype=BF16, device=DEV))
    assert Y.shape == (0, 16)
