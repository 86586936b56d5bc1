"""The expert path in the single-plane precision: operands rounded once to bfloat16, corrections exact."""
import pytest
import torch

import paper_2609_15039_amd as sp
import workloads as WL

from tests import expert_ref as R
from tests.test_gpu_epilogue import BF16, DEV, F32, ints
from tests.test_gpu_expert_path import pair_logits

pytestmark = pytest.mark.gpu

PB, PX = sp.SPLITEE_PREC_BF16, sp.SPLITEE_PREC_BF16X3
HALF = torch.finfo(BF16).eps / 2


def tiled(W, layout):
    return sp.tile_experts(W) if layout == "tiled" else W


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (9, 16, 4), (300, 8, 2)])
def test_integers_are_exact(T, E, k, out, layout):
    """Inputs, gated products (64 at most) and sums are integers, halves or quarters that bfloat16 or binary32 hold."""
    K, N, D = 8, 24, 40
    X, L = ints((T, K), -1, 1, T), pair_logits(T, E, k, T)
    Wgu, Wd, res = ints((E, 2 * N, K), -1, 1, 2), ints((E, D, N), -1, 1, 3), ints((T, D), -9, 9, 4)
    H = torch.zeros((T, D), dtype=torch.float64)
    for t in range(T):
        for e in torch.nonzero(L[t] > -1).flatten().tolist():
            z = X[t].double() @ Wgu[e].double().T
            H[t] += (torch.relu(z[:N]) * z[N:]) @ Wd[e].double().T / k
    Y = sp.expert_ffn(X.to(DEV), L.to(DEV), k, tiled(Wgu.to(DEV, BF16), layout), tiled(Wd.to(DEV, BF16), layout), prec=PB,
                      act="relu", residual=res.to(DEV, out), out_dtype=out)
    assert Y.dtype == out and torch.equal(Y.cpu(), (H + res.double()).float().to(out))


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("mech", ["gaussian", "laplace", "none"])
@pytest.mark.parametrize("T", [3, 130, 700])
def test_each_stage(T, mech, layout):
    """The path equals its stages, and each stage is within the bound of an operand rounded to bfloat16."""
    E, k, K, N, D = 8, 2, 256, 64, 128
    mech, scale = sp.MECHS[mech], 0.5
    masked = mech != sp.SPLITEE_MECH_NONE
    X = torch.from_numpy(WL.gen_x(T, K, seed=T)).to(DEV)
    g = torch.Generator(device=DEV).manual_seed(T)
    L = torch.randn((T, E), generator=g, device=DEV)
    Wgu = (torch.randn((E, 2 * N, K), generator=g, device=DEV) * 0.06).to(BF16)
    Wd = (torch.randn((E, D, N), generator=g, device=DEV) * 0.1).to(BF16)
    res = torch.randn((T, D), generator=g, device=DEV)
    Y = sp.expert_ffn(X, L, k, tiled(Wgu, layout), tiled(Wd, layout), mech, scale, 1.0, seed=5, stream_id=9, row0=7, prec=PB, residual=res)

    r = sp.route(L, k)
    off = r.offsets.cpu()

    def stage(A, W, sid, first, index, **ep):
        rows, width = A.shape
        eta = sp.noise(rows, width, mech, scale, 1.0, 5, sid, first) if masked else torch.zeros_like(A)
        C = sp.grouped_linear(sp.mask(torch.zeros_like(A), eta, PX), PX, tiled(W, layout), r.offsets, row_index=index) if masked else None
        out = sp.grouped_linear(sp.mask(A, eta, PB), PB, tiled(W, layout), r.offsets, row_index=index, C=C, **ep)
        a, e, w, ix = A.cpu().double(), eta.cpu().double(), W.cpu().double(), None if index is None else index.cpu()
        P, _ = R.grouped64(a, w, off, ix)
        # fl32(x + eta) is off by u of itself and its rounding to bfloat16 by HALF of it; the products sum |x + eta| |w|
        # (half a step more of it) and |eta| |w|, each width terms
        _, both = R.grouped64((a + e).abs() * (1 + HALF) + e.abs(), w, off, ix)
        _, once = R.grouped64((a + e).abs(), w, off, ix)
        terms = width + 2
        S = both + HALF * once / ((terms + 8) * R.U * 1.01)
        want, bound = R.epilogue64(P, S, terms, None, None, ep.get("act", "none"), ep.get("gated", False), None, F32)
        off_by = (out.cpu().double() - want).abs()
        print(T, mech, layout, "off / bound %.2g" % float((off_by / bound).max()), flush=True)
        assert (off_by <= bound).all()
        return out

    H = stage(X, Wgu, 9, 7, r.row_index, act="silu", gated=True)
    Z = stage(H, Wd, 10, 7 * k, None)
    assert torch.equal(Y, sp.combine(Z, r.slot, r.weights, residual=res))
