"""splitee_route and splitee_combine against plain references, masks and ties included."""
import numpy as np
import pytest
import torch

import paper_2609_15039_amd as sp

from tests import expert_ref as R
from tests.test_gpu_epilogue import BF16, DEV, F32, padded

pytestmark = pytest.mark.gpu

NAMES = ("experts", "weights", "offsets", "row_index", "slot")


def check(logits, k, score="softmax", renorm=True, got=None):
    want = R.route_ref(logits, k, score, renorm)
    got = sp.route(logits.to(DEV), k, score=score, renorm=renorm) if got is None else got
    for name, w, g in zip(NAMES, want, got):
        g = g.cpu().numpy()
        if name != "weights":
            assert g.dtype == np.int32 and np.array_equal(g, w), name
            continue
        # exp of a binary32 difference (rounded: up to |l - m| 2^-24 of the value, |l - m| <= 88 before it
        # vanishes) within 4 units, E terms summed (gamma), one quotient
        bound = (88 + 4 + logits.shape[1] + 4) * R.U * w + 1e-37
        assert (np.abs(g - w) <= bound).all(), name
    return got


@pytest.mark.parametrize("score", list(sp.SCORES))
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (3, 2, 2), (63, 5, 3), (64, 64, 64), (65, 65, 6), (129, 128, 8), (257, 200, 16),
                                   (500, 256, 8), (1000, 300, 2), (70, 513, 10), (130, 1024, 64), (5000, 8, 2), (20000, 16, 1)])
def test_route(T, E, k, score, renorm):
    print(T, E, k, score, renorm, flush=True)
    g = torch.Generator().manual_seed(T + E)
    check(torch.randn(T, E, generator=g) * 2, k, score, renorm)


@pytest.mark.parametrize("T,E,k", [(40, 8, 4), (300, 100, 8), (200, 600, 5)])
@pytest.mark.parametrize("score", list(sp.SCORES))
def test_ties_and_masks(T, E, k, score):
    """Few values, so most rows have ties; masked experts, rows with fewer than k left, rows with none,
    rows of the type's lowest value, a NaN among numbers."""
    g = torch.Generator().manual_seed(E)
    L = torch.randint(-2, 3, (T, E), generator=g).float()
    L[torch.rand(T, E, generator=g) < 0.3] = float("-inf")
    L[::7] = float("-inf")
    L[1::7] = torch.finfo(F32).min
    L[2::7, 1:] = float("-inf")
    L[3::7, E // 2] = float("nan")
    L[4::7] = 0.0
    L[5::7, ::2] = -0.0
    for renorm in (True, False):
        r = check(L, k, score, renorm)
        assert (r.experts[::7] == -1).all() and (r.weights[::7] == 0).all() and (r.slot[::7] == -1).all()


@pytest.mark.parametrize("T", [3, 100])
@pytest.mark.parametrize("renorm", [True, False])
def test_infinite_logits(T, renorm):
    """+inf before every number, two of them by index; softmax weights NaN, a sigmoid's 1; tokens beside it as ever."""
    L = torch.arange(20.0).repeat(T, 1) / 8
    L[0, 5] = L[0, 11] = float("inf")
    L[0, 2] = float("nan")
    other = R.route_ref(L[1:], 3, "softmax", renorm)[1]
    r = sp.route(L.to(DEV), 3, renorm=renorm)
    assert r.experts[0].tolist() == [5, 11, 19] and torch.isnan(r.weights[0]).all()
    bound = (88 + 4 + 20 + 4) * R.U * other + 1e-37  # as in check
    assert (np.abs(r.weights[1:].cpu().numpy() - other) <= bound).all()
    s = sp.route(L.to(DEV), 3, score="sigmoid", renorm=False)
    assert s.experts[0].tolist() == [5, 11, 19] and s.weights[0, :2].tolist() == [1.0, 1.0]


def test_no_tokens_and_all_masked():
    r = sp.route(torch.empty((0, 9), device=DEV), 3)
    assert torch.equal(r.offsets.cpu(), torch.zeros(10, dtype=torch.int32))
    check(torch.full((100, 9), float("-inf")), 3)


def test_logits_in_a_wider_array():
    g = torch.Generator().manual_seed(5)
    wide = torch.full((150, 77), 1e30)
    wide[:, :70] = torch.randn(150, 70, generator=g)
    check(wide[:, :70], 4, got=sp.route(wide.to(DEV)[:, :70], 4))


@pytest.mark.parametrize("T,E,k", [(5, 64, 8), (700, 128, 8)])
def test_replays(T, E, k):
    L = torch.zeros((T, E), device=DEV)
    ws = sp._aligned_bytes(sp.splitee_route_workspace_bytes(T, E, k), DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = sp.route(L, k, ws=(ws, ws.numel()))
    g = torch.Generator().manual_seed(T)
    for _ in range(3):
        new = torch.randn(T, E, generator=g)
        L.copy_(new)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check(new, k, got=r)
        check(new, k)


@pytest.mark.parametrize("h", [F32, BF16])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (3, 2, 7), (16, 8, 2048), (5, 9, 130), (100, 4, 2050), (33, 64, 24), (2, 3, 4099)])
def test_combine(T, k, N, h, out):
    """Negative and too large slots add nothing, whatever H holds; the same slot may come twice."""
    g = torch.Generator().manual_seed(T + N)
    h_rows = max(1, T * k // 2)
    H = torch.randn(h_rows, N, generator=g).to(h)
    slot = torch.randint(-2, h_rows + 2, (T, k), generator=g, dtype=torch.int32)
    slot[:, 0] = torch.arange(T) % h_rows
    w = torch.randn(T, k, generator=g)
    for res in (None, torch.randn(T, N, generator=g).to(out)):
        live = (slot >= 0) & (slot < h_rows)
        used = torch.zeros(h_rows, dtype=torch.bool)
        used[slot[live].long()] = True
        Hd = padded(H, h)
        Hd[~used.to(DEV)] = float("nan")
        terms = torch.where(live[..., None], H[slot.clamp(0, h_rows - 1).long()].double() * w.double()[..., None], 0.0)
        want, size = terms.sum(1), terms.abs().sum(1)
        if res is not None:
            want, size = want + res.double(), size + res.double().abs()
        bound = (k + 2) * R.U * 1.01 * size
        bound = bound + torch.finfo(out).eps / 2 * (want.abs() + bound)
        Y = padded(torch.zeros(T, N), out, extra=1)
        Y.fill_(float("nan"))
        sp.combine(Hd, slot.to(DEV), w.to(DEV), residual=None if res is None else padded(res, out), out_dtype=out, Y=Y)
        assert ((Y.cpu().double() - want).abs() <= bound).all()
        assert torch.isnan(Y._base[:, N:]).all()


def test_combine_in_place_and_of_no_rows():
    slot, w = torch.full((6, 2), -1, dtype=torch.int32, device=DEV), torch.full((6, 2), float("nan"), device=DEV)
    Y = torch.arange(6 * 16, device=DEV).float().reshape(6, 16)
    want = Y.clone()
    sp.combine(torch.empty((0, 16), device=DEV), slot, w, residual=Y, Y=Y)
    assert torch.equal(Y, want)
    assert torch.equal(sp.combine(torch.empty((0, 16), device=DEV), slot, w), torch.zeros_like(Y))
