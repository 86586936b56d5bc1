"""Three planes, none of them zero, through every kernel of the products with an epilogue, bit for bit: the planes are independent
small integers, so that the sum of the three products is an integer below 2^24, exact in any order, and no plane can be
left out, taken twice or taken from another row unseen (the reference is held to that)."""
import numpy as np
import pytest
import torch

import paper_2609_15039_amd as sp

from tests import expert_ref as R
from tests.linear_shapes import DENSE, GROUPED
from tests.test_gpu_epilogue import BF16, DEV, F32, SHAPES
from tests.test_gpu_far import FAR
from tests.test_gpu_linear_plans import fresh, ints, rows_of

pytestmark = pytest.mark.gpu

X3 = sp.SPLITEE_PREC_BF16X3


def planes(rows, K, seed, ld=None):
    """3 x rows x K of 1 .. 8 and -1 .. -8, inside rows of ld whose rest is NaN (K + 16)."""
    p = ints((3, rows, K), 1, 8, seed) * (2 * ints((3, rows, K), 0, 1, seed + 1) - 1)
    wide = torch.full((3, rows, K + 16 if ld is None else ld), float("nan"), dtype=BF16, device=DEV)
    wide[:, :, :K] = p
    return wide[:, :, :K]


def weights(W, layout):
    if layout == "rows":
        return W
    return sp.tile_weights(W) if W.dim() == 2 else sp.tile_experts(W)


def product(p, W):
    return p.double().sum(0) @ W.double().T


def held_to_each_plane(p, W):
    """The planes' own products differ, and none is zero."""
    one = [q.double() @ W.double().T for q in p]
    assert all(bool((o != 0).any()) for o in one) and not torch.equal(one[0], one[1]) and not torch.equal(one[1], one[2])


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("M,N,K", DENSE + SHAPES)
def test_dense(M, N, K, layout):
    A, W2 = planes(M, K, M), ints((2 * N, K), -4, 4, N).to(BF16)
    held_to_each_plane(A, W2)
    for gated, out, parts in ((False, F32, ""), (True, F32, "C"), (False, BF16, "Cr")):
        W = W2 if gated else W2[:N]
        C = rows_of(ints((M, W.shape[0]), -50, 50, 1), F32) if "C" in parts else None
        res = rows_of(ints((M, N), -99, 99, 3), out) if "r" in parts else None
        print(M, N, K, layout, gated, out, sp.splitee_linear_plan_probe(M, 1, True, N, K, X3, gated), flush=True)
        want = R.epilogue_bits(product(A, W), C, None, "none", gated, res, out)
        Y = sp.linear_epilogue(A, X3, weights(W, layout), C=C, gated=gated, residual=res, out_dtype=out, Y=fresh(M, N, out))
        assert torch.equal(Y, want)


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("at", range(len(GROUPED)))
def test_by_expert(at, layout):
    n, N, K = GROUPED[at]
    rows, E = sum(n), len(n)
    offsets, begin = R.counts_to_offsets(n).to(DEV), np.concatenate([[0], np.cumsum(n)])
    W2 = ints((E, 2 * N, K), -4, 4, N).to(BF16)
    tokens = max(1, rows // 2)
    index = torch.from_numpy(np.random.default_rng(at).integers(0, tokens, rows).astype(np.int32)).to(DEV)
    for gated, gather in ((False, True), (True, False), (True, True)):
        A = planes(tokens if gather else rows, K, rows)
        W = W2 if gated else W2[:, :N].contiguous()
        print(rows, E, N, K, layout, gated, gather, sp.splitee_linear_plan_probe(rows, E, False, N, K, X3, gated), flush=True)
        X = A[:, index.long()] if gather else A
        P = torch.cat([product(X[:, begin[e]:begin[e + 1]], W[e]) for e in range(E)])
        held_to_each_plane(A, W[0])
        Y = sp.grouped_linear(A, X3, weights(W, layout), offsets, row_index=index if gather else None, gated=gated, Y=fresh(rows, N, F32))
        assert torch.equal(Y, R.epilogue_bits(P, gated=gated))


@pytest.mark.parametrize("M", [9, 1200])
def test_far_planes(M):
    """Planes up to 2.5 GB, the third one's rows more than 2^31 bytes and 2^32 elements from the first's."""
    N, K = 1100, 72
    A, W = planes(M, K, 1, FAR), ints((N, K), -4, 4, 2).to(BF16)
    assert torch.equal(sp.linear_epilogue(A, X3, W), R.epilogue_bits(product(A, W)))


@pytest.mark.parametrize("rows", [5, 40, 900])
def test_far_planes_by_expert(rows):
    """Gathered from planes of 2^31 bytes less some rows, in an order that the rows do not have."""
    N, K, tokens = 200, 72, (1 << 31) // (FAR * 2)
    A, W = planes(tokens, K, 1, FAR), ints((2, N, K), -4, 4, 2).to(BF16)
    n = [rows // 3, rows - rows // 3]
    index = (tokens - 1 - torch.arange(rows, device=DEV)).to(torch.int32)
    X = A[:, index.long()]
    P = torch.cat([product(X[:, :n[0]], W[0]), product(X[:, n[0]:], W[1])])
    Y = sp.grouped_linear(A, X3, W, R.counts_to_offsets(n).to(DEV), row_index=index)
    assert torch.equal(Y, R.epilogue_bits(P))


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("M,N,K", [(1, 300, 264), (12, 2050, 2056), (40, 515, 1032), (333, 1000, 2560), (1500, 770, 136), (4500, 600, 72)])
def test_the_split_of_a_value_comes_back(M, N, K, layout):
    """Odd integers of 24 bits, whose split has three planes, times weight rows with one 1 or -1 each: the integers themselves."""
    X = (ints((M, K), 1 << 22, (1 << 23) - 1, M) * 2 + 1) * (2 * ints((M, K), 0, 1, M + 1) - 1)
    at = (torch.arange(N, device=DEV) * 37 + K - 1) % K  # every part of K, the last columns among them
    sign = 2 * ints((N,), 0, 1, N) - 1
    W = torch.zeros((N, K), device=DEV)
    W[torch.arange(N, device=DEV), at] = sign
    Xt = sp.mask(X, torch.zeros_like(X), X3)
    assert all(float((q.view(BF16) != 0).float().mean()) > 0.9 for q in Xt)
    Y = sp.linear_epilogue(Xt, X3, weights(W.to(BF16), layout))
    assert torch.equal(Y, X[:, at] * sign)
    offsets = torch.tensor([0, M // 2, M], dtype=torch.int32, device=DEV)
    W2 = torch.stack([W, -W]).to(BF16)
    Y = sp.grouped_linear(Xt, X3, weights(W2, layout), offsets)
    assert torch.equal(Y, X[:, at] * sign * torch.where(torch.arange(M, device=DEV) < M // 2, 1.0, -1.0)[:, None])
