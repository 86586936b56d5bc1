"""Every kernel of the products with an epilogue on integers, bit for bit (the exact product comes from a binary64
matrix product of integers on the GPU)."""
import numpy as np
import pytest
import torch

import paper_2609_15039_amd as sp

from tests import expert_ref as R
from tests.linear_shapes import DENSE, GROUPED
from tests.test_gpu_epilogue import BF16, DEV, F32

pytestmark = pytest.mark.gpu


def ints(shape, lo, hi, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV).float()


def rows_of(x, dtype):
    """x with 16-byte rows."""
    per = 16 // dtype.itemsize
    out = torch.empty((x.shape[0], -(-x.shape[1] // per) * per), dtype=dtype, device=DEV)[:, :x.shape[1]]
    out.copy_(x)
    return out


def fresh(rows, N, out):
    return rows_of(torch.full((rows, N), float("nan"), device=DEV), out)


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("prec", ["bf16", "bf16x3"])
@pytest.mark.parametrize("M,N,K", DENSE)
def test_dense(M, N, K, prec, layout):
    A, W2 = ints((M, K), -8, 8, M), ints((2 * N, K), -4, 4, N)
    planes = R.split(A, prec)
    for gated, out, parts in ((False, BF16, "Cbr"), (True, F32, "Cbr"), (True, BF16, "b"), (False, F32, "")):
        NW = 2 * N if gated else N
        print(M, N, K, prec, layout, gated, out, sp.splitee_linear_plan_probe(M, 1, True, N, K, sp.PRECS[prec], gated), flush=True)
        W = W2[:NW].to(BF16)
        C = rows_of(ints((M, NW), -50, 50, 1), F32) if "C" in parts else None
        bias = ints((NW,), -9, 9, 2) if "b" in parts else None
        res = rows_of(ints((M, N), -99, 99, 3), out) if "r" in parts else None
        want = R.epilogue_bits(A.double() @ W.double().T, C, bias, "relu", gated, res, out)
        Y = sp.linear_epilogue(planes, sp.PRECS[prec], sp.tile_weights(W) if layout == "tiled" else W, C=C, bias=bias, act="relu",
                               gated=gated, residual=res, out_dtype=out, Y=fresh(M, N, out))
        assert torch.equal(Y, want)


# few tiles under a long K: every tile is split, by tiles of one to seven 16-row blocks and one or two 64-column blocks,
# and some that are not (the first, and gated widths that are no multiple of 4)
@pytest.mark.parametrize("w", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(5, 40, 64), (1, 17, 1032), (2, 2052, 4096), (17, 1000, 4096), (33, 1036, 2056), (49, 2052, 4096),
                                   (65, 2052, 4096), (97, 2052, 4096), (257, 515, 2056), (257, 2052, 4096), (300, 2052, 4096),
                                   (300, 2600, 4096)])
def test_dense_binary32(M, N, K, w):
    A, W2 = ints((M, K), -8, 8, M), ints((2 * N, K), -4, 4, N).to(w)
    for gated, out, parts in ((False, BF16, "Cbr"), (True, F32, "Cbr"), (True, BF16, "b"), (False, F32, "r")):
        print(M, N, K, w, gated, out, parts, flush=True)
        NW = 2 * N if gated else N
        C = rows_of(ints((M, NW), -50, 50, 1), F32) if "C" in parts else None
        bias = ints((NW,), -9, 9, 2) if "b" in parts else None
        res = rows_of(ints((M, N), -99, 99, 3), out) if "r" in parts else None
        want = R.epilogue_bits(A.double() @ W2[:NW].double().T, C, bias, "relu", gated, res, out)
        Y = fresh(M, N, out) if res is None else res  # the residual in place
        beside = Y._base[:, N:].clone()
        sp.linear_epilogue(A, sp.SPLITEE_PREC_F32, W2[:NW], C=C, bias=bias, act="relu", gated=gated, residual=res, out_dtype=out, Y=Y)
        assert torch.equal(Y, want)
        assert torch.equal(Y._base[:, N:].view(torch.uint8), beside.view(torch.uint8))


@pytest.mark.parametrize("layout", ["rows", "tiled"])
@pytest.mark.parametrize("prec", ["bf16", "bf16x3"])
@pytest.mark.parametrize("at", range(len(GROUPED)))
def test_by_expert(at, prec, layout):
    n, N, K = GROUPED[at]
    rows, E = sum(n), len(n)
    offsets = R.counts_to_offsets(n).to(DEV)
    expert = torch.repeat_interleave(torch.arange(E), torch.tensor(n)).to(DEV)
    A, W2 = ints((rows, K), -8, 8, rows), ints((E, 2 * N, K), -4, 4, N).to(BF16)
    index = torch.from_numpy(np.random.default_rng(at).integers(0, rows, rows).astype(np.int32)).to(DEV)
    planes = R.split(A, prec)
    for gated, out, parts, gather in ((False, F32, "Cb", True), (True, BF16, "Cbr", False)):
        NW = 2 * N if gated else N
        print(rows, E, N, K, prec, layout, gated, out, sp.splitee_linear_plan_probe(rows, E, False, N, K, sp.PRECS[prec], gated), flush=True)
        W = W2[:, :NW].contiguous()
        P = torch.zeros((rows, NW), dtype=torch.float64, device=DEV)
        X = A[index.long()] if gather else A
        begin = 0
        for e in range(E):
            P[begin:begin + n[e]] = X[begin:begin + n[e]].double() @ W[e].double().T
            begin += n[e]
        C = rows_of(ints((rows, NW), -50, 50, 1), F32) if "C" in parts else None
        bias = ints((E, NW), -9, 9, 2) if "b" in parts else None
        res = rows_of(ints((rows, N), -99, 99, 3), out) if "r" in parts else None
        want = R.epilogue_bits(P, C, None if bias is None else bias[expert], "relu", gated, res, out)
        Y = sp.grouped_linear(planes, sp.PRECS[prec], sp.tile_experts(W) if layout == "tiled" else W, offsets,
                              row_index=index if gather else None, C=C, bias=bias, act="relu", gated=gated, residual=res, out_dtype=out,
                              Y=fresh(rows, N, out))
        assert torch.equal(Y, want)
