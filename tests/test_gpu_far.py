"""Operands whose parts lie more than 2^31 bytes, or elements, apart: leading dimensions and strides near
their limits, of which only the first columns are used."""
import pytest
import torch

import paper_2609_15039_amd as sp

from tests import expert_ref as R
from tests.test_gpu_epilogue import BF16, DEV, F32
from tests.test_gpu_linear_plans import ints

pytestmark = pytest.mark.gpu

FAR = (1 << 20) - 8


def far(x, dtype, ld=FAR):
    """x with a leading dimension of ld (the rest uninitialised)."""
    out = torch.empty((x.shape[0], ld), dtype=dtype, device=DEV)[:, :x.shape[1]]
    out.copy_(x)
    return out


@pytest.mark.parametrize("M,prec,wd", [(1200, "bf16", BF16), (9, "bf16", BF16), (600, "f32", F32), (600, "f32", BF16)])
def test_dense(M, prec, wd):
    N, K = 1100, 72
    A, W, C, res = ints((M, K), -8, 8, 1), ints((N, K), -4, 4, 2), ints((M, N), -50, 50, 3), ints((M, N), -99, 99, 4)
    want = R.epilogue_bits(A.double() @ W.double().T, C, None, "relu", False, res)
    Y = far(torch.zeros((M, N), device=DEV), F32)
    sp.linear_epilogue(far(A, F32 if prec == "f32" else BF16), sp.PRECS[prec], far(W, wd), C=far(C, F32), act="relu",
                       residual=far(res, F32), Y=Y)
    assert torch.equal(Y, want)


@pytest.mark.parametrize("rows,prec", [(5, "bf16"), (1500, "bf16"), (40, "bf16x3"), (700, "f32")])
def test_by_expert(rows, prec):
    """Two experts' W 2^31 elements apart; rows in order and gathered (a plane of A near 2^31 bytes)."""
    N, K, wd = 200, 72, F32 if prec == "f32" else BF16
    n = [rows // 3, rows - rows // 3]
    offsets = R.counts_to_offsets(n).to(DEV)
    gap = (1 << 31) + 64
    store = torch.empty(gap + N * K, dtype=wd, device=DEV)
    W = store.as_strided((2, N, K), (gap, K, 1))
    W[0], W[1] = ints((N, K), -4, 4, 2), ints((N, K), -4, 4, 3)
    A, C = ints((rows, K), -8, 8, 1), ints((rows, N), -50, 50, 3)
    P = torch.cat([A[:n[0]].double() @ W[0].double().T, A[n[0]:].double() @ W[1].double().T])
    want = R.epilogue_bits(P, C)
    planes = R.split(A, prec)
    far_a = torch.empty(planes.shape[:2] + (FAR if planes.shape[0] == 1 else K,), dtype=planes.dtype, device=DEV)[:, :, :K]
    far_a.copy_(planes)
    assert torch.equal(sp.grouped_linear(far_a, sp.PRECS[prec], W, offsets, C=far(C, F32), Y=far(torch.zeros_like(C), F32)), want)
    # gathered: 1024 rows of (2^20 - 8) bfloat16 are just below 2^31 bytes (binary32: half as many)
    tokens = (1 << 31) // (FAR * planes.element_size())
    tall = torch.empty((planes.shape[0], tokens, FAR if planes.shape[0] == 1 else K), dtype=planes.dtype, device=DEV)[:, :, :K]
    index = (tokens - 1 - torch.arange(rows, device=DEV) % tokens).to(torch.int32)
    tall[:, index.long()] = planes[:, :rows]
    if rows <= tokens:
        assert torch.equal(sp.grouped_linear(tall, sp.PRECS[prec], W, offsets, row_index=index, C=C), want)


def test_combine():
    T, k, N, ld = 800, 3, 40, 1 << 20
    H = far(ints((T * k, N), -9, 9, 1), F32, ld)
    slot = torch.randperm(T * k, device=DEV).to(torch.int32).reshape(T, k)
    want = sum(H[slot[:, j].long()] for j in range(k))
    Y = far(torch.zeros((T, N), device=DEV), F32, ld)
    assert torch.equal(sp.combine(H, slot, torch.ones((T, k), device=DEV), Y=Y), want)
