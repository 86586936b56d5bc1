"""Binary32 by expert on both sides of the border between 16- and 64-row tiles, bit for bit on integers."""
import numpy as np
import pytest
import torch

import paper_2609_15039_amd as sp

from tests import expert_ref as R
from tests.test_gpu_epilogue import BF16, DEV, F32
from tests.test_gpu_linear_plans import fresh, ints, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", [F32, BF16])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("per", [1, 24, 25, 32, 33, 48, 49, 64])
@pytest.mark.parametrize("N,K", [(70, 264), (260, 1032)])
def test_both_sides(N, K, per, gated, w):
    """`per` rows an expert on average, spread unevenly over five, one with none."""
    n = [per * 5 // 4, 0, per * 5 // 2, 1, 0]
    n[4] = per * 5 - sum(n)
    rows, begin = sum(n), np.concatenate([[0], np.cumsum(n)])
    offsets = R.counts_to_offsets(n).to(DEV)
    A, W = ints((rows, K), -8, 8, per), ints((5, 2 * N if gated else N, K), -4, 4, N).to(w)
    C, bias = ints((rows, W.shape[1]), -50, 50, 1), ints((5, W.shape[1]), -9, 9, 2)
    P = torch.cat([A[begin[e]:begin[e + 1]].double() @ W[e].double().T for e in range(5)])
    expert = torch.repeat_interleave(torch.arange(5), torch.tensor(n)).to(DEV)
    for index in (None, torch.arange(rows - 1, -1, -1, dtype=torch.int32, device=DEV)):
        X = A if index is None else A.flip(0).contiguous()  # gathered back into the same order
        Y = sp.grouped_linear(X, sp.SPLITEE_PREC_F32, W, offsets, row_index=index, C=rows_of(C, F32), bias=bias, act="relu", gated=gated,
                              Y=fresh(rows, N, F32))
        assert torch.equal(Y, R.epilogue_bits(P, C, bias[expert], "relu", gated))
