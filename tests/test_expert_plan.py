"""Which kernel a product with an epilogue takes: every one that any shape takes is among those that the GPU
tests run (tests/test_gpu_linear_plans.py).  Host only."""
import math
import random

import pytest

import paper_2609_15039_amd as sp

from tests.linear_shapes import DENSE, GROUPED

BF16, X3 = sp.SPLITEE_PREC_BF16, sp.SPLITEE_PREC_BF16X3


def variant(rows, groups, dense, N, K, prec, gated):
    kind, bm, tn, nw, ksplit, halve = sp.splitee_linear_plan_probe(rows, groups, dense, N, K, prec, gated)
    assert 1 <= ksplit <= 8 and (dense or ksplit == 1) and (kind == 0) == (bm > 0)
    return prec, gated, dense, kind, bm, tn, nw, ksplit > 1, halve


def test_every_kernel_is_run_by_a_test():
    run = set()
    for prec in (BF16, X3):
        for gated in (False, True):
            run |= {variant(M, 1, True, N, K, prec, gated) for M, N, K in DENSE}
            run |= {variant(sum(n), len(n), False, N, K, prec, gated) for n, N, K in GROUPED}
    rng = random.Random(2)

    def log(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    missing = {}
    for _ in range(30000):
        dense = rng.random() < 0.5
        shape = (log(1, 9000), 1 if dense else log(2, 200), dense, log(1, 10000), log(8, 10000) // 8 * 8)
        for prec in (BF16, X3):
            for gated in (False, True):
                v = variant(*shape, prec, gated)
                if v not in run:
                    missing.setdefault(v, shape)
    assert not missing


@pytest.mark.parametrize("bad", [(0, 1, True, 8, 8, BF16, 0), (8, 0, False, 8, 8, BF16, 0), (8, 1, True, 8, 12, BF16, 0),
                                 (8, 1, True, 8, 8, sp.SPLITEE_PREC_F32, 0)])
def test_probe_refuses(bad):
    with pytest.raises(sp.SpliteeError):
        sp.splitee_linear_plan_probe(*bad)


@pytest.mark.parametrize("prec", [sp.SPLITEE_PREC_F32, BF16, X3])
def test_workspace_covers_the_splits(prec):
    """Partial products of every split, gate and up columns apart; binary32 has the GEMM's and the product."""
    for M, N, K in DENSE:
        for gated in (0, 1):
            need = sp.splitee_epilogue_workspace_bytes(M, N, K, prec, gated)
            row = -(-N // 4) * 4 * (1 + gated) * 4
            if prec == sp.SPLITEE_PREC_F32:
                assert need >= M * row
            else:
                ks = sp.splitee_linear_plan_probe(M, 1, True, N, K, prec, gated)[4]
                assert need == (ks * M * row if ks > 1 else 0)
