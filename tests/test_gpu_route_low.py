"""Sigmoid scores far below binary32's smallest number, renormalised: their quotients are those of exp."""
import pytest
import torch

import paper_2609_15039_amd as sp

from tests.test_gpu_epilogue import DEV
from tests.test_gpu_route import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", [(1, 8, 4), (70, 64, 8), (300, 300, 5), (2100, 16, 16)])
@pytest.mark.parametrize("top", [-20.0, -80.0, -86.0, -89.0, -104.0, -500.0])
def test_low_logits(T, E, k, top):
    """Logits from `top` down by a few units: exp(-x) of binary32 overflows from 88.7 on, and from 87.3 to there the scores have fewer bits."""
    g = torch.Generator().manual_seed(T + E)
    L = top - 6 * torch.rand(T, E, generator=g)
    r = check(L, k, "sigmoid", True)
    assert (r.weights.sum(1).cpu() - 1).abs().max() < 1e-5


@pytest.mark.parametrize("renorm", [True, False])
def test_from_one_end_to_the_other(renorm):
    """Each token's largest logit somewhere from 100 down to -699, the others any distance below; some below -700, whose
    score is 0."""
    g = torch.Generator().manual_seed(7)
    T, E = 1000, 32
    first = 100 - 799 * torch.rand(T, 1, generator=g)
    L = first - torch.rand(T, E, generator=g) ** 4 * 300
    L[:, 3] = first[:, 0]
    check(L, 6, "sigmoid", renorm)


@pytest.mark.parametrize("T", [5, 200])
def test_no_score_at_all(T):
    """Logits below -700 only, the type's lowest value among them: chosen, with weights of 0."""
    L = torch.full((T, 12), torch.finfo(torch.float32).min)
    L[:, 5], L[:, 7] = -700.5, -2e4
    r = check(L, 4, "sigmoid", True)
    assert r.experts[0].tolist() == [5, 7, 0, 1] and (r.weights == 0).all()
    assert (sp.route(L.to(DEV), 4, score="sigmoid", renorm=False).weights == 0).all()
