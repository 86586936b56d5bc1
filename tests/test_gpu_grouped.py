"""splitee_grouped_linear against a plain reference in 64 bits, and bit for bit on integers."""
import numpy as np
import pytest
import torch

import paper_2609_15039_amd as sp
import workloads as WL

from tests import expert_ref as R
from tests.test_gpu_epilogue import BF16, DEV, F32, KINDS, ints, padded

pytestmark = pytest.mark.gpu

# rows of each expert: one row, none, few, ragged, one expert with all, more experts than a wave has lanes
COUNTS = {"one": [0, 0, 1, 0], "few": [1, 0, 3, 2, 0, 1, 1, 4], "ragged": [5, 17, 0, 33, 64, 1, 100, 16], "all-in-one": [0, 300, 0],
          "large": [257, 0, 600, 31], "single": [140], "many": [(7 * i) % 5 for i in range(150)], "none": [0, 0, 0]}


def weights(W, layout):
    if layout == "f32":
        return W.to(DEV)
    W = W.to(BF16).to(DEV)
    return sp.tile_experts(W) if layout == "tiled" else W


@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("N,K", [(40, 72), (257, 200), (128, 1032)])
@pytest.mark.parametrize("counts", list(COUNTS))
def test_integers_are_exact(counts, N, K, prec, layout):
    """Gathered and in order; rows before the first expert's and behind the last's are left as they were."""
    n = COUNTS[counts]
    E, before, behind = len(n), 2, 3
    offsets = R.counts_to_offsets(n) + before
    rows = int(offsets[-1]) + behind
    tokens = max(1, rows // 2)
    rng = np.random.default_rng(N + rows)
    W2 = ints((E, 2 * N, K), -4, 4, N + K)
    for gather, gated, out, parts in ((True, True, BF16, "Cb"), (False, False, F32, "br"), (True, False, F32, ""), (False, True, BF16, "r")):
        print(counts, N, K, prec, layout, gather, gated, out, parts, flush=True)
        X = ints((tokens if gather else rows, K), -8, 8, rows)
        index = torch.from_numpy(rng.integers(0, tokens, rows).astype(np.int32)) if gather else None
        W = W2 if gated else W2[:, :N].contiguous()
        NW = W.shape[1]
        P, _ = R.grouped64(X.double(), W.double(), offsets, index)
        expert = torch.repeat_interleave(torch.arange(E), torch.tensor(n))
        C = ints((rows, NW), -50, 50, 1) if "C" in parts else None
        bias = ints((E, NW), -9, 9, 2) if "b" in parts else None
        res = ints((rows, N), -99, 99, 3).to(out) if "r" in parts else None
        live = slice(before, rows - behind)
        want = torch.full((rows, N), 7.0, dtype=out)
        want[live] = R.epilogue_bits(P[live], None if C is None else C[live], None if bias is None else bias[expert],
                                     "relu", gated, None if res is None else res[live], out)
        Y = padded(torch.zeros(rows, N), out, extra=1)
        Y.fill_(7.0)
        sp.grouped_linear(R.split(X, prec).to(DEV), sp.PRECS[prec], weights(W, layout), offsets.to(DEV),
                          row_index=None if index is None else index.to(DEV), C=None if C is None else padded(C, extra=1),
                          bias=None if bias is None else bias.to(DEV), act="relu", gated=gated,
                          residual=None if res is None else padded(res, out), out_dtype=out, Y=Y)
        assert torch.equal(Y.cpu(), want)
        assert torch.isnan(Y._base[:, N:]).all()


@pytest.mark.parametrize("act", list(sp.ACTS))
@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("counts", ["few", "ragged"])
def test_within_the_bound(counts, prec, layout, act):
    n, N, K = COUNTS[counts], 90, 328
    offsets = R.counts_to_offsets(n)
    rows, E = int(offsets[-1]), len(n)
    g = torch.Generator().manual_seed(rows)
    X = torch.randn(rows, K, generator=g)
    X = X.to(BF16).float() if prec == "bf16" else X
    W = torch.randn(E, 2 * N, K, generator=g) * 0.1
    W = W if layout == "f32" else W.to(BF16).float()
    P, S = R.grouped64(X.double(), W.double(), offsets, None)
    C, bias = torch.randn(rows, 2 * N, generator=g), torch.randn(E, 2 * N, generator=g)
    expert = torch.repeat_interleave(torch.arange(E), torch.tensor(n))
    for out in (F32, BF16):
        want, bound = R.epilogue64(P, S, K, C, bias[expert], act, True, None, out)
        Y = sp.grouped_linear(R.split(X, prec).to(DEV), sp.PRECS[prec], weights(W, layout), offsets.to(DEV), C=padded(C),
                              bias=bias.to(DEV), act=act, gated=True, out_dtype=out)
        off = (Y.cpu().double() - want).abs()
        print(counts, prec, layout, act, out, "off / bound %.2g" % float((off / bound).max()), flush=True)
        assert (off <= bound).all()


@pytest.mark.parametrize("prec,layout", [("bf16", "rows"), ("bf16x3", "tiled"), ("f32", "f32")])
def test_indices_and_offsets_out_of_range_are_clamped(prec, layout):
    """An index past A takes its first or last row; offsets past the rows end there."""
    rows, tokens, N, K = 40, 10, 33, 136
    X, W = ints((tokens, K), -8, 8, 1), ints((3, N, K), -4, 4, 2)
    index = torch.arange(rows, dtype=torch.int32) - 15  # -15 .. 24
    offsets = torch.tensor([-5, 7, 30, 2 ** 31 - 1], dtype=torch.int32)
    want, _ = R.grouped64(X.double(), W.double(), offsets.clamp(0, rows), index.clamp(0, tokens - 1))
    Y = sp.grouped_linear(R.split(X, prec).to(DEV), sp.PRECS[prec], weights(W, layout), offsets.to(DEV), row_index=index.to(DEV))
    assert torch.equal(Y.cpu().double(), want)


@pytest.mark.parametrize("prec,layout", [("bf16", "rows"), ("bf16", "tiled"), ("bf16x3", "rows"), ("f32", "rows")])
@pytest.mark.parametrize("counts", ["few", "large"])
def test_values_of_other_rows_and_experts_do_not_reach_the_result(counts, prec, layout):
    """Experts without rows hold NaN, and so do tokens that no row takes and the padding of A and W."""
    n, N, K, wide = COUNTS[counts], 70, 200, 232
    offsets = R.counts_to_offsets(n)
    rows, E = int(offsets[-1]), len(n)
    X, W = ints((rows, K), -8, 8, 1), ints((E, N, K), -4, 4, 2)
    P, _ = R.grouped64(X.double(), W.double(), offsets, None)
    planes = R.split(X, prec)
    A = torch.full((planes.shape[0], 2 * rows, wide), float("nan"), dtype=planes.dtype, device=DEV)
    A[:, 1::2, :K] = planes.to(DEV)
    Wd = torch.full((E, N + 3, wide), float("nan"), dtype=BF16, device=DEV)
    for e in range(E):
        if n[e]:
            Wd[e, :N, :K] = W[e].to(DEV, BF16)
    Wv = sp.tile_experts(Wd[:, :N, :K]) if layout == "tiled" else Wd[:, :N, :K]
    index = (2 * torch.arange(rows) + 1).to(torch.int32).to(DEV)
    Y = sp.grouped_linear(A[:, :, :K], sp.PRECS[prec], Wv, offsets.to(DEV), row_index=index)
    assert torch.equal(Y.cpu().double(), P)


def test_repeats_and_replays_with_other_groups():
    """A captured call goes by the offsets that are on the device when it is replayed."""
    E, N, K, rows = 8, 200, 264, 90
    X, W = ints((rows, K), -8, 8, 1), ints((E, N, K), -4, 4, 2)
    A, Wd = R.split(X, "bf16").to(DEV), weights(W, "rows")
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    Y = torch.empty((rows, N), device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.grouped_linear(A, sp.SPLITEE_PREC_BF16, Wd, off, Y=Y)
    rng = np.random.default_rng(0)
    for _ in range(4):
        n = rng.multinomial(rows, np.full(E, 1 / E))
        offsets = R.counts_to_offsets(n)
        off.copy_(offsets)
        Y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, _ = R.grouped64(X.double(), W.double(), offsets, None)
        assert torch.equal(Y.cpu().double(), want)
        assert torch.equal(sp.grouped_linear(A, sp.SPLITEE_PREC_BF16, Wd, off), Y)
