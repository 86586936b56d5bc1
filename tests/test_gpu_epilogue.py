"""splitee_linear_epilogue against a plain reference in 64 bits, and bit for bit on integers."""
import pytest
import torch

import paper_2609_15039_amd as sp
import workloads as WL

from tests import expert_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
# precision, weights
KINDS = [("bf16", "rows"), ("bf16", "tiled"), ("bf16x3", "rows"), ("bf16x3", "tiled"), ("f32", "rows"), ("f32", "f32")]


def weights(W, layout):
    if layout == "f32":
        return W.to(DEV)
    W = W.to(BF16).to(DEV)
    return sp.tile_weights(W) if layout == "tiled" else W


def padded(x, dtype=F32, extra=0, fill=float("nan")):
    """x on the device inside a wider array, whose rest holds `fill`."""
    per = 16 // dtype.itemsize
    ld = (-(-x.shape[-1] // per) + extra) * per
    out = torch.full((x.shape[0], ld), fill, dtype=dtype, device=DEV)
    out[:, :x.shape[1]] = x.to(DEV, dtype)
    return out[:, :x.shape[1]]


def ints(shape, lo, hi, seed):
    return torch.from_numpy(WL.gen_int(shape, lo, hi, seed))


SHAPES = [(1, 1, 8), (1, 100, 72), (2, 33, 64), (3, 257, 136), (15, 64, 2560), (16, 640, 520), (17, 130, 1032), (31, 96, 200),
          (33, 515, 392), (64, 128, 512), (65, 300, 1096), (100, 2050, 128), (129, 257, 648), (255, 512, 72), (257, 300, 256),
          (300, 1000, 2056), (513, 770, 64), (1025, 264, 328), (700, 2600, 136)]


@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_integers_are_exact(M, N, K, prec, layout):
    """Every part of the epilogue on, gated and not, into arrays wider than the result."""
    X, W2 = ints((M, K), -8, 8, M + K), ints((2 * N, K), -4, 4, N + K)
    for gated, out, parts in ((False, F32, "Cbr"), (True, BF16, "Cbr"), (True, F32, ""), (False, BF16, "b")):
        print(M, N, K, prec, layout, gated, out, parts, flush=True)
        W = W2 if gated else W2[:N]
        NW = W.shape[0]
        C = ints((M, NW), -50, 50, 1) if "C" in parts else None
        bias = ints((1, NW), -9, 9, 2)[0] if "b" in parts else None
        res = ints((M, N), -99, 99, 3) if "r" in parts else None
        want = R.epilogue_bits(X.double() @ W.double().T, C, bias, "relu", gated, res.to(out) if "r" in parts else None, out)
        Y = padded(torch.zeros(M, N), out, extra=1)
        Y.fill_(float("nan"))
        sp.linear_epilogue(R.split(X, prec).to(DEV), sp.PRECS[prec], weights(W, layout),
                           C=padded(C, extra=1) if "C" in parts else None, bias=bias.to(DEV) if "b" in parts else None,
                           act="relu", gated=gated, residual=padded(res, out, extra=2) if "r" in parts else None,
                           out_dtype=out, Y=Y)
        assert torch.equal(Y.cpu(), want)
        assert torch.isnan(Y._base[:, N:]).all()  # nothing past column N


@pytest.mark.parametrize("act", list(sp.ACTS))
@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("M,N,K", [(1, 70, 264), (16, 96, 1096), (40, 200, 520), (200, 140, 712), (330, 520, 136)])
def test_within_the_bound(M, N, K, prec, layout, act):
    g = torch.Generator().manual_seed(M + N)
    X = torch.randn(M, K, generator=g)
    X = X.to(BF16).float() if prec == "bf16" else X
    W = torch.randn(2 * N, K, generator=g) * 0.1
    W = W if layout == "f32" else W.to(BF16).float()
    C, bias = torch.randn(M, 2 * N, generator=g), torch.randn(2 * N, generator=g)
    for gated, out in ((True, F32), (True, BF16), (False, F32)):
        NW = 2 * N if gated else N
        res = torch.randn(M, N, generator=g).to(out)
        want, bound = R.epilogue64(X.double() @ W[:NW].double().T, X.double().abs() @ W[:NW].double().abs().T, K, C[:, :NW],
                                   bias[:NW], act, gated, res, out)
        Y = sp.linear_epilogue(R.split(X, prec).to(DEV), sp.PRECS[prec], weights(W[:NW], layout), C=padded(C[:, :NW]),
                               bias=bias[:NW].to(DEV), act=act, gated=gated, residual=padded(res, out), out_dtype=out)
        off = (Y.cpu().double() - want).abs()
        print(M, N, K, prec, layout, act, gated, out, "off / bound %.2g" % float((off / bound).max()), flush=True)
        assert (off <= bound).all()


@pytest.mark.parametrize("M,N,K", [(5, 64, 0), (200, 300, 0), (0, 64, 64), (4, 0, 64)])
@pytest.mark.parametrize("prec,layout", [("bf16", "rows"), ("bf16x3", "tiled"), ("f32", "f32")])
def test_empty(M, N, K, prec, layout):
    """K = 0 is a product of zeros; no rows or columns is an empty call."""
    A = R.split(torch.zeros(M, K), prec).to(DEV)
    W = torch.zeros((N, K), dtype=F32 if layout == "f32" else BF16, device=DEV)
    if layout == "tiled":
        W = sp.TiledWeights(torch.zeros(1, dtype=BF16, device=DEV), N, K)
    bias = torch.arange(N, dtype=F32, device=DEV)
    Y = sp.linear_epilogue(A, sp.PRECS[prec], W, bias=bias if N else None)
    assert Y.shape == (M, N) and torch.equal(Y, bias[:N].expand(M, N))


@pytest.mark.parametrize("prec,layout", [("bf16", "rows"), ("bf16", "tiled"), ("bf16x3", "tiled"), ("f32", "rows")])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_values_past_the_operands_do_not_reach_the_result(M, prec, layout):
    """A and W as parts of wider arrays of NaN: a ragged K tile, row padding, rows past the last."""
    N, K, wide = 70, 200, 216
    X, W = ints((M, K), -8, 8, 1), ints((N, K), -4, 4, 2)
    planes = R.split(X, prec)
    A = torch.full((planes.shape[0], M, wide), float("nan"), dtype=planes.dtype, device=DEV)
    A[:, :, :K] = planes.to(DEV)
    Wd = torch.full((N + 40, wide), float("nan"), dtype=BF16, device=DEV)
    Wd[:N, :K] = W.to(DEV, BF16)
    Wv = sp.tile_weights(Wd[:N, :K]) if layout == "tiled" else Wd[:N, :K]
    Y = sp.linear_epilogue(A[:, :, :K], sp.PRECS[prec], Wv)
    assert torch.equal(Y.cpu().double(), X.double() @ W.double().T)


@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("M", [3, 50, 400])
def test_infinities_and_nan_stay_in_their_row(M, prec, layout):
    N, K = 100, 136
    X, W = ints((M, K), -8, 8, 1), ints((N, K), 1, 4, 2)
    X[0, 5], X[M - 1, 7] = float("inf"), float("nan")
    planes = R.split(X, prec)
    if planes.shape[0] == 3:
        planes[1:, 0, 5] = 0  # the split of an infinity: the first plane alone
    Y = sp.linear_epilogue(planes.to(DEV), sp.PRECS[prec], weights(W, layout)).cpu().double()
    assert torch.equal(Y[1:M - 1], (X.double() @ W.double().T)[1:M - 1])
    assert torch.isinf(Y[0]).all() and torch.isnan(Y[M - 1]).all()


@pytest.mark.parametrize("act", list(sp.ACTS))
@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("M", [1, 40, 400])
def test_activations_at_the_ends_of_the_range(M, prec, layout, act):
    """A product of zeros, so that z is the bias: infinities, NaN and values whose squares or cubes overflow give what
    the formula gives (+inf stays +inf, -inf is 0 of a ReLU and else NaN), the others 16 u of |z|."""
    inf, low = float("inf"), torch.finfo(F32).min
    z = torch.tensor([inf, -inf, float("nan"), -low, low, 1e20, -1e20, 1e13, -1e13, 100.0, -100.0, 20.0, -20.0, 5.0, -5.0, 0.0, 1e-30])
    z = z.repeat(11)
    W = weights(torch.ones(z.numel(), 64), layout)
    Y = sp.linear_epilogue(R.split(torch.zeros(M, 64), prec).to(DEV), sp.PRECS[prec], W, bias=z.to(DEV), act=act).cpu().double()
    want = R.act64(z.double(), act).expand(M, -1)
    assert torch.equal(torch.isnan(Y), torch.isnan(want))
    ends = torch.isinf(want)
    assert torch.equal(Y[ends], want[ends])
    rest = ~ends & ~torch.isnan(want)
    bound = 16 * R.U * z.double().abs().expand(M, -1) + torch.finfo(F32).tiny
    assert ((Y - want)[rest].abs() <= bound[rest]).all()


@pytest.mark.parametrize("M,N,K,prec", [(2, 512, 2560, "bf16x3"), (60, 256, 4096, "bf16"), (300, 640, 2048, "bf16x3")])
def test_residual_in_place(M, N, K, prec):
    X, W, res = ints((M, K), -8, 8, 1), ints((N, K), -4, 4, 2), ints((M, N), -99, 99, 3)
    for out in (F32, BF16):
        want = R.epilogue_bits(X.double() @ W.double().T, residual=res.to(out), out=out)
        Y = res.to(DEV, out)
        sp.linear_epilogue(R.split(X, prec).to(DEV), sp.PRECS[prec], weights(W, "rows"), residual=Y, Y=Y, out_dtype=out)
        assert torch.equal(Y.cpu(), want)


def test_same_product_as_masked_linear_unmask():
    """The unmask alone: the values of splitee_masked_linear_unmask, up to the order of the sums."""
    M, N, K = 77, 600, 1032
    X, W = torch.from_numpy(WL.gen_x(M, K)).to(DEV), torch.from_numpy(WL.gen_w(N, K)).to(DEV).to(BF16)
    eta = sp.noise(M, K, sp.SPLITEE_MECH_GAUSSIAN, 1.0, 1.0, 0, 1)
    Xt = sp.mask(X, eta, sp.SPLITEE_PREC_BF16X3)
    C = sp.correction(W, M, sp.SPLITEE_MECH_GAUSSIAN, 1.0, 1.0, 0, 1)
    a, b = sp.masked_linear_unmask(Xt, sp.SPLITEE_PREC_BF16X3, W, C), sp.linear_epilogue(Xt, sp.SPLITEE_PREC_BF16X3, W, C=C)
    S = (X + eta).double().abs() @ W.double().abs().T
    assert ((a.double() - b.double()).abs() <= 2 * (K + 8) * R.U * 1.01 * S).all()


@pytest.mark.parametrize("M,N,K,prec,layout", [(1, 2560, 9728, "bf16x3", "tiled"), (40, 2560, 4096, "f32", "rows"),
                                               (333, 2560, 9728, "bf16", "rows"), (600, 1030, 2056, "bf16x3", "rows")])
def test_repeats_and_replays(M, N, K, prec, layout):
    """The same bits again, on another stream, and from a captured graph replayed between eager calls."""
    g = torch.Generator(device=DEV).manual_seed(M)
    A = R.split(torch.randn(M, K, generator=g, device=DEV), prec)
    W = weights(torch.randn(N, K, generator=g, device=DEV).cpu(), layout)
    bias = torch.randn(N, generator=g, device=DEV)
    nbytes = sp.splitee_epilogue_workspace_bytes(M, N, K, sp.PRECS[prec], False)

    def call(Y, ws):
        return sp.linear_epilogue(A, sp.PRECS[prec], W, bias=bias, act="silu", ws=(ws, nbytes), Y=Y)

    def space():
        return padded(torch.full((M, N), float("nan"))), sp._aligned_bytes(nbytes, DEV).fill_(255)
    first = call(*space())
    again = call(*space())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = call(*space())
    torch.cuda.synchronize()
    assert torch.equal(first, again) and torch.equal(first, other)
    Y, ws = space()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(Y, ws)
    for _ in range(3):
        Y.zero_()
        ws.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, first)
        assert torch.equal(call(*space()), first)
