"""The GELU's own error, apart from the product's: a product of zeros, so that z is the bias, exact.

The largest error allowed relative to the GELU, in halves of a step of binary32 (u = 2^-24): Phi(z) is 1/2 + z p(z^2), or an
exponential times t q(t).
 1/2 + z p, |z| < 1.4: p lies in 1/4 .. 1/2, so its last step rounds by u / 4, those before by less than as much again after
   their powers of z^2, and the rounding of z^2 moves p by 0.11 u at most; times 1.4 with 0.03 u of the fit and the last sum's
   u Phi / 2 that is 0.9 u, 11.1 u of Phi(-1.4) = 0.0808; z times it another u: 12.1 u.
 beyond: t has a sum and a reciprocal of one unit (1 + 2 u), of which t q(t) takes at most 1.3 times, 1.3 x 3 u; q's seven
   steps u each on terms that sum to 1.12 q at most, the larger ones last, 3 u; the fit 0.5 u; the exponential of one unit
   2 u; two products and that with z 3 u: 12.4 u.  Its exponent, z^2 / 2, has two roundings and a constant off by 0.23 u: 2.23 u
   z^2 / 2.
On the positive side this is an error of 1 - Phi(z) < 0.081, and the rest is two roundings.
"""
import pytest
import torch

import paper_2609_15039_amd as sp

from tests.test_gpu_epilogue import DEV, F32, KINDS

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def points():
    g = torch.Generator().manual_seed(3)
    spread = [(-13.0, -6.0), (-6.0, -4.0), (-4.0, -2.0), (-2.0, -1.0), (-1.0, 0.0), (0.0, 1.0), (1.0, 2.0), (2.0, 13.0)]
    z = [lo + (hi - lo) * torch.rand(500, generator=g) for lo, hi in spread]
    edge = torch.tensor(1.4)
    tiny = [torch.tensor([s * 10.0 ** e for s in (1, -1) for e in range(-30, 0)])]
    return torch.cat(z + tiny + [torch.stack([edge, -edge, torch.nextafter(edge, 2 * edge), -torch.nextafter(edge, 2 * edge),
                                              torch.nextafter(edge, 0 * edge), -torch.nextafter(edge, 0 * edge)])])


def run(z, prec, layout, M, **kw):
    W = torch.zeros((z.numel(), 64), device=DEV, dtype=F32 if layout == "f32" else torch.bfloat16)
    A = torch.zeros((3 if prec == "bf16x3" else 1, M, 64), device=DEV, dtype=F32 if prec == "f32" else torch.bfloat16)
    return sp.linear_epilogue(A, sp.PRECS[prec], sp.tile_weights(W) if layout == "tiled" else W, bias=z.to(DEV), act="gelu", **kw)


@pytest.mark.parametrize("prec,layout", KINDS)
@pytest.mark.parametrize("M", [1, 40, 400])
def test_error_relative_to_the_gelu(M, prec, layout):
    z = points()
    Y = run(z, prec, layout, M).cpu().double()
    zd = z.double()
    want = 0.5 * zd * torch.erfc(-zd * 0.5 ** 0.5)
    allowed = torch.where(zd < 0, 12.5 + torch.where(zd <= -1.4, 1.12 * zd ** 2, 0.0), 4.0) * 1.01 * U * want.abs()
    off = (Y - want).abs() / (allowed + torch.finfo(F32).tiny)
    print(M, prec, layout, "off / allowed %.2g at z = %.9g" % (float(off.max()), float(z[int(off.max(0).values.argmax())])), flush=True)
    assert (off <= 1).all()


@pytest.mark.parametrize("prec,layout", KINDS)
def test_no_less_exact_than_the_formula_in_binary32(prec, layout):
    """Root mean square over each range, against z (1 + erf(z / sqrt 2)) / 2 step by step in binary32; where the last product's
    rounding is all that both have, 20000 of them agree to a few hundredths, for which a tenth is left."""
    g = torch.Generator().manual_seed(9)
    for lo, hi in ((-8.0, -4.0), (-4.0, -3.0), (-3.0, -2.0), (-2.0, -1.0), (-1.0, -0.01), (-0.01, 0.01), (0.01, 1.0), (1.0, 2.0), (2.0, 8.0)):
        z = lo + (hi - lo) * torch.rand(20000, generator=g)
        want = 0.5 * z.double() * torch.erfc(-z.double() * 0.5 ** 0.5)
        plain = 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
        rms = [float((y.cpu().double() - want).square().mean().sqrt()) for y in (run(z, prec, layout, 1)[0], plain)]
        print(lo, hi, "%.3g, step by step %.3g" % tuple(rms), flush=True)
        assert rms[0] <= 1.1 * rms[1]
