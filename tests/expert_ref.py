"""Plain references of the projections with an epilogue and of the expert path.

Values in 64 bits with a bound of the binary32 kernels' error beside them, and, for integers, the
very bits: sums of small integers are exact in any order, and what follows the sum (C, bias, a
ReLU, the gate's product, the residual, the rounding to the output's type) is one rounding each.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24  # half a step of binary32


def act64(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return torch.relu(z) if act == "relu" else z


def epilogue64(R, S, terms, C=None, bias=None, act="none", gated=False, residual=None, out=torch.float32):
    """(value, bound) in 64 bits of the epilogue on the exact product R, where a binary32 sum of `terms`
    products whose absolute values sum to S stands in for R.

    z is off by at most terms u S (any order of a sum: gamma_n) plus u |.| for each of C and bias.  The
    activations' slopes are below 1.13, their own evaluation (expf, erff, tanhf, a quotient, up to five
    products) is taken as 16 u of |z|: each factor but z is at most 2 and the device functions' errors are a few
    units in the last place of theirs.  A product of two such values is off by the sum of
    each error times the other's magnitude and u of itself, the residual's sum by u of itself, and
    the last rounding by half a step of the output's type."""
    z, dz = R, (terms + 8) * U * 1.01 * S
    if C is not None:
        z = z - C.double()
        dz = dz + U * (z.abs() + dz)
    if bias is not None:
        z = z + bias.double()
        dz = dz + U * (z.abs() + dz)
    N = z.shape[-1] // (2 if gated else 1)
    h, dh = act64(z[..., :N], act), dz[..., :N]
    if act != "none":
        dh = 1.13 * dh + 16 * U * z[..., :N].abs()
    if gated:
        up, du = z[..., N:], dz[..., N:]
        dh = dh * (up.abs() + du) + du * h.abs() + U * (h * up).abs()
        h = h * up
    if residual is not None:
        h = h + residual.double()
        dh = dh + U * (h.abs() + dh)
    step = torch.finfo(out).eps / 2
    return h, dh + step * (h.abs() + dh) + torch.finfo(torch.float32).tiny


def epilogue_bits(R, C=None, bias=None, act="none", gated=False, residual=None, out=torch.float32):
    """The epilogue on a product R of integers below 2^24 (float64), step by step in binary32; act none or relu."""
    assert act in ("none", "relu") and float(R.abs().max() if R.numel() else 0) < 2 ** 24
    z = R.float()
    if C is not None:
        z = z - C
    if bias is not None:
        z = z + bias
    N = z.shape[-1] // (2 if gated else 1)
    h = torch.relu(z[..., :N]) if act == "relu" else z[..., :N]
    if gated:
        h = h * z[..., N:]
    if residual is not None:
        h = h + residual.float()
    return h.to(out)


def split(X, prec):
    """The planes of splitee_mask for a mask of zeros: "f32", "bf16" (X must be bfloat16 values) or "bf16x3"."""
    if prec == "f32":
        return X[None].contiguous()
    hi = X.to(torch.bfloat16)
    if prec == "bf16":
        return hi[None].contiguous()
    mid = (X - hi.float()).to(torch.bfloat16)
    lo = (X - hi.float() - mid.float()).to(torch.bfloat16)
    return torch.stack([hi, mid, lo])


def counts_to_offsets(counts):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))


def grouped64(X, W, offsets, row_index):
    """(R, S) of the grouped product by expert, zeros for rows of no expert; X rows x K and W float64."""
    rows = X.shape[0] if row_index is None else row_index.numel()
    R = torch.zeros((rows, W.shape[1]), dtype=torch.float64)
    S = torch.zeros_like(R)
    for e in range(W.shape[0]):
        b, n = int(offsets[e]), int(offsets[e + 1])
        if n > b:
            x = X[b:n] if row_index is None else X[row_index[b:n].long()]
            R[b:n], S[b:n] = x @ W[e].T, x.abs() @ W[e].abs().T
    return R, S


def route_ref(logits, k, score, renorm):
    """Row by row in Python and 64 bits: experts, weights, offsets, row_index, slot as numpy arrays."""
    L = logits.double().numpy()
    T, E = L.shape
    experts, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    rows = [[] for _ in range(E)]
    for t in range(T):
        live = [e for e in range(E) if not math.isnan(L[t, e]) and L[t, e] != -math.inf]
        best = sorted(live, key=lambda e: (-L[t, e], e))[:k]
        if not best:
            continue
        m = L[t, best[0]]
        w = [math.exp(L[t, e] - m) if score == "softmax" else 0.0 if L[t, e] < -700 else 1 / (1 + math.exp(-L[t, e]))
             for e in best]
        if renorm:
            w = [x / sum(w) if sum(w) else 0.0 for x in w]
        elif score == "softmax":
            total = sum(math.exp(L[t, e] - m) for e in live)
            w = [x / total for x in w]
        for j, (e, x) in enumerate(zip(best, w)):
            experts[t, j], weights[t, j] = e, x
            rows[e].append((t, j))
    offsets = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int32)
    row_index, slot = np.full(T * k, -1, np.int32), np.full((T, k), -1, np.int32)
    for e in range(E):
        for i, (t, j) in enumerate(rows[e]):
            row_index[offsets[e] + i] = t
            slot[t, j] = offsets[e] + i
    return experts, weights, offsets, row_index, slot
