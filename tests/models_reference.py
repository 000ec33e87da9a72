"""Local models in float64 on the CPU, from their definitions, each value with a bound on what float32 sums and one rounding to
the element type may be off by.

A rounding is off by half a step at most: u(t) = eps(t) / 2 of the value, half the least subnormal below the normal range.  A sum of n
terms in float32 in any order is off by n 2^-24 of the sum of their magnitudes; terms that are themselves rounded add
their own.  First-order bounds are doubled nowhere: second-order terms are covered by the factor (1 + 2^-6) at the end.
"""
import math

import torch

F32 = 2.0 ** -24
SLACK = 1.0 + 2.0 ** -6
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# Shapes (M, K, Din, Dout) whose products and gradients take every size of tile, with rows that are aligned and that are not
TILES = [(2000, 16, 136, 2304), (2001, 16, 137, 2303), (3000, 16, 1536, 136), (3001, 16, 1535, 137), (4500, 16, 136, 2560), (4501, 16, 133, 2559),
         (6000, 16, 2048, 136), (6001, 16, 2047, 139), (700, 16, 264, 1032), (701, 16, 263, 1033), (700, 16, 1024, 648), (701, 16, 1023, 649),
         (700, 3, 136, 136), (701, 3, 133, 135), (4100, 1, 512, 4096), (6000, 3, 520, 2304), (6001, 3, 521, 2303), (7000, 6, 1800, 1800)]
# and narrow ones, whose gradients take every block of results and features in several runs a group
NARROW = [(5000, 3, 64, 64), (5001, 7, 33, 32), (3000, 2, 17, 40), (70_000, 5, 37, 24), (2000, 1, 3, 5), (4000, 9, 1, 64), (4000, 9, 64, 1), (3001, 4, 50, 47)]
ACTIVATIONS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def half_step(t):
    return torch.finfo(t).eps / 2


def least(t):
    """Half the distance of two subnormals."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def rounded(value, error, t):
    """Bound after rounding value (known to within error) to t."""
    return SLACK * (error + half_step(t) * (value.abs() + error)) + least(t)


def check(got, want, bound, what):
    got, want, bound = got.detach().cpu().double(), want.cpu(), bound.cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    odd = ~finite & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), f"{what}: infinities differ"
    off = ((got - want).abs() - bound)[finite]
    assert off.numel() == 0 or bool((off <= 0).all()), \
        f"{what}: {int((off > 0).sum())} of {off.numel()} values beyond their bound, worst by {float(off.max()):.3e}"


def group(node, K):
    flat = node.reshape(-1).tolist()
    members = [[] for _ in range(K)]
    for p, e in enumerate(flat):
        if 0 <= e < K:
            members[e].append(p)
    offsets, order = [0], []
    for m in members:
        order += m
        offsets.append(len(order))
    slot = [-1] * len(flat)
    for s, p in enumerate(order):
        slot[p] = s
    order += [-1] * (len(flat) - len(order))
    i32 = dict(dtype=torch.int32)
    return torch.tensor(offsets, **i32), torch.tensor(order, **i32), torch.tensor(slot, **i32).reshape(node.shape)


def _two(slot):
    return slot if slot.dim() == 2 else slot[:, None]


def dispatch(X, slot, weight, out):
    """out (the places' contents before the call) with the rows in their places, and its bound."""
    want, bound = out.double().clone(), torch.zeros_like(out, dtype=torch.float64)
    s = _two(slot)
    w = None if weight is None else weight.double().reshape(s.shape)
    for t in range(s.shape[0]):
        for j in range(s.shape[1]):
            at = int(s[t, j])
            if 0 <= at < out.shape[0]:
                want[at] = X[t].double() * (1.0 if w is None else w[t, j])
                if w is not None:
                    bound[at] = rounded(want[at], F32 * want[at].abs() + least(torch.float32), out.dtype)
    return want, bound


def combine(Y, slot, weight):
    s = _two(slot)
    T, k = s.shape
    w = torch.ones((T, k), dtype=torch.float64) if weight is None else weight.double().reshape(T, k)
    want, size = (torch.zeros((T, Y.shape[1]), dtype=torch.float64) for _ in range(2))
    for t in range(T):
        for j in range(k):
            if 0 <= int(s[t, j]) < Y.shape[0]:
                term = w[t, j] * Y[int(s[t, j])].double()
                want[t] += term
                size[t] += term.abs()
    return want, rounded(want, k * F32 * size + k * least(torch.float32), Y.dtype)


def combine_grad(dout, Y, slot, weight, dY):
    """(dY, its bound, dweight, its bound); dY: the places' contents before the call."""
    s = _two(slot)
    want, bound = dispatch(dout, slot, weight, dY)
    dw, size = (torch.zeros(s.shape, dtype=torch.float64) for _ in range(2))
    for t in range(s.shape[0]):
        for j in range(s.shape[1]):
            if 0 <= int(s[t, j]) < Y.shape[0]:
                terms = dout[t].double() * Y[int(s[t, j])].double()
                dw[t, j] = terms.sum()
                size[t, j] = terms.abs().sum()
    n = Y.shape[1]
    return want, bound, dw.reshape(slot.shape), SLACK * (n * F32 * size + n * least(torch.float32)).reshape(slot.shape)


def activation(z, act):
    """The activation and its derivative; in the limits of infinite arguments what the function tends to."""
    one, zero = torch.ones_like(z), torch.zeros_like(z)
    if act == "none":
        return z, one
    if act == "relu":
        return torch.where(z < 0, zero, z), torch.where(torch.isnan(z), z, (z > 0).double())
    zf = torch.where(torch.isinf(z), zero, z)
    if act == "silu":
        g = torch.special.expit(zf)
        y, d = zf * g, g + zf * g * (1 - g)
    elif act == "gelu":
        g = 0.5 * torch.special.erfc(-zf / math.sqrt(2.0))
        y, d = zf * g, g + zf * torch.exp(-zf * zf / 2) / math.sqrt(2 * math.pi)
    else:
        c = 2 * math.sqrt(2 / math.pi)
        g = torch.special.expit(c * (zf + 0.044715 * zf ** 3))
        y, d = zf * g, g + zf * g * (1 - g) * c * (1 + 3 * 0.044715 * zf * zf)
    y = torch.where(z == math.inf, z, torch.where(z == -math.inf, zero, y))
    return y, torch.where(z == math.inf, one, torch.where(z == -math.inf, zero, d))


def product(X, A, offsets, bias, act, residual, out, pre):
    """(Y, its bound, z, its bound); out, pre: the rows' contents before the call."""
    A3 = A if A.dim() == 3 else A[None]
    K, dout, din = A3.shape
    bounds = [0, X.shape[0]] if offsets is None else offsets.tolist()
    want, bound = out.double().clone(), torch.zeros(out.shape, dtype=torch.float64)
    z, zb = pre.double().clone(), torch.zeros(out.shape, dtype=torch.float64)
    b = None if bias is None else bias.double().reshape(K, dout)
    for e in range(K):
        rows = slice(bounds[e], bounds[e + 1])
        x, a = X[rows].double(), A3[e].double()
        v = x @ a.t()
        size = x.abs() @ a.abs().t()
        if b is not None:
            v, size = v + b[e], size + b[e].abs()
        err = (din + 2) * (F32 * size + least(torch.float32))
        y, _ = activation(v, act)
        # no activation grows faster than 1.13 |z|; its factors are at most one and take sixteen roundings
        yerr = 1.13 * err + (0 if act in ("none", "relu") else 16 * F32 * v.abs())
        if residual is not None:
            r = residual[rows].double()
            y = y + r
            yerr = yerr + F32 * (y.abs() + r.abs())
        z[rows], zb[rows] = v, rounded(v, err, X.dtype)
        want[rows], bound[rows] = y, rounded(y, yerr, X.dtype)
    return want, bound, z, zb


def product_grad(dY, X, A, offsets, pre, act, dX):
    """(dX, bound, dA, bound, dbias, bound); dX: the rows' contents before the call."""
    A3 = A if A.dim() == 3 else A[None]
    K, dout, din = A3.shape
    t = X.dtype
    bounds = [0, X.shape[0]] if offsets is None else offsets.tolist()
    gx, bx = dX.double().clone(), torch.zeros(dX.shape, dtype=torch.float64)
    gA, bA = (torch.zeros(A3.shape, dtype=torch.float64) for _ in range(2))
    gb, bb = (torch.zeros((K, dout), dtype=torch.float64) for _ in range(2))
    for e in range(K):
        rows = slice(bounds[e], bounds[e + 1])
        n = max(0, bounds[e + 1] - bounds[e])
        x, a, dz = X[rows].double(), A3[e].double(), dY[rows].double()
        err = torch.zeros_like(dz)
        if act != "none":
            s = activation(pre[rows].double(), act)[1]
            if act != "relu":
                # thirty-two roundings of terms that stay below one: the arguments' errors meet falling exponentials
                err = 32 * F32 * dz.abs()
            dz = dz * s
            err = rounded(dz, err + F32 * dz.abs() + least(torch.float32), t)         # the operand of the products has type t
        tiny = least(torch.float32)
        gx[rows] = dz @ a
        bx[rows] = rounded(gx[rows], err @ a.abs() + (dout + 2) * (F32 * (dz.abs() + err) @ a.abs() + tiny), t)
        gA[e] = dz.t() @ x
        bA[e] = rounded(gA[e], err.t() @ x.abs() + (n + 2) * (F32 * (dz.abs() + err).t() @ x.abs() + tiny), t)
        gb[e] = dz.sum(0)
        bb[e] = rounded(gb[e], err.sum(0) + (n + 2) * (F32 * (dz.abs() + err).sum(0) + tiny), t)
    return gx, bx, gA.reshape(A.shape), bA.reshape(A.shape), gb.reshape(*A.shape[:-2], dout), bb.reshape(*A.shape[:-2], dout)
