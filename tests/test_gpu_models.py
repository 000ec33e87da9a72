"""Local models on the GPU against the float64 reference: rows sorted by node and back, products with the nodes' matrices, gradients."""
import math

import pytest
import torch

import models_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def som():
    from paper_2604_26555_amd import Som
    s = Som(0)
    yield s
    s.close()


def normal(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def padded(t, extra=0, lead=0):
    """The same matrix on the GPU with a leading dimension of its own and an offset of `lead` elements."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + extra) + lead + 8,), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[lead:lead + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
    view.copy_(t)
    return view


def draw_nodes(gen, T, k, K, how="even"):
    if how == "one":
        return torch.full((T, k), min(3, K - 1), dtype=torch.int32)
    if how == "none":
        return torch.full((T, k), -1, dtype=torch.int32)
    node = torch.randint(0, K, (T, k), generator=gen)
    if how == "skew":
        node = (torch.rand(T, k, generator=gen) ** 6 * K).long().clamp(max=K - 1)
    if how == "holes":
        node = torch.where(torch.rand(T, k, generator=gen) < 0.2, torch.randint(-5, 0, (T, k), generator=gen), node)
        node = torch.where(torch.rand(T, k, generator=gen) < 0.1, torch.randint(K, K + 9, (T, k), generator=gen), node)
        node[::7] = -1
    return node.int()


GROUPS = [(1, 1, 1, "even"), (1, 8, 128, "even"), (3, 2, 5, "none"), (63, 1, 2, "even"), (64, 1, 64, "one"), (65, 3, 7, "holes"), (257, 2, 1, "even"),
          (1000, 8, 100, "holes"), (2048, 1, 1024, "skew"), (4099, 4, 61, "holes"), (9001, 1, 8192, "even"), (5000, 2, 32768, "holes"),
          (70001, 2, 437, "skew"), (300_000, 1, 1024, "holes"), (100_000, 8, 3, "one"), (40_000, 1, 20_000, "skew")]


@pytest.mark.parametrize("T, k, K, how", GROUPS)
def test_group(som, T, k, K, how):
    gen = torch.Generator().manual_seed(T + K)
    node = draw_nodes(gen, T, k, K, how)
    want = ref.group(node, K)
    got = som.som_group(node.cuda(), K)
    for g, w, name in zip(got, want, ("offsets", "order", "slot")):
        assert torch.equal(g.cpu(), w), name
    if k == 1:                                     # a plain list of units
        offsets, order, slot = som.som_group(node[:, 0].contiguous().cuda(), K)
        assert torch.equal(slot.cpu(), want[2][:, 0]) and torch.equal(order.cpu(), want[1]) and torch.equal(offsets.cpu(), want[0])


def test_group_of_nothing(som):
    offsets, order, slot = som.som_group(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 9)
    assert offsets.tolist() == [0] * 10 and order.numel() == 0 and slot.shape == (0, 4)


#       T, k, K, D, extra, lead, how
ROWS = [(1, 1, 1, 1, 0, 0, "even"), (1, 8, 16, 2048, 0, 0, "even"), (5, 2, 3, 3, 2, 1, "holes"), (7, 3, 4, 7, 0, 3, "even"), (33, 2, 9, 8, 0, 0, "holes"),
        (19, 4, 6, 50, 0, 0, "skew"), (23, 1, 6, 51, 6, 5, "holes"), (64, 2, 8, 64, 8, 0, "even"), (12, 8, 40, 1001, 1, 1, "holes"), (9, 5, 7, 129, 0, 0, "none"),
        (17, 2, 4, 4096, 0, 0, "one"), (6, 3, 9, 2600, 3, 2, "holes")]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("T, k, K, D, extra, lead, how", ROWS)
def test_dispatch_combine_and_gradient(som, T, k, K, D, extra, lead, how, dtype):
    gen = torch.Generator().manual_seed(D)
    node = draw_nodes(gen, T, k, K, how)
    _, _, slot = ref.group(node, K)
    X, Y, dout = normal(gen, T, D, dtype=dtype), normal(gen, T * k + 2, D, dtype=dtype), normal(gen, T, D, dtype=dtype)
    weight = torch.softmax(torch.randn(T, k, generator=gen), 1)
    slot_d, weight_d = slot.cuda(), weight.cuda()
    Xd, Yd, gd = padded(X, extra, lead), padded(Y, extra, lead), padded(dout, 0, lead)
    before = normal(gen, T * k + 2, D, dtype=dtype)
    for w, wd in ((None, None), (weight, weight_d)):
        out = padded(before, extra, lead)
        assert som.som_dispatch(Xd, slot_d, weight=wd, out=out) is out
        want, bound = ref.dispatch(X, slot, w, before)
        ref.check(out, want, bound, "dispatch")
        ref.check(som.som_combine(Yd, slot_d, weight=wd), *ref.combine(Y, slot, w), "combine")
        dY = padded(before, extra, lead)
        dweight = som.som_combine_grad(gd, Yd, slot_d, weight=wd, dY=dY)[1]
        want, bound, dw, dwb = ref.combine_grad(dout, Y, slot, w, before)
        ref.check(dY, want, bound, "dY")
        ref.check(dweight, dw, dwb, "dweight")
        only_y, none = som.som_combine_grad(gd, Yd, slot_d, weight=wd, dY=padded(before, extra, lead), dweight=False)
        assert none is None and torch.equal(only_y, dY)
        none, only_w = som.som_combine_grad(gd, Yd, slot_d, weight=wd, dY=False)
        assert none is None and torch.equal(only_w, dweight)
    if T * k:
        assert som.som_dispatch(Xd, slot_d).shape == (T * k, D)


def test_rows_that_are_no_numbers_stay_where_they_are(som):
    """A row of NaN or infinities reaches its own places and results only; a pair without a place reads nothing."""
    node = torch.tensor([[0, 1], [1, -1], [0, 1]], dtype=torch.int32)
    _, _, slot = ref.group(node, 2)
    X = torch.ones(3, 40)
    X[1, 3], X[2, 5] = float("nan"), float("inf")
    Y = som.som_dispatch(X.cuda(), slot.cuda(), out=torch.zeros(6, 40, device="cuda"))
    assert torch.equal(torch.isnan(Y.cpu()).any(1), torch.tensor([False, False, False, True, False, False]))
    poisoned = torch.full((6, 40), float("nan"))
    poisoned[:5] = 1.0                                                     # the sixth place is nobody's
    out = som.som_combine(poisoned.cuda(), slot.cuda())
    assert torch.equal(out.cpu(), torch.tensor([2.0, 1.0, 2.0])[:, None].expand(3, 40))


def test_slots_outside_the_places_are_not_followed(som):
    slot = torch.tensor([[0, 99], [-7, 1], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32)
    X, Y = torch.randn(3, 33).bfloat16(), torch.randn(4, 33).bfloat16()
    out = torch.zeros(4, 33, dtype=torch.bfloat16)
    ref.check(som.som_dispatch(X.cuda(), slot.cuda(), out=out.cuda()), *ref.dispatch(X, slot, None, out), "dispatch")
    ref.check(som.som_combine(Y.cuda(), slot.cuda()), *ref.combine(Y, slot, None), "combine")
    dY, dw = som.som_combine_grad(X.cuda(), Y.cuda(), slot.cuda(), dY=out.cuda())
    want = ref.combine_grad(X, Y, slot, None, out)
    ref.check(dY, want[0], want[1], "dY")
    ref.check(dw, want[2], want[3], "dweight")


def cut(gen, M, K, how):
    """Offsets of K nodes over M rows."""
    if how == "one":
        counts = torch.zeros(K, dtype=torch.long)
        counts[K // 2] = M
    else:
        share = torch.rand(K, generator=gen) ** (8 if how == "skew" else 1) + 1e-9
        if K > 2:
            share[torch.rand(K, generator=gen) < 0.2] = 0
            share[0] += 1e-6
        counts = torch.floor(share / share.sum() * M).long()
        counts[int(counts.argmax())] += M - int(counts.sum())
    if how == "tail":                               # rows behind the last node's
        counts[int(counts.argmax())] -= min(int(counts.max()), 5)
    return torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]).int()


#           M, K, Din, Dout, extra, lead, how, act, bias, residual, pre
PRODUCTS = [(1, 1, 1, 1, 0, 0, "whole", "none", False, False, False), (1, 4, 64, 64, 0, 0, "even", "silu", True, True, True),
            (3, 5, 7, 5, 3, 1, "even", "gelu", True, False, True), (40, 8, 128, 96, 0, 0, "tail", "gelu_tanh", True, True, True),
            (70, 3, 50, 16, 0, 0, "even", "none", True, False, False), (200, 37, 37, 24, 0, 0, "tail", "relu", True, True, False),
            (130, 1, 100, 257, 0, 0, "whole", "silu", False, True, False), (300, 4, 264, 136, 8, 0, "skew", "gelu_tanh", True, False, True),
            (257, 2, 513, 300, 1, 1, "even", "relu", False, False, True), (515, 3, 256, 512, 0, 0, "one", "gelu", True, True, True),
            (64, 64, 512, 64, 0, 0, "even", "none", False, True, False), (16, 200, 72, 40, 0, 8, "even", "silu", True, False, False),
            (1030, 2, 192, 320, 0, 0, "tail", "none", True, False, True), (900, 700, 16, 8, 0, 0, "skew", "relu", True, True, True),
            (31, 1, 1024, 24, 0, 0, "whole", "gelu", True, True, True), (600, 1, 64, 1024, 64, 64, "whole", "gelu_tanh", True, True, True),
            (2, 1, 4096, 130, 0, 0, "whole", "none", False, False, False), (5, 1, 33, 2050, 0, 0, "whole", "silu", True, False, True)]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("M, K, Din, Dout, extra, lead, how, act, bias, residual, pre", PRODUCTS)
def test_product_and_gradient(som, M, K, Din, Dout, extra, lead, how, act, bias, residual, pre, dtype):
    gen = torch.Generator().manual_seed(M + Din)
    offsets = None if how == "whole" else cut(gen, M, K, how)
    X, A = normal(gen, M, Din, dtype=dtype), normal(gen, K, Dout, Din, dtype=dtype, scale=Din ** -0.5)
    if offsets is None:
        A = A[0]
    c = normal(gen, *A.shape[:-2], Dout, dtype=dtype) if bias else None
    R = normal(gen, M, Dout, dtype=dtype) if residual else None
    before, before_x = normal(gen, M, Dout, dtype=dtype), normal(gen, M, Din, dtype=dtype)
    dev = lambda t: None if t is None else t.cuda()
    Xd, Ad, offd = padded(X, extra, lead), A.cuda(), dev(offsets)
    out, z = padded(before, extra, lead), padded(before, extra, 0) if pre else None
    som.som_node_product(Xd, Ad, offsets=offd, bias=dev(c), activation=act, residual=None if R is None else padded(R, extra, lead), pre=z, out=out)
    want, bound, wz, bz = ref.product(X, A, offsets, c, act, R, before, before)
    ref.check(out, want, bound, "Y")
    if pre:
        ref.check(z, wz, bz, "pre")
    dY, Z = normal(gen, M, Dout, dtype=dtype), normal(gen, M, Dout, dtype=dtype, scale=2.0)
    dX = padded(before_x, extra, lead)
    got = som.som_node_product_grad(padded(dY, extra, lead), Xd, Ad, offsets=offd, pre=padded(Z, extra, 0) if act != "none" else None, activation=act, dX=dX)
    want = ref.product_grad(dY, X, A, offsets, Z, act, before_x)
    for g, i, name in zip(got, (0, 2, 4), ("dX", "dA", "dbias")):
        ref.check(g, want[i], want[i + 1], name)
    # each alone, and again: the same bits
    zd = padded(Z, 0, 0) if act != "none" else None
    for which in range(3):
        args = [False, False, False]
        args[which] = padded(before_x, extra, lead) if which == 0 else None
        alone = som.som_node_product_grad(padded(dY, 0, 0), Xd, Ad, offsets=offd, pre=zd, activation=act, dX=args[0], dA=args[1], dbias=args[2])
        assert torch.equal(alone[which], got[which]) and [t is None for t in alone] == [i != which for i in range(3)]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("M, K, Din, Dout, how, act", [(20_000, 1, 64, 48, "whole", "silu"), (30_001, 1, 9, 5, "whole", "none"), (12_345, 3, 24, 272, "one", "relu"),
                                                      (9000, 2, 300, 16, "skew", "gelu_tanh"), (70_000, 20, 8, 8, "one", "none"), (5000, 40, 40, 33, "skew", "gelu")])
def test_gradient_of_long_groups(som, M, K, Din, Dout, how, act, dtype):
    """Groups whose sums over rows are taken in runs and joined."""
    gen = torch.Generator().manual_seed(M)
    offsets = None if how == "whole" else cut(gen, M, K, how)
    X, A, dY, Z = (normal(gen, *s, dtype=dtype) for s in ((M, Din), (K, Dout, Din), (M, Dout), (M, Dout)))
    got = som.som_node_product_grad(dY.cuda(), X.cuda(), A.cuda(), offsets=None if offsets is None else offsets.cuda(), pre=Z.cuda(), activation=act)
    want = ref.product_grad(dY, X, A, offsets, Z, act, torch.zeros(M, Din, dtype=dtype))
    for g, i, name in zip(got, (0, 2, 4), ("dX", "dA", "dbias")):
        ref.check(g, want[i], want[i + 1], name)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("M, K, Din, Dout", ref.TILES + ref.NARROW)
def test_every_size_of_tile(som, M, K, Din, Dout, dtype):
    """Larger products, against float64 on the GPU: tiles of every size, uneven groups, rows behind the last; twice, to the same bits."""
    gen = torch.Generator().manual_seed(M + Din)
    offsets = None if K == 1 else cut(gen, M, K, "tail")
    with torch.device("cuda"):
        g = torch.Generator(device="cuda").manual_seed(M)
        rnd = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).to(dtype)
        X, A, c, R = rnd(M, Din), rnd(K, Dout, Din, scale=Din ** -0.5), rnd(K, Dout), rnd(M, Dout)
        dY, Z, before, before_x = rnd(M, Dout), rnd(M, Dout, scale=2.0), rnd(M, Dout), rnd(M, Din)
        off = None if offsets is None else offsets.cuda()
        outs = []
        for _ in range(2):
            out, pre, dX = before.clone(), before.clone(), before_x.clone()
            som.som_node_product(X, A, offsets=off, bias=c, activation="gelu", residual=R, pre=pre, out=out)
            outs.append([out, pre, *som.som_node_product_grad(dY, X, A, offsets=off, pre=Z, activation="silu", dX=dX)])
        for a, b in zip(*outs):
            assert torch.equal(a, b)
        out, pre, dX, dA, dbias = outs[0]
        y, yb, z, zb = ref.product(X, A, offsets, c, "gelu", R, before, before)
        ref.check(out, y, yb, "Y")
        ref.check(pre, z, zb, "pre")
        grads = ref.product_grad(dY, X, A, offsets, Z, "silu", before_x)
        for got, i, name in ((dX, 0, "dX"), (dA, 2, "dA"), (dbias, 4, "dbias")):
            ref.check(got, grads[i], grads[i + 1], name)


def test_offsets_behind_four_billion_bytes(som):
    """Places, rows and matrices further than 2^31 values and 2^32 bytes from their tensors' starts."""
    M, D = 600_000, 4096                                             # 2.5e9 values, 4.9 GB
    with torch.device("cuda"):
        Y = torch.zeros(M, D, dtype=torch.bfloat16)
        X = torch.randn(3, D).bfloat16()
        slot = torch.tensor([[M - 1], [7], [550_001]], dtype=torch.int32)
        som.som_dispatch(X, slot, out=Y)
        som.som_sync()
        assert torch.equal(Y[slot[:, 0].long()], X) and int((Y[524_288:] != 0).any(1).sum()) == 2
        assert torch.equal(som.som_combine(Y, slot), X)
        A = (torch.randn(2, 8, D) / 64).bfloat16()
        offsets = torch.tensor([M - 70, M - 5, M], dtype=torch.int32)         # the last seventy rows
        out = torch.zeros(M, 8, dtype=torch.bfloat16)
        som.som_node_product(Y, A, offsets=offsets, out=out)
        x, a = Y[M - 1].double(), A[1].double()
        assert ((out[M - 1].double() - a @ x).abs() <= 2.0 ** -8 * (a @ x).abs() + D * ref.F32 * (a.abs() @ x.abs())).all() and not out[:M - 70].any()
        dY = torch.zeros(M, 8, dtype=torch.bfloat16)
        dY[M - 1] = 1.0
        _, dA, dbias = som.som_node_product_grad(dY, Y, A, offsets=offsets, dX=False)
        assert torch.equal(dA[1], Y[M - 1].expand(8, D)) and not dA[0].any() and torch.equal(dbias, torch.tensor([[0.0], [1.0]]).expand(2, 8).bfloat16())
        dX = som.som_node_product_grad(dY, Y, A, offsets=offsets, dX=torch.zeros_like(Y), dA=False, dbias=False)[0]
        want = a.sum(0)
        assert ((dX[M - 1].double() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * ref.F32 * a.abs().sum(0)).all() and int((dX != 0).any(1).sum()) == 1
    del Y, dX, out, dY
    torch.cuda.empty_cache()


@pytest.mark.parametrize("Din, Dout, M", [(64, 40, 300), (2048, 64, 9), (256, 256, 300)])
def test_small_half_precision_values_count(som, Din, Dout, M):
    """float16 rows below its normal range (6e-5) are not taken for zeros."""
    gen = torch.Generator().manual_seed(9)
    X, A = normal(gen, M, Din, dtype=torch.float16, scale=2.0 ** -18), normal(gen, Dout, Din, dtype=torch.float16)
    zero = torch.zeros(M, Dout, dtype=torch.float16)
    Y = som.som_node_product(X.cuda(), A.cuda())
    want, bound, _, _ = ref.product(X, A, None, None, "none", None, zero, zero)
    ref.check(Y, want, bound, "Y")
    assert float(want.abs().mean()) > 4 * float(bound.mean())
    dX, dA, _ = som.som_node_product_grad(normal(gen, M, Dout, dtype=torch.float16).cuda(), X.cuda(), A.cuda())
    assert float(dA.float().abs().mean()) > 0


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_product_without_rows(som, dtype):
    X, A = torch.empty(0, 24, dtype=dtype, device="cuda"), torch.randn(3, 8, 24, device="cuda").to(dtype)
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert som.som_node_product(X, A, offsets=offsets).shape == (0, 8)
    dX, dA, dbias = som.som_node_product_grad(torch.empty(0, 8, dtype=dtype, device="cuda"), X, A, offsets=offsets)
    assert dX.shape == (0, 24) and not dA.any() and not dbias.any() and dA.shape == A.shape and dbias.shape == (3, 8)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("Din, Dout", [(72, 40), (37, 21), (256, 256)])
def test_rows_behind_a_group_do_not_reach_it(som, Din, Dout, dtype):
    """NaN in one node's rows, and in rows that are no node's, stays out of every other node's results and gradients."""
    gen = torch.Generator().manual_seed(3)
    offsets = torch.tensor([0, 5, 5, 75, 80], dtype=torch.int32)
    X, A, dY = normal(gen, 90, Din, dtype=dtype), normal(gen, 4, Dout, Din, dtype=dtype, scale=Din ** -0.5), normal(gen, 90, Dout, dtype=dtype)
    X[75:], dY[75:] = float("nan"), float("nan")
    A[3] = float("inf")
    before, before_x = torch.zeros(90, Dout, dtype=dtype), torch.zeros(90, Din, dtype=dtype)
    Y = som.som_node_product(X.cuda(), A.cuda(), offsets=offsets.cuda(), out=before.cuda()).cpu()
    dX, dA, dbias = (t.cpu() for t in som.som_node_product_grad(dY.cuda(), X.cuda(), A.cuda(), offsets=offsets.cuda(), dX=before_x.cuda()))
    live = torch.arange(90) < 75
    want, bound, _, _ = ref.product(X[:75], A[:3], offsets[:4], None, "none", None, before[:75], before[:75])
    ref.check(Y[live], want, bound, "Y")
    assert torch.isnan(Y[75:80]).all() and not Y[80:].any() and not dX[80:].any()
    grads = ref.product_grad(dY[:75], X[:75], A[:3], offsets[:4], None, "none", before_x[:75])
    ref.check(dX[live], grads[0], grads[1], "dX")
    ref.check(dA[:3], grads[2], grads[3], "dA")
    ref.check(dbias[:3], grads[4], grads[5], "dbias")
    assert torch.isnan(dA[3]).all() and torch.isnan(dbias[3]).all()


def test_offsets_outside_the_rows_are_cut_off(som):
    """Offsets beyond the rows, or falling ones: the rows that exist are taken, nothing beyond them."""
    gen = torch.Generator().manual_seed(4)
    X, A = normal(gen, 20, 24, dtype=torch.bfloat16), normal(gen, 3, 16, 24, dtype=torch.bfloat16)
    before = torch.zeros(20, 16, dtype=torch.bfloat16)
    Y = som.som_node_product(X.cuda(), A.cuda(), offsets=torch.tensor([-5, 8, 8, 1000], dtype=torch.int32).cuda(), out=before.cuda())
    want, bound, _, _ = ref.product(X, A, torch.tensor([0, 8, 8, 20]), None, "none", None, before, before)
    ref.check(Y, want, bound, "Y")
    dX, dA, dbias = som.som_node_product_grad(before.cuda(), X.cuda(), A.cuda(), offsets=torch.tensor([9, 3, 99, 50], dtype=torch.int32).cuda())
    assert not dA.any() and not dbias.any()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_activations_over_their_whole_range(som, act, dtype):
    """One feature, one matrix of one entry: the activation of every value from far left to far right, infinities and NaN among them."""
    v = torch.cat([torch.linspace(-12, 12, 1501), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 40, -40, 200, -200, 6e4, -6e4, math.inf, -math.inf, math.nan])])
    X = v[:, None].to(dtype)
    A = torch.ones(1, 1, dtype=dtype)
    zero = torch.zeros_like(X)
    Y = som.som_node_product(X.cuda(), A.cuda(), activation=act)
    want, bound, _, _ = ref.product(X, A, None, None, act, None, zero, zero)
    ref.check(Y, want, bound, "Y")
    dX, _, _ = som.som_node_product_grad(torch.ones_like(X).cuda(), X.cuda(), A.cuda(), pre=X.cuda(), activation=act)
    want = ref.product_grad(torch.ones_like(X), X, A, None, X, act, zero)
    ref.check(dX, want[0], want[1], "dX")


def test_a_training_step_of_local_models_on_a_map(som):
    """As they are used together: units of a trained map and their neighbours route rows through two layers of local models,
    then the whole way back; every stage against the reference on the stage's own inputs."""
    from paper_2604_26555_amd.topology import lattice_distances
    gen = torch.Generator().manual_seed(12)
    T, D, H, O, K, k = 700, 50, 40, 6, 30, 3
    X, W = normal(gen, T, D), normal(gen, K, D)
    G = torch.from_numpy(lattice_distances(5, 6, "hex"))
    Xd = X.cuda()
    bmu, _, _ = som.som_bmu(Xd, W.cuda())
    near = torch.sort(G, dim=1, stable=True).indices[:, :k].int()          # every node and its two nearest
    node = near.cuda()[bmu.long()].contiguous()
    node[::50] = -1
    weight = torch.softmax(-G.cuda()[bmu.long()[:, None], node.long().clamp(min=0)], 1).contiguous()
    A1, c1, A2, c2 = normal(gen, K, H, D, scale=D ** -0.5), normal(gen, K, H), normal(gen, K, O, H, scale=H ** -0.5), normal(gen, K, O)
    target = normal(gen, T, O).cuda()
    A1d, c1d, A2d, c2d = A1.cuda(), c1.cuda(), A2.cuda(), c2.cuda()

    offsets, _, slot = som.som_group(node, K)
    Xg = som.som_dispatch(Xd, slot, out=torch.zeros(T * k, D, device="cuda"))
    pre = torch.zeros(T * k, H, device="cuda")
    Hg = som.som_node_product(Xg, A1d, offsets=offsets, bias=c1d, activation="gelu_tanh", pre=pre, out=torch.zeros(T * k, H, device="cuda"))
    Yg = som.som_node_product(Hg, A2d, offsets=offsets, bias=c2d, out=torch.zeros(T * k, O, device="cuda"))
    out = som.som_combine(Yg, slot, weight=weight)
    dout = out - target
    dYg, dweight = som.som_combine_grad(dout, Yg, slot, weight=weight, dY=torch.zeros(T * k, O, device="cuda"))
    dHg, dA2, dc2 = som.som_node_product_grad(dYg, Hg, A2d, offsets=offsets, dX=torch.zeros(T * k, H, device="cuda"))
    dXg, dA1, dc1 = som.som_node_product_grad(dHg, Xg, A1d, offsets=offsets, pre=pre, activation="gelu_tanh", dX=torch.zeros(T * k, D, device="cuda"))
    dX = som.som_combine(dXg, slot)
    som.som_sync()

    c = lambda t: t.cpu()
    zero = lambda n: torch.zeros(T * k, n)
    off, _, sl = ref.group(c(node), K)
    assert torch.equal(c(offsets), off) and torch.equal(c(slot), sl) and int(off[-1]) == 3 * (T - 14)
    ref.check(Xg, *ref.dispatch(X, sl, None, zero(D)), "rows")
    y, b, z, zb = ref.product(c(Xg), A1, off, c1, "gelu_tanh", None, zero(H), zero(H))
    ref.check(Hg, y, b, "hidden")
    ref.check(pre, z, zb, "pre")
    y, b, _, _ = ref.product(c(Hg), A2, off, c2, "none", None, zero(O), zero(O))
    ref.check(Yg, y, b, "results")
    ref.check(out, *ref.combine(c(Yg), sl, c(weight)), "out")
    y, b, dw, dwb = ref.combine_grad(c(dout), c(Yg), sl, c(weight), zero(O))
    ref.check(dYg, y, b, "dYg")
    ref.check(dweight, dw, dwb, "dweight")
    for got, want in (((dHg, dA2, dc2), ref.product_grad(c(dYg), c(Hg), A2, off, None, "none", zero(H))),
                      ((dXg, dA1, dc1), ref.product_grad(c(dHg), c(Xg), A1, off, c(pre), "gelu_tanh", zero(D)))):
        for g, i in zip(got, (0, 2, 4)):
            ref.check(g, want[i], want[i + 1], "gradient")
    ref.check(dX, *ref.combine(c(dXg), sl, None), "dX")


def test_captured_and_replayed_on_changing_inputs(som):
    """Group, dispatch, product and gradients in one graph, replayed on other rows with eager calls in between."""
    gen = torch.Generator().manual_seed(7)
    T, k, K, D, H = 300, 2, 11, 72, 40
    X, node = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda")
    A = normal(gen, K, H, D, dtype=torch.bfloat16, scale=D ** -0.5).cuda()
    dY = normal(gen, T * k, H, dtype=torch.bfloat16).cuda()
    from paper_2604_26555_amd import Som
    stream = torch.cuda.Stream()
    mine = Som(0, stream)
    z = lambda n: torch.zeros(T * k, n, dtype=torch.bfloat16, device="cuda")
    bufs = dict(Xg=z(D), pre=z(H), Y=z(H), dX=z(D))

    def step(s, b):
        offsets, order, slot = s.som_group(node, K)
        s.som_dispatch(X, slot, out=b["Xg"])
        s.som_node_product(b["Xg"], A, offsets=offsets, activation="silu", pre=b["pre"], out=b["Y"])
        _, dA, dbias = s.som_node_product_grad(dY, b["Xg"], A, offsets=offsets, pre=b["pre"], activation="silu", dX=b["dX"])
        return [offsets, order, slot, b["Xg"], b["pre"], b["Y"], b["dX"], dA, dbias]

    def fill(i):
        g = torch.Generator().manual_seed(100 + i)
        X.copy_(normal(g, T, D, dtype=torch.bfloat16))
        node.copy_(draw_nodes(g, T, k, K, ("even", "holes", "one")[i % 3]))

    fill(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(mine, bufs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = step(mine, bufs)
    for i in range(4):
        fill(i)
        for b in bufs.values():
            b.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = step(som, {n: torch.zeros_like(b) for n, b in bufs.items()})
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b), f"replay {i}"
    mine.close()


def test_outputs_made_for_a_stream_of_their_own(som):
    """A context on a stream other than the current one: its outputs' memory comes from that stream's pool."""
    from paper_2604_26555_amd import Som
    side = torch.cuda.Stream()
    mine = Som(0, side)
    X = torch.randn(2000, 256, device="cuda")
    node = torch.randint(0, 16, (2000, 2), device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    offsets, _, slot = mine.som_group(node, 16)
    Y = mine.som_combine(mine.som_dispatch(X, slot), slot)
    mine.som_sync()
    assert torch.equal(Y, X + X) and int(offsets[-1]) == 4000
    mine.close()


@pytest.mark.parametrize("D", [2, 40, 300])
def test_the_same_place_twice(som, D):
    """Pairs of one row that share a place: read twice by the sum, written twice with the same values; a single row of any stride."""
    X = torch.randn(50, D, device="cuda")
    slot = torch.arange(50, dtype=torch.int32, device="cuda")[:, None].repeat(1, 3)
    assert torch.equal(som.som_dispatch(X, slot, out=torch.empty_like(X)), X)
    assert torch.equal(som.som_combine(X, slot), X + X + X)
    dY, dw = som.som_combine_grad(X, X, slot)
    assert torch.equal(dY, X) and torch.equal(dw[:, 0], dw[:, 2])
    row = torch.as_strided(torch.randn(D, device="cuda"), (1, D), (2 ** 22, 1))
    assert torch.equal(som.som_dispatch(row, slot[:1, :1]), row)
    assert torch.equal(som.som_node_product(row, torch.eye(D, device="cuda")), row)


def test_python_refusals(som):
    X, A = torch.zeros(6, 8, device="cuda"), torch.zeros(2, 4, 8, device="cuda")
    off, slot = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda"), torch.zeros(6, 1, dtype=torch.int32, device="cuda")
    for error, f in [
        (TypeError, lambda: som.som_group(slot.long(), 2)), (ValueError, lambda: som.som_group(slot.cpu(), 2)),
        (ValueError, lambda: som.som_group(torch.zeros(4, 4, dtype=torch.int32, device="cuda").t()[:2], 2)),
        (ValueError, lambda: som.som_group(slot, 2, offsets=off[:2])),
        (TypeError, lambda: som.som_dispatch(X.double(), slot)), (ValueError, lambda: som.som_dispatch(X.t(), slot)),
        (ValueError, lambda: som.som_dispatch(X[:5], slot)), (ValueError, lambda: som.som_dispatch(X, slot, weight=torch.zeros(6, 2, device="cuda"))),
        (TypeError, lambda: som.som_dispatch(X, slot, out=X.half())), (ValueError, lambda: som.som_dispatch(X, slot, out=X[:, :7])),
        (ValueError, lambda: som.som_combine(X, slot, out=torch.zeros(5, 8, device="cuda"))), (TypeError, lambda: som.som_combine(X, slot.float())),
        (ValueError, lambda: som.som_combine_grad(X[:5], X, slot)), (TypeError, lambda: som.som_combine_grad(X.half(), X, slot)),
        (ValueError, lambda: som.som_node_product(X, A)), (ValueError, lambda: som.som_node_product(X, A, offsets=off[:2])),
        (ValueError, lambda: som.som_node_product(X[:, :7], A, offsets=off)), (TypeError, lambda: som.som_node_product(X, A.half(), offsets=off)),
        (ValueError, lambda: som.som_node_product(X, A, offsets=off, bias=torch.zeros(2, 3, device="cuda"))),
        (ValueError, lambda: som.som_node_product(X, A, offsets=off, residual=torch.zeros(6, 5, device="cuda"))),
        (ValueError, lambda: som.som_node_product(X, A.transpose(1, 2), offsets=off)), (KeyError, lambda: som.som_node_product(X, A, offsets=off, activation="x")),
        (ValueError, lambda: som.som_node_product_grad(X, X, A, offsets=off)),
        (Exception, lambda: som.som_node_product_grad(torch.zeros(6, 4, device="cuda"), X, A, offsets=off, activation="relu")),
    ]:
        with pytest.raises(error):
            f()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_left_tails_of_16_bit_activations_to_a_rounding(som, act, dtype):
    """What is left of an activation far to the left, and its slope there, are as exact as their type and not only small beside z.
    A result may be off by half a step of its type, and by 2^-13 of itself: the fit of the error function's complement 2^-14.5, the
    exponents (128 at most in base 2, three roundings of 2^-24) 2^-15.4.  Float32's range ends at 2^-126, where the factors beside the exponential
    are below 2^8."""
    X = torch.linspace(-12, -2, 2001)[:, None].to(dtype)
    A, zero = torch.ones(1, 1, dtype=dtype), torch.zeros_like(X)
    want, slope = ref.activation(X.double(), act)
    bound = lambda v: (ref.half_step(dtype) + 2.0 ** -13) * v.abs() + ref.least(dtype) + 2.0 ** -118
    for rows in (1, 2001):                          # (few rows and many take different kernels)
        Y = som.som_node_product(X[:rows].cuda(), A.cuda(), activation=act)
        ref.check(Y, want[:rows], bound(want[:rows]), "Y")
    dX, _, _ = som.som_node_product_grad(torch.ones_like(X).cuda(), X.cuda(), A.cuda(), pre=X.cuda(), activation=act)
    ref.check(dX, slope, bound(slope), "dX")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Din, Dout", [(24, 24), (40, 30), (20, 61), (64, 64), (3, 5), (48, 100), (200, 300), (200, 6)])
def test_bias_gradients_add_up_what_is_not_rounded_yet(som, Din, Dout, dtype, act):
    """The products take dz in 16 bits; the biases' gradients are sums of float32 values, and so nearer than dz's roundings would leave them."""
    gen = torch.Generator().manual_seed(Dout)
    offsets = torch.tensor([0, 100, 100, 190, 260], dtype=torch.int32)
    X, A, dY, Z = (normal(gen, *s, dtype=dtype) for s in ((260, Din), (4, Dout, Din), (260, Dout), (260, Dout)))
    dz = dY.double() * ref.activation(Z.double(), act)[1]
    dev = (dY.cuda(), X.cuda(), A.cuda(), offsets.cuda(), Z.cuda(), act)
    dbias = som.som_node_product_grad(*dev)[2]
    for e in range(4):
        d = dz[int(offsets[e]):int(offsets[e + 1])]
        # a slope is off by 32 roundings, the sum by one for each of its terms and two for the product and the joined sums
        want, size = d.sum(0), (1.2 * dY[int(offsets[e]):int(offsets[e + 1])].double().abs()).sum(0)
        ref.check(dbias[e], want, ref.rounded(want, (d.shape[0] + 34) * (ref.F32 * size + ref.least(torch.float32)), dtype), f"dbias of node {e}")
    assert torch.equal(som.som_node_product_grad(*dev, dX=False, dA=False)[2], dbias)


def test_new_outputs_hold_zeros_where_nothing_belongs(som):
    """Rows without a place and rows of no node, in memory that held NaN before."""
    gen = torch.Generator().manual_seed(2)
    T, k, K, D, H = 500, 2, 7, 64, 40
    node = draw_nodes(gen, T, k, K, "holes").cuda()
    X, A = torch.randn(T, D, device="cuda"), torch.randn(K, H, D, device="cuda")
    offsets, _, slot = som.som_group(node, K)
    end = int(offsets[-1])
    assert 0 < end < T * k
    calls = [lambda: som.som_dispatch(X, slot), lambda: som.som_node_product(torch.ones(T * k, D, device="cuda"), A, offsets=offsets),
             lambda: som.som_combine_grad(X, torch.ones(T * k, D, device="cuda"), slot)[0],
             lambda: som.som_node_product_grad(torch.ones(T * k, H, device="cuda"), torch.ones(T * k, D, device="cuda"), A, offsets=offsets)[0]]
    for f in calls:
        for n in (D, H):
            held = [torch.full((T * k, n), float("nan"), device="cuda") for _ in range(4)]
            del held
        out = f()
        assert out[:end].any(1).all() and not out[end:].any()


def test_new_outputs_are_cleared_in_every_replay(som):
    """Outputs that the wrapper makes inside a captured graph: rows of no node are zeros again in each replay."""
    from paper_2604_26555_amd import Som
    gen = torch.Generator().manual_seed(8)
    T, K, D, H = 400, 5, 48, 24
    X, A, node = torch.randn(T, D, device="cuda"), torch.randn(K, H, D, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    mine = Som(0, stream)

    def step(s):
        offsets, _, slot = s.som_group(node, K)
        Xg = s.som_dispatch(X, slot)
        return offsets, Xg, s.som_node_product(Xg, A, offsets=offsets), s.som_combine_grad(X, Xg, slot)[0]

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(mine)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = step(mine)
    for i, how in enumerate(("even", "holes", "none", "holes")):
        node.copy_(draw_nodes(gen, T, 1, K, how)[:, 0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = step(som)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b), f"replay {i}"
        assert not outs[1][int(outs[0][-1]):].any() and not outs[2][int(outs[0][-1]):].any()
    mine.close()


def test_more_tiles_than_a_row_of_the_grid(som):
    """134 million rows of one value and their gradient's 65: more than the 2^20 workgroups that a row of the grid holds, 17 GB of results."""
    M, D, step = 2 ** 27 + 3, 65, 2 ** 22
    with torch.device("cuda"):
        dY, A = torch.randn(M, 1, dtype=torch.float16), torch.randn(1, D).half()
        dX = som.som_node_product_grad(dY, torch.empty(M, D, dtype=torch.float16), A, dA=False, dbias=False)[0]
        for lo in range(0, M, step):                 # one product a result: exact in float32, rounded once
            assert torch.equal(dX[lo:lo + step], (dY[lo:lo + step].float() * A.float()).half()), lo
    del dX, dY
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("M, K, Din, Dout, how", [(200, 40, 600, 70, "one"), (95, 10, 512, 33, "skew"), (300, 64, 1029, 48, "skew"), (64, 7, 300, 130, "one"), (77, 1, 520, 40, "one")])
def test_few_rows_on_uneven_nodes(som, M, K, Din, Dout, how, dtype):
    """Products whose mean number of rows a node is small, with most rows on one node: several workgroups share a node's rows."""
    gen = torch.Generator().manual_seed(M)
    offsets = cut(gen, M, K, how)
    X, A, c = normal(gen, M, Din, dtype=dtype), normal(gen, K, Dout, Din, dtype=dtype, scale=Din ** -0.5), normal(gen, K, Dout, dtype=dtype)
    R, before = normal(gen, M, Dout, dtype=dtype), normal(gen, M, Dout, dtype=dtype)
    out, z = padded(before, 3, 1), padded(before, 1, 0)
    som.som_node_product(padded(X, 1, 1), A.cuda(), offsets=offsets.cuda(), bias=c.cuda(), activation="silu", residual=padded(R, 2, 1), pre=z, out=out)
    want, bound, wz, bz = ref.product(X, A, offsets, c, "silu", R, before, before)
    ref.check(out, want, bound, "Y")
    ref.check(z, wz, bz, "pre")


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("M, Din, Dout", [(33, 512, 70), (49, 517, 41), (64, 1024, 130), (64, 1031, 33), (40, 300, 17), (57, 640, 16), (17, 600, 50), (32, 513, 24)])
def test_up_to_64_rows_of_one_node(som, M, Din, Dout, dtype):
    """Two and four blocks of sixteen rows to a workgroup: partial last blocks, contractions that end inside a step, results that are no multiple
    of sixteen, all of the epilogue, matrices with leading dimensions of their own."""
    gen = torch.Generator().manual_seed(M + Din)
    X, A, c = normal(gen, M, Din, dtype=dtype), normal(gen, Dout, Din, dtype=dtype, scale=Din ** -0.5), normal(gen, Dout, dtype=dtype)
    R, before = normal(gen, M, Dout, dtype=dtype), normal(gen, M, Dout, dtype=dtype)
    for act in ("none", "gelu"):
        out, z = padded(before, 3, 1), padded(before, 1, 3)
        som.som_node_product(padded(X, 5, 1), A.cuda(), bias=c.cuda(), activation=act, residual=padded(R, 2, 1), pre=z, out=out)
        want, bound, wz, bz = ref.product(X, A, None, c, act, R, before, before)
        ref.check(out, want, bound, "Y")
        ref.check(z, wz, bz, "pre")


@pytest.mark.parametrize("M, Din, Dout", [(4136, 1024, 4096), (4160, 2048, 4096), (4115, 1024, 4096)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_last_rows_of_one_node_apart(som, M, Din, Dout, dtype):
    """A large product whose last rows go through the kernel of few rows: every matrix with a leading dimension of its own, so that the last rows'
    places are theirs."""
    with torch.device("cuda"):
        g = torch.Generator(device="cuda").manual_seed(M)
        rnd = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).to(dtype)
        wide = lambda t, extra: torch.cat([t, torch.full((M, extra), float("nan"), dtype=dtype)], 1)[:, :t.shape[1]]
        X, A, c, R, before = rnd(M, Din), rnd(Dout, Din, scale=Din ** -0.5), rnd(Dout), rnd(M, Dout), rnd(M, Dout)
        out, z = wide(before, 8), wide(before, 24)
        som.som_node_product(wide(X, 16), A, bias=c, activation="silu", residual=wide(R, 32), pre=z, out=out)
        want, bound, wz, bz = ref.product(X, A, None, c, "silu", R, before, before)
        ref.check(out, want, bound, "Y")
        ref.check(z, wz, bz, "pre")


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("Din, Dout", [(24, 16), (200, 136), (37, 70), (136, 3)])
def test_gradients_with_offsets_outside_the_rows(som, Din, Dout, dtype):
    """Offsets before the first row and behind the last: the gradients are those of the rows that exist.  Falling ones: nothing outside the
    matrices' own memory is written."""
    gen = torch.Generator().manual_seed(Din)
    M, K = 60, 3
    X, A, dY, Z = (normal(gen, *s, dtype=dtype) for s in ((M, Din), (K, Dout, Din), (M, Dout), (M, Dout)))
    before = normal(gen, M, Din, dtype=dtype)
    for offsets, inside in (([-5, 8, 8, 1000], [0, 8, 8, 60]), ([-100, -7, 60, 2 ** 31 - 1], [0, 0, 60, 60]), ([3, 70, 80, 90], [3, 60, 60, 60])):
        dX = padded(before, 2, 1)
        got = som.som_node_product_grad(dY.cuda(), X.cuda(), A.cuda(), offsets=torch.tensor(offsets, dtype=torch.int32).cuda(), pre=Z.cuda(), activation="silu", dX=dX)
        want = ref.product_grad(dY, X, A, torch.tensor(inside), Z, "silu", before)
        for g, i, name in zip(got, (0, 2, 4), ("dX", "dA", "dbias")):
            ref.check(g, want[i], want[i + 1], name)
    guard = 4096

    def guarded(*shape):
        n = math.prod(shape)
        buf = torch.full((n + 2 * guard,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[guard:guard + n].view(*shape)

    bufs = [guarded(M, Din), guarded(K, Dout, Din), guarded(K, Dout)]
    for offsets in ([9, 3, 99, 50], [60, 0, 60, 0], [50, 60, 5, 60]):
        som.som_node_product_grad(dY.cuda(), X.cuda(), A.cuda(), offsets=torch.tensor(offsets, dtype=torch.int32).cuda(), pre=Z.cuda(), activation="silu",
                                  dX=bufs[0][1], dA=bufs[1][1], dbias=bufs[2][1])
        for buf, _ in bufs:
            assert (buf[:guard] == 7).all() and (buf[-guard:] == 7).all()


@pytest.mark.parametrize("Din, Dout", [(2048, 1024), (2050, 1022)])
def test_matrices_behind_two_billion_values(som, Din, Dout):
    """The last nodes' matrices lie further than 2^31 values from the first one's start: products by few rows and by tiles, gradients."""
    K = 2 ** 31 // (Din * Dout) + 6
    with torch.device("cuda"):
        A = torch.zeros(K, Dout, Din, dtype=torch.bfloat16)
        A[-2:] = torch.randn(2, Dout, Din) / 45
        assert (K - 2) * Dout * Din > 2 ** 31
        for M in (20, 40_000):                          # rows of the last two nodes: five, and the others
            X, dY = torch.randn(M, Din).bfloat16(), torch.randn(M, Dout).bfloat16()
            offsets = torch.zeros(K + 1, dtype=torch.int32)
            offsets[-2], offsets[-1] = 5, M
            Y = som.som_node_product(X, A, offsets=offsets)
            cut = (slice(0, 5), slice(5, min(M, 400)))
            for e, rows in zip((-2, -1), cut):
                x, a = X[rows].double(), A[e].double()
                want = x @ a.t().contiguous()
                ref.check(Y[rows], want, ref.rounded(want, Din * ref.F32 * (x.abs() @ a.abs().t().contiguous()), X.dtype), "Y")
            dX, dA, _ = som.som_node_product_grad(dY, X, A, offsets=offsets)
            for e, rows in zip((-2, -1), cut):
                g, a = dY[rows].double(), A[e].double()
                want = g @ a
                ref.check(dX[rows], want, ref.rounded(want, Dout * ref.F32 * (g.abs() @ a.abs()), X.dtype), "dX")
            g, x = dY[:5].double(), X[:5].double()
            want = g.t().contiguous() @ x
            ref.check(dA[-2], want, ref.rounded(want, 5 * ref.F32 * (g.abs().t().contiguous() @ x.abs()), X.dtype), "dA")
            assert not dA[:-2].any() and dA[-1].any()
            del dA, dX, Y
    del A
    torch.cuda.empty_cache()
