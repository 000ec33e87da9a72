"""Local models on a machine without a GPU: what the entry points refuse, and what the reference of their GPU tests is."""
import ctypes as C

import pytest
import torch

import models_reference as ref
import stub_library
from paper_2604_26555_amd import SOM_EINVAL, SOM_OK

i32, i64 = C.c_int32, C.c_int64


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    return stub_library.link(str(tmp_path_factory.mktemp("stub")))


@pytest.fixture
def ctx(stub):
    c = stub_library.StubContext(stub)
    yield c
    c.close()


GROUP = dict(node="p", T=7, k=2, K=5, offsets="p", order="p", slot="p")
DISPATCH = dict(type=1, X="p", T=7, D=16, ldx=16, slot="p", k=2, weight="p", Y="p", M=14, ldy=16)
COMBINE = dict(type=1, Y="p", M=14, D=16, ldy=16, slot="p", T=7, k=2, weight="p", out="p", ldo=16)
COMBINE_GRAD = dict(type=2, dout="p", T=7, D=16, lddo=16, Y="p", M=14, ldy=16, slot="p", k=2, weight="p", dY="p", lddy=16, dweight="p")
PRODUCT = dict(type=0, X="p", M=14, Din=16, ldx=16, offsets="p", K=5, A="p", Dout=8, bias="p", act=2, residual="p", ldr=8, pre="p", ldpre=8, Y="p", ldy=8)
PRODUCT_GRAD = dict(type=0, dY="p", M=14, Dout=8, lddy=8, X="p", Din=16, ldx=16, offsets="p", K=5, A="p", pre="p", ldpre=8, act=2, dX="p", lddx=16,
                    dA="p", dbias="p")
CALLS = dict(som_group=GROUP, som_dispatch=DISPATCH, som_combine=COMBINE, som_combine_grad=COMBINE_GRAD, som_node_product=PRODUCT,
             som_node_product_grad=PRODUCT_GRAD)
WIDE = {"T", "M", "ldx", "ldy", "ldo", "lddo", "lddy", "lddx", "ldr", "ldpre"}


def call(ctx, name, **changes):
    args = []
    for key, v in {**CALLS[name], **changes}.items():
        if v == "p":
            args.append(ctx._p)
        elif v == "odd":
            args.append(C.c_void_p(ctx._p.value + 1))
        elif v is None:
            args.append(C.c_void_p(None))
        else:
            args.append(i64(v) if key in WIDE else i32(v))
    return ctx._run(getattr(ctx.lib, name), *args)


@pytest.mark.parametrize("name", CALLS)
def test_plain_calls_launch(ctx, name):
    rc, kernels = call(ctx, name)
    assert rc == SOM_OK and kernels, ctx.error()


REFUSED = [
    ("som_group", dict(node=None), "node"), ("som_group", dict(offsets=None), "offsets"), ("som_group", dict(T=-1), "negative"),
    ("som_group", dict(k=0), "k=0"), ("som_group", dict(K=0), "K (0)"), ("som_group", dict(K=32769), "32768"),
    ("som_group", dict(T=2 ** 30, k=2), "2^31-1"), ("som_group", dict(T=2 ** 62, k=4), "2^31-1"), ("som_group", dict(node="odd"), "aligned"),
    ("som_dispatch", dict(type=3), "type"), ("som_dispatch", dict(X=None), "X"), ("som_dispatch", dict(Y=None), "Y"),
    ("som_dispatch", dict(slot=None), "slot"), ("som_dispatch", dict(D=0), "width"), ("som_dispatch", dict(ldx=15), "X: leading"),
    ("som_dispatch", dict(ldy=15), "Y: leading"), ("som_dispatch", dict(M=-1), "negative"), ("som_dispatch", dict(M=2 ** 31), "2^31-1"),
    ("som_dispatch", dict(D=2 ** 20 + 1, ldx=2 ** 20 + 1, ldy=2 ** 20 + 1), "width"), ("som_dispatch", dict(ldx=2 ** 21 + 1), "above"),
    ("som_dispatch", dict(X="odd"), "aligned"),
    ("som_combine", dict(out=None), "out"), ("som_combine", dict(Y=None), "Y"), ("som_combine", dict(ldo=1), "out: leading"),
    ("som_combine", dict(type=-1), "type"), ("som_combine", dict(k=-3), "k=-3"),
    ("som_combine_grad", dict(dY=None, dweight=None), "neither"), ("som_combine_grad", dict(dout=None), "dout"),
    ("som_combine_grad", dict(Y=None), "Y"), ("som_combine_grad", dict(lddy=7), "dY: leading"), ("som_combine_grad", dict(lddo=7), "dout: leading"),
    ("som_node_product", dict(X=None), "X"), ("som_node_product", dict(A=None), "A"), ("som_node_product", dict(Y=None), "Y"),
    ("som_node_product", dict(offsets=None), "one node"), ("som_node_product", dict(act=5), "activation"), ("som_node_product", dict(act=-1), "activation"),
    ("som_node_product", dict(K=0), "K (0)"), ("som_node_product", dict(Dout=0), "width"), ("som_node_product", dict(ldr=7), "residual: leading"),
    ("som_node_product", dict(ldpre=7), "pre: leading"), ("som_node_product", dict(ldy=7), "Y: leading"),
    ("som_node_product_grad", dict(dX=None, dA=None, dbias=None), "none of"), ("som_node_product_grad", dict(pre=None), "pre"),
    ("som_node_product_grad", dict(dY=None), "dY"), ("som_node_product_grad", dict(X=None), "X"), ("som_node_product_grad", dict(A=None), "A"),
    ("som_node_product", dict(M=2 ** 31 - 65535), "2^31-65536"), ("som_node_product_grad", dict(M=2 ** 31 - 1), "2^31-65536"),
    ("som_node_product_grad", dict(lddx=15), "dX: leading"), ("som_node_product_grad", dict(offsets=None), "one node"),
]


@pytest.mark.parametrize("name, changes, says", REFUSED)
def test_refusals_name_their_reason_and_launch_nothing(ctx, name, changes, says):
    rc, kernels = call(ctx, name, **changes)
    assert rc == SOM_EINVAL and kernels == [] and says in ctx.error(), (rc, kernels, ctx.error())


def test_optional_arguments(ctx):
    assert call(ctx, "som_group", order=None, slot=None)[0] == SOM_OK
    assert call(ctx, "som_dispatch", weight=None)[0] == SOM_OK
    assert call(ctx, "som_combine_grad", Y=None, dweight=None)[0] == SOM_OK               # Y serves the weights' gradient only
    assert call(ctx, "som_node_product", bias=None, residual=None, pre=None)[0] == SOM_OK
    assert call(ctx, "som_node_product", offsets=None, K=1)[0] == SOM_OK
    assert call(ctx, "som_node_product_grad", pre=None, act=0)[0] == SOM_OK
    assert call(ctx, "som_node_product_grad", A=None, dX=None)[0] == SOM_OK
    assert call(ctx, "som_node_product_grad", X=None, dA=None)[0] == SOM_OK


def test_calls_on_nothing(ctx):
    """No rows: nothing is launched but what clears the outputs that have a value of their own."""
    rc, kernels = call(ctx, "som_group", T=0, node=None, order=None, slot=None)
    assert rc == SOM_OK and len(kernels) == 1
    assert call(ctx, "som_dispatch", T=0, X=None, slot=None, weight=None) == (SOM_OK, [])
    assert call(ctx, "som_combine", T=0, out=None, slot=None) == (SOM_OK, [])
    assert call(ctx, "som_combine", M=0, Y=None)[0] == SOM_OK                               # rows of zeros
    assert call(ctx, "som_node_product", M=0, X=None, Y=None) == (SOM_OK, [])
    rc, kernels = call(ctx, "som_node_product_grad", M=0, X=None, dY=None, pre=None, dX=None)
    assert rc == SOM_OK and kernels                                                        # zeros for dA and dbias


def test_null_context(stub):
    lib = C.CDLL(stub)
    for name, call_args in CALLS.items():
        assert getattr(lib, name)(None, *[C.c_void_p(None) if v == "p" else (i64(v) if key in WIDE else i32(v)) for key, v in call_args.items()]) == SOM_EINVAL


def test_without_memory_for_the_workspace(ctx):
    ctx.limit(16)
    rc, kernels = call(ctx, "som_group", T=100_000)
    assert rc == -2 and kernels == [] and "workspace" in ctx.error()
    rc, kernels = call(ctx, "som_node_product_grad", Din=300, ldx=300, lddx=300)
    assert rc == -2 and kernels == []
    ctx.limit()
    assert call(ctx, "som_group", T=100_000)[0] == SOM_OK


@pytest.mark.parametrize("T, k, K, launches", [(1, 8, 128, 1), (8192, 2, 64, 1), (8193, 2, 64, 3), (100, 1, 8205, 1), (100, 1, 8300, 4), (50_000, 1, 2047, 3),
                                               (50_000, 1, 2048, 4), (50_000, 1, 32768, 4)])
def test_group_routes(ctx, T, k, K, launches):
    """One launch up to 16384 pairs (where four wavefronts' counters fit LDS), beyond it three up to 2047 nodes and four above."""
    rc, kernels = call(ctx, "som_group", T=T, k=k, K=K)
    assert rc == SOM_OK and len(kernels) == launches, kernels


def tiles_of(ctx, name, **changes):
    """Rows of the tiles that a call launches (a workgroup's LDS is 512 bytes a row), in order."""
    call(ctx, name, **changes)
    return [lds // 512 for kernel, _, _, _, _, lds in ctx.launches if "product_tile" in kernel]


def test_shapes_take_every_tile(ctx):
    """The shapes of the GPU tests reach tiles of 64, 128 and 256 rows in the product and in both gradients, aligned and not."""
    seen = set()
    for M, K, Din, Dout in ref.TILES:
        off = "p" if K > 1 else None
        for t, E in ((0, 4), (1, 8), (2, 8)):
            aligned = Din % E == 0 and Dout % E == 0
            for b in tiles_of(ctx, "som_node_product", type=t, M=M, K=K, offsets=off, Din=Din, ldx=Din, Dout=Dout, ldr=Dout, ldpre=Dout, ldy=Dout):
                seen.add((t > 0, "product", b, aligned))
            grad = dict(type=t, M=M, K=K, offsets=off, Din=Din, ldx=Din, lddx=Din, Dout=Dout, lddy=Dout, ldpre=Dout, act=0, pre=None, dbias=None)
            for b in tiles_of(ctx, "som_node_product_grad", dA=None, **grad):
                seen.add((t > 0, "dX", b, aligned))
            for b in tiles_of(ctx, "som_node_product_grad", dX=None, **grad):
                seen.add((t > 0, "dA", b, aligned))
    want = {(half, form, b, aligned) for half in (True, False) for form in ("product", "dX", "dA") for b in (64, 128, 256) for aligned in (True, False)}
    assert want - seen == set()


@pytest.mark.parametrize("M, Din, Dout", [(22_076, 192, 1344), (25_792, 176, 784)])
def test_a_unit_holds_four_workgroups_of_64_rows(ctx, M, Din, Dout):
    """Between four and five tiles of 64 x 64 a unit: one round if five workgroups fitted its LDS, and two as four do, so tiles of 128 (of
    bfloat16 gradients 23 us instead of 34, and 19 instead of 25)."""
    assert 4 * 256 < -(-M // 64) * -(-Din // 64) <= 5 * 256
    assert tiles_of(ctx, "som_node_product_grad", type=1, M=M, K=1, offsets=None, Din=Din, ldx=Din, lddx=Din, Dout=Dout, lddy=Dout, act=0, pre=None,
                    dA=None, dbias=None) == [128]


@pytest.mark.parametrize("M", [60_000, 100_000, 130_000, 200_000])
def test_narrow_float32_gradients_fill_the_chip_once(ctx, M):
    """64 values both ways in float32: a workgroup's LDS leaves room for one a unit, so as many runs as there are units at most."""
    rc, _ = call(ctx, "som_node_product_grad", type=0, M=M, K=1, offsets=None, Din=64, ldx=64, lddx=64, Dout=64, lddy=64, ldpre=64)
    name, x, _, _, _, lds = ctx.launches[0]
    assert rc == SOM_OK and "gradient_narrow" in name and 160 * 1024 // lds == 1 and 128 < x <= 256
    rc, _ = call(ctx, "som_node_product_grad", type=1, M=M, K=1, offsets=None, Din=64, ldx=64, lddx=64, Dout=64, lddy=64, ldpre=64)
    assert rc == SOM_OK and 160 * 1024 // ctx.launches[0][5] >= 2 and 128 < ctx.launches[0][1] <= 512


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("M, Din, Dout, blocks", [(33, 512, 70, 4), (49, 517, 41, 4), (64, 1024, 130, 4), (64, 1031, 33, 4), (40, 300, 17, 4), (57, 640, 16, 4),
                                                  (17, 600, 50, 2), (32, 513, 24, 2)])
def test_blocks_of_one_nodes_few_rows(ctx, type, M, Din, Dout, blocks):
    """The shapes of the GPU tests of few rows take kernels of two and four blocks of sixteen rows."""
    rc, kernels = call(ctx, "som_node_product", type=type, M=M, K=1, offsets=None, Din=Din, ldx=Din, Dout=Dout, ldr=Dout, ldpre=Dout, ldy=Dout)
    assert rc == SOM_OK and len(kernels) == 1 and "product_few" in kernels[0] and f"Li{blocks}E" in kernels[0].replace(f",{blocks}>", f"Li{blocks}E")


def test_only_what_is_read_decides_how_gradients_are_read(ctx):
    """The slopes' pass reads the values before the activation; the products of dz that follow do not, and take the direct way to LDS whatever
    the leading dimension of those values."""
    for ldpre in (1024, 1025):
        rc, kernels = call(ctx, "som_node_product_grad", type=2, M=3000, Din=1024, ldx=1024, lddx=1024, Dout=1024, lddy=1024, ldpre=ldpre)
        assert rc == SOM_OK and [k for k in kernels if "product_tile" in k] and all("Lb1E" in k for k in kernels if "product_tile" in k), kernels
    rc, kernels = call(ctx, "som_node_product_grad", type=2, M=3000, Din=1024, ldx=1025, lddx=1024, Dout=1024, lddy=1024, ldpre=1024)
    assert rc == SOM_OK and ["Lb1E" in k for k in kernels if "product_tile" in k] == [True, False], kernels
    rc, kernels = call(ctx, "som_node_product", type=2, M=3000, Din=1024, ldx=1024, Dout=1024, ldy=1024, residual=None, ldr=1, pre=None, ldpre=3)
    assert rc == SOM_OK and len(kernels) == 1 and "product_tile" in kernels[0] and "Lb1E" in kernels[0], kernels


@pytest.mark.parametrize("K, Din, Dout, few", [(62, 264, 768, True), (63, 264, 768, False), (200, 1240, 512, False), (200, 1256, 512, True), (40, 248, 64, False), (40, 256, 64, True)])
def test_where_few_rows_have_a_kernel_of_their_own(ctx, K, Din, Dout, few):
    """Rows of 512 bytes and more; up to 3000 workgroups of sixteen results, or any number of them where the rows have 2500 bytes."""
    rc, kernels = call(ctx, "som_node_product", type=1, M=4 * K, K=K, Din=Din, ldx=Din, Dout=Dout, ldr=Dout, ldpre=Dout, ldy=Dout)
    assert rc == SOM_OK and len(kernels) == 1 and ("product_few" if few else "product_tile") in kernels[0], kernels


@pytest.mark.parametrize("type", [1, 2])
@pytest.mark.parametrize("M, Din, Dout, blocks", [(4136, 1024, 4096, 4), (4160, 2048, 4096, 4), (4115, 1024, 4096, 2)])
def test_last_rows_apart_take_blocks(ctx, type, M, Din, Dout, blocks):
    """The large products of the GPU tests leave their last rows to the kernel of few rows."""
    rc, kernels = call(ctx, "som_node_product", type=type, M=M, K=1, offsets=None, Din=Din, ldx=Din + 16, Dout=Dout, ldr=Dout + 32, ldpre=Dout + 24, ldy=Dout + 8)
    assert rc == SOM_OK and len(kernels) == 2 and "product_few" in kernels[1] and f"Li{blocks}E" in kernels[1].replace(f",{blocks}>", f"Li{blocks}E")


ROUTES = [  # call, changes, kernels in order
    # narrow rows: up to 64 results and 256 bytes of the contraction
    ("som_node_product", dict(M=5000, Din=64, ldx=64, Dout=64, ldr=64, ldpre=64, ldy=64), ["product_narrow"]),
    ("som_node_product", dict(M=5000, Din=65, ldx=65, Dout=64, ldr=64, ldpre=64, ldy=64), ["product_tile"]),
    ("som_node_product", dict(M=5000, Din=64, ldx=64, Dout=65, ldr=65, ldpre=65, ldy=65), ["product_tile"]),
    ("som_node_product", dict(type=1, M=5000, Din=128, ldx=128, Dout=64, ldr=64, ldpre=64, ldy=64), ["product_narrow"]),
    ("som_node_product", dict(type=1, M=5000, Din=129, ldx=129, Dout=64, ldr=64, ldpre=64, ldy=64), ["product_tile"]),
    # few rows: ten a node, or 64 of one
    ("som_node_product", dict(type=1, M=50, Din=2048, ldx=2048, Dout=256, ldr=256, ldpre=256, ldy=256), ["product_few"]),
    ("som_node_product", dict(type=1, M=51, Din=2048, ldx=2048, Dout=256, ldr=256, ldpre=256, ldy=256), ["product_tile"]),
    ("som_node_product", dict(type=1, M=64, K=1, offsets=None, Din=512, ldx=512, Dout=256, ldr=256, ldpre=256, ldy=256), ["product_few"]),
    ("som_node_product", dict(type=1, M=65, K=1, offsets=None, Din=512, ldx=512, Dout=256, ldr=256, ldpre=256, ldy=256), ["product_tile"]),
    ("som_node_product", dict(type=1, M=64, K=1, offsets=None, Din=255, ldx=255, Dout=256, ldr=256, ldpre=256, ldy=256), ["product_tile"]),
    # one node's last rows apart where they would start another round, and in the tiles where they would not
    ("som_node_product", dict(type=2, M=4099, K=1, offsets=None, Din=4096, ldx=4096, Dout=4096, ldr=4096, ldpre=4096, ldy=4096), ["product_tile", "product_few"]),
    ("som_node_product", dict(type=2, M=4000, K=1, offsets=None, Din=4096, ldx=4096, Dout=4096, ldr=4096, ldpre=4096, ldy=4096), ["product_tile"]),
    # gradients: slopes and biases in a pass of their own, joins where a group can have more than one run; narrow ones at once
    ("som_node_product_grad", dict(type=1, M=300, Din=300, ldx=300, lddx=300), ["slope", "product_tile", "product_tile"]),
    ("som_node_product_grad", dict(type=1, M=9000, Din=300, ldx=300, lddx=300), ["slope", "product_tile", "product_tile", "runs_join", "runs_join"]),
    ("som_node_product_grad", dict(type=1, M=300, Din=300, ldx=300, lddx=300, act=0, dbias=None), ["product_tile", "product_tile"]),
    ("som_node_product_grad", dict(type=1, M=300, Din=16, dA=None, dbias=None), ["gradient_narrow"]),
    ("som_node_product_grad", dict(type=1, M=300, Dout=65, lddy=65, ldpre=65, dA=None, dbias=None), ["product_narrow"]),
    ("som_node_product_grad", dict(type=1, M=0, dA=None, dbias=None), []),
    ("som_node_product_grad", dict(type=0, M=200, Din=64, ldx=64, lddx=64), ["gradient_narrow"]),
    ("som_node_product_grad", dict(type=2, M=9000, Din=64, ldx=64, lddx=64), ["gradient_narrow", "runs_join", "runs_join"]),
    ("som_node_product_grad", dict(type=0, M=200, Din=64, ldx=64, lddx=64, dX=None, dA=None), ["gradient_narrow"]),
    ("som_node_product_grad", dict(type=0, M=200, Din=65, ldx=65, lddx=65, act=0, dbias=None), ["product_tile", "product_tile"]),
    ("som_node_product_grad", dict(type=1, M=200, Dout=65, lddy=65, ldpre=65, act=0, dbias=None), ["product_narrow", "product_tile"]),
]


@pytest.mark.parametrize("name, changes, kernels", ROUTES)
def test_routes(ctx, name, changes, kernels):
    rc, got = call(ctx, name, **changes)
    assert rc == SOM_OK and len(got) == len(kernels) and all(k in g for k, g in zip(kernels, got)), got


def test_a_failed_launch_is_reported(ctx):
    for name in CALLS:
        rc, kernels = call(ctx, name)
        ctx.fail(kernels[-1].split("<")[0])
        rc, _ = call(ctx, name)
        assert rc == -3 and "launch" in ctx.error(), name
        ctx.fail()


def test_reference_group_by_hand():
    offsets, order, slot = ref.group(torch.tensor([[2, 0], [0, -1], [7, 2]], dtype=torch.int32), 3)
    assert offsets.tolist() == [0, 2, 2, 4] and order.tolist() == [1, 2, 0, 5, -1, -1] and slot.tolist() == [[2, 0], [1, -1], [-1, 3]]


@pytest.mark.parametrize("act", ref.ACTIVATIONS)
def test_reference_gradients_against_autograd_and_differences(act):
    """The reference's formulas: sorted rows, products and the way back, against torch's derivatives and central differences."""
    gen = torch.Generator().manual_seed(5)
    node = torch.randint(-1, 4, (9, 2), generator=gen).int()
    offsets, _, slot = ref.group(node, 4)
    w = torch.rand(9, 2, generator=gen, dtype=torch.float64)
    X, A, c, g = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((9, 5), (4, 3, 5), (4, 3), (9, 3)))
    off = offsets.tolist()

    def loss(X, A, c, w):
        total = 0.0
        for t in range(9):
            for j in range(2):
                if slot[t, j] >= 0:
                    e = int(node[t, j])
                    total = total + w[t, j] * (g[t] * ref.activation(A[e] @ X[t] + c[e], act)[0]).sum()
        return total

    places = torch.zeros(18, 5, dtype=torch.float64)
    Xg = ref.dispatch(X, slot, None, places)[0]
    empty = torch.zeros(18, 3, dtype=torch.float64)
    Y, _, pre, _ = ref.product(Xg, A, offsets, c, act, None, empty, empty)
    dY, _, dw, _ = ref.combine_grad(g, Y, slot, w, empty)
    dXg, _, dA, _, dc, _ = ref.product_grad(dY, Xg, A, offsets, pre, act, places)
    dX = ref.combine(dXg, slot, None)[0]
    leaves = [v.clone().requires_grad_() for v in (X, A, c, w)]
    auto = torch.autograd.grad(loss(*leaves), leaves)
    # float64 throughout, but for dz, whose bound and not value is rounded: agreement to 2^-40 of the largest entry
    for got, want in zip((dX, dA, dc, dw), auto):
        assert (got - want).abs().max() <= 2.0 ** -40 * want.abs().max().clamp(min=1)
    step = 2.0 ** -13
    for got, i in zip((dX, dA, dc, dw), range(4)):
        args = [X, A, c, w]
        d = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * d, args[i] - step * d
        slope = (loss(*up) - loss(*down)) / (2 * step)
        if act == "relu":
            continue                                     # (not differentiable where a step crosses zero)
        # the third derivative of a term is below 4 |d . A|^3 |g w|: of some forty terms of size 5 a thousandth of 2^-6 remains
        assert abs(float((got * d).sum() - slope)) <= 2.0 ** -12 * (1 + abs(float(slope)))
    assert off[-1] == int((slot >= 0).sum())


@pytest.mark.parametrize("Din", [65, 200])
@pytest.mark.parametrize("type", [0, 1, 2])
def test_as_many_rows_as_a_product_takes(ctx, type, Din):
    """2^31 - 65536 rows, with matrices that go through tiles: their launch holds them in rows of 2^20 workgroups, no dimension 2^32 work-items."""
    M = 2 ** 31 - 65536
    for name, changes in (("som_node_product", dict(Dout=1, ldy=1, act=0, bias=None, residual=None, pre=None)),
                          ("som_node_product_grad", dict(Dout=1, lddy=1, act=0, pre=None, dA=None, dbias=None)),
                          ("som_node_product_grad", dict(Dout=1, lddy=1, act=0, pre=None, dX=None, dbias=None))):
        if name == "som_node_product" and type > 0 and Din < 129:
            continue                                 # (a narrow product)
        for K, offsets in ((1, None), (32768, "p")):
            rc, kernels = call(ctx, name, type=type, M=M, Din=Din, ldx=Din, lddx=Din, offsets=offsets, K=K, **changes)
            assert rc == SOM_OK and "product_tile" in kernels[0], (rc, kernels, ctx.error())
            _, x, y, z, threads, lds = ctx.launches[0]
            assert x * threads < 2 ** 32 and y < 65536 and z == 1 and (y == 1 or x % 8 == 0)
            if changes.get("dX", "p"):
                rows, width = lds // 512, Din if name.endswith("grad") else 1
                assert x * y >= (-(-M // rows) + (K if K > 1 else 0)) * -(-width // rows)
    # the rows of the GPU test that goes beyond one row of the grid
    M = 2 ** 27 + 3
    call(ctx, "som_node_product_grad", type=2, M=M, K=1, offsets=None, Din=65, ldx=65, lddx=65, Dout=1, lddy=1, act=0, pre=None, dA=None, dbias=None)
    assert ctx.launches[0][2] > 1


@pytest.mark.parametrize("M, K, Din, Dout", [(640, 64, 2048, 1024), (10_000, 1000, 2048, 1024), (37, 5, 600, 70), (64, 1, 512, 256), (33, 1, 512, 256)])
def test_few_rows_have_a_workgroup_for_every_sixteen(ctx, M, K, Din, Dout):
    """However the rows of few-row products lie on the nodes, all on one among them, each sixteen of a node have workgroups of their own
    (one node's rows go sixteen, 32 or 64 to one)."""
    rc, kernels = call(ctx, "som_node_product", type=1, M=M, K=K, offsets="p" if K > 1 else None, Din=Din, ldx=Din, Dout=Dout, ldr=Dout, ldpre=Dout, ldy=Dout)
    assert rc == SOM_OK and len(kernels) == 1 and "product_few" in kernels[0]
    across = -(-Dout // 16)
    if K == 1:
        assert ctx.launches[0][1] == across
        return
    gen = torch.Generator().manual_seed(M)
    even, one = torch.full((K,), M // K), torch.zeros(K, dtype=torch.long)
    even[:M % K] += 1
    one[K // 2] = M
    for counts in (even, one, torch.bincount((torch.rand(M, generator=gen) ** 6 * K).long(), minlength=K)):
        assert ctx.launches[0][1] >= int(((counts + 15) // 16).sum()) * across


@pytest.mark.parametrize("name", ["som_dispatch", "som_combine", "som_combine_grad"])
def test_places_of_a_row_are_bounded(ctx, name):
    """A row's places are counted in steps of four by one group of lanes, whose count would pass 2^31 - 1 for a single row of as many."""
    assert call(ctx, name, T=1, k=2 ** 20, M=2 ** 20)[0] == SOM_OK
    for k in (2 ** 20 + 1, 2 ** 31 - 3, 2 ** 31 - 1):
        rc, kernels = call(ctx, name, T=1, k=k, M=2 ** 20)
        assert rc == SOM_EINVAL and kernels == [] and "places of a row" in ctx.error()
    assert call(ctx, "som_group", T=1, k=2 ** 20 + 1)[0] == SOM_OK              # the sort has pairs only


class Recorder:
    """Stands for the library behind the Python wrapper: every call is noted and succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or SOM_OK


@pytest.fixture
def wrapper(monkeypatch):
    """The Python wrapper on CPU tensors, without a library."""
    from paper_2604_26555_amd import som as module
    monkeypatch.setattr(module, "_raw_stream", lambda index: 0)
    s = module.Som.__new__(module.Som)
    s.lib, s.device, s._raw, s._h = Recorder(), torch.device("cpu"), 0, None
    return s


def test_group_writes_offsets_only_where_they_lie_side_by_side(wrapper):
    """K + 1 integers are written from the first entry's address on: a column of a matrix or an expanded number does not hold them."""
    node, order, slot = (torch.zeros(6, dtype=torch.int32) for _ in range(3))
    table = torch.zeros(5, 3, dtype=torch.int32)
    for offsets in (table[:, 1:2], table[:, 1], table[:1, :1].expand(5, 1), table[0, :1].expand(5), table.view(15)[::3], torch.zeros(4, dtype=torch.int32)):
        with pytest.raises(ValueError):
            wrapper.som_group(node, 4, offsets=offsets, order=order, slot=slot)
    assert wrapper.lib.calls == []
    offsets = torch.zeros(5, dtype=torch.int32)
    assert wrapper.som_group(node, 4, offsets=offsets, order=order, slot=slot)[0] is offsets
    assert wrapper.lib.calls[0][1][5] == offsets.data_ptr()


def test_rows_that_a_call_leaves_are_zeros_in_new_outputs(wrapper):
    """What is no pair's place, or no node's row, is not written: in a tensor that the wrapper makes it holds zeros, not what was in memory."""
    slot, offsets = torch.tensor([[0], [-1], [1]], dtype=torch.int32), torch.tensor([0, 1, 2], dtype=torch.int32)
    X, A, dY = torch.ones(3, 8), torch.ones(2, 4, 8), torch.ones(3, 4)
    torch.use_deterministic_algorithms(True)                  # (new memory is filled with NaN then)
    try:
        assert torch.isnan(torch.empty(3)).all()
        new = [wrapper.som_dispatch(X, slot), wrapper.som_combine_grad(X, X, slot)[0], wrapper.som_node_product(X, A, offsets=offsets),
               wrapper.som_node_product_grad(dY, X, A, offsets=offsets)[0]]
    finally:
        torch.use_deterministic_algorithms(False)
    assert [tuple(t.shape) for t in new] == [(3, 8), (3, 8), (3, 4), (3, 8)] and not any(t.any() for t in new)
    assert [name for name, _ in wrapper.lib.calls] == ["som_dispatch", "som_combine_grad", "som_node_product", "som_node_product_grad"]
