"""The operators of local models on a map as cases that can be timed: rows sorted by node and back, and the product of
every row with its node's matrix.

A map (or any router) gives each row one or more nodes.  ``som_group`` puts the (row, node) pairs in the nodes' order,
``som_dispatch`` brings the rows there, ``som_node_product`` takes each row through its node's matrix with bias, activation
and residual, and ``som_combine`` adds a row's results up again with its weights; the ``_grad`` calls are the way back of a
training step.  Sizes are this repository's workloads (50 features on 32 x 32 nodes, 37 on 19 x 23, 200 features) and, for
half-precision rows, generic widths from one row to some ten thousand.

With ``own`` false, ``run`` computes the same in elementary torch operations in float32.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTIVATIONS = ["none", "relu", "silu", "gelu", "gelu_tanh"]

# Fields of a case:
#   op       sort          pairs sorted by node and the rows brought into that order
#            combine       rows back, with weights
#            combine_grad  the gradient of that for the sorted rows and the weights
#            product       every sorted row times its node's matrix, with bias, activation and residual
#            product_grad  its gradient for the rows, the matrices and the biases
#   type     of rows and matrices; weights of rows are float32
#   t, k     rows, and nodes a row has (the sorted form holds t * k rows);  nodes: nodes of the map
#   d, dout  features of a row, and of a product's result
#   drop     share of rows that are padding, and half as many single pairs that found no place (node -1)
#   act, bias, residual, pre   the product's epilogue; pre: the values before the activation are kept for the gradient


def _case(name, op, type, t, k, nodes, d, dout=0, drop=0.0, act="none", bias=False, residual=False, pre=False):
    c = dict(op=op, type=type, t=int(t), k=int(k), nodes=int(nodes), d=int(d), dout=int(dout), drop=float(drop), act=act,
             bias=bool(bias), residual=bool(residual), pre=bool(pre))
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one row on its way to eight nodes' models, as a serving loop sends it: all latency
        _case("sort_one_row", "sort", "bf16", 1, 8, 128, 2048),
        # a batch of prompts with padding
        _case("sort_prompts", "sort", "bf16", 16384, 4, 64, 2048, drop=0.04),
        # the headline table (cfg1): every row to its unit
        _case("sort_1m_d50", "sort", "f32", 1_000_000, 1, 1024, 50),
        # sixteen sequences in flight, one row each
        _case("combine_16_rows", "combine", "f16", 16, 8, 128, 2048),
        # the way back of a batch of prompts
        _case("combine_prompts", "combine", "bf16", 16384, 4, 64, 2048),
        # and its gradient in a training step
        _case("combine_grad_prompts", "combine_grad", "bf16", 16384, 4, 64, 2048),
        # a wide table of odd size, each row with its two nearest nodes, some rows left out
        _case("combine_grad_30k_d200", "combine_grad", "f32", 30_011, 2, 437, 200, drop=0.05),
        # four rows of a serving loop through eight models each: the models' matrices are what is read
        _case("product_32_rows", "product", "bf16", 32, 1, 64, 2048, 1024, act="silu", bias=True),
        # a training batch through its models, values before the activation kept
        _case("product_64k_rows", "product", "bf16", 65536, 1, 64, 2048, 1536, act="gelu_tanh", bias=True, residual=True, pre=True),
        # one model for all rows, an odd number of them
        _case("product_one_node", "product", "f16", 4099, 1, 1, 4096, 4096, act="gelu", bias=True),
        # the gradient of a training batch
        _case("product_grad_32k_rows", "product_grad", "bf16", 32768, 1, 64, 2048, 1536, act="silu", bias=True, pre=True),
        # local models of a table in float32: 37 features to 24 values on 19 x 23 nodes
        _case("product_grad_250k_d37", "product_grad", "f32", 250_013, 1, 437, 37, 24, act="relu", bias=True, pre=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sort", "sort", "combine", "combine_grad", "product", "product", "product_grad", "product_grad"])
    type = rng.choice(["f32", "bf16", "bf16", "f16"])
    nodes = _log(rng, 1, 1200)
    size = 4 if type == "f32" else 2
    if not op.startswith("product"):
        d = _log(rng, 8, 4096)
        k = min(nodes, rng.choice([1, 1, 2, 4, 6, 8]))
        t = _log(rng, 1, min(1_000_000, 2.5e8 / (d * size * (k + 0.25))))
        return _case(None, op, type, t, k, nodes, d, drop=rng.choice([0.0, 0.0, 0.03]))
    d, dout = _log(rng, 8, 4096), _log(rng, 4, 4096)
    if rng.random() < 0.6:                         # widths of half-precision models are mostly multiples of something
        d, dout = max(8, d - d % 16), max(8, dout - dout % 16)
    nodes = max(1, min(nodes, int(2e8 / (d * dout))))
    most = 1.9e11 / (d * dout) / (2 if op == "product_grad" else 1) / (8 if type == "f32" else 1)
    t = _log(rng, 1, max(2, min(1_000_000, most, 4e8 / (size * (d + dout)))))
    act = rng.choice(ACTIVATIONS)
    return _case(None, op, type, t, 1, nodes, d, dout, drop=rng.choice([0.0, 0.0, 0.03]), act=act, bias=rng.random() < 0.6,
                 residual=op == "product" and rng.random() < 0.4, pre=act != "none" and (op == "product_grad" or rng.random() < 0.5))


def _nodes(case, gen):
    """Nodes of every row, distinct within a row, some nodes sought far more often than others."""
    t, k, nodes = case["t"], case["k"], case["nodes"]
    popular = torch.empty(nodes, device=DEVICE).exponential_(generator=gen) + 0.2
    if k == 1:
        edges = torch.cumsum((popular / popular.sum()).double(), 0)
        u = torch.rand(t, device=DEVICE, generator=gen, dtype=torch.float64)
        node = torch.searchsorted(edges, u).clamp_(max=nodes - 1)[:, None]
    else:
        node = torch.empty((t, k), device=DEVICE, dtype=torch.int64)
        step = max(1, (1 << 24) // nodes)
        for lo in range(0, t, step):
            n = min(step, t - lo)
            score = torch.log(popular) - torch.log(torch.empty((n, nodes), device=DEVICE).exponential_(generator=gen))
            node[lo:lo + n] = torch.topk(score, k, dim=1).indices
    node = node.int()
    if case["drop"]:
        gone = torch.rand((t, 1), device=DEVICE, generator=gen) < case["drop"]
        gone = gone | (torch.rand((t, k), device=DEVICE, generator=gen) < 0.5 * case["drop"])
        node = torch.where(gone, torch.full_like(node, -1), node)
    return node.contiguous()


def _places(node, nodes):
    """Stable sort of the pairs by node: offsets, order, slot (elementary operations, nothing read back)."""
    flat = node.reshape(-1).long()
    kept = (flat >= 0) & (flat < nodes)
    key, order = torch.sort(torch.where(kept, flat, nodes), stable=True)
    offsets = torch.searchsorted(key, torch.arange(nodes + 1, device=node.device))
    slot = torch.empty_like(order)
    slot[order] = torch.arange(order.numel(), device=node.device)
    slot = torch.where(kept, slot, -1)
    order = torch.where(key < nodes, order, -1)
    return offsets.int(), order.int(), slot.reshape(node.shape).int()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    type, t, k, d = TYPES[case["type"]], case["t"], case["k"], case["d"]

    def normal(*shape, scale=1.0, of=type):
        out = torch.empty(shape, device=DEVICE, dtype=of)
        rows = max(1, (1 << 26) // max(1, out[0].numel()))
        for lo in range(0, shape[0], rows):
            part = out[lo:lo + rows]
            part.copy_(torch.randn(part.shape, device=DEVICE, generator=gen).mul_(scale))
        return out

    s = dict(case=case)
    node = _nodes(case, gen)
    if case["op"] == "sort":
        s.update(node=node, X=normal(t, d), Y=torch.zeros((t * k, d), device=DEVICE, dtype=type))
        return s
    offsets, _, slot = _places(node, case["nodes"])
    if case["op"] in ("combine", "combine_grad"):
        weight = torch.softmax(torch.randn((t, k), device=DEVICE, generator=gen), 1)
        s.update(slot=slot, weight=weight.contiguous(), Y=normal(t * k, d))
        if case["op"] == "combine_grad":
            s.update(dout=normal(t, d), dY=torch.zeros((t * k, d), device=DEVICE, dtype=type))
        return s
    nodes, dout = case["nodes"], case["dout"]
    s.update(X=normal(t, d), A=normal(nodes, dout, d, scale=1.0 / math.sqrt(d)))
    s["offsets"] = None if nodes == 1 and not case["drop"] else offsets
    s["bounds"] = offsets.tolist()               # the plain form's loop over the nodes, known before the call
    s["bias"] = normal(nodes, dout, scale=0.5) if case["bias"] else None
    if case["op"] == "product":
        s["residual"] = normal(t, dout) if case["residual"] else None
        s["pre"] = torch.zeros((t, dout), device=DEVICE, dtype=type) if case["pre"] else None
        s["Y"] = torch.zeros((t, dout), device=DEVICE, dtype=type)
        return s
    s["dY"] = normal(t, dout)
    s["pre"] = normal(t, dout) if case["pre"] else None
    s["dX"] = torch.zeros((t, d), device=DEVICE, dtype=type)
    return s


_contexts = {}


def _context():
    """The program's library context on the stream it works on, kept."""
    key = torch.cuda.current_stream().cuda_stream
    if key not in _contexts:
        import paper_2604_26555_amd as pkg
        _contexts[key] = pkg.Som(0)
    return _contexts[key]


def _activate(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    c = math.sqrt(2.0 / math.pi)
    th = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + th) + 0.5 * z * (1.0 - th * th) * c * (1.0 + 3.0 * 0.044715 * z * z)


def _run_own(s):
    case, som = s["case"], _context()
    op = case["op"]
    if op == "sort":
        offsets, order, slot = som.som_group(s["node"], case["nodes"])
        return [offsets, order, slot, som.som_dispatch(s["X"], slot, out=s["Y"])]
    if op == "combine":
        return [som.som_combine(s["Y"], s["slot"], weight=s["weight"])]
    if op == "combine_grad":
        return list(som.som_combine_grad(s["dout"], s["Y"], s["slot"], weight=s["weight"], dY=s["dY"]))
    if op == "product":
        som.som_node_product(s["X"], s["A"], offsets=s["offsets"], bias=s["bias"], activation=case["act"], residual=s["residual"],
                             pre=s["pre"], out=s["Y"])
        return [s["Y"]] if s["pre"] is None else [s["Y"], s["pre"]]
    dX, dA, dbias = som.som_node_product_grad(s["dY"], s["X"], s["A"], offsets=s["offsets"], pre=s["pre"], activation=case["act"],
                                              dX=s["dX"], dbias=None if case["bias"] else False)
    return [dX, dA] if dbias is None else [dX, dA, dbias]


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op, type, k = case["op"], TYPES[case["type"]], case["k"]
    if op == "sort":
        offsets, order, slot = _places(s["node"], case["nodes"])
        rows = s["X"][order.long().clamp(min=0) // k]
        return [offsets, order, slot, torch.where((order >= 0)[:, None], rows, torch.zeros_like(rows))]
    if op in ("combine", "combine_grad"):
        held = (s["slot"] >= 0)[:, :, None]
        at = s["slot"].long().clamp(min=0)
        rows = torch.where(held, s["Y"][at].float(), 0.0)
        if op == "combine":
            return [(rows * s["weight"][:, :, None]).sum(1).to(type)]
        dout = s["dout"].float()
        dweight = (rows * dout[:, None, :]).sum(2)
        scaled = (dout[:, None, :] * s["weight"][:, :, None]).to(type)
        # pairs without a place go to a row behind the last, which is cut off
        dY = torch.zeros((at.numel() + 1, case["d"]), device=DEVICE, dtype=type)
        dY[torch.where(s["slot"] >= 0, at, at.numel()).reshape(-1)] = scaled.reshape(-1, case["d"])
        return [dY[:-1], dweight]
    X, A, bounds, act = s["X"], s["A"], s["bounds"], case["act"]
    if op == "product":
        Y = torch.zeros((case["t"], case["dout"]), device=DEVICE, dtype=type)
        pre = torch.zeros_like(Y) if case["pre"] else None
        for e in range(case["nodes"]):
            lo, hi = bounds[e], bounds[e + 1]
            if lo == hi:
                continue
            z = X[lo:hi].float() @ A[e].float().t()
            if s["bias"] is not None:
                z = z + s["bias"][e].float()
            if pre is not None:
                pre[lo:hi] = z.to(type)
            y = _activate(z, act)
            if s["residual"] is not None:
                y = y + s["residual"][lo:hi].float()
            Y[lo:hi] = y.to(type)
        return [Y] if pre is None else [Y, pre]
    dz = s["dY"].float()
    if act != "none":
        dz = dz * _slope(s["pre"].float(), act)
    dX = torch.zeros((case["t"], case["d"]), device=DEVICE, dtype=type)
    dA = torch.zeros_like(A)
    dbias = torch.zeros((case["nodes"], case["dout"]), device=DEVICE, dtype=type)
    for e in range(case["nodes"]):
        lo, hi = bounds[e], bounds[e + 1]
        if lo == hi:
            continue
        dX[lo:hi] = (dz[lo:hi] @ A[e].float()).to(type)
        dA[e] = (dz[lo:hi].t() @ X[lo:hi].float()).to(type)
        if case["bias"]:
            dbias[e] = dz[lo:hi].sum(0).to(type)
    return [dX, dA, dbias] if case["bias"] else [dX, dA]


def work(case):
    t, k, d, dout, nodes = (float(case[x]) for x in ("t", "k", "d", "dout", "nodes"))
    b = 4.0 if case["type"] == "f32" else 2.0
    kept = (1.0 - case["drop"]) * (1.0 - 0.5 * case["drop"])
    pairs = t * k * kept
    op = case["op"]
    if op == "sort":
        return {"bytes": 12.0 * t * k + 4.0 * (nodes + 1) + b * d * (t + pairs), "flops": t * k}
    if op == "combine":
        return {"bytes": 8.0 * t * k + b * d * (pairs + t), "flops": 2.0 * pairs * d}
    if op == "combine_grad":
        return {"bytes": 12.0 * t * k + b * d * (t + 2.0 * pairs), "flops": 3.0 * pairs * d}
    read = min(nodes, pairs)                       # matrices that some row asks for
    if op == "product":
        results = 1 + int(case["residual"]) + int(case["pre"])
        return {"bytes": b * (pairs * d + read * dout * (d + int(case["bias"])) + pairs * dout * results), "flops": 2.0 * pairs * d * dout}
    return {"bytes": b * (2.0 * pairs * d + pairs * dout * (1 + int(case["pre"])) + (read + nodes) * dout * d + nodes * dout * int(case["bias"])),
            "flops": 4.0 * pairs * d * dout}


def exact(case, seed):
    """From the definitions, pair by pair and node by node, in float64."""
    s = prepare(case, seed)
    op, k = case["op"], case["k"]
    if op == "sort":
        node = s["node"].cpu().numpy().reshape(-1).astype(np.int64)
        members = np.flatnonzero((node >= 0) & (node < case["nodes"]))
        members = members[np.argsort(node[members], kind="stable")]
        offsets = np.concatenate([[0], np.cumsum(np.bincount(node[members], minlength=case["nodes"]))])
        order = np.full(node.size, -1)
        order[:members.size] = members
        slot = np.full(node.size, -1)
        slot[members] = np.arange(members.size)
        Y = torch.zeros((node.size, case["d"]), device=DEVICE, dtype=torch.float64)
        Y[:members.size] = s["X"].double()[torch.from_numpy(members // k).to(DEVICE)]
        return [torch.from_numpy(offsets), torch.from_numpy(order), torch.from_numpy(slot.reshape(case["t"], k)), Y]
    if op in ("combine", "combine_grad"):
        Y = s["Y"].double()
        out = torch.zeros((case["t"], case["d"]), device=DEVICE, dtype=torch.float64)
        dY = torch.zeros_like(Y) if op == "combine_grad" else None
        dweight = torch.zeros((case["t"], k), device=DEVICE, dtype=torch.float64)
        for j in range(k):
            rows = torch.nonzero(s["slot"][:, j] >= 0)[:, 0]
            at = s["slot"][rows, j].long()
            w = s["weight"][rows, j].double()[:, None]
            if op == "combine":
                out.index_add_(0, rows, w * Y[at])
            else:
                g = s["dout"][rows].double()
                dY[at] = w * g
                dweight[rows, j] = torch.linalg.vecdot(g, Y[at])
        return [out] if op == "combine" else [dY, dweight]
    act, X, A = case["act"], s["X"], s["A"]
    outs = {"product": ["Y", "pre"], "product_grad": ["dX", "dA", "dbias"]}[op]
    r = dict(Y=torch.zeros((case["t"], case["dout"]), device=DEVICE, dtype=torch.float64),
             pre=torch.zeros((case["t"], case["dout"]), device=DEVICE, dtype=torch.float64) if case["pre"] else None,
             dX=torch.zeros((case["t"], case["d"]), device=DEVICE, dtype=torch.float64), dA=torch.zeros(A.shape, device=DEVICE, dtype=torch.float64),
             dbias=torch.zeros((case["nodes"], case["dout"]), device=DEVICE, dtype=torch.float64) if case["bias"] else None)

    def parts(z):
        """The activation and its slope."""
        if act == "relu":
            return z.clamp(min=0.0), torch.heaviside(z, torch.zeros_like(z))
        if act == "silu":
            g = torch.special.expit(z)
            return z * g, g + z * g * (1.0 - g)
        if act == "gelu":
            phi = torch.special.ndtr(z)
            return z * phi, phi + z * torch.exp(-z * z / 2.0) * 0.3989422804014327
        if act == "gelu_tanh":
            u = 1.5957691216057308 * (z + 0.044715 * z ** 3)         # (1 + tanh(u / 2)) / 2 is the logistic function of u
            g = torch.special.expit(u)
            return z * g, g + z * g * (1.0 - g) * 1.5957691216057308 * (1.0 + 0.134145 * z * z)
        return z, torch.ones_like(z)

    for e in range(case["nodes"]):
        rows = slice(s["bounds"][e], s["bounds"][e + 1])
        if rows.start == rows.stop:
            continue
        x, a = X[rows].double(), A[e].double()
        if op == "product":
            z = torch.mm(a, x.t().contiguous()).t()
            if s["bias"] is not None:
                z = z + s["bias"][e].double()
            if case["pre"]:
                r["pre"][rows] = z
            y = parts(z)[0]
            r["Y"][rows] = y if s["residual"] is None else y + s["residual"][rows].double()
        else:
            dz = s["dY"][rows].double()
            if act != "none":
                dz = dz * parts(s["pre"][rows].double())[1]
            r["dX"][rows] = torch.mm(dz, a)
            r["dA"][e] = torch.mm(x.t().contiguous(), dz).t()
            if case["bias"]:
                r["dbias"][e] = dz.sum(0)
    return [r[o] for o in outs if r[o] is not None]
