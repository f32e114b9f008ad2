"""The operators of a mini-batch step around the layers, as they are measured: rows that are looked up by vertex id and the gradient of
the table they come from, rows kept in 8 bits, and the step that orthogonalises the update of a weight matrix.

A case is a dict of plain values.  "kind" names the operator and its direction:
  lookup       rows of a table by id, scaled
  lookup_grad  the gradient of the table: the rows that came back, summed by id
  store        rows quantised into a store of 8-bit rows, at the places that ids name
  load         rows of such a store by id, as numbers again
  orthogonal   matrices orthogonalised by Newton-Schulz products
  muon         one optimizer step over a model's weight matrices with updates orthogonalised like that
Sizes: "v" rows of the table or store, "n" ids, "f" columns; "ids" says how the ids are spread: "uniform", "hubs" (few ids come often, as
the sources of a graph do), "each" (every row once, in random order); "padded" is the share of ids that name no row.  "table" and
"dtype" are the types of the table and of the looked-up rows.  "shapes" are matrices, as rows x columns.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the plain forms below; True: the framework's entry points

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SCALE = 0.125                            # of a lookup
BLOCK = 32                               # columns of a stored row that share an exponent
TOP = 448.0                              # the largest number of the 8-bit type
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
HYPER = dict(lr=0.02, momentum=0.95)
DECAY = 0.01


def listed():
    return [
        # a small batch on the smallest graph in use: launches and the host path count
        dict(name="lookup_small", kind="lookup", v=4096, n=1021, f=64, ids="uniform", padded=0.0, table="f32", dtype="f32"),
        # a large batch's vertices from bf16 embeddings of the 2.4-million-vertex graph, in the layers' type
        dict(name="lookup_batch", kind="lookup", v=2449029, n=1224515, f=256, ids="hubs", padded=0.0, table="bf16", dtype="f32"),
        # the gradient of the small batch
        dict(name="grad_small", kind="lookup_grad", v=4096, n=1021, f=64, ids="uniform", padded=0.0, table="f32", dtype="f32"),
        # learned embeddings of the 2.4-million-vertex graph: most rows come once or not at all, some thousands of times
        dict(name="grad_vertices", kind="lookup_grad", v=2449029, n=1224515, f=100, ids="hubs", padded=0.0, table="f32", dtype="f32"),
        # one of 47 categories for every vertex, unknown for some: long sums
        dict(name="grad_categories", kind="lookup_grad", v=47, n=2449029, f=256, ids="uniform", padded=0.08, table="bf16", dtype="bf16"),
        # hidden rows of a small batch, written
        dict(name="store_small", kind="store", v=4096, n=1021, f=64, ids="uniform", padded=0.0, dtype="f32"),
        # hidden rows of a large batch's vertices in bf16, some vertices more than once
        dict(name="store_batch", kind="store", v=2449029, n=1224515, f=256, ids="hubs", padded=0.0, dtype="bf16"),
        # a small batch's neighbours, read
        dict(name="load_small", kind="load", v=4096, n=1021, f=100, ids="hubs", padded=0.0, dtype="f32"),
        # a large batch from stored features beyond every cache
        dict(name="load_capacity", kind="load", v=27764989, n=2449029, f=128, ids="uniform", padded=0.01, dtype="bf16"),
        # the weight matrices of the three-layer model: launches count
        dict(name="orthogonal_model", kind="orthogonal", shapes="100x256,256x256,256x47", dtype="f32"),
        # wide layers in bf16, the step with momentum
        dict(name="muon_wide", kind="muon", shapes="602x1000,1000x1000,1000x41", dtype="bf16"),
        # one large matrix: the matrix cores decide
        dict(name="orthogonal_large", kind="orthogonal", shapes="2560x4000", dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _matrices(case):
    return [tuple(int(d) for d in s.split("x")) for s in case["shapes"].split(",")]


def draw(rng):
    """A case of the same ranges: sizes over their logarithms, odd ones among them, below the largest listed one's work."""
    kind = rng.choice(["lookup", "lookup_grad", "lookup_grad", "store", "load", "orthogonal", "muon"])
    if kind in ("orthogonal", "muon"):
        most = rng.choice([64, 300, 1200, 2400])
        widths = [_log_int(rng, 8, most) for _ in range(rng.randrange(2, 6))]
        return dict(kind=kind, shapes=",".join(f"{a}x{b}" for a, b in zip(widths, widths[1:])), dtype=rng.choice(["f32", "bf16"]))
    f = _log_int(rng, 4, 602)
    n = _log_int(rng, 16, min(2449029, 300000000 // f))
    v = _log_int(rng, 16, min(2449029, 300000000 // f))
    ids = rng.choice(["uniform", "hubs", "each"])
    if ids == "each":
        v = n
    case = dict(kind=kind, v=v, n=n, f=f, ids=ids, padded=rng.choice([0.0, 0.0, 0.05, 0.5]), dtype=rng.choice(["f32", "bf16"]))
    if kind.startswith("lookup"):
        case["table"] = rng.choice(["f32", "bf16"])
    return case


# ---------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(generator=gen)


def _ids(case, gen):
    v, n = case["v"], case["n"]
    if case["ids"] == "each":
        ids = torch.randperm(v, device="cuda", generator=gen)
    else:
        u = torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)
        ids = ((u ** 2.5 if case["ids"] == "hubs" else u) * v).to(torch.int64).clamp(max=v - 1)
    ids[torch.rand(n, device="cuda", generator=gen) < case["padded"]] = -1
    return ids.to(torch.int32)


def _stride(f):
    """Bytes of a stored row: the codes, an exponent for each block of them, up to a multiple of 16."""
    return -(-(f + -(-f // BLOCK)) // 16) * 16


def _stored(s):
    """The codes and the exponents of a store as tensors of their own types."""
    f = s["case"]["f"]
    return s["store"][:, :f].view(torch.float8_e4m3fn), s["store"][:, f:f + -(-f // BLOCK)]


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    s = dict(case=case)
    if kind in ("orthogonal", "muon"):
        dtype = DTYPES[case["dtype"]]
        s["tensors"] = []
        for rows, cols in _matrices(case):
            # a gradient is a sum over vertices of which a part of the directions has most
            k = min(rows, cols)
            size = 10.0 ** (-1.0 * torch.rand(k, device="cuda", generator=gen))
            g = (_normal(gen, rows, k) * size) @ _normal(gen, k, cols) * (1e-3 / k ** 0.5)
            t = dict(g=g.to(dtype))
            if kind == "muon":
                w = _normal(gen, rows, cols) / rows ** 0.5
                t.update(p=w.to(dtype), m=_normal(gen, rows, cols) * 5e-3, scale=max(1.0, cols / rows) ** 0.5)
            else:
                t["o"] = torch.empty_like(t["g"])
            s["tensors"].append(t)
    else:
        v, n, f, dtype = case["v"], case["n"], case["f"], DTYPES[case["dtype"]]
        s["ids"] = _ids(case, gen)
        if kind == "lookup":
            s.update(table=_normal(gen, v, f, dtype=DTYPES[case["table"]]), y=torch.empty(n, f, device="cuda", dtype=dtype))
        elif kind == "lookup_grad":
            s.update(dy=_normal(gen, n, f, dtype=dtype).mul_(1e-2), dtable=torch.empty(v, f, device="cuda", dtype=DTYPES[case["table"]]))
        else:
            s["store"] = torch.zeros(v, _stride(f), device="cuda", dtype=torch.uint8)
            if kind == "store":
                x = _normal(gen, n, f, dtype=dtype)
                s["x"] = x * (x > -0.5) * (_normal(gen, f).abs() + 0.1).to(dtype)  # behind a rectifier many values are 0
            else:
                codes, exponents = _stored(s)
                for a in range(0, v, 1 << 20):
                    b = min(v, a + (1 << 20))
                    codes[a:b], exponents[a:b] = _quantised(_normal(gen, b - a, f) * (_normal(gen, f).abs() + 0.1))
                s["y"] = torch.empty(n, f, device="cuda", dtype=dtype)
    if own:
        _keep(s)
    return s


def _keep(s):
    """What a program keeps between its steps: workspaces, and the list of a model's matrices."""
    import paper_2104_06700_amd as gnn
    case = s["case"]
    kind = case["kind"]
    if kind == "lookup_grad":
        nbytes = gnn.gnn_lookup_workspace_bytes(case["v"], case["n"], case["f"])
    elif kind == "store":
        nbytes = gnn.gnn_store_rows_workspace_bytes(case["v"], case["n"])
    elif kind == "muon":
        ts = s["tensors"]
        s["handle"] = gnn.MuonTensors([t["p"] for t in ts], [t["g"] for t in ts], [t["m"] for t in ts], weight_decay=DECAY,
                                      update_scale=[t["scale"] for t in ts])
        nbytes = gnn.gnn_muon_workspace_bytes(s["handle"])
    elif kind == "orthogonal":
        s["handle"] = gnn.OrthogonalizeTensors([t["g"] for t in s["tensors"]], [t["o"] for t in s["tensors"]])
        nbytes = gnn.gnn_orthogonalize_workspace_bytes(s["handle"])
    else:
        return
    s["workspace"] = torch.empty(max(nbytes, 1), device="cuda", dtype=torch.uint8)


# ---------------------------------------------------------------- passes

def run(s):
    if own:
        return _run_own(s)
    return {"lookup": _plain_lookup, "lookup_grad": _plain_lookup_grad, "store": _plain_store, "load": _plain_load,
            "orthogonal": _plain_orthogonal, "muon": _plain_muon}[s["case"]["kind"]](s)


def _run_own(s):
    import paper_2104_06700_amd as gnn
    kind = s["case"]["kind"]
    if kind == "lookup":
        gnn.gnn_lookup_fwd(s["table"], s["ids"], s["y"], scale=SCALE)
        return s["y"]
    if kind == "lookup_grad":
        gnn.gnn_lookup_bwd(s["ids"], s["dy"], s["dtable"], scale=SCALE, workspace=s["workspace"])
        return s["dtable"]
    if kind == "store":
        gnn.gnn_store_rows(s["x"], s["store"], s["ids"], workspace=s["workspace"])
        return list(_stored(s))
    if kind == "load":
        gnn.gnn_load_rows(s["store"], s["y"], s["ids"])
        return s["y"]
    if kind == "muon":
        gnn.gnn_muon_step(s["handle"], HYPER["lr"], momentum=HYPER["momentum"], steps=STEPS, workspace=s["workspace"])
        return [[t["p"], t["m"]] for t in s["tensors"]]
    gnn.gnn_orthogonalize(s["handle"], steps=STEPS, workspace=s["workspace"])
    return [t["o"] for t in s["tensors"]]


# ---------------------------------------------------------------- plain forms

def _plain_lookup(s):
    v, ids = s["case"]["v"], s["ids"].long()
    there = (ids >= 0) & (ids < v)
    rows = s["table"][ids.clamp(0, v - 1)].float() * SCALE
    s["y"].copy_(rows * there[:, None])
    return s["y"]


def _plain_lookup_grad(s):
    case = s["case"]
    v, ids = case["v"], s["ids"].long()
    ids = torch.where((ids >= 0) & (ids < v), ids, v)  # the last row is for ids that name none
    long_sums = case["n"] > 256 * v  # they lose too much in 32 bits
    if long_sums and case["n"] * (v + 1) <= 1 << 28:
        total = _sums_of_few(ids, s["dy"], v + 1)
    else:
        total = torch.zeros(v + 1, case["f"], device="cuda", dtype=torch.float64 if long_sums else torch.float32)
        total.index_add_(0, ids, s["dy"].to(total.dtype))
    s["dtable"].copy_(total[:v] * SCALE)
    return s["dtable"]


def _sums_of_few(ids, dy, v):
    """Sums by id as products with the ids' zeros and ones, 2,048 rows at a time, and their sums in 64 bits: additions one by one
    would wait for each other where many rows have the same id."""
    pad = -len(ids) % 2048
    ids = torch.cat([ids, ids.new_full((pad,), v - 1)]).view(-1, 1, 2048)
    dy = torch.cat([dy, dy.new_zeros(pad, dy.shape[1])]).view(-1, 2048, dy.shape[1]).float()
    chosen = (ids == torch.arange(v, device="cuda")[:, None]).float()
    return torch.bmm(chosen, dy).double().sum(0)


def _quantised(x):
    """Rows in 8 bits: e4m3 codes, and for every block of columns the least exponent that takes its values below the type's
    largest number."""
    n, f = x.shape
    b = x.float()
    if f % BLOCK:
        b = torch.cat([b, b.new_zeros(n, -f % BLOCK)], 1)
    b = b.view(n, -1, BLOCK)
    m, e = torch.frexp(b.abs().amax(2))  # amax = m 2^e with 0.5 <= m < 1, and 448 = 0.875 2^9
    e = torch.where(m > 0, torch.where(m > 0.875, e - 8, e - 9).clamp(min=-127), -127)
    codes = (b * torch.exp2(-e.float())[:, :, None]).to(torch.float8_e4m3fn)
    return codes.view(n, -1)[:, :f], (e + 127).to(torch.uint8)


def _plain_store(s):
    case, ids = s["case"], s["ids"].long()
    v, n = case["v"], case["n"]
    codes, exponents = _quantised(s["x"])
    there = (ids >= 0) & (ids < v)
    at = torch.arange(n, device="cuda")
    last = torch.full((v + 1,), -1, device="cuda").scatter_reduce_(0, torch.where(there, ids, v), at, "amax")
    keep = there & (last[ids.clamp(0, v - 1)] == at)  # an id that comes again: the last row stays
    to_codes, to_exponents = _stored(s)
    to_codes.view(torch.uint8)[ids[keep]] = codes[keep].view(torch.uint8)
    to_exponents[ids[keep]] = exponents[keep]
    return [to_codes, to_exponents]


def _plain_load(s):
    case, ids = s["case"], s["ids"].long()
    v, f = case["v"], case["f"]
    codes, exponents = _stored(s)
    there = (ids >= 0) & (ids < v)
    at = ids.clamp(0, v - 1)
    size = torch.exp2(exponents[at].float() - 127).repeat_interleave(BLOCK, 1)[:, :f]
    s["y"].copy_(codes.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * size * there[:, None])
    return s["y"]


def _newton_schulz(u):
    a, b, c = COEFFICIENTS
    x = u.t() if u.shape[0] > u.shape[1] else u
    x = x / (x.square().sum().sqrt() + EPS)
    for _ in range(STEPS):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _plain_orthogonal(s):
    for t in s["tensors"]:
        t["o"].copy_(_newton_schulz(t["g"].float()))
    return [t["o"] for t in s["tensors"]]


def _plain_muon(s):
    lr, mu = HYPER["lr"], HYPER["momentum"]
    for t in s["tensors"]:
        g = t["g"].float()
        t["m"].mul_(mu).add_(g)
        o = _newton_schulz(g + mu * t["m"])
        t["p"].copy_(t["p"].float() * (1 - lr * DECAY) - lr * t["scale"] * o)
    return [[t["p"], t["m"]] for t in s["tensors"]]


# ---------------------------------------------------------------- work

def _distinct(n, v, spread):
    """How many rows n ids name at all, on average."""
    if spread == "each":
        return n
    if spread == "uniform":
        return int(v * (1 - math.exp(-n / v)))
    total, edges = 0.0, [v ** (k / 200) - 1 for k in range(201)] + [v]
    for a, b in zip(edges, edges[1:]):  # ids below x are a share (x / v)^(1 / 2.5) of all
        p = ((b / v) ** 0.4 - (a / v) ** 0.4) / (b - a)
        total += (b - a) * (1 - math.exp(-n * p))
    return max(1, int(total))


def work(case):
    kind = case["kind"]
    if kind in ("orthogonal", "muon"):
        size = DTYPES[case["dtype"]].itemsize
        flops = nbytes = 0
        for rows, cols in _matrices(case):
            m, n = min(rows, cols), max(rows, cols)
            flops += STEPS * (m * m * n + m * m * m + 2 * m * m * n)  # half of what is symmetric
            nbytes += rows * cols * (2 * size if kind == "orthogonal" else 3 * size + 8)
        return dict(bytes=nbytes, flops=flops)
    v, n, f, size = case["v"], case["n"], case["f"], DTYPES[case["dtype"]].itemsize
    named = int(n * (1 - case["padded"]))
    touched = _distinct(named, v, case["ids"])
    stored = f + -(-f // BLOCK)
    if kind == "lookup":
        return dict(bytes=4 * n + touched * f * DTYPES[case["table"]].itemsize + n * f * size, flops=n * f)
    if kind == "lookup_grad":
        return dict(bytes=4 * n + named * f * size + v * f * DTYPES[case["table"]].itemsize, flops=n * f)
    if kind == "store":
        return dict(bytes=4 * n + touched * (f * size + stored), flops=2 * n * f)
    return dict(bytes=4 * n + touched * stored + n * f * size, flops=n * f)


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """Each operator from its definition, in 64 bits."""
    s = prepare(case, seed)
    return {"lookup": _exact_lookup, "lookup_grad": _exact_lookup_grad, "store": _exact_store, "load": _exact_load,
            "orthogonal": _exact_orthogonal, "muon": _exact_muon}[case["kind"]](s)


def _named(s):
    """Positions whose id names a row, and those ids."""
    at = torch.nonzero((s["ids"] >= 0) & (s["ids"] < s["case"]["v"])).squeeze(1)
    return at, s["ids"][at].long()


def _exact_lookup(s):
    at, ids = _named(s)
    y = torch.zeros(s["y"].shape, device="cuda", dtype=torch.float64)
    y[at] = s["table"][ids].double() * SCALE
    return y


def _exact_lookup_grad(s):
    at, ids = _named(s)
    case = s["case"]
    total = torch.zeros(case["v"], case["f"], device="cuda", dtype=torch.float64)
    for part in torch.arange(len(at), device="cuda").split(max(1, (1 << 27) // case["f"])):
        total.index_add_(0, ids[part], s["dy"][at[part]].double() * SCALE)
    return total


def _exact_code(x):
    """A number of at most TOP to the nearest of the 8-bit type, ties to the even one: three bits behind the leading one, steps of
    2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_store(s):
    case = s["case"]
    v, f = case["v"], case["f"]
    at, ids = _named(s)
    order = torch.argsort(ids, stable=True)  # of equal ids the last position comes last
    ids, at = ids[order], at[order]
    final = torch.ones(len(ids), device="cuda", dtype=torch.bool)
    final[:-1] = ids[1:] != ids[:-1]
    ids, at = ids[final], at[final]
    codes = torch.zeros(v, f, device="cuda", dtype=torch.float64)
    exponents = torch.zeros(v, -(-f // BLOCK), device="cuda", dtype=torch.int64)
    for j in range(0, f, BLOCK):
        x = s["x"][at, j:j + BLOCK].double()
        top = x.abs().amax(1)
        e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / TOP)), -127.0).clamp(min=-127)
        exponents[ids, j // BLOCK] = (e + 127).long()
        codes[ids, j:j + BLOCK] = _exact_code(x * torch.exp2(-e)[:, None])
    return [codes, exponents]


def _exact_load(s):
    case = s["case"]
    at, ids = _named(s)
    codes, exponents = _stored(s)
    y = torch.zeros(case["n"], case["f"], device="cuda", dtype=torch.float64)
    for j in range(case["f"]):
        y[at, j] = torch.ldexp(codes[:, j][ids].double(), exponents[:, j // BLOCK][ids].int() - 127)
    return y


def _exact_orthogonalized(u):
    """The same polynomial of the singular values, by products of the smaller side first."""
    a, b, c = COEFFICIENTS
    tall = u.shape[0] > u.shape[1]
    x = u / (torch.linalg.vector_norm(u) + EPS)
    for _ in range(STEPS):
        g = x.t() @ x if tall else x @ x.t()
        q = b * g + c * torch.linalg.matrix_power(g, 2)
        q.diagonal().add_(a)
        x = x @ q if tall else q @ x
    return x


def _exact_orthogonal(s):
    return [_exact_orthogonalized(t["g"].double()) for t in s["tensors"]]


def _exact_muon(s):
    lr, mu = HYPER["lr"], HYPER["momentum"]
    out = []
    for t in s["tensors"]:
        g, p = t["g"].double(), t["p"].double()
        m = mu * t["m"].double() + g
        out.append([p - lr * DECAY * p - lr * t["scale"] * _exact_orthogonalized(mu * m + g), m])
    return out
