"""Operators of a graph transformer with learned vertex features, as cases that can be timed and compared.

Three operators, each with its gradient: the embedding lookup that gives vertices (or tokens) their features, dot-product attention
over the entries of a CSR (scores capped by a tanh, a bias by the distance of an edge's ends, the graph as the mask) and
group norm with an activation over the graphs of a batch.  ``run`` computes them in plain torch operations in 32 bits where ``own`` is
false, and by the package's entry points where it is true; ``exact`` evaluates the definitions in 64 bits.

A case's fields.  All: ``op`` ("lookup", "lookup_grad", "attend", "attend_train", "norm", "norm_train"), ``dtype`` of the features
and of what comes out ("f32" or "bf16").  Lookups: ``n`` ids, ``vocab`` rows of the table, ``f`` columns, ``ids`` id type, ``skew`` how
unevenly rows are drawn (0: evenly), ``scale``.  Attention: ``graph`` ("power": ``n`` vertices, ``e`` edges with power-law in-degrees; "batch":
``n`` vertices in graphs of up to ``e`` vertices, every pair of a graph an edge), ``heads``, ``dim``, ``softcap`` (0: none), ``buckets``
of the distance bias (0: none).  Norm: ``n`` rows of ``f`` columns, ``ld`` row pitch, ``graphs`` in the batch, ``groups``, ``act``.
"""
import math

import torch

own = False

FIELDS = {"op": "lookup", "dtype": "f32", "n": 0, "vocab": 0, "f": 0, "ids": "i32", "skew": 0.0, "scale": 1.0, "graph": "power", "e": 0,
          "heads": 0, "dim": 0, "softcap": 0.0, "buckets": 0, "ld": 0, "graphs": 1, "groups": 1, "act": "none"}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
EPS = 1e-5
LONGEST = 20_000                                    # in-degree of a vertex, at most
MOST_LOOKED_UP = 2_000_000 * 128                    # ids x columns, edges x columns and rows x columns of the largest listed cases
MOST_ATTENDED = 39_561_252 * 64
MOST_NORMED = 232_965 * 602


def _case(name=None, **fields):
    c = dict(FIELDS, **fields)
    c["f"] = c["f"] or c["heads"] * c["dim"]
    c["ld"] = c["ld"] or c["f"]
    return dict(c, name=name) if name else c


def listed():
    return [
        # the features of the few hundred vertices of one request, out of a citation-sized table: what counts is the latency of the call
        _case("lookup_512_f32", n=512, vocab=19_717, f=32, scale=32 ** 0.5),
        # learned features of a training batch on a large skewed graph: 64-bit ids, few rows drawn often
        _case("lookup_1m_f128_bf16", n=1_000_003, vocab=1 << 21, f=128, dtype="bf16", ids="i64", skew=3.0, scale=128 ** 0.5),
        # the gradient of a small batch: nearly all of the table's rows stay zero; odd number of columns
        _case("lookup_grad_4k_f41", op="lookup_grad", n=4_096, vocab=19_717, f=41, skew=1.0, scale=0.5),
        # the gradient of a large batch, some rows drawn a hundred thousand times
        _case("lookup_grad_2m_f128", op="lookup_grad", n=2_000_000, vocab=232_965, f=128, skew=3.0, scale=128 ** 0.5),
        # one attention layer on a few thousand vertices: latency
        _case("attend_4k_4x8", op="attend", n=4_096, e=40_000, heads=4, dim=8),
        # a hidden attention layer of 64 bf16 columns on a large graph with hub vertices, scores capped
        _case("attend_133k_8x8_bf16", op="attend", n=132_534, e=39_561_252, heads=8, dim=8, dtype="bf16", softcap=30.0),
        # a batch of small graphs, each attended as a whole (the mask keeps graphs apart), with a bias by distance: a training pass
        _case("attend_train_batch_8x16_bf16", op="attend_train", graph="batch", n=50_000, e=48, heads=8, dim=16, dtype="bf16", buckets=16),
        # a training pass of a sparse graph of ordinary size, capped scores and a bias by distance
        _case("attend_train_100k_8x16", op="attend_train", n=100_000, e=2_000_000, heads=8, dim=16, softcap=20.0, buckets=8),
        # the norm between two layers of a citation-sized graph: latency
        _case("norm_20k_f32", op="norm", n=19_717, f=32, groups=4, act="relu"),
        # a batch of many small graphs
        _case("norm_batch_f128_bf16", op="norm", n=500_000, f=128, graphs=20_000, groups=8, act="silu", dtype="bf16"),
        # the input features of one large graph, rows padded to 608
        _case("norm_233k_f602", op="norm", n=232_965, f=602, ld=608, groups=7, act="gelu"),
        # a training pass over a batch of graphs of very different sizes
        _case("norm_train_133k_f256_bf16", op="norm_train", n=132_534, f=256, graphs=64, groups=32, act="silu", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "lookup_grad", "attend", "attend_train", "attend_train", "norm", "norm", "norm_train"])
    dtype = rng.choice(["f32", "f32", "bf16"])
    if op.startswith("lookup"):
        f = rng.choice([8, 16, 32, 64, 128, 256, _log(rng, 3, 602), _log(rng, 3, 602)])
        n = min(_log(rng, 300, 3_000_000), MOST_LOOKED_UP // f)
        return _case(op=op, dtype=dtype, n=n, vocab=min(_log(rng, 2_000, 2_000_000), MOST_LOOKED_UP // f), f=f, ids=rng.choice(["i32", "i64"]),
                     skew=rng.choice([0.0, 1.0, 3.0]), scale=rng.choice([1.0, round(f ** 0.5, 3)]))
    if op.startswith("attend"):
        heads, dim = rng.choice([1, 2, 4, 6, 8]), rng.choice([4, 7, 8, 16, 32, 64])
        most = MOST_ATTENDED // (16 if op == "attend_train" else 1) // (heads * dim)
        n = _log(rng, 4_000, 200_000)
        c = dict(op=op, dtype=dtype, n=n, heads=heads, dim=dim, softcap=rng.choice([0.0, 20.0, 50.0]), buckets=rng.choice([0, 5, 16, 64]))
        if rng.random() < 0.3:
            return _case(graph="batch", **dict(c, n=min(n, most // 32)), e=_log(rng, 4, 64))
        return _case(e=min(int(n * math.exp(rng.uniform(math.log(4), math.log(300)))), most), **c)
    groups = rng.choice([1, 2, 4, 8, 14, 32])
    f = groups * max(1, _log(rng, 16, 602) // groups)
    n = min(_log(rng, 4_000, 500_000), MOST_NORMED // f // (2 if op == "norm_train" else 1))
    align = 4 if dtype == "f32" else 8
    return _case(op=op, dtype=dtype, n=n, f=f, ld=f if rng.random() < 0.6 else -(-f // align) * align, graphs=rng.choice([1, 1, _log(rng, 2, n // 20)]),
                 groups=rng.choice([groups, groups, f]),
                 # (the slope of relu jumps at 0, where 32 and 64 bits need not agree about the side)
                 act=rng.choice(["none", "elu", "silu", "gelu", "elu" if op == "norm_train" else "relu"]))


# ---------------------------------------------------------------- inputs

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(seed * 64 + stream)


def _matrix(rows, cols, ld, dtype, seed, stream, scale=1.0, mean=0.0):
    """Normal values in the first `cols` of `ld` columns; the padding is left as zeros."""
    t = torch.zeros((rows, ld), dtype=torch.float32, device="cuda")
    t[:, :cols] = torch.randn((rows, cols), generator=_gen(seed, stream), device="cuda") * scale + mean
    return t.to(TYPES[dtype])[:, :cols]


def _ids(c, seed):
    """Row numbers vocab * u^(1 + skew), relabelled: evenly drawn, or a few rows most of the time."""
    rnd = _gen(seed, 1)
    u = torch.rand(c["n"], generator=rnd, device="cuda", dtype=torch.float64) ** (1 + c["skew"])
    label = torch.randperm(c["vocab"], generator=rnd, device="cuda")
    return label[(u * c["vocab"]).long().clamp_(max=c["vocab"] - 1)].to(TYPES[c["ids"]])


def _edges(c, seed):
    """(sources, destinations, distance bucket) of the edges, in no order."""
    rnd = _gen(seed, 1)
    n, buckets = c["n"], max(1, c["buckets"])
    if c["graph"] == "batch":
        size = torch.randint(1, c["e"] + 1, (n,), generator=rnd, device="cuda")
        first = torch.cat([size.new_zeros(1), size.cumsum(0)])
        first = torch.cat([first[first < n], first.new_full((1,), n)])
        size = first[1:] - first[:-1]
        own_size, own_first = torch.repeat_interleave(size, size), torch.repeat_interleave(first[:-1], size)
        dst = torch.repeat_interleave(torch.arange(n, device="cuda"), own_size)
        at = torch.arange(dst.numel(), device="cuda") - torch.repeat_interleave(own_size.cumsum(0) - own_size, own_size)
        src = own_first[dst] + at
        return src.int(), dst.int(), (src - dst).abs().clamp_(max=buckets - 1).int()      # the vertices of a chain
    u = torch.rand(n, generator=rnd, device="cuda", dtype=torch.float64).clamp_min(1e-12).pow_(-1 / 1.1)
    top = float(min(LONGEST, n - 1))
    lo, hi = 1e-3, top
    for _ in range(50):
        x0 = (lo + hi) / 2
        lo, hi = (x0, hi) if float((u * x0).clamp_(0, top).floor_().sum()) < c["e"] else (lo, x0)
    dst = torch.repeat_interleave(torch.arange(n, device="cuda"), (u * hi).clamp_(0, top).long())
    dst = dst[torch.randperm(dst.numel(), generator=rnd, device="cuda")]
    dst = torch.cat([dst, torch.randint(n, (max(0, c["e"] - dst.numel()),), generator=rnd, device="cuda")])[:c["e"]]
    src = dst[torch.randint(dst.numel(), (dst.numel(),), generator=rnd, device="cuda")]
    dist = torch.randint(buckets, (dst.numel(),), generator=rnd, device="cuda")
    return src.int(), dst.int(), dist.int()


def _graph_ptr(c, seed):
    """Row offsets of the graphs: cut points drawn at random, so that some graphs are many times longer than others and some empty."""
    cuts = torch.randint(c["n"] + 1, (c["graphs"] - 1,), generator=_gen(seed, 1), device="cuda").sort().values
    return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), c["n"])]).int()


def _inputs(c, seed):
    s = {}
    if c["op"].startswith("lookup"):
        s["id"] = _ids(c, seed)
        if c["op"] == "lookup":
            s["table"] = _matrix(c["vocab"], c["f"], c["f"], c["dtype"], seed, 2, c["f"] ** -0.5)
        else:
            s["dout"] = _matrix(c["n"], c["f"], c["f"], c["dtype"], seed, 2)
    elif c["op"].startswith("attend"):
        s["src"], s["dst"], s["dist"] = _edges(c, seed)
        s["q"], s["k"], s["v"] = (_matrix(c["n"], c["f"], c["f"], c["dtype"], seed, i) for i in (2, 3, 4))
        s["bias"] = _matrix(c["buckets"], c["heads"], c["heads"], "f32", seed, 5) if c["buckets"] else None
        if c["op"] == "attend_train":
            s["dout"] = _matrix(c["n"], c["f"], c["f"], c["dtype"], seed, 6)
    else:
        s["x"] = _matrix(c["n"], c["f"], c["ld"], c["dtype"], seed, 2, 2.0, 1.0)
        s["weight"], s["shift"] = (_matrix(1, c["f"], c["f"], "f32", seed, i, 0.2, m)[0] for i, m in ((3, 1.0), (4, 0.0)))
        s["ptr"] = _graph_ptr(c, seed)
        if c["op"] == "norm_train":
            s["dout"] = _matrix(c["n"], c["f"], c["ld"], c["dtype"], seed, 6)
    return s


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    if case["op"].startswith("attend"):
        if own:
            import paper_2104_03058_b200 as g
            # a program keeps the handle of a graph it goes on using; for training that of the reversed edges too
            s["csr"] = g.build_csr(case["n"], s["src"], s["dst"])
            s["slot_dist"] = g.edge_values(s["csr"], s["dist"]) if case["buckets"] else None
            if case["op"] == "attend_train":
                s["csr_t"] = g.build_csr(case["n"], s["dst"], s["src"])
                s["slot_dist_t"] = g.edge_values(s["csr_t"], s["dist"]) if case["buckets"] else None
        else:
            s["src"], s["dst"], s["dist"] = s["src"].long(), s["dst"].long(), s["dist"].long()
    elif case["op"].startswith("norm") and not own:
        s["graph"] = torch.repeat_interleave(torch.arange(case["graphs"], device="cuda"), (s["ptr"][1:] - s["ptr"][:-1]).long())
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2104_03058_b200 as g
    out = TYPES[s["dtype"]]
    if s["op"] == "lookup":
        return g.embedding(s["table"], s["id"], scale=s["scale"], out_dtype=out)
    if s["op"] == "lookup_grad":
        return g.embedding_backward(s["id"], s["dout"], s["vocab"], scale=s["scale"])
    if s["op"] == "attend":
        return g.aggregate_attention(s["csr"], s["q"], s["k"], s["v"], s["heads"], s["dim"], softcap=s["softcap"], dist=s["slot_dist"],
                                     bias=s["bias"], out_dtype=out)
    if s["op"] == "attend_train":
        y, lse = g.aggregate_attention(s["csr"], s["q"], s["k"], s["v"], s["heads"], s["dim"], softcap=s["softcap"], dist=s["slot_dist"],
                                       bias=s["bias"], out_dtype=out, with_lse=True)
        grads = g.aggregate_attention_backward(s["csr"], s["csr_t"], s["q"], s["k"], s["v"], s["dout"], lse, s["heads"], s["dim"],
                                               softcap=s["softcap"], dist=s["slot_dist"], dist_t=s["slot_dist_t"], bias=s["bias"],
                                               out_dtype=out)
        return (y, *(d for d in grads if d is not None))
    if s["op"] == "norm":
        return g.group_norm(s["x"], s["groups"], s["weight"], s["shift"], s["ptr"], EPS, s["act"], out_dtype=out)
    y, mean, rstd = g.group_norm(s["x"], s["groups"], s["weight"], s["shift"], s["ptr"], EPS, s["act"], out_dtype=out, with_stats=True)
    return (y, *g.group_norm_backward(s["dout"], s["x"], s["groups"], mean, rstd, s["weight"], s["shift"], s["ptr"], s["act"], out_dtype=out))


def _plain(s):
    if s["op"] == "lookup":
        return (s["table"][s["id"]].float() * s["scale"]).to(TYPES[s["dtype"]])
    if s["op"] == "lookup_grad":
        grad = torch.zeros((s["vocab"], s["f"]), device="cuda")
        return grad.index_add_(0, s["id"], s["dout"].float()).mul_(s["scale"])
    return _plain_attend(s) if s["op"].startswith("attend") else _plain_norm(s)


def _plain_attend(s):
    """Edge by edge: scores, softmax over the edges that end in a vertex, weighted sum; then the gradients."""
    n, src, dst, shape, out = s["n"], s["src"], s["dst"], (-1, s["heads"], s["dim"]), TYPES[s["dtype"]]
    scale = s["dim"] ** -0.5
    q, k, v = (s[name].float().reshape(shape) for name in "qkv")
    score = (q[dst] * k[src]).sum(2) * scale
    slope = None
    if s["softcap"]:
        tanh = torch.tanh(score / s["softcap"])
        score, slope = tanh * s["softcap"], 1 - tanh * tanh
    if s["buckets"]:
        score = score + s["bias"][s["dist"]]
    index = dst[:, None].expand_as(score)
    top = torch.full((n, s["heads"]), -math.inf, device="cuda").scatter_reduce_(0, index, score, "amax")
    p = torch.exp(score - top[dst])
    p = p / torch.zeros((n, s["heads"]), device="cuda").index_add_(0, dst, p)[dst]
    y = torch.zeros(q.shape, device="cuda").index_add_(0, dst, p[:, :, None] * v[src]).reshape(n, -1)
    if s["op"] == "attend":
        return y.to(out)
    dout = s["dout"].float().reshape(shape)
    dv = torch.zeros(q.shape, device="cuda").index_add_(0, src, p[:, :, None] * dout[dst])
    dp = (dout[dst] * v[src]).sum(2)
    ds = p * (dp - torch.zeros((n, s["heads"]), device="cuda").index_add_(0, dst, p * dp)[dst])
    dbias = []
    if s["buckets"]:                                   # a few sums of millions of terms of either sign: 64 bits
        dbias = [torch.zeros((s["buckets"], s["heads"]), dtype=torch.float64, device="cuda").index_add_(0, s["dist"], ds.double()).float()]
    ds = (ds if slope is None else ds * slope) * scale
    dq = torch.zeros(q.shape, device="cuda").index_add_(0, dst, ds[:, :, None] * k[src])
    dk = torch.zeros(q.shape, device="cuda").index_add_(0, src, ds[:, :, None] * q[dst])
    return (y.to(out), *(d.reshape(n, -1).to(out) for d in (dq, dk, dv)), *dbias)


def _activation(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "elu":
        return torch.where(z > 0, z, torch.expm1(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _slope(z, act):
    """Derivative of the activation."""
    if act == "relu":
        return (z > 0).float()
    if act == "elu":
        return torch.where(z > 0, 1.0, torch.exp(z))
    if act == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _graph_sums(s, values):
    """[graphs, groups, 1] sums over a graph's rows and a group's columns (64 bits: up to a hundred million terms)."""
    sums = torch.zeros((s["graphs"], s["groups"]), dtype=torch.float64, device="cuda")
    return sums.index_add_(0, s["graph"], values.sum(2).double())[:, :, None]


def _plain_norm(s):
    x, out = s["x"].float().reshape(s["n"], s["groups"], -1), TYPES[s["dtype"]]
    count = ((s["ptr"][1:] - s["ptr"][:-1]).double() * x.shape[2]).clamp_min(1)[:, None, None]
    mean = (_graph_sums(s, x) / count).float()
    centred = x - mean[s["graph"]]
    rstd = torch.rsqrt(_graph_sums(s, centred * centred) / count + EPS).float()
    xhat = centred * rstd[s["graph"]]
    weight, shift = s["weight"].reshape(s["groups"], -1), s["shift"].reshape(s["groups"], -1)
    z = xhat * weight + shift
    y = _activation(z, s["act"]).reshape(s["n"], -1).to(out)
    if s["op"] == "norm":
        return y
    dz = s["dout"].float().reshape(x.shape) * _slope(z, s["act"])
    g = dz * weight
    mean_g, mean_gx = ((_graph_sums(s, t) / count).float()[s["graph"]] for t in (g, g * xhat))
    dx = (g - mean_g - xhat * mean_gx) * rstd[s["graph"]]
    # (the sums over all rows in 64 bits)
    return y, dx.reshape(s["n"], -1).to(out), *(t.double().sum(0).reshape(-1).float() for t in (dz * xhat, dz))


# ---------------------------------------------------------------- the same results in 64 bits

def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"] == "lookup":
        return torch.index_select(s["table"].double(), 0, s["id"].long()) * c["scale"]
    if c["op"] == "lookup_grad":
        order = s["id"].long().argsort(stable=True)
        row_ptr = torch.searchsorted(s["id"].long()[order], torch.arange(c["vocab"] + 1, device="cuda"))
        take = torch.sparse_csr_tensor(row_ptr, order, torch.full((c["n"],), c["scale"], dtype=torch.float64, device="cuda"),
                                       size=(c["vocab"], c["n"]))
        return torch.cat([take @ part.double().contiguous() for part in s["dout"].split(64, dim=1)], dim=1)
    return _exact_attend(c, s) if c["op"].startswith("attend") else _exact_norm(c, s)


def _exact_attend(c, s):
    """One head after the other, the gradients by differentiation."""
    src, dst, dist = s["src"].long(), s["dst"].long(), s["dist"].long()
    parts = []
    for h in range(c["heads"]):
        cols = slice(h * c["dim"], (h + 1) * c["dim"])
        leaves = [s[name][:, cols].double() for name in "qkv"]
        if c["buckets"]:
            leaves.append(s["bias"][:, h].double())
        with torch.set_grad_enabled(c["op"] == "attend_train"):
            for t in leaves:
                t.requires_grad_(c["op"] == "attend_train")
            q, k, v = leaves[:3]
            score = torch.einsum("ed,ed->e", q[dst], k[src]) / c["dim"] ** 0.5
            if c["softcap"]:
                score = c["softcap"] * torch.tanh(score / c["softcap"])
            if c["buckets"]:
                score = score + leaves[3][dist]
            weight = torch.exp(score - score.detach().max())              # scores of one head are within a few tens of each other
            total = torch.zeros(c["n"], dtype=torch.float64, device="cuda").index_add(0, dst, weight)
            top = torch.zeros((c["n"], c["dim"]), dtype=torch.float64, device="cuda").index_add(0, dst, weight[:, None] * v[src])
            y = top / torch.where(total > 0, total, 1.0)[:, None]
        grads = torch.autograd.grad(y, leaves, s["dout"][:, cols].double()) if c["op"] == "attend_train" else []
        parts.append([t.detach() for t in (y, *grads)])
    joined = [torch.cat(list(t), dim=1) if t[0].dim() == 2 else torch.stack(list(t), dim=1) for t in zip(*parts)]
    return joined[0] if c["op"] == "attend" else tuple(joined)


def _exact_norm(c, s):
    """Sums over a graph as products with the matrix that says which rows it holds; the gradients by differentiation."""
    size = (s["ptr"][1:] - s["ptr"][:-1]).long()
    graph = torch.repeat_interleave(torch.arange(c["graphs"], device="cuda"), size)
    x, weight, shift = (t.double() for t in (s["x"], s["weight"], s["shift"]))
    leaves = [x, weight, shift]
    with torch.set_grad_enabled(c["op"] == "norm_train"):
        for t in leaves:
            t.requires_grad_(c["op"] == "norm_train")
        grouped = x.reshape(c["n"], c["groups"], -1)
        zeros = torch.zeros((c["graphs"], c["groups"]), dtype=torch.float64, device="cuda")
        count = (size.double() * grouped.shape[2]).clamp_min(1)[:, None]
        mean = zeros.index_add(0, graph, grouped.sum(2)) / count
        off = grouped - mean[graph][:, :, None]
        var = zeros.index_add(0, graph, (off ** 2).sum(2)) / count
        z = (off / torch.sqrt(var + EPS)[graph][:, :, None]).reshape(c["n"], -1) * weight + shift
        if c["act"] == "silu":
            y = torch.nn.functional.silu(z)
        elif c["act"] == "gelu":
            y = torch.nn.functional.gelu(z)
        elif c["act"] == "elu":
            y = torch.nn.functional.elu(z)
        else:
            y = z.clamp_min(0) if c["act"] == "relu" else z
    if c["op"] == "norm":
        return y
    return (y.detach(), *torch.autograd.grad(y, leaves, s["dout"].double()))


# ---------------------------------------------------------------- floors

def work(case):
    c = case
    n, f, elem, idx = c["n"], c["f"], 2 if c["dtype"] == "bf16" else 4, 8 if c["ids"] == "i64" else 4
    if c["op"] == "lookup":                                       # ids, the rows drawn (each once, were all of them different), the output
        return {"bytes": n * idx + min(n, c["vocab"]) * f * elem + n * f * elem, "flops": n * f}
    if c["op"] == "lookup_grad":                                  # ids, the gradients that came in, the whole table's gradient
        return {"bytes": n * idx + n * f * elem + c["vocab"] * f * 4, "flops": n * f}
    if c["op"].startswith("attend"):
        nnz = n * (2 * c["e"] + 1) // 3 if c["graph"] == "batch" else c["e"]          # graphs of 1 .. e vertices, evenly: E[s^2] / E[s]
        graph = 4 * (n + 1) + nnz * (8 if c["buckets"] else 4)
        forward = {"bytes": graph + 4 * n * f * elem, "flops": nnz * (4 * f + 8 * c["heads"])}
        if c["op"] == "attend":
            return forward
        # q, k, v, the output's gradient in, three gradients out, and the reversed graph
        return {"bytes": forward["bytes"] + 2 * graph + 7 * n * f * elem, "flops": forward["flops"] + nnz * (10 * f + 16 * c["heads"])}
    moved = n * f * elem
    return {"bytes": 2 * moved, "flops": 10 * n * f} if c["op"] == "norm" else {"bytes": 5 * moved, "flops": 30 * n * f}
