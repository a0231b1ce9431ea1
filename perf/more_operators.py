"""The parts of a sequence-aware graph transformer beside its attention, as cases that can be timed and compared.

Three operators, each with its gradient: layer norm (every row by itself), rotary positions of queries and keys, and a gated
linear recurrence over the rows of each graph of a batch.  ``run`` computes them in plain torch operations in 32 bits where ``own`` is false, and by
the package's entry points where it is true; ``exact`` evaluates the definitions in 64 bits.

A case's fields.  All: ``op`` ("norm", "norm_train", "rotate", "rotate_train", "scan", "scan_train"), ``dtype`` of the inputs and of
what comes out ("f32" or "bf16"), ``n`` rows, ``f`` columns, ``ld`` row pitch.  Rotary: ``heads`` of ``dim`` columns, ``part`` of them rotated,
``pairs`` ("half": column i turns with i + part / 2, "interleaved": 2i with 2i + 1), ``ids`` type of the positions, ``far`` the first position
that does not occur, ``scaling`` of the frequencies beyond ``length`` positions by ``factor``, ``scale`` of the rotated columns.  Recurrence: ``graphs`` in the
batch (``graphs == n``: single tokens), ``form`` ("sigmoid": h = s h + (1 - s) x with s the gate's logistic function, "factor": h = gate h + x).
"""
import math

import torch

own = False

FIELDS = {"op": "norm", "dtype": "f32", "n": 0, "f": 0, "ld": 0, "heads": 0, "dim": 0, "part": 0, "pairs": "half", "ids": "i32", "far": 0,
          "scaling": "none", "length": 0, "factor": 1.0, "scale": 1.0, "graphs": 1, "form": "sigmoid"}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
EPS = 1e-5
BASE = 10_000.0
TURNS = (1.0, 32.0)                                  # frequencies with fewer turns than the first over `length` are scaled as a whole, with more than the second not
MOST_NORMED = 232_965 * 602                          # rows x columns of the largest listed cases
MOST_ROTATED = 500_009 * 12 * 64
MOST_SCANNED = 1_000_003 * 128


def _case(name=None, **fields):
    c = dict(FIELDS, **fields)
    c["f"] = c["f"] or c["heads"] * c["dim"]
    c["ld"] = c["ld"] or c["f"]
    c["part"] = c["part"] or c["dim"]
    return dict(c, name=name) if name else c


def listed():
    return [
        # the norm of the few hundred vertices of one request: latency
        _case("norm_512_f128", n=512, f=128),
        # the norm ahead of an attention layer on a large graph
        _case("norm_133k_f256_bf16", n=132_534, f=256, dtype="bf16"),
        # a training pass over the input features of one large graph, rows padded to 608
        _case("norm_train_233k_f602", op="norm_train", n=232_965, f=602, ld=608),
        # a training pass of a batch of small graphs, odd number of rows
        _case("norm_train_500k_f128_bf16", op="norm_train", n=500_003, f=128, dtype="bf16"),
        # the queries and keys of 64 tokens, one for each sequence that is being answered, at far positions: latency
        _case("rotate_64_16x64_bf16", op="rotate", n=64, heads=16, dim=64, dtype="bf16", ids="i64", far=1_000_000, scaling="ramp", length=4_096, factor=32.0),
        # queries and keys (the first 16 of 24 heads of a joint projection) of a large graph's vertices, half layout
        _case("rotate_133k_16x16", op="rotate", n=132_534, heads=16, dim=16, ld=384, far=4_096),
        # a training pass over long documents: half of each head is rotated, neighbouring columns, there and back
        _case("rotate_train_500k_12x64_bf16", op="rotate_train", n=500_009, heads=12, dim=64, part=32, pairs="interleaved", dtype="bf16",
              ids="i64", far=131_072, scaling="position", factor=8.0, scale=1.1),
        # one more token for each of 256 sequences
        _case("scan_step_256_f512", op="scan", n=256, f=512, graphs=256),
        # a batch of graphs of very different sizes
        _case("scan_133k_f256_bf16", op="scan", n=132_534, f=256, graphs=64, dtype="bf16"),
        # one sequence of a million rows
        _case("scan_1m_f128", op="scan", n=1_000_003, f=128, form="factor"),
        # a training pass over many short sequences
        _case("scan_train_50k_f128_bf16", op="scan_train", n=50_000, f=128, graphs=2_000, dtype="bf16"),
        # a training pass over a few long ones, odd number of columns
        _case("scan_train_233k_f301", op="scan_train", n=232_965, f=301, graphs=5, form="factor"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_train", "rotate", "rotate_train", "scan", "scan", "scan_train", "scan_train"])
    dtype = rng.choice(["f32", "bf16"])
    align = 4 if dtype == "f32" else 8
    if op.startswith("norm"):
        f = rng.choice([32, 64, 128, 256, 512, 1024, _log(rng, 16, 4_096), _log(rng, 16, 4_096)])
        n = _log(rng, 500, min(500_000, MOST_NORMED // f // (1 if op == "norm_train" else 2)))
        return _case(op=op, dtype=dtype, n=n, f=f, ld=f if rng.random() < 0.6 else -(-f // align) * align)
    if op.startswith("rotate"):
        heads, dim = rng.choice([1, 2, 4, 8, 12, 16, 24, 32]), rng.choice([8, 16, 32, 48, 64, 80, 96, 128])
        scaling = rng.choice(["none", "none", "position", "base", "ramp"])
        return _case(op=op, dtype=dtype, n=_log(rng, 16, min(1_000_000, MOST_ROTATED // (heads * dim))), heads=heads, dim=dim,
                     part=rng.choice([dim, dim, dim // 2]), pairs=rng.choice(["half", "interleaved"]), ld=heads * dim * rng.choice([1, 1, 3]),
                     ids=rng.choice(["i32", "i64"]), far=_log(rng, 512, 1_000_000), scaling=scaling, length=4_096,
                     factor=1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]), scale=rng.choice([1.0, 1.1]))
    f = rng.choice([16, 32, 64, 128, 256, 512, _log(rng, 8, 602), _log(rng, 8, 602)])
    n = _log(rng, 500, min(1_000_000, MOST_SCANNED // f // (2 if op == "scan_train" else 1)))
    graphs = rng.choice([1, 1, _log(rng, 2, n // 20), _log(rng, 2, n // 20), n if n < 10_000 else 16])
    return _case(op=op, dtype=dtype, n=n, f=f, ld=f if rng.random() < 0.6 else -(-f // align) * align, graphs=graphs,
                 form=rng.choice(["sigmoid", "factor"]))


# ---------------------------------------------------------------- inputs

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(seed * 64 + stream)


def _matrix(rows, cols, ld, dtype, seed, stream, scale=1.0, mean=0.0):
    """Normal values in the first `cols` of `ld` columns; the padding is left as zeros."""
    t = torch.zeros((rows, ld), dtype=torch.float32, device="cuda")
    t[:, :cols] = torch.randn((rows, cols), generator=_gen(seed, stream), device="cuda") * scale + mean
    return t.to(TYPES[dtype])[:, :cols]


def _graph_ptr(c, seed):
    """Row offsets of the graphs: cut points drawn at random, so that some graphs are many times longer than others and some empty."""
    cuts = torch.randint(c["n"] + 1, (c["graphs"] - 1,), generator=_gen(seed, 1), device="cuda").sort().values
    return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), c["n"])]).int()


def _inputs(c, seed):
    n, f, ld, dtype = c["n"], c["f"], c["ld"], c["dtype"]
    s = {}
    if c["op"].startswith("norm"):
        s["x"] = _matrix(n, f, ld, dtype, seed, 2, 2.0, 0.5)
        s["weight"], s["shift"] = (_matrix(1, f, f, "f32", seed, i, 0.2, m)[0] for i, m in ((3, 1.0), (4, 0.0)))
    elif c["op"].startswith("rotate"):
        s["x"] = _matrix(n, f, ld, dtype, seed, 2)
        s["positions"] = torch.randint(c["far"], (n,), generator=_gen(seed, 1), device="cuda").to(TYPES[c["ids"]])
    else:
        s["x"] = _matrix(n, f, ld, dtype, seed, 2)
        # a state's weight of a fifth to a few thousand rows; as factors in the inputs' own type, some of them 1
        s["gate"] = _matrix(n, f, ld, "f32", seed, 3, 2.0, 2.0)
        if c["form"] == "factor":
            s["gate"] = torch.sigmoid(s["gate"])
        s["gate"] = torch.cat([s["gate"], s["gate"].new_zeros((n, ld - f))], dim=1).to(TYPES[dtype])[:, :f]
        s["ptr"] = None if c["graphs"] == n else _graph_ptr(c, seed)
        s["initial"] = _matrix(c["graphs"], f, f, "f32", seed, 4)
        if c["op"] == "scan_train":
            s["dfinal"] = _matrix(c["graphs"], f, f, "f32", seed, 5)
    if c["op"].endswith("_train"):
        s["dout"] = _matrix(n, f, ld, dtype, seed, 6)
    return s


def _frequencies(c):
    """Radians per position of each pair, in 64 bits."""
    r = c["part"]
    base = BASE * c["factor"] ** (r / (r - 2)) if c["scaling"] == "base" else BASE
    freq = base ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    if c["scaling"] == "position":
        freq = freq / c["factor"]
    if c["scaling"] == "ramp":
        kept = ((freq * c["length"] / (2 * math.pi) - TURNS[0]) / (TURNS[1] - TURNS[0])).clamp(0, 1)
        freq = freq * (kept + (1 - kept) / c["factor"])
    return freq


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    if case["op"].startswith("rotate"):
        if own:
            import paper_2104_03058_b200 as g
            # a program makes the frequencies once
            s["freq"] = g.rotary_frequencies(case["part"], BASE, case["scaling"], case["factor"], case["length"], TURNS, device="cuda")
        else:
            s["freq"] = _frequencies(case)
    elif case["op"].startswith("scan") and not own:
        ptr = torch.arange(case["n"] + 1, device="cuda") if s["ptr"] is None else s["ptr"].long()
        s["length_of"] = ptr[1:] - ptr[:-1]
        s["first"], s["last"] = ptr[:-1], ptr[1:] - 1
        s["graph"] = torch.repeat_interleave(torch.arange(case["graphs"], device="cuda"), s["length_of"])
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2104_03058_b200 as g
    out = TYPES[s["dtype"]]
    if s["op"] == "norm":
        return g.layer_norm(s["x"], s["weight"], s["shift"], EPS, out_dtype=out)
    if s["op"] == "norm_train":
        y, mean, rstd = g.layer_norm(s["x"], s["weight"], s["shift"], EPS, out_dtype=out, with_stats=True)
        return (y, *g.layer_norm_backward(s["dout"], s["x"], mean, rstd, s["weight"], out_dtype=out))
    if s["op"].startswith("rotate"):
        turn = dict(positions=s["positions"], interleaved=s["pairs"] == "interleaved", scale=s["scale"], out_dtype=out)
        y = g.rotary(s["x"], s["freq"], s["heads"], s["dim"], **turn)
        return y if s["op"] == "rotate" else (y, g.rotary(s["dout"], s["freq"], s["heads"], s["dim"], inverse=True, **turn))
    batch = dict(graph_ptr=s["ptr"], graphs=s["graphs"], initial=s["initial"])
    if s["op"] == "scan":
        return g.linear_recurrence(s["x"], s["gate"], s["form"], out_dtype=out, with_final=True, **batch)
    y, final, states = g.linear_recurrence(s["x"], s["gate"], s["form"], out_dtype=out, with_final=True, with_states=True, **batch)
    return (y, final, *g.linear_recurrence_backward(s["dout"], s["x"], s["gate"], states, s["form"], dfinal=s["dfinal"], out_dtype=out, **batch))


def _plain(s):
    if s["op"].startswith("norm"):
        return _plain_norm(s)
    return _plain_rotate(s) if s["op"].startswith("rotate") else _plain_scan(s)


def _plain_norm(s):
    x, out = s["x"].float(), TYPES[s["dtype"]]
    centred = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xhat = centred * rstd
    y = (xhat * s["weight"] + s["shift"]).to(out)
    if s["op"] == "norm":
        return y
    dout = s["dout"].float()
    g = dout * s["weight"]
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
    # (the sums over all rows in 64 bits)
    return y, dx.to(out), (dout * xhat).double().sum(0).float(), dout.double().sum(0).float()


def _plain_rotate(s):
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = ((t * s["scale"]).float()[:, None, :] for t in (torch.cos(angle), torch.sin(angle)))
    there = _plain_turn(s, s["x"], cos, sin)
    return there if s["op"] == "rotate" else (there, _plain_turn(s, s["dout"], cos, -sin))


def _plain_turn(s, x, cos, sin):
    r, shape = s["part"], (s["n"], s["heads"], s["dim"])
    x = x.float().reshape(shape)
    y = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if s["pairs"] == "interleaved" else (slice(0, r // 2), slice(r // 2, r))
    y[:, :, a] = x[:, :, a] * cos - x[:, :, b] * sin
    y[:, :, b] = x[:, :, a] * sin + x[:, :, b] * cos
    return y.reshape(s["n"], -1).to(TYPES[s["dtype"]])


def _doubled(a, b):
    """h[t] = a[t] h[t - 1] + b[t] along the rows (h[-1] = 0): after k steps a and b say how a row depends on the one 2^k rows ahead of it."""
    a, h, d = a.clone(), b.clone(), 1
    while d < a.shape[0]:
        h[d:] += a[d:] * h[:-d]
        a[d:] *= a[:-d].clone()
        d *= 2
    return h


def _plain_scan(s):
    n, out = s["n"], TYPES[s["dtype"]]
    x, gate = s["x"].float(), s["gate"].float()
    some = (s["length_of"] > 0)[:, None]
    if s["form"] == "factor":
        a, rest = gate, None
    else:
        a, rest = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    b = x if rest is None else rest * x
    starts = torch.zeros((n, 1), dtype=torch.bool, device="cuda")
    starts[s["first"][some[:, 0]]] = True
    entering = torch.where(starts, s["initial"][s["graph"]], 0.0)
    h = _doubled(torch.where(starts, 0.0, a), torch.where(starts, b + a * entering, b))
    final = torch.where(some, h[s["last"].clamp_min(0)], s["initial"])
    if s["op"] == "scan":
        return h.to(out), final
    ends = torch.zeros((n, 1), dtype=torch.bool, device="cuda")
    ends[s["last"][some[:, 0]]] = True
    arriving = s["dout"].float() + torch.where(ends, s["dfinal"][s["graph"]], 0.0)
    onward = torch.where(ends, 0.0, torch.cat([a[1:], torch.zeros_like(a[:1])]))
    g = _doubled(onward.flip(0), arriving.flip(0)).flip(0)
    before = torch.where(starts, entering, torch.cat([torch.zeros_like(h[:1]), h[:-1]]))
    dx, dgate = (g, g * before) if rest is None else (rest * g, g * (before - x) * a * rest)
    dinitial = torch.where(some, (a * g)[s["first"].clamp_max(n - 1)], s["dfinal"])
    return h.to(out), final, dx.to(out), dgate.to(out), dinitial


# ---------------------------------------------------------------- the same results in 64 bits

def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"].startswith("norm"):
        return _exact_norm(c, s)
    return _exact_rotate(c, s) if c["op"].startswith("rotate") else _exact_scan(c, s)


def _exact_norm(c, s):
    leaves = [s[name].double() for name in ("x", "weight", "shift")]
    with torch.set_grad_enabled(c["op"] == "norm_train"):
        for t in leaves:
            t.requires_grad_(c["op"] == "norm_train")
        y = torch.nn.functional.layer_norm(leaves[0], (c["f"],), leaves[1], leaves[2], EPS)
    return y if c["op"] == "norm" else (y.detach(), *torch.autograd.grad(y, leaves, s["dout"].double()))


def _exact_rotate(c, s):
    """As products of complex numbers, a stretch of rows after the other."""
    n, r = c["n"], c["part"]
    turn = torch.polar(torch.full((1,), c["scale"], dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * _frequencies(c))[:, None, :]

    def turned(x, turn):
        done = []
        for rows, by in zip(x.split(1 << 16), turn.split(1 << 16)):
            heads = rows.double().unflatten(1, (c["heads"], c["dim"]))
            pairs, rest = heads[:, :, :r], heads[:, :, r:]
            pairs = pairs.unflatten(2, (r // 2, 2)) if c["pairs"] == "interleaved" else pairs.unflatten(2, (2, r // 2)).transpose(2, 3)
            pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
            pairs = pairs if c["pairs"] == "interleaved" else pairs.transpose(2, 3)
            done.append(torch.cat([pairs.flatten(2), rest], dim=2).flatten(1))
        return torch.cat(done)

    y = turned(s["x"], turn)
    return y if c["op"] == "rotate" else (y, turned(s["dout"], turn.conj()))


def _exact_scan(c, s):
    """Row after row inside of stretches of the rows, all stretches side by side, then from one stretch to the next; the gradients by differentiation."""
    n, f, graphs = c["n"], c["f"], c["graphs"]
    train = c["op"] == "scan_train"
    size = (torch.ones(n, device="cuda") if s["ptr"] is None else s["ptr"][1:] - s["ptr"][:-1]).long()
    graph = torch.repeat_interleave(torch.arange(graphs, device="cuda"), size)
    starts = torch.cat([graph.new_full((1,), -1), graph[:-1]]) != graph
    ends = torch.cat([graph[1:], graph.new_full((1,), -1)]) != graph
    leaves = [s[name].double() for name in ("x", "gate", "initial")]
    with torch.set_grad_enabled(train):
        for t in leaves:
            t.requires_grad_(train)
        x, gate, initial = leaves
        a = gate if c["form"] == "factor" else torch.sigmoid(gate)
        b = x if c["form"] == "factor" else torch.sigmoid(-gate) * x
        a, b = torch.where(starts[:, None], 0.0, a), torch.where(starts[:, None], b + a * initial[graph], b)
        width = max(1, math.isqrt(n))
        count = -(-n // width)
        pad = count * width - n
        a, b = (torch.cat([t, t.new_zeros((pad, f))]).reshape(count, width, f).unbind(1) for t in (a, b))
        h, through = [b[0]], [a[0]]
        for t in range(1, width):
            h.append(torch.addcmul(b[t], a[t], h[-1]))
            through.append(through[-1] * a[t])
        state = [torch.zeros((f,), dtype=torch.float64, device="cuda")]
        for k in range(count - 1):
            state.append(torch.addcmul(h[-1][k], through[-1][k], state[-1]))
        y = torch.addcmul(torch.stack(h, 1), torch.stack(through, 1), torch.stack(state)[:, None, :]).reshape(count * width, f)[:n]
        final = initial.index_copy(0, graph[ends], y[ends])
    if not train:
        return y, final
    return (y.detach(), final.detach(), *torch.autograd.grad((y, final), leaves, (s["dout"].double(), s["dfinal"].double())))


# ---------------------------------------------------------------- floors

def work(case):
    c = case
    n, f, elem = c["n"], c["f"], 2 if c["dtype"] == "bf16" else 4
    moved = n * f * elem
    if c["op"] == "norm":                                         # x in, the result out
        return {"bytes": 2 * moved + 8 * f, "flops": 8 * n * f}
    if c["op"] == "norm_train":                                   # and again x and the result's gradient in, that of x out
        return {"bytes": 5 * moved + 16 * f, "flops": 20 * n * f}
    if c["op"].startswith("rotate"):
        passes, turned = 1 + (c["op"] == "rotate_train"), n * c["heads"] * c["part"]
        return {"bytes": passes * (2 * moved + n * (8 if c["ids"] == "i64" else 4)), "flops": passes * 3 * turned}
    states = c["graphs"] * f * 4
    forward = {"bytes": 3 * moved + 2 * states, "flops": (2 if c["form"] == "factor" else 6) * n * f}
    if c["op"] == "scan":                                         # x and gates in, the result out; the states in and out
        return forward
    # x, gates and the result's gradient in, two gradients out; the first states, the last ones' gradient in, the first ones' out
    return {"bytes": forward["bytes"] + 5 * moved + 3 * states, "flops": forward["flops"] + (6 if c["form"] == "factor" else 14) * n * f}
