"""The operators around the KAN blocks of a language model, as cases that can be timed.

Three operators, each with its gradient, all through the package's public entry points:

  lookup  kan_lookup_forward / kan_lookup_backward: rows of a table by token id, times a scale; the table's
          gradient, the sum over the tokens of each id
  norm    kan_block_norm_forward / kan_block_norm_backward: the norm in front of a block and the norm behind
          it with gate and residual scale, in one pass over the residual stream
  loss    kan_vocab_loss_forward / kan_vocab_loss_backward: softmax cross entropy of rows against a table of
          outputs, in pieces of the table, without the logits

A case is a dict of plain values.  "pass" is "forward", "backward" or "step" (a loss and its gradient).
Keys of the operators:

  lookup  rows (of the table), width, tokens, table "f32" | "f16" | "bf16" (the gradient's type too), out:
          type of the looked-up rows and of their gradient, ids "u16" | "i32" | "i64", use "uniform" | "zipf":
          how the tokens spread over the rows, pad: share of the ids that name no row (i32, i64)
  norm    tokens, width, stream: type of x, y, block: type of u, v and gate, gate, first (no block in front:
          the norm before the first block alone)
  loss    tokens, rows, width, type, pad: share of the targets that are left out
  buffers "kept": outputs live as long as the program (a server's loop); "plain": the call brings its own

With `own` the calls are the package's; without, the same operators as elementary torch operations in 32 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "u16": 2, "i32": 4, "i64": 8}
EPS = 1e-6

# The most that a drawn case may cost: the largest listed one of its operator.
MOST_LOOKUP = 65536 * 4096           # values of the table, and of the looked-up rows
MOST_NORM = 8192 * 4096              # values of the stream
MOST_LOSS = 8192 * 131072 * 2048     # products of one of the three matrix products


def _lookup(name, which, tokens, rows, width, *, table="bf16", out="bf16", ids="i64", use="zipf", pad=0.0, scale=1.0,
            buffers="plain"):
    return {"name": name, "op": "lookup", "pass": which, "tokens": tokens, "rows": rows, "width": width, "table": table,
            "out": out, "ids": ids, "use": use, "pad": pad, "scale": scale, "buffers": buffers}


def _norm(name, which, tokens, width, *, stream="bf16", block="f32", gate=True, first=False, buffers="plain"):
    return {"name": name, "op": "norm", "pass": which, "tokens": tokens, "width": width, "stream": stream, "block": block,
            "gate": gate, "first": first, "scale": 0.5, "buffers": buffers}


def _loss(name, which, tokens, rows, width, *, type="bf16", ids="i64", pad=0.0, scale=1.0, buffers="plain"):
    return {"name": name, "op": "loss", "pass": which, "tokens": tokens, "rows": rows, "width": width, "type": type,
            "ids": ids, "pad": pad, "scale": scale, "buffers": buffers}


def listed():
    return [
        # Decoding: the input of the first block for the token that was just chosen.
        _lookup("lookup, one token", "forward", 1, 65536, 2048, out="f32", scale=0.5, buffers="kept"),
        # A training batch or a long prompt, handed to fp32 blocks.
        _lookup("lookup, 16384 tokens", "forward", 16384, 65536, 4096, out="f32", scale=0.5),
        # The gradient of that table, tokens as texts use them, some of the batch padding.
        _lookup("lookup gradient, 16384 tokens", "backward", 16384, 65536, 4096, pad=0.05, scale=0.5),
        # Learning a codebook: the gradient of its ten-entry rows from every edge of a 2048 x 512 layer.
        _lookup("codebook gradient, 2048 x 512 edges", "backward", 2048 * 512, 65536, 10, table="f32", out="f32", ids="u16"),
        # Decoding: between two blocks, for one token.
        _norm("norms, one token", "forward", 1, 2048, buffers="kept"),
        # Between two fp32 blocks on a 16-bit residual stream, a training batch or a prompt.
        _norm("norms, 8192 tokens", "forward", 8192, 2048),
        # The way back through the same place, wide rows, everything in 16 bits.
        _norm("norms gradient, 8192 tokens", "backward", 8192, 4096, block="bf16"),
        # A width and a batch that come from a data set; full precision, no gate.
        _norm("norms gradient, ragged fp32", "backward", 999, 1000, stream="f32", gate=False),
        # Scoring one token that was proposed elsewhere.
        _loss("loss, one token", "forward", 1, 65536, 2048, buffers="kept"),
        # The training step of a large vocabulary.
        _loss("loss step, 8192 tokens x 131072", "step", 8192, 131072, 2048),
        # Fine-tuning on short ragged batches with prompts masked out, fp16.
        _loss("loss step, ragged fp16", "step", 1111, 50021, 1000, type="f16", pad=0.3),
        # A validation or a small study in full precision, on the fp32 outputs of a head.
        _loss("loss step, fp32", "step", 500, 10007, 256, type="f32", ids="i32", scale=2.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width between lo and hi: half of them whole multiples of 64, the others as they fall."""
    n = _log_int(rng, lo, hi)
    return min(hi, max(64, (n + 32) // 64 * 64)) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["lookup", "norm", "loss"])
    if op == "lookup":
        which = rng.choice(["forward", "backward"])
        codebook = rng.random() < 0.25
        width = 10 if codebook else _width(rng, 64, 8192)
        rows = _log_int(rng, 256, min(262144, MOST_LOOKUP // width))
        tokens = _log_int(rng, 1, min(1 << 20 if codebook else 1 << 16, MOST_LOOKUP // width))
        table = "f32" if codebook else rng.choice(["bf16", "bf16", "f16", "f32"])
        ids = rng.choice(["i32", "i64"] + (["u16"] if rows <= 65536 else []))
        case = _lookup("", which, tokens, rows, width, table=table, out=rng.choice([table, "f32"]), ids=ids,
                       use=rng.choice(["uniform", "zipf"]), pad=0.0 if ids == "u16" else rng.choice([0.0, 0.1]),
                       scale=rng.choice([1.0, 0.5, math.sqrt(width)]), buffers=rng.choice(["kept", "plain"]))
    elif op == "norm":
        width = _width(rng, 64, 8192)
        stream = rng.choice(["bf16", "bf16", "f16", "f32"])
        case = _norm("", rng.choice(["forward", "backward"]), _log_int(rng, 1, min(16384, MOST_NORM // width)), width,
                     stream=stream, block=rng.choice([stream, "f32"]), gate=rng.random() < 0.5, first=rng.random() < 0.2,
                     buffers=rng.choice(["kept", "plain"]))
    else:
        type = rng.choice(["bf16", "bf16", "f16", "f32"])
        most = MOST_LOSS // (8 if type == "f32" else 1)       # (fp32 products cost the most)
        width = _width(rng, 64, 4096)
        rows = _log_int(rng, 1000, 131072)
        tokens = _log_int(rng, 1, max(1, min(8192, most // (rows * width))))
        case = _loss("", rng.choice(["forward", "step", "step"]), tokens, rows, width, type=type, ids=rng.choice(["i32", "i64"]),
                     pad=rng.choice([0.0, 0.2]), scale=rng.choice([1.0, 0.5]), buffers=rng.choice(["kept", "plain"]))
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------------


def _tokens(g, n, rows, use, pad, ids):
    if use == "zipf":                    # P(rank r) ~ 1 / r, the ranks scattered over the table
        upto = (1.0 / torch.arange(1, rows + 1, device="cuda", dtype=torch.float64)).cumsum(0)
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * upto[-1]
        t = torch.randperm(rows, generator=g, device="cuda")[torch.searchsorted(upto, u).clamp_(max=rows - 1)]
    else:
        t = torch.randint(0, rows, (n,), generator=g, device="cuda")
    if pad:
        t = torch.where(torch.rand(n, generator=g, device="cuda") < pad, -1, t)
    if ids == "u16":                     # (16-bit ids are carried in int16)
        return torch.where(t >= 32768, t - 65536, t).to(torch.int16)
    return t.to(torch.int32 if ids == "i32" else torch.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, type, mul=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(mul).to(TYPES[type])

    n, d = case["tokens"], case["width"]
    kept = case["buffers"] == "kept"
    s = {"case": case, "scale": case["scale"]}
    if case["op"] == "lookup":
        s["ids"] = _tokens(g, n, case["rows"], case["use"], case["pad"], case["ids"])
        if case["pass"] == "forward":
            s["table"] = normal(case["rows"], d, type=case["table"], mul=0.5)
            s["y"] = torch.empty((n, d), dtype=TYPES[case["out"]], device="cuda") if kept else None
        else:
            s["dy"] = normal(n, d, type=case["out"], mul=1.0 / 64)
            s["dtable"] = torch.empty((case["rows"], d), dtype=TYPES[case["table"]], device="cuda") if kept else None
    elif case["op"] == "norm":
        st, bl = case["stream"], case["block"]
        s["w_before"] = normal(d, type=st, mul=0.1).add_(0.3)       # (KAN layers take inputs of [-1, 1])
        s["w_after"] = None if case["first"] else normal(d, type=st, mul=0.2).add_(1.0)
        s["x"] = normal(n, d, type=st, mul=2.0)                    # (backward: the stream behind the block, y)
        s["v"] = None if case["first"] else normal(n, d, type=bl, mul=0.7)
        s["gate"] = normal(n, d, type=bl) if case["gate"] and not case["first"] else None
        s["y"] = s["u"] = None
        if case["pass"] == "backward":
            s["dy"] = normal(n, d, type=st, mul=1.0 / 64)
            s["du"] = normal(n, d, type=bl, mul=1.0 / 64)
        elif kept:
            s["y"] = None if case["first"] else torch.empty_like(s["x"])
            s["u"] = torch.empty((n, d), dtype=TYPES[bl], device="cuda")
    else:
        V = case["rows"]
        s["table"] = normal(V, d, type=case["type"], mul=2.0 / math.sqrt(d))
        s["targets"] = _tokens(g, n, V, "zipf", case["pad"], case["ids"])
        # rows that a trained model hands on: they favour their target
        h = torch.randn((n, d), generator=g, device="cuda")
        favour = torch.rand((n, 1), generator=g, device="cuda") * 2.0
        s["h"] = (h + favour * s["table"][s["targets"].long().clamp(min=0)].float()).to(TYPES[case["type"]])
        s["dloss"] = torch.full((n,), 1.0 / n, device="cuda")
        s["loss"] = torch.empty(n, device="cuda") if kept else None
        s["lse"] = torch.empty(n, device="cuda") if kept else None
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------


def _row_ids(ids, rows):
    """Row of every id, and whether it names one."""
    t = ids.long() & 0xFFFF if ids.dtype == torch.int16 else ids.long()
    ok = (t >= 0) & (t < rows)
    return torch.where(ok, t, 0), ok


def _plain_lookup(s):
    case = s["case"]
    t, ok = _row_ids(s["ids"], case["rows"])
    if case["pass"] == "forward":
        y = s["table"][t].float() * s["scale"]
        return torch.where(ok[:, None], y, 0.0).to(TYPES[case["out"]])
    dy = torch.where(ok[:, None], s["dy"].float() * s["scale"], 0.0)
    grad = torch.zeros((case["rows"], case["width"]), device="cuda")
    return grad.index_add_(0, t, dy).to(TYPES[case["table"]])


def _plain_norm(s):
    case = s["case"]
    st, bl, alpha = TYPES[case["stream"]], TYPES[case["block"]], s["scale"]
    x, wb = s["x"].float(), s["w_before"].float()
    if not case["first"]:
        v, wa = s["v"].float(), s["w_after"].float()
        rv = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
        sig = 1.0 / (1.0 + torch.exp(-s["gate"].float())) if s["gate"] is not None else 1.0
    if case["pass"] == "forward":
        y = x if case["first"] else x + alpha * sig * (wa * (v * rv))
        u = wb * (y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS))
        return (None if case["first"] else y.to(st)), u.to(bl)
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    hat, du = x * r, s["du"].float()
    t = du * wb
    gy = s["dy"].float() + r * (t - hat * (t * hat).mean(1, keepdim=True))
    dwb = (du * hat).sum(0).to(st)
    if case["first"]:
        return gy.to(st), None, None, dwb, None
    m = v * rv
    dn = alpha * sig * gy
    dwa = (dn * m).sum(0).to(st)
    q = dn * wa
    dv = rv * (q - m * (q * m).mean(1, keepdim=True))
    dgate = None if s["gate"] is None else (alpha * gy * (wa * m) * sig * (1.0 - sig)).to(bl)
    return gy.to(st), dv.to(bl), dgate, dwb, dwa


def _plain_loss(s):
    case = s["case"]
    t, ok = _row_ids(s["targets"], case["rows"])
    h, w = s["h"].float(), s["table"].float()
    z = (h @ w.t()) * s["scale"]
    top = z.amax(1, keepdim=True)
    lse = top[:, 0] + (z - top).exp().sum(1).log()
    loss = torch.where(ok, lse - z.gather(1, t[:, None])[:, 0], 0.0)
    if case["pass"] == "forward":
        return loss, lse
    weight = torch.where(ok, s["dloss"], 0.0) * s["scale"]
    p = (z - lse[:, None]).exp()
    p.scatter_add_(1, t[:, None], torch.full_like(lse, -1.0)[:, None])
    p = p * weight[:, None]
    type = TYPES[case["type"]]
    return loss, lse, (p @ w).to(type), (p.t() @ h).to(type)


def _own_lookup(s):
    from paper_2512_15742_amd import binding as kb
    case = s["case"]
    if case["pass"] == "forward":
        return kb.kan_lookup_forward(s["table"], s["ids"], scale=s["scale"], dtype=TYPES[case["out"]], y=s["y"])
    return kb.kan_lookup_backward(s["dy"], s["ids"], case["rows"], scale=s["scale"], dtype=TYPES[case["table"]], dtable=s["dtable"])


def _own_norm(s):
    from paper_2512_15742_amd import binding as kb
    case = s["case"]
    if case["pass"] == "forward":
        return kb.kan_block_norm_forward(s["x"], v=s["v"], gate=s["gate"], w_after=s["w_after"], w_before=s["w_before"],
                                         scale=s["scale"], eps=EPS, dtype=TYPES[case["block"]], y=s["y"], u=s["u"])
    return kb.kan_block_norm_backward(s["x"], dy=s["dy"], du=s["du"], v=s["v"], gate=s["gate"], w_after=s["w_after"],
                                      w_before=s["w_before"], scale=s["scale"], eps=EPS)


def _own_loss(s):
    from paper_2512_15742_amd import binding as kb
    loss, lse = kb.kan_vocab_loss_forward(s["h"], s["table"], s["targets"], scale=s["scale"], loss=s["loss"], lse=s["lse"])
    if s["case"]["pass"] == "forward":
        return loss, lse
    dh, dtable = kb.kan_vocab_loss_backward(s["h"], s["table"], s["targets"], lse, s["dloss"], scale=s["scale"])
    return loss, lse, dh, dtable


PLAIN = {"lookup": _plain_lookup, "norm": _plain_norm, "loss": _plain_loss}
OWN = {"lookup": _own_lookup, "norm": _own_norm, "loss": _own_loss}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---- what a pass cannot do without, and its exact outputs ------------------------------------------------------------


def work(case):
    n, d = case["tokens"], case["width"]
    if case["op"] == "lookup":
        ids, row, out = BYTES[case["ids"]] * n, BYTES[case["table"]] * d, BYTES[case["out"]] * d
        if case["pass"] == "forward":
            return {"bytes": ids + n * out + min(n, case["rows"]) * row, "flops": n * d}
        return {"bytes": ids + n * out + case["rows"] * row, "flops": n * d}
    if case["op"] == "norm":
        st, bl = BYTES[case["stream"]], BYTES[case["block"]]
        parts, gate = 1 if case["first"] else 2, case["gate"] and not case["first"]
        if case["pass"] == "forward":      # x, v, gate in; y, u out
            values = st * parts + bl * (parts + gate)
            return {"bytes": n * d * values + parts * d * st, "flops": n * d * (4 + 5 * (parts - 1) + 4 * gate)}
        values = 3 * st + bl + 2 * bl * (parts - 1 + gate)      # y, dy, du, v, gate in; dx, dv, dgate out
        return {"bytes": n * d * values + 2 * parts * d * st, "flops": n * d * (10 + 10 * (parts - 1) + 6 * gate)}
    V, b = case["rows"], BYTES[case["type"]]
    io, products = b * (n + V) * d, 2 * n * V * d
    if case["pass"] == "forward":
        return {"bytes": io + n * (8 + BYTES[case["ids"]]), "flops": products}
    return {"bytes": 2 * io + n * (12 + BYTES[case["ids"]]), "flops": 3 * products}


def _exact_norm(case, s):
    """The definition in 64 bits; gradients by differentiating it."""
    def at(k):
        return None if s[k] is None else s[k].double()

    def rms(a, w):
        return a / (a.pow(2).sum(1, keepdim=True) / a.shape[1] + EPS).sqrt() * w

    def behind(v, gate, w):
        y = rms(v, w) * case["scale"]
        return y if gate is None else y * torch.sigmoid(gate)

    if case["pass"] == "forward":
        y = at("x") if case["first"] else at("x") + behind(at("v"), at("gate"), at("w_after"))
        return (None if case["first"] else y), rms(y, at("w_before"))
    y, wb = at("x").requires_grad_(), at("w_before").requires_grad_()
    gy, dwb = torch.autograd.grad((rms(y, wb) * at("du")).sum(), (y, wb))
    gy = gy + at("dy")
    if case["first"]:
        return gy, None, None, dwb, None
    v, wa = at("v").requires_grad_(), at("w_after").requires_grad_()
    gate = None if s["gate"] is None else at("gate").requires_grad_()
    leaves = (v, wa) if gate is None else (v, wa, gate)
    got = torch.autograd.grad((behind(v, gate, wa) * gy).sum(), leaves)
    return gy, got[0], got[2] if gate is not None else None, dwb, got[1]


def exact(case, seed):
    """What run returns for these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    rows = case["rows"]
    ids = s["ids"] if case["op"] == "lookup" else s["targets"]
    ids = ids.to(torch.int64) % 65536 if case["ids"] == "u16" else ids.to(torch.int64)
    named = ((ids >= 0) & (ids < rows)).nonzero()[:, 0]
    if case["op"] == "lookup":
        if case["pass"] == "forward":
            y = torch.zeros((case["tokens"], case["width"]), dtype=torch.float64, device="cuda")
            y[named] = s["table"][ids[named]].double() * case["scale"]
            return y
        grad = torch.zeros((rows, case["width"]), dtype=torch.float64, device="cuda")
        grad.index_add_(0, ids[named], s["dy"][named].double())
        return grad * case["scale"]
    w, step = s["table"].double(), case["pass"] == "step"
    loss = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")
    lse = torch.empty_like(loss)
    dh, dw = torch.zeros_like(s["h"], dtype=torch.float64), torch.zeros_like(w) if step else None
    for a in range(0, case["tokens"], 1024):
        h = s["h"][a:a + 1024].double()
        z = torch.mm(h, w.t()).mul_(case["scale"])
        lse[a:a + 1024] = torch.logsumexp(z, 1)
        at = named[(named >= a) & (named < a + 1024)]
        loss[at] = lse[at] - z[at - a, ids[at]]
        if step:
            p = torch.softmax(z, 1)[at - a]
            p[torch.arange(len(at), device="cuda"), ids[at]] -= 1.0
            p *= s["dloss"][at].double()[:, None] * case["scale"]
            dh[at] = torch.mm(p, w)
            dw += torch.mm(p.t(), h[at - a])
    return (loss, lse, dh, dw) if step else (loss, lse)
