"""The operators between the layers and at both ends of a model that is trained or served, as cases that can be timed: embedding lookup
and its gradient, the root-mean-square norm of a residual sum (in 8 bits too) and its gradient, the loss of a student against a teacher's
top logits and its gradient.

With `own` false, `run` computes them in elementary torch operations; with `own` true it calls the package.  Both get the same tensors.
Widths and vocabularies are those of the package's model configurations (256 in fp32 with 4096 ids; 4096, 8192 with 128256; 5120 with
32000; draft vocabularies of 1024 and 32000) or generic, rows those of its workloads.

Layouts: ids int32 [tokens], -1 for padding; weights [vocabulary][width]; activations [rows][width]; logits [rows][student's vocabulary];
the teacher's entries [rows][K] as ids (int32, -1 for none) and logits (fp32); id_map int32 [teacher's vocabulary]: the student's id or -1.
"""
import math

import numpy as np
import torch

own = False

TOP = {"e4m3": 448.0, "int8": 127.0}      # largest magnitude of the 8-bit formats, and the least scale
FLOOR = 2.0 ** -120
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
BYTES = {"fp32": 4, "bf16": 2, "e4m3": 1, "int8": 1}
EPS = 1e-5


def _embed(name, tokens, vocab, width, dtype, out, scale, pad):
    """pad: share of the ids that are -1"""
    case = {"op": "embed", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "out": out, "scale": scale, "pad": pad}
    return {"name": name, **case} if name else case


def _embed_grad(name, tokens, vocab, width, dtype, out, scale, pad):
    return {**_embed(name, tokens, vocab, width, dtype, out, scale, pad), "op": "embed_grad"}


def _norm(name, rows, width, dtype, residual, out, group):
    """residual: its type, or "none"; group: columns that share a scale in 8 bits, 0 for the whole row"""
    case = {"op": "norm", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "out": out, "group": group}
    return {"name": name, **case} if name else case


def _norm_grad(name, rows, width, dtype, grad, carried):
    """grad: the type of the output's gradient; carried: whether the residual sum has a gradient of its own"""
    case = {"op": "norm_grad", "rows": rows, "width": width, "dtype": dtype, "grad": grad, "carried": carried}
    return {"name": name, **case} if name else case


def _distill(name, mode, rows, vocab, K, dtype, out, teacher, temperature, kind, pad):
    """mode: "loss", "grad" (from the statistics that the loss left) or "both" at once; teacher: its vocabulary, 0 where it is the student's"""
    case = {"op": "distill", "mode": mode, "rows": rows, "vocab": vocab, "K": K, "dtype": dtype, "out": out, "teacher": teacher,
            "temperature": temperature, "kind": kind, "pad": pad}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one new token of an 8B-shaped model on its way into an fp32 residual stream: nothing but latency
        _embed("embed-token", 1, 128256, 4096, "bf16", "fp32", 1.0, 0.0),
        # a 16k-token prompt of a 70B-shaped model, rows scaled by the width's root
        _embed("embed-prompt", 16384, 128256, 8192, "bf16", "bf16", 8192 ** 0.5, 0.0),
        # the embedding's gradient for a batch of padded training sequences of an 8B-shaped model
        _embed_grad("embed-grad", 8192, 128256, 4096, "bf16", "bf16", 1.0, 0.1),
        # the same of the small fp32 model, an odd number of tokens
        _embed_grad("embed-grad-tiny-fp32", 2003, 4096, 256, "fp32", "fp32", 16.0, 0.0),
        # a decoding step of one sequence: a projection's fp32 output joins the fp32 residual stream
        _norm("norm-token", 1, 4096, "fp32", "fp32", "bf16", 0),
        # a 16k-token prompt on its way into products in e4m3
        _norm("norm-prompt-e4m3", 16384, 4096, "bf16", "bf16", "e4m3", 128),
        # a decoding step of a serving batch of 64 of a 70B-shaped model, into products in int8
        _norm("norm-batch-int8", 64, 8192, "bf16", "bf16", "int8", 0),
        # the norm's gradient in training, with what the residual stream carries back
        _norm_grad("norm-grad", 8192, 4096, "bf16", "bf16", True),
        # an odd number of rows of a 13B-shaped model in fp32; a first norm, whose input has no other use
        _norm_grad("norm-grad-odd-fp32", 1001, 5120, "fp32", "fp32", False),
        # validation loss of the small fp32 model's draft over one short sequence
        _distill("distill-loss-tiny", "loss", 61, 1024, 16, "fp32", "fp32", 4096, 1.0, "kl", 0.0),
        # a training step's loss and gradient of a draft with a reduced vocabulary, one row in ten padding
        _distill("distill-draft", "both", 8192, 32000, 64, "bf16", "bf16", 128256, 1.0, "kl", 0.1),
        # the gradient alone, for a student with the teacher's whole vocabulary, fp32 logits, a softer target
        _distill("distill-grad-whole", "grad", 2048, 128256, 16, "fp32", "bf16", 0, 2.0, "ce", 0.0),
    ]


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "distill", "distill"])
    dtype, vocab, width = rng.choice([("fp32", 4096, 256), ("bf16", 128256, 4096), ("bf16", 128256, 4096), ("bf16", 32000, 5120), ("bf16", 128256, 8192),
                                      ("fp32", 32000, 4096), ("bf16", 5003, 1000), ("fp32", 50257, 1002)])
    pad = rng.choice([0.0, 0.0, 0.1, 0.5])
    if op == "embed":
        return _embed("", _log(rng, 1, 16384), vocab, width, dtype, rng.choice([dtype, "fp32"]), rng.choice([1.0, width ** 0.5]), pad)
    if op == "embed_grad":
        return _embed_grad("", _log(rng, 1, 16384), vocab, width, dtype, rng.choice([dtype, "fp32"]), rng.choice([1.0, width ** 0.5]), pad)
    if op == "norm":
        return _norm("", _log(rng, 1, 16384), width, dtype, rng.choice(["none", dtype, dtype, "fp32"]), rng.choice([dtype, "bf16", "e4m3", "e4m3", "int8"]),
                     rng.choice([0, 32, 128]))
    if op == "norm_grad":
        return _norm_grad("", _log(rng, 1, 16384), width, dtype, rng.choice([dtype, "bf16"]), rng.random() < 0.6)
    dtype = rng.choice(["fp32", "bf16"])
    vocab, teacher = rng.choice([(1024, 4096), (32000, 128256), (32000, 0), (128256, 0), (50257, 0), (10007, 32000)])
    return _distill("", rng.choice(["loss", "grad", "both"]), _log(rng, 1, 8192), vocab, rng.choice([1, 7, 16, 64, 200]), dtype, rng.choice([dtype, "bf16"]),
                    teacher, rng.choice([1.0, 1.0, 2.0, 0.7]), rng.choice(["kl", "ce"]), pad)


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"case": case, **{"embed": _prepare_embed, "embed_grad": _prepare_embed_grad, "norm": _prepare_norm, "norm_grad": _prepare_norm_grad,
                             "distill": _prepare_distill}[case["op"]](case, g)}


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _without(g, n, share):
    """Which of n are padding: the last ones of a batch's shuffled sequences, as many for every seed"""
    return torch.randperm(n, generator=g, device="cuda") < int(n * share)


def _ids(case, g):
    """Ids as a text has them: the i-th most frequent about 1 / i as often as the first, in an order of their own."""
    T, V = case["tokens"], case["vocab"]
    rank = (float(V) ** _uniform(g, T).double() - 1.0).long().clamp(0, V - 1)
    ids = torch.randperm(V, generator=g, device="cuda")[rank]
    return ids.masked_fill(_without(g, T, case["pad"]), -1).to(torch.int32)


def _prepare_embed(case, g):
    return {"ids": _ids(case, g), "weight": _normal(g, case["vocab"], case["width"]).to(DTYPE[case["dtype"]])}


def _prepare_embed_grad(case, g):
    return {"ids": _ids(case, g), "grad": _normal(g, case["tokens"], case["width"]).mul_(1e-3).to(DTYPE[case["dtype"]])}


def _stream(g, rows, width, dtype):
    """A residual stream as trained models have it: some dimensions many times larger than the others."""
    gain = torch.ones(width, device="cuda")
    gain[torch.randperm(width, generator=g, device="cuda")[: max(1, width // 256)]] = 20.0
    return _normal(g, rows, width).mul_(gain).to(dtype)


def _prepare_norm(case, g):
    rows, k, dt = case["rows"], case["width"], DTYPE[case["dtype"]]
    st = {"gain": (1 + 0.1 * _normal(g, k)).to(dt), "residual": None}
    if case["residual"] == "none":
        st["x"] = _stream(g, rows, k, dt)
    else:
        st["x"], st["residual"] = _normal(g, rows, k).to(dt), _stream(g, rows, k, DTYPE[case["residual"]])
    return st


def _prepare_norm_grad(case, g):
    rows, k, dt = case["rows"], case["width"], DTYPE[case["dtype"]]
    st = {"gain": (1 + 0.1 * _normal(g, k)).to(dt), "x": _stream(g, rows, k, dt), "grad": _normal(g, rows, k).mul_(1e-3).to(DTYPE[case["grad"]])}
    st["carried"] = _normal(g, rows, k).mul_(1e-3).to(dt) if case["carried"] else None
    return st


def _prepare_distill(case, g):
    """A student that has learned part of the way: its logits at the teacher's entries are the teacher's with noise."""
    rows, V, K = case["rows"], case["vocab"], case["K"]
    Vt = case["teacher"] or V
    # K different ids a row: steps of a number that shares no divisor with the vocabulary
    step = next(s for s in range(7919, 8919) if math.gcd(s, Vt) == 1)
    ids = (torch.randint(0, Vt, (rows, 1), generator=g, device="cuda") + step * torch.arange(K, device="cuda")) % Vt
    values = 14.0 - 0.6 * _uniform(g, rows, K).mul_(-1.0).add_(1.0).log_().neg_().cumsum(-1)
    st = {"id_map": None}
    mapped = ids
    if case["teacher"]:
        st["id_map"] = torch.full((Vt,), -1, dtype=torch.int32, device="cuda")
        st["id_map"][torch.randperm(Vt, generator=g, device="cuda")[:V].sort().values] = torch.arange(V, dtype=torch.int32, device="cuda")
        mapped = st["id_map"][ids].long()
    z = _normal(g, rows, V + 1).mul_(2.0)
    z.scatter_(1, mapped.where(mapped >= 0, torch.full_like(mapped, V)), values + _normal(g, rows, K))
    st["logits"] = z[:, :V].to(DTYPE[case["dtype"]], copy=True).contiguous()
    del z
    st["ids"] = ids.masked_fill(_without(g, rows, case["pad"])[:, None], -1).to(torch.int32)
    st["values"] = values
    if case["mode"] != "loss":
        st["grad"] = torch.full((rows,), 1.0 / rows, device="cuda")
    if case["mode"] == "grad":
        x = st["logits"].float()
        st["stats"] = torch.stack([x.amax(1), ((x - x.amax(1, keepdim=True)) / case["temperature"]).exp().sum(1)], 1).contiguous()
    return st


# ------------------------------------------------------------------------------------------------ a pass
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _plain_embed(st):
    rows = st["weight"][st["ids"].clamp_min(0).long()].float() * st["case"]["scale"]
    return rows.masked_fill((st["ids"] < 0)[:, None], 0.0).to(DTYPE[st["case"]["out"]])


def _plain_embed_grad(st):
    c = st["case"]
    live = st["ids"] >= 0
    total = torch.zeros(c["vocab"], c["width"], device="cuda")
    total.index_add_(0, st["ids"][live].long(), st["grad"][live].float())
    return (total * c["scale"]).to(DTYPE[c["out"]])


def _plain_norm(st):
    c = st["case"]
    s = st["x"].float()
    if st["residual"] is not None:
        s = s + st["residual"].float()
    y = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + EPS) * st["gain"].float()
    out = {"sum": None if st["residual"] is None else s.to(st["residual"].dtype)}
    if c["out"] not in TOP:
        return {**out, "y": y.to(DTYPE[c["out"]])}
    rows, k = y.shape
    n = c["group"] or k
    y = torch.nn.functional.pad(y, (0, -k % n)).view(rows, -1, n)
    scale = (y.abs().amax(-1) * (1.0 / TOP[c["out"]])).clamp_min(FLOOR)
    code = (y * (1.0 / scale)[..., None]).clamp(-TOP[c["out"]], TOP[c["out"]])
    if c["out"] == "int8":
        return _normed(st, (code.round() * scale[..., None]).view(rows, -1)[:, :k].bfloat16(), scale, out["sum"])
    return _normed(st, code.to(torch.float8_e4m3fn).view(rows, -1)[:, :k], scale, out["sum"])


def _normed(st, codes, scale, total):
    """What a pass of "norm" in 8 bits returns: the codes and scales, or for whole-number codes the values that they stand for, in bf16."""
    return {"values" if st["case"]["out"] == "int8" else "codes": codes, "scale": scale, "sum": total}


def _plain_norm_grad(st):
    x, g, w = st["x"].float(), st["grad"].float(), st["gain"].float()
    u = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    h, gw = x * u, g * w
    dx = u * (gw - h * (gw * h).mean(-1, keepdim=True))
    if st["carried"] is not None:
        dx = dx + st["carried"].float()
    return {"x": dx.to(st["x"].dtype), "gain": (g * h).sum(0).to(st["gain"].dtype)}


def _target(st):
    """(the student's ids, 0 where there is none; p; ln p, 0 where p is 0; rows with an entry)"""
    ids = st["ids"].long()
    if st["id_map"] is not None:
        ids = st["id_map"][ids.clamp_min(0)].long().masked_fill(ids < 0, -1)
    v = (st["values"] / st["case"]["temperature"]).masked_fill(ids < 0, -math.inf)
    some = (ids >= 0).any(1)
    top = v.amax(1, keepdim=True).masked_fill(~some[:, None], 0.0)
    e = (v - top).exp()
    total = e.sum(1, keepdim=True).masked_fill(~some[:, None], 1.0)
    p = e / total
    return ids.clamp_min(0), p, (v - top - total.log()).masked_fill(p == 0, 0.0), some


def _plain_distill(st):
    c, T = st["case"], st["case"]["temperature"]
    x = st["logits"].float()
    if c["mode"] == "grad":
        top, total = st["stats"][:, :1], st["stats"][:, 1:]
        e = ((x - top) / T).exp()
    else:
        top = x.amax(1, keepdim=True)
        e = ((x - top) / T).exp()
        total = e.sum(1, keepdim=True)
    ids, p, lnp, some = _target(st)
    out = {}
    if c["mode"] != "grad":
        lnq = (x.gather(1, ids) - top) / T - total.log()
        out["loss"] = (p * (lnp - lnq if c["kind"] == "kl" else -lnq)).sum(1)
    if c["mode"] != "loss":
        w = st["grad"][:, None] / T
        dz = e.mul_(w * p.sum(1, keepdim=True) / total).masked_fill_(~some[:, None], 0.0).scatter_add_(1, ids, p * -w)
        out["logits"] = dz.to(DTYPE[c["out"]])
    return out


_run_plain = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "distill": _plain_distill}


def _own_embed(st):
    from paper_2503_01840_b200 import binding as sb
    return sb.embedding(st["ids"], st["weight"], scale=st["case"]["scale"], dtype=DTYPE[st["case"]["out"]])


def _own_embed_grad(st):
    from paper_2503_01840_b200 import binding as sb
    return sb.embedding_backward(st["grad"], st["ids"], st["case"]["vocab"], scale=st["case"]["scale"], dtype=DTYPE[st["case"]["out"]])


def _own_norm(st):
    from paper_2503_01840_b200 import binding as sb
    c = st["case"]
    got = sb.rms_norm(st["x"], st["gain"], EPS, residual=st["residual"], dtype=DTYPE[c["out"]], group=c["group"])
    got = (got,) if isinstance(got, torch.Tensor) else got
    total = None if st["residual"] is None else got[-1]
    if c["out"] not in TOP:
        return {"sum": total, "y": got[0]}
    codes, scale = got[:2]
    if c["out"] == "int8":
        wide = scale if c["group"] == 0 else scale.repeat_interleave(c["group"], 1)[:, : c["width"]]
        codes = (codes * wide).bfloat16()
    return _normed(st, codes, scale, total)


def _own_norm_grad(st):
    from paper_2503_01840_b200 import binding as sb
    dx, dgain = sb.rms_norm_backward(st["grad"], st["x"], st["gain"], EPS, grad_sum=st["carried"])
    return {"x": dx, "gain": dgain}


def _own_distill(st):
    from paper_2503_01840_b200 import binding as sb
    c = st["case"]
    kw = dict(id_map=st["id_map"], temperature=c["temperature"])
    if c["mode"] == "loss":
        return {"loss": sb.distill_loss(st["logits"], st["ids"], st["values"], kind=c["kind"], **kw)}
    if c["mode"] == "grad":
        return {"logits": sb.distill_loss_backward(st["grad"], st["logits"], st["stats"], st["ids"], st["values"], dtype=DTYPE[c["out"]], **kw)}
    loss, dz = sb.distill_loss_and_grad(st["grad"], st["logits"], st["ids"], st["values"], kind=c["kind"], dtype=DTYPE[c["out"]], **kw)
    return {"loss": loss, "logits": dz}


_run_own = {"embed": _own_embed, "embed_grad": _own_embed_grad, "norm": _own_norm, "norm_grad": _own_norm_grad, "distill": _own_distill}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, op = case, case["op"]
    if op in ("embed", "embed_grad"):
        T, k = c["tokens"], c["width"]
        live = T - int(T * c["pad"])
        if op == "embed":
            return {"bytes": 4 * T + live * k * BYTES[c["dtype"]] + T * k * BYTES[c["out"]], "flops": live * k}
        return {"bytes": 4 * T + live * k * BYTES[c["dtype"]] + c["vocab"] * k * BYTES[c["out"]], "flops": live * k}
    if op == "norm":
        n = c["rows"] * c["width"]
        r = 0 if c["residual"] == "none" else BYTES[c["residual"]]
        scales = c["rows"] * -(-c["width"] // (c["group"] or c["width"])) if c["out"] in TOP else 0
        return {"bytes": n * (BYTES[c["dtype"]] + 2 * r + BYTES[c["out"]]) + 4 * scales + c["width"] * BYTES[c["dtype"]], "flops": 5 * n}
    if op == "norm_grad":
        n = c["rows"] * c["width"]
        return {"bytes": n * (BYTES[c["grad"]] + (3 if c["carried"] else 2) * BYTES[c["dtype"]]) + 2 * c["width"] * BYTES[c["dtype"]], "flops": 10 * n}
    live = c["rows"] - int(c["rows"] * c["pad"])
    n = live * c["vocab"]
    nbytes = n * BYTES[c["dtype"]] + c["rows"] * (c["K"] * 8 + 4) + 4 * c["teacher"]
    if c["mode"] != "loss":
        nbytes += c["rows"] * (c["vocab"] * BYTES[c["out"]] + (12 if c["mode"] == "grad" else 4))
    return {"bytes": nbytes, "flops": n * {"loss": 4, "grad": 3, "both": 6}[c["mode"]]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "norm": _exact_norm, "norm_grad": _exact_norm_grad, "distill": _exact_distill}[case["op"]](st)


def _exact_embed(st):
    out = torch.zeros(st["case"]["tokens"], st["case"]["width"], dtype=torch.float64, device="cuda")
    live = (st["ids"] != -1).nonzero().flatten()
    out[live] = torch.index_select(st["weight"], 0, st["ids"][live]).double() * st["case"]["scale"]
    return out


def _exact_embed_grad(st):
    """Sums of runs of equal ids, as differences of running sums where they are sorted."""
    c = st["case"]
    out = torch.zeros(c["vocab"], c["width"], dtype=torch.float64, device="cuda")
    ids, order = st["ids"].sort(stable=True)
    order = order[ids >= 0]
    present, counts = ids[ids >= 0].unique_consecutive(return_counts=True)
    if len(present):
        run = st["grad"].double()[order].cumsum(0)[counts.cumsum(0) - 1]
        out[present.long()] = torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1])) * c["scale"]
    return out


def _exact_norm(st):
    """Codes as the reals that they round; whole-number codes, of which a few steps cover most values, as what their roundings stand for."""
    c = st["case"]
    s = st["x"].double() + (st["residual"].double() if st["residual"] is not None else 0.0)
    y = st["gain"].double() * s / ((s * s).sum(1) / s.shape[1] + EPS).sqrt()[:, None]
    total = s if st["residual"] is not None else None
    if c["out"] not in TOP:
        return {"sum": total, "y": y}
    k, n = c["width"], c["group"] or c["width"]
    scale = torch.stack([y[:, i: i + n].abs().amax(1) / TOP[c["out"]] for i in range(0, k, n)], 1)
    wide = scale.repeat_interleave(n, 1)[:, :k]
    return _normed(st, (y / wide).round() * wide if c["out"] == "int8" else y / wide, scale, total)


def _exact_norm_grad(st):
    """As the Jacobian of w s / |s|: the part of the gradient along s is taken out, up to eps."""
    x, g, w = st["x"].double(), st["grad"].double(), st["gain"].double()
    k = x.shape[1]
    r2 = (x * x).sum(1, keepdim=True) / k + EPS
    along = ((g * w) * x).sum(1, keepdim=True) / (k * r2)
    dx = (g * w - along * x) / r2.sqrt()
    if st["carried"] is not None:
        dx = dx + st["carried"].double()
    return {"x": dx, "gain": torch.einsum("rk,rk->k", g, x / r2.sqrt())}


def _exact_distill(st):
    c, T = st["case"], st["case"]["temperature"]
    rows, V = c["rows"], c["vocab"]
    back = st["id_map"].cpu().numpy() if st["id_map"] is not None else np.arange(V)
    ids, values = st["ids"].cpu().numpy(), st["values"].double().cpu().numpy()
    has = np.where(ids >= 0, back[np.maximum(ids, 0)], -1)
    with np.errstate(invalid="ignore", divide="ignore"):
        p = np.where(has >= 0, np.exp((values - values.max(1, keepdims=True)) / T), 0.0)
        p = p / np.maximum(p.sum(1, keepdims=True), 1e-300)
        entropy = -np.where(p > 0, p * np.log(p), 0.0).sum(1)
    dense = torch.zeros(rows, V, dtype=torch.float64, device="cuda")
    dense.scatter_add_(1, torch.from_numpy(np.maximum(has, 0)).long().cuda(), torch.from_numpy(p).cuda())
    lnq = torch.log_softmax(st["logits"].double() / T, 1)
    out = {}
    if c["mode"] != "grad":
        out["loss"] = -(dense * lnq).sum(1) - (torch.from_numpy(entropy).cuda() if c["kind"] == "kl" else 0.0)
    if c["mode"] != "loss":
        share = torch.from_numpy(p.sum(1)).cuda()[:, None]
        out["logits"] = lnq.exp_().mul_(share).sub_(dense).mul_(st["grad"].double()[:, None] / T)
    return out
