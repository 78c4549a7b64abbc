"""The operators of serving with a quantised key-value cache, as cases that can be timed: rotary positions and their gradient, writing
keys and values into a paged cache (rotating and quantising them on the way), reading positions of it back, and the attention of one
new token per sequence over it.

With `own` false, `run` computes them in elementary torch operations; with `own` true it calls the package.  Both get the same
tensors.  Shapes are those of the package's model configurations (4 / 2 heads of 64 in fp32; 32 / 8, 64 / 8 and 40 / 40 heads of 128 in
bf16; pages of 16), lengths and batches those of its workloads, or generic.

Layouts: x [tokens][heads][head_dim]; pools [pages][kv heads][page size][head_dim] of bf16, fp32, e4m3 or int8; scales fp32 [pages][kv
heads][page size], one for each token and head, of the two 8-bit formats; page_table int32 [sequences][pages per sequence].
"""
import math

import numpy as np
import torch

own = False

# largest magnitude of the 8-bit formats, and the least scale
TOP = {"e4m3": 448.0, "int8": 127.0}
FLOOR = 2.0 ** -120
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
BYTES = {"fp32": 4, "bf16": 2, "e4m3": 1, "int8": 1}


def _rotary(name, tokens, heads, hd, rot, layout, dtype, theta, scaling, grad):
    """heads: of the rotated view; the tokens lie 1.2 times as far apart, as the queries and keys of a fused projection do."""
    case = {"op": "rotary", "tokens": tokens, "heads": heads, "hd": hd, "rot": rot, "layout": layout, "dtype": dtype, "theta": theta,
            "scaling": scaling, "grad": grad}
    return {"name": name, **case} if name else case


def _append(name, seqs, lo, hi, behind, H, G, hd, rot, layout, dtype, fmt, page, theta, scaling, idle):
    """Sequences that hold `behind` tokens get lo .. hi new ones; `idle` rows belong to no sequence."""
    case = {"op": "append", "seqs": seqs, "lo": lo, "hi": hi, "behind": behind, "H": H, "G": G, "hd": hd, "rot": rot, "layout": layout,
            "dtype": dtype, "fmt": fmt, "page": page, "theta": theta, "scaling": scaling, "idle": idle}
    return {"name": name, **case} if name else case


def _read(name, seqs, lo, hi, G, hd, fmt, page, dtype):
    case = {"op": "read", "seqs": seqs, "lo": lo, "hi": hi, "G": G, "hd": hd, "fmt": fmt, "page": page, "dtype": dtype}
    return {"name": name, **case} if name else case


def _attend(name, seqs, lo, hi, H, G, hd, dtype, fmt, page, idle):
    """Lengths lo .. hi; the last `idle` sequences are empty."""
    case = {"op": "attend", "seqs": seqs, "lo": lo, "hi": hi, "H": H, "G": G, "hd": hd, "dtype": dtype, "fmt": fmt, "page": page, "idle": idle}
    return {"name": name, **case} if name else case


def listed():
    return [
        # the queries and keys of one new token of an 8B-shaped model: nothing but latency
        _rotary("rotary-token", 1, 40, 128, 128, "half", "bf16", 5e5, "none", False),
        # those of a 16k-token prompt, positions scaled for a context eight times the trained one
        _rotary("rotary-prompt", 16384, 40, 128, 128, "half", "bf16", 5e5, "wavelength", False),
        # the gradient in training: a 13B-shaped model with multi-head attention, fp32, half of each head rotated in neighbouring pairs
        _rotary("rotary-grad", 4096, 80, 128, 64, "interleaved", "fp32", 1e4, "rotations", True),
        # a decoding step of a serving batch of 64, two slots idle: one token each
        _append("append-step-b64", 64, 1, 1, 1024, 32, 8, 128, 128, "half", "bf16", "e4m3", 16, 5e5, "none", 2),
        # an odd chunk of a prompt of a multi-head-attention model, and the chunk read back as the next kernel wants it
        _append("append-chunk-int8", 1, 1001, 1001, 517, 40, 40, 128, 64, "interleaved", "bf16", "int8", 64, 1e4, "linear", 0),
        # a whole 16k-token prompt
        _append("append-prompt", 1, 16384, 16384, 0, 32, 8, 128, 128, "half", "bf16", "e4m3", 16, 5e5, "wavelength", 0),
        # a 16k-token prefix that a prompt shares, read back for its prefill
        _read("read-prefix", 1, 16384, 16384, 8, 128, "e4m3", 16, "bf16"),
        # a few short sequences of a small fp32 model
        _read("read-tiny-fp32", 3, 61, 400, 2, 64, "int8", 16, "fp32"),
        # one chat user
        _attend("attend-chat", 1, 613, 613, 32, 8, 128, "bf16", "e4m3", 16, 0),
        # one user with a long document
        _attend("attend-16k", 1, 16384, 16384, 32, 8, 128, "bf16", "e4m3", 16, 0),
        # a serving batch of ragged lengths, one slot idle
        _attend("attend-b64", 64, 256, 2048, 32, 8, 128, "bf16", "int8", 16, 1),
        # long contexts of a 70B-shaped model in an unquantised cache
        _attend("attend-long-70b", 16, 4097, 32768, 64, 8, 128, "bf16", "bf16", 16, 0),
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


def _heads(rng):
    """(dtype, query heads, KV heads, head_dim)"""
    return rng.choice([("bf16", 32, 8, 128), ("bf16", 32, 8, 128), ("bf16", 64, 8, 128), ("bf16", 40, 40, 128), ("bf16", 16, 2, 64),
                       ("bf16", 16, 8, 256), ("fp32", 4, 2, 64), ("fp32", 32, 8, 128)])


def _draw(rng):
    op = rng.choice(["rotary", "append", "read", "attend", "attend"])
    dtype, H, G, hd = _heads(rng)
    page = rng.choice([16, 16, 32, 64])
    layout, scaling = rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "wavelength", "rotations"])
    rot, theta = rng.choice([hd, hd, hd // 2]), rng.choice([1e4, 5e5])
    fmt = rng.choice(["e4m3", "e4m3", "int8", dtype])
    if op == "rotary":
        return _rotary("", _log(rng, 1, 16384), H + G, hd, rot, layout, dtype, theta, scaling, rng.random() < 0.4)
    if op == "append":
        seqs = _log(rng, 1, 64)
        lo = 1 if rng.random() < 0.5 else _log(rng, 1, 2048)
        return _append("", seqs, lo, lo if lo == 1 else lo + rng.randint(0, lo), _log(rng, 1, 2048) - 1, H, G, hd, rot, layout, dtype, fmt, page,
                       theta, scaling, rng.choice([0, 0, 1, 3]))
    if op == "read":
        lo = _log(rng, 1, 8192)
        return _read("", _log(rng, 1, 32), lo, lo + rng.randint(0, lo), G, hd, fmt, page, rng.choice([dtype, "bf16"]))
    seqs, lo = _log(rng, 1, 64), _log(rng, 1, 16384)
    return _attend("", seqs, lo, lo + rng.randint(0, lo), H, G, hd, dtype, fmt, page, rng.choice([0, 0, 1]) if seqs > 1 else 0)


# ------------------------------------------------------------------------------------------------ inputs
def _frequencies(rot, theta, scaling):
    """Radians a position turns each pair by (float64), and the factor on cosine and sine."""
    f = float(theta) ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "wavelength":    # kept above 4 turns in 8192 positions, an eighth below one, between them in proportion to the turns
        turns = 8192 * f / (2 * np.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * keep + f / 8.0 * (1 - keep), 1.0
    if scaling == "rotations":     # kept above 32 turns in 4096 positions, a quarter below one, between them in proportion to the pair's index
        def at(turns):
            return rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), rot - 1)
        keep = 1.0 - np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f * keep + f / 4.0 * (1 - keep), 0.1 * math.log(4.0) + 1.0
    return f, 1.0


def _lengths(lo, hi, n, seed):
    """Spread evenly over the range in a random order: another seed is other inputs, but not another amount of work."""
    return np.random.default_rng(seed).permutation(np.linspace(lo, hi, n).round().astype(np.int64))


def _keys(g, *shape):
    """Keys as trained models have them: some dimensions of a head several times larger than the others."""
    x = torch.randn(*shape, generator=g, device="cuda")
    gain = torch.ones(shape[-1], device="cuda")
    gain[torch.randperm(shape[-1], generator=g, device="cuda")[: max(1, shape[-1] // 32)]] = 6.0
    return x.mul_(gain)


def _quantised(x, fmt):
    """(codes, scales) of x float32 [..., hd]"""
    scale = (x.abs().amax(-1) * (1.0 / TOP[fmt])).clamp_min(FLOOR)
    y = (x * (1.0 / scale)[..., None]).clamp(-TOP[fmt], TOP[fmt])
    return (y.round() if fmt == "int8" else y).to(DTYPE[fmt]), scale


def _pool(x, fmt):
    return _quantised(x, fmt) if fmt in TOP else (x.to(DTYPE[fmt]), None)


def _table(g, per_seq):
    """Pages of the sequences in random order out of one pool: (table int32 [sequences][most], pages)."""
    total = int(sum(per_seq))
    ids = torch.randperm(total + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(per_seq), max(1, int(max(per_seq))), dtype=torch.int32)
    at, host = 0, ids.cpu()
    for s, n in enumerate(per_seq):
        table[s, : int(n)] = host[at: at + int(n)]
        at += int(n)
    return table.cuda(), total + 3


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"case": case, **{"rotary": _prepare_rotary, "append": _prepare_append, "read": _prepare_read, "attend": _prepare_attend}[case["op"]](case, seed, g)}


def _prepare_rotary(case, seed, g):
    T, n, hd = case["tokens"], case["heads"], case["hd"]
    wide = torch.randn(T, n + n // 5, hd, generator=g, device="cuda").to(DTYPE[case["dtype"]])
    f, m = _frequencies(case["rot"], case["theta"], case["scaling"])
    first = np.random.default_rng(seed).integers(0, 16384)       # a prompt's positions follow what the cache holds
    return {"x": wide[:, :n], "pos": torch.arange(first, first + T, dtype=torch.int32, device="cuda"), "freq": torch.from_numpy(f).cuda(), "mscale": m}


def _prepare_append(case, seed, g):
    H, G, hd, ps, fmt = case["H"], case["G"], case["hd"], case["page"], case["fmt"]
    lens = _lengths(case["lo"], case["hi"], case["seqs"], seed)
    table, pages = _table(g, [-(-(case["behind"] + n) // ps) for n in lens])
    seq = np.concatenate([np.full(n, s) for s, n in enumerate(lens)] + [np.full(case["idle"], -1)]).astype(np.int32)
    pos = np.concatenate([case["behind"] + np.arange(n) for n in lens] + [np.zeros(case["idle"])]).astype(np.int32)
    T = len(seq)
    qkv = torch.empty(T, H + 2 * G, hd, dtype=DTYPE[case["dtype"]], device="cuda")
    qkv[:, :H] = torch.randn(T, H, hd, generator=g, device="cuda")
    qkv[:, H: H + G] = _keys(g, T, G, hd)
    qkv[:, H + G:] = torch.randn(T, G, hd, generator=g, device="cuda")
    f, m = _frequencies(case["rot"], case["theta"], case["scaling"])
    st = {"qkv": qkv, "seq": torch.from_numpy(seq).cuda(), "pos": torch.from_numpy(pos).cuda(), "table": table, "freq": torch.from_numpy(f).cuda(), "mscale": m,
          "live": torch.from_numpy(np.flatnonzero(seq >= 0)).cuda()}
    for x in ("k", "v"):
        st[x + "_pool"] = torch.zeros(pages, G, ps, hd, dtype=torch.uint8 if fmt in TOP else DTYPE[fmt], device="cuda")
        st[x + "_pool"] = st[x + "_pool"].view(DTYPE[fmt])
        st[x + "_scale"] = torch.zeros(pages, G, ps, device="cuda") if fmt in TOP else None
    return st


def _prepare_pools(case, per_seq, g):
    table, pages = _table(g, per_seq)
    kp, ks = _pool(_keys(g, pages, case["G"], case["page"], case["hd"]), case["fmt"])
    vp, vs = _pool(torch.randn(pages, case["G"], case["page"], case["hd"], generator=g, device="cuda"), case["fmt"])
    return {"table": table, "k_pool": kp, "k_scale": ks, "v_pool": vp, "v_scale": vs}


def _prepare_read(case, seed, g):
    lens = _lengths(case["lo"], case["hi"], case["seqs"], seed)
    seq = np.concatenate([np.full(n, s) for s, n in enumerate(lens)]).astype(np.int32)
    pos = np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
    return {"seq": torch.from_numpy(seq).cuda(), "pos": torch.from_numpy(pos).cuda(), **_prepare_pools(case, -(-lens // case["page"]), g)}


def _prepare_attend(case, seed, g):
    lens = _lengths(case["lo"], case["hi"], case["seqs"], seed)
    if case["idle"]:
        lens[-case["idle"]:] = 0
    q = torch.randn(case["seqs"], case["H"], case["hd"], generator=g, device="cuda").to(DTYPE[case["dtype"]])
    return {"q": q, "len": torch.from_numpy(lens.astype(np.int32)).cuda(), **_prepare_pools(case, -(-lens // case["page"]), g)}


# ------------------------------------------------------------------------------------------------ a pass
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _cos_sin(st):
    """float32 [rows][1][pairs]; the angles are formed in 64 bits, as positions times frequencies go to thousands of turns"""
    a = st["pos"].double()[:, None, None] * st["freq"]
    return a.cos().float() * st["mscale"], a.sin().float() * st["mscale"]


def _turned(x, cos, sin, layout):
    """x float32 [rows][heads][hd], its first dimensions rotated by pairs."""
    n = cos.shape[-1]
    if layout == "half":
        a, b = x[..., :n], x[..., n: 2 * n]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * n:]], -1)
    a, b = x[..., 0: 2 * n: 2], x[..., 1: 2 * n: 2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., 2 * n:]], -1)


def _plain_rotary(st):
    cos, sin = _cos_sin(st)
    return _turned(st["x"].float(), cos, -sin if st["case"]["grad"] else sin, st["case"]["layout"]).to(st["x"].dtype)


def _plain_append(st):
    c = st["case"]
    H, G, ps, fmt, live = c["H"], c["G"], c["page"], c["fmt"], st["live"]
    cos, sin = _cos_sin(st)
    qk = _turned(st["qkv"][:, : H + G].float(), cos, sin, c["layout"])
    pos, seq = st["pos"][live].long(), st["seq"][live].long()
    page, off = st["table"][seq, pos // ps].long(), pos % ps
    back = {}
    for x, rows in (("k", qk[:, H:]), ("v", st["qkv"][:, H + G:].float())):
        code, scale = _pool(rows[live], fmt)
        as_bytes = torch.uint8 if fmt in TOP else DTYPE[fmt]
        st[x + "_pool"].view(as_bytes)[page, :, off] = code.view(as_bytes)
        if scale is not None:
            st[x + "_scale"][page, :, off] = scale
            back[x] = torch.zeros(rows.shape, device="cuda")
            back[x][live] = code.float() * scale[..., None]
    return _appended(st, qk[:, :H].to(st["qkv"].dtype), {x: t.to(torch.bfloat16) for x, t in back.items()})


def _appended(st, q, back):
    """What a pass of "append" returns: the queries; the pools and scales, or for whole-number codes the values that they stand for."""
    if st["case"]["fmt"] == "int8":
        return {"q": q, "k": back["k"], "v": back["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    return {"q": q, "k_pool": st["k_pool"], "v_pool": st["v_pool"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _plain_read(st):
    c = st["case"]
    seq, pos = st["seq"].long(), st["pos"].long()
    page, off = st["table"][seq, pos // c["page"]].long(), pos % c["page"]
    out = {}
    for x in ("k", "v"):
        rows = st[x + "_pool"].view(torch.uint8)[page, :, off].view(DTYPE[c["fmt"]]) if c["fmt"] in TOP else st[x + "_pool"][page, :, off]
        rows = rows.float()
        out[x] = (rows * st[x + "_scale"][page, :, off][..., None] if c["fmt"] in TOP else rows).to(DTYPE[c["dtype"]])
    return out


def _plain_attend(st):
    c = st["case"]
    B, H, G, hd, ps = c["seqs"], c["H"], c["G"], c["hd"], c["page"]
    table = st["table"].long()
    n = table.shape[1] * ps

    def rows(x):
        t = st[x + "_pool"].view(torch.uint8)[table].view(DTYPE[c["fmt"]]) if c["fmt"] in TOP else st[x + "_pool"][table]
        t = t.float()
        if c["fmt"] in TOP:
            t = t * st[x + "_scale"][table][..., None]
        return t.transpose(1, 2).reshape(B, G, n, hd)

    hidden = torch.arange(n, device="cuda")[None, :] >= st["len"][:, None]
    empty = (st["len"] == 0)[:, None]
    s = torch.matmul(st["q"].float().view(B, G, H // G, hd), rows("k").transpose(2, 3)).view(B, H, n) * hd ** -0.5
    s = s.masked_fill(hidden[:, None], -math.inf)
    top = s.amax(-1).masked_fill(empty, 0.0)
    p = (s - top[..., None]).exp()
    total = p.sum(-1)
    v = rows("v").masked_fill(hidden[:, None, :, None], 0.0)
    out = torch.matmul(p.view(B, G, H // G, n), v).view(B, H, hd) / total.masked_fill(empty, 1.0)[..., None]
    return {"out": out.to(st["q"].dtype), "lse": total.log() + top}


_run_plain = {"rotary": _plain_rotary, "append": _plain_append, "read": _plain_read, "attend": _plain_attend}


def _own_rotary(st):
    from paper_2503_01840_b200 import binding as sb
    f = sb.rotary_backward if st["case"]["grad"] else sb.rotary
    return f(st["x"], st["pos"], st["freq"], layout=st["case"]["layout"], mscale=st["mscale"])


def _own_append(st):
    from paper_2503_01840_b200 import binding as sb
    c, qkv = st["case"], st["qkv"]
    H, G = c["H"], c["G"]
    q = sb.kv_append(qkv[:, H: H + G], qkv[:, H + G:], st["k_pool"], st["v_pool"], st["table"], st["seq"], st["pos"], k_scale=st["k_scale"],
                     v_scale=st["v_scale"], q=qkv[:, :H], inv_freq=st["freq"], layout=c["layout"], mscale=st["mscale"])
    back = {}
    if c["fmt"] == "int8":
        back["k"], back["v"] = sb.kv_read(st["k_pool"], st["v_pool"], st["table"], st["seq"], st["pos"], k_scale=st["k_scale"], v_scale=st["v_scale"])
    return _appended(st, q, back)


def _own_read(st):
    from paper_2503_01840_b200 import binding as sb
    k, v = sb.kv_read(st["k_pool"], st["v_pool"], st["table"], st["seq"], st["pos"], k_scale=st["k_scale"], v_scale=st["v_scale"],
                      dtype=DTYPE[st["case"]["dtype"]])
    return {"k": k, "v": v}


def _own_attend(st):
    from paper_2503_01840_b200 import binding as sb
    out, lse = sb.decode_attention(st["q"], st["k_pool"], st["v_pool"], st["table"], st["len"], k_scale=st["k_scale"], v_scale=st["v_scale"],
                                   want_lse=True)
    return {"out": out, "lse": lse}


_run_own = {"rotary": _own_rotary, "append": _own_append, "read": _own_read, "attend": _own_attend}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, op = case, case["op"]
    if op == "rotary":
        n = c["tokens"] * c["heads"] * c["hd"]
        return {"bytes": 2 * n * BYTES[c["dtype"]] + 4 * c["tokens"] + 4 * c["rot"], "flops": 3 * c["tokens"] * c["heads"] * c["rot"]}
    a_row = c["G"] * (c["hd"] * BYTES[c["fmt"]] + (4 if c["fmt"] in TOP else 0))          # a token's keys, or its values, in the cache
    lens = np.linspace(c["lo"], c["hi"], c["seqs"]).round()
    if op == "append":
        T, live = float(lens.sum()) + c["idle"], float(lens.sum())
        e = BYTES[c["dtype"]]
        nbytes = T * ((2 * c["H"] + 2 * c["G"]) * c["hd"] * e + 8) + live * 2 * a_row
        if c["fmt"] == "int8":
            nbytes += live * 2 * a_row + T * 2 * c["G"] * c["hd"] * 2
        return {"bytes": nbytes, "flops": T * (3 * (c["H"] + c["G"]) * c["rot"] + (4 * c["G"] * c["hd"] if c["fmt"] in TOP else 0))}
    tokens = float(lens[: c["seqs"] - c["idle"]].sum()) if op == "attend" else float(lens.sum())
    if op == "read":
        return {"bytes": tokens * (2 * a_row + 2 * c["G"] * c["hd"] * BYTES[c["dtype"]] + 8), "flops": tokens * 2 * c["G"] * c["hd"]}
    return {"bytes": tokens * 2 * a_row + c["seqs"] * c["H"] * (2 * c["hd"] * BYTES[c["dtype"]] + 4), "flops": 4 * tokens * c["H"] * c["hd"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"rotary": _exact_rotary, "append": _exact_append, "read": _exact_read, "attend": _exact_attend}[case["op"]](st)


def _rotate64(x, st, layout, sign=1.0):
    """As complex numbers: a pair (a, b) is a + bi, and a position multiplies it by m exp(i angle)."""
    w = torch.polar(torch.full((), st["mscale"], dtype=torch.float64, device="cuda"), sign * torch.outer(st["pos"].double(), st["freq"]))[:, None]
    n = w.shape[-1]
    y = x.double()
    pairs = y[..., : 2 * n].unflatten(-1, (2, n) if layout == "half" else (n, 2))
    pairs = pairs.transpose(-1, -2) if layout == "half" else pairs
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * w)
    z = z.transpose(-1, -2) if layout == "half" else z
    y[..., : 2 * n] = z.reshape(y[..., : 2 * n].shape)
    return y


def _exact_rotary(st):
    return _rotate64(st["x"].clone(), st, st["case"]["layout"], -1.0 if st["case"]["grad"] else 1.0)


def _exact_append(st):
    """Codes as the reals that they round."""
    c, qkv = st["case"], st["qkv"]
    H, G = c["H"], c["G"]
    out = {"q": _rotate64(qkv[:, :H].clone(), st, c["layout"])}
    new = {"k": _rotate64(qkv[:, H: H + G].clone(), st, c["layout"]), "v": qkv[:, H + G:].double()}
    seq, pos, table = st["seq"].cpu().numpy(), st["pos"].cpu().numpy(), st["table"].cpu().numpy()
    live = np.flatnonzero(seq >= 0)
    page = torch.from_numpy(table[seq[live], pos[live] // c["page"]].astype(np.int64)).cuda()
    off = torch.from_numpy((pos[live] % c["page"]).astype(np.int64)).cuda()
    live = torch.from_numpy(live).cuda()
    for x, rows in new.items():
        scale = None
        if c["fmt"] in TOP:
            scale = rows[live].abs().amax(-1) / TOP[c["fmt"]]
            out[x + "_scale"] = torch.zeros(st[x + "_scale"].shape, dtype=torch.float64, device="cuda")
            out[x + "_scale"][page, :, off] = scale
        else:
            out[x + "_scale"] = None
        if c["fmt"] == "int8":
            out[x] = torch.zeros_like(rows)
            out[x][live] = rows[live]
        else:
            out[x + "_pool"] = torch.zeros(st[x + "_pool"].shape, dtype=torch.float64, device="cuda")
            out[x + "_pool"][page, :, off] = rows[live] / scale[..., None] if scale is not None else rows[live]
    return out


def _exact_read(st):
    c, out = st["case"], {}
    seq, pos, table = st["seq"].cpu().numpy(), st["pos"].cpu().numpy(), st["table"].cpu().numpy()
    page = torch.from_numpy(table[seq, pos // c["page"]].astype(np.int64)).cuda()
    off = torch.from_numpy((pos % c["page"]).astype(np.int64)).cuda()
    for x in ("k", "v"):
        out[x] = st[x + "_pool"].double()[page, :, off]
        if c["fmt"] in TOP:
            out[x] *= st[x + "_scale"].double()[page, :, off][..., None]
    return out


def _exact_attend(st):
    c = st["case"]
    H, G, hd = c["H"], c["G"], c["hd"]
    out = torch.zeros(c["seqs"], H, hd, dtype=torch.float64, device="cuda")
    lse = torch.full((c["seqs"], H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["len"].tolist()):
        if n == 0:
            continue
        pages = st["table"][b, : -(-n // c["page"])].long()
        for g in range(G):
            k, v = ((st[x + "_pool"][:, g].view(torch.uint8)[pages].view(DTYPE[c["fmt"]]) if c["fmt"] in TOP else st[x + "_pool"][:, g][pages]).double()
                    .reshape(-1, hd)[:n] for x in ("k", "v"))
            if c["fmt"] in TOP:
                k, v = (t * st[x + "_scale"][:, g][pages].double().reshape(-1)[:n, None] for x, t in (("k", k), ("v", v)))
            heads = slice(g * (H // G), (g + 1) * (H // G))
            s = st["q"][b, heads].double() @ k.T / math.sqrt(hd)
            lse[b, heads] = torch.logsumexp(s, -1)
            out[b, heads] = (s - lse[b, heads, None]).exp() @ v
    return {"out": out, "lse": lse}
