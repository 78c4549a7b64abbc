"""Embedding lookup, norms of a residual sum and distillation from a teacher's top logits, with their gradients, against plain forms in 64 bits on the CPU."""
import ctypes as C
import math
import zlib

import pytest
import torch

from paper_2503_01840_b200 import binding as sb

gpu = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}       # half a step of a rounding, relative (bf16: of its eight bits)
E = 2.0 ** -24
FLOOR = 2.0 ** -120


def gen(*seed):
    return torch.Generator().manual_seed(zlib.crc32(repr(seed).encode()))


def randn(g, *shape):
    return torch.randn(*shape, generator=g)


def strided(x, more, device="cuda"):
    """x [rows][columns] as a view of wider rows, one element in from an allocation's beginning where `more` is odd"""
    wide = torch.zeros(x.shape[0], x.shape[1] + more, dtype=x.dtype, device=device)
    view = wide[:, more % 2: more % 2 + x.shape[1]]
    view.copy_(x)
    return view


def within(got, want, tol):
    """Element by element; where want is infinite or NaN, got is the same."""
    got, fine = got.cpu().double(), want.isfinite()
    assert got.shape == want.shape
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()])
    off = ((got - want).abs() - tol)[fine]
    assert off.numel() == 0 or off.max() <= 0, float(off.max())


# ------------------------------------------------------------------------------------------------ embedding
def lookup(ids, w, scale):
    out = torch.zeros(len(ids), w.shape[1], dtype=torch.float64)
    live = (ids >= 0) & (ids < len(w))
    out[live] = w.double()[ids[live].long()] * scale
    return out


@gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("T,V,k", [(1, 1, 1), (1, 1000, 4096), (3, 7, 2), (129, 50, 250), (64, 300, 1002), (33, 5003, 1000), (700, 900, 136), (5, 64, 8192), (2, 9, 20000)])
def test_embedding(dtype, out, T, V, k):
    """Ids of both sizes, padding, strided weights and outputs, a scale that is no power of two."""
    g = gen(T, V, k)
    w, ids = randn(g, V, k).to(DT[dtype]), torch.randint(0, V, (T,), generator=g)
    ids[torch.rand(T, generator=g) < 0.2] = -1
    want = lookup(ids, w, 1.7)
    tol = want.abs() * (2 * E + HALF[out])             # the scale's own rounding, the product's, the output's
    a = sb.embedding(ids.cuda(), w.cuda(), scale=1.7, dtype=DT[out])
    assert a.dtype == DT[out] and a.is_contiguous()
    within(a, want, tol)
    for more in (8, 3):
        room = torch.full((T, k + 2 * more), 5.0, dtype=DT[out], device="cuda")
        sb.embedding(ids.int().cuda(), strided(w, more), scale=1.7, out=room[:, more: more + k])
        assert torch.equal(room[:, more: more + k], a) and (room[:, :more] == 5).all() and (room[:, more + k:] == 5).all()
    assert torch.equal(sb.embedding(ids.cuda(), w.cuda()).cpu(), lookup(ids, w, 1.0).to(DT[dtype]))


@gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("T,V,k,ids", [(1, 1, 1, "any"), (7, 5, 3, "any"), (8, 3, 8, "same"), (9, 3, 8, "same"), (65, 2, 130, "any"), (300, 4097, 64, "any"), (1000, 300, 250, "few"),
                                       (4096, 600, 72, "same"), (4200, 40000, 16, "few"), (5000, 9, 40, "any"), (33, 128256, 24, "any"), (260, 70, 1000, "few"), (64, 50, 4096, "any"),
                                       (31, 40, 20, "none"), (6000, 2000000, 4, "few")])
def test_embedding_gradient(dtype, out, T, V, k, ids):
    """Runs of every length, inside chunks and over many; added to what is there; rows without a token; the same bits every time."""
    g = gen(T, V, k, ids)
    grad = randn(g, T, k).to(DT[dtype])
    i = {"any": lambda: torch.randint(0, V, (T,), generator=g), "same": lambda: torch.full((T,), V - 1), "none": lambda: torch.full((T,), -1),
         "few": lambda: (torch.rand(T, generator=g) ** 6 * V).long().clamp(0, V - 1)}[ids]()
    if ids == "any":
        i[torch.rand(T, generator=g) < 0.1] = -1
    live = i >= 0
    want = torch.zeros(V, k, dtype=torch.float64).index_add_(0, i[live], grad[live].double()) * 1.7
    mass = torch.zeros(V, k, dtype=torch.float64).index_add_(0, i[live], grad[live].double().abs()) * 1.7
    n = torch.bincount(i[live], minlength=V)[:, None].double()
    tol = mass * (n + 2) * E + want.abs() * HALF[out]
    got = sb.embedding_backward(grad.cuda(), i.cuda(), V, scale=1.7, dtype=DT[out])
    assert got.dtype == DT[out]
    within(got, want, tol)
    assert not got[(n[:, 0] == 0).cuda()].any()
    again = sb.embedding_backward(strided(grad, 5), i.int().cuda(), V, scale=1.7, out=torch.full((V, k + 3), 5.0, dtype=DT[out], device="cuda")[:, 1:1 + k])
    assert torch.equal(again, got)
    had = randn(g, V, k).to(DT[out])
    more = sb.embedding_backward(grad.cuda(), i.cuda(), V, scale=1.7, out=had.cuda(), accumulate=True)
    total = had.double() + want
    within(more, total, mass * (n + 2) * E + total.abs() * (E + HALF[out]))
    assert torch.equal(more.cpu()[n[:, 0] == 0], had[n[:, 0] == 0])
    one = sb.embedding_backward(grad[:1].cuda().expand(T, k), i.cuda(), V, dtype=DT[out])               # rows that lie in one place
    within(one, n * grad[0].double(), n * grad[0].double().abs() * (n * E + HALF[out]))


@gpu
def test_embedding_of_no_tokens_and_bad_ids():
    w = torch.ones(10, 16, device="cuda")
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert sb.embedding(none, w).shape == (0, 16)
    assert not sb.embedding_backward(torch.zeros(0, 16, device="cuda"), none, 10).any()
    keep = torch.ones(10, 16, device="cuda")
    assert torch.equal(sb.embedding_backward(torch.zeros(0, 16, device="cuda"), none, 10, out=keep, accumulate=True), w)
    for bad in (10, -2, 1 << 40, -(1 << 33), (1 << 32) + 3):
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        ids = torch.tensor([3, bad, 4], device="cuda")
        out = sb.embedding(ids, w, status=status)
        assert out[0].all() and out[2].all() and not out[1].any() and status.tolist()[:3] == [2, 64, 1]
        status.zero_()
        got = sb.embedding_backward(torch.ones(3, 16, device="cuda"), ids, 10, status=status)
        assert got.sum() == 32 and got[3].all() and got[4].all() and status.tolist()[:3] == [2, 64, 1]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_embedding_autograd(dtype):
    """Through a sum (whose gradient is expanded) and a product; fp32 rows of a bf16 table; by differences: the map is linear."""
    g = gen(3)
    w = randn(g, 50, 40).to(DT[dtype]).cuda().requires_grad_()
    ids = torch.randint(-1, 50, (77,), generator=g).cuda()
    c = randn(g, 77, 40).cuda()
    y = sb.embedding(ids, w, 2.0, torch.float32)
    with torch.no_grad():
        assert not sb.embedding(ids, w, 2.0, torch.float32).requires_grad
    assert y.requires_grad
    (y * c).sum().backward()
    assert torch.equal(w.grad, sb.embedding_backward(c, ids, 50, 2.0, DT[dtype]))
    d = randn(g, 50, 40).to(DT[dtype]).cuda()
    moved = (sb.embedding(ids, d, 2.0, torch.float32).double() * c.double()).sum()
    exact = sb.embedding_backward(c, ids, 50, 2.0, torch.float32)
    assert abs(float(moved - (exact.double() * d.double()).sum())) <= 77 * 4 * E * float((sb.embedding(ids, d.abs(), 2.0, torch.float32).double() * c.double().abs()).sum())
    w.grad = None
    sb.embedding(ids, w).sum().backward()
    assert torch.equal(w.grad[:, 0].cpu().double(), torch.bincount(ids[ids >= 0].cpu(), minlength=50).double())
    with pytest.raises(ValueError):
        sb.embedding(ids, w, out=torch.empty(77, 40, dtype=DT[dtype], device="cuda"))


# ------------------------------------------------------------------------------------------------ norm
def normed(x, res, gain, eps):
    s = x.double() + (res.double() if res is not None else 0.0)
    return s, s / (s.square().mean(1, keepdim=True) + eps).sqrt() * gain.double()


def norm_error(y, k):
    """Relative: the sum of squares (a thread adds k / 256 of them, then a tree), half of that in the root; the root's two last places; sum, two products."""
    return y.abs() * E * ((k / 256 + 16) / 2 + 4 + 4)


TYPES = [("bf16", None, "bf16", "bf16"), ("bf16", "bf16", "bf16", "bf16"), ("fp32", "fp32", "bf16", "bf16"), ("fp32", None, "fp32", "fp32"), ("bf16", "fp32", "fp32", "fp32"),
         ("fp32", "bf16", "bf16", "fp32")]
SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 64), (130, 256), (2, 250), (33, 1000), (9, 1002), (65, 1024), (4, 5120), (300, 136), (7, 8192), (2, 12000), (3, 20001), (64, 2048)]


@gpu
@pytest.mark.parametrize("x,res,gain,out", TYPES)
@pytest.mark.parametrize("rows,k", SHAPES)
def test_norm(x, res, gain, out, rows, k):
    """Contiguous, strided, off their alignment; in place of the residual and of x."""
    g = gen(rows, k)
    xs, w = randn(g, rows, k).to(DT[x]), (1 + 0.3 * randn(g, k)).to(DT[gain])
    rs = (20 * randn(g, rows, k)).to(DT[res]) if res else None
    s, y = normed(xs, rs, w, 1e-5)
    tol = norm_error(y, k) + y.abs() * HALF[out]
    cuda = lambda t: None if t is None else t.cuda()
    got = sb.rms_norm(xs.cuda(), w.cuda(), 1e-5, cuda(rs), DT[out])
    a, total = got if res else (got, None)
    within(a, y, tol)
    if res:
        assert total.dtype == DT[res]
        within(total, s, s.abs() * (E + HALF[res]))
    for more in (8, 3):
        r = strided(rs, more) if res else None
        b = sb.rms_norm(strided(xs, more), w.cuda(), 1e-5, r, DT[out], sum_out=r)
        b, t = b if res else (b, None)
        within(b, y, tol)
        if res:
            assert t is r and torch.equal(t, total)
    if res == x:
        into = xs.cuda()
        b, t = sb.rms_norm(into, w.cuda(), 1e-5, cuda(rs), DT[out], sum_out=into)
        assert torch.equal(b, a) and torch.equal(into, total) and t is into
    if rows > 1:                                         # one row for all
        wide = sb.rms_norm(xs.cuda()[1:2].expand(rows, k), w.cuda(), 1e-5, None, DT[out])
        assert torch.equal(wide, sb.rms_norm(xs.cuda()[1:2], w.cuda(), 1e-5, None, DT[out]).expand(rows, k))


@gpu
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("x,res", [("bf16", "bf16"), ("fp32", None), ("fp32", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("rows,k,group", [(1, 4096, 0), (3, 7, 0), (33, 1000, 32), (9, 1002, 128), (65, 1024, 128), (4, 5120, 256), (5, 5120, 0), (40, 256, 64), (7, 8192, 32), (2, 12000, 128),
                                          (3, 20001, 0), (3, 96, 16), (2, 480, 48), (5, 130, 128), (6, 64, 512), (3, 8184, 0)])
def test_norm_in_8_bits(fmt, x, res, rows, k, group):
    """What the codes and scales stand for is within half a step of the norm; a group of zeros; one far above the others."""
    g = gen(rows, k, group)
    top = 448.0 if fmt == "e4m3" else 127.0
    xs, w = randn(g, rows, k).to(DT[x]), (1 + 0.3 * randn(g, k)).to(torch.bfloat16)
    xs[0, : min(k, 128)] = 0
    if k > 300:
        xs[-1, 300] = 1000.0
    rs = randn(g, rows, k).to(DT[res]) if res else None
    if res:
        rs[0, : min(k, 128)] = 0
    s, y = normed(xs, rs, w, 1e-5)
    n = group or k
    groups = -(-k // n)
    amax = torch.stack([y[:, i * n: (i + 1) * n].abs().amax(1) for i in range(groups)], 1)
    scale = (amax / top).clamp_min(FLOOR)
    for more in (0, 3):
        view = (lambda t: strided(t, more)) if more else (lambda t: t.cuda())
        got = sb.rms_norm(view(xs), w.cuda(), 1e-5, view(rs) if res else None, DT[fmt], group)
        codes, sc = got[:2]
        assert codes.dtype == DT[fmt] and codes.is_contiguous() and sc.shape == (rows, groups)
        rel = norm_error(torch.ones(1, dtype=torch.float64), k)
        within(sc, scale, scale * (rel + 3 * E))
        wide = scale.repeat_interleave(n, 1)[:, :k]
        value = codes.cpu().double() * sc.cpu().double().repeat_interleave(n, 1)[:, :k]
        # half a step: of e4m3 2^-4 of the value or 2^-10 scales below its normal numbers, of int8 half a scale; a scale that is off shifts the value by as much of itself
        step = torch.maximum(y.abs() * 2.0 ** -4, wide * 2.0 ** -10) if fmt == "e4m3" else wide * 0.5
        within(value, y, step * (1 + 2.0 ** -10) + y.abs() * (rel + 8 * E) * 8)
        assert codes.cpu().float().abs().max() <= top
        if res:
            within(got[2], s, s.abs() * (E + HALF[res]))


@gpu
@pytest.mark.parametrize("k", [96, 1002, 4096])
def test_norm_of_rows_that_are_no_numbers(k):
    """Zeros, infinities, NaN, numbers whose squares overflow; the rows beside them are as they would be."""
    g = gen(k)
    x = randn(g, 6, k)
    x[1] = 0
    x[2, 5] = math.inf
    x[3, 7] = math.nan
    x[4] *= 1e30
    w = torch.ones(k)
    y = sb.rms_norm(x.cuda(), w.cuda(), 1e-5)
    within(y[[0, 5]], normed(x[[0, 5]], None, w, 1e-5)[1], norm_error(normed(x[[0, 5]], None, w, 1e-5)[1], k) * 2)
    assert not y[1].any() and y[2, 5].isnan() and y[2, :5].abs().max() == 0 and y[3].isnan().all() and not y[4].any()
    for fmt, group in (("e4m3", 0), ("int8", 32), ("e4m3", 128)):
        codes, scale = sb.rms_norm(x.cuda(), w.cuda(), 1e-5, dtype=DT[fmt], group=group)
        value = codes.float() * scale.repeat_interleave(group or k, 1)[:, :k]
        assert value[3].isnan().all() and value[2, 5].isnan() and not value[1].any() and not value[4].any() and value[[0, 5]].isfinite().all()
    bf = sb.rms_norm(x.bfloat16().cuda(), w.bfloat16().cuda(), 1e-5)
    assert bf[3].isnan().all() and not bf[1].any()


def norm_gradient(g, s, gain, eps, carried):
    s, gw = s.double(), g.double() * gain.double()
    u = (s.square().mean(1, keepdim=True) + eps).rsqrt()
    h = s * u
    dx = u * (gw - h * (gw * h).mean(1, keepdim=True))
    size = u * (gw.abs() + h.abs() * (gw * h).abs().mean(1, keepdim=True))
    if carried is not None:
        dx, size = dx + carried.double(), size + carried.double().abs()
    return dx, size, (g.double() * h).sum(0), (g.double() * h).abs().sum(0)


@gpu
@pytest.mark.parametrize("grad,x,gain,carried", [("bf16", "bf16", "bf16", True), ("bf16", "bf16", "bf16", False), ("fp32", "fp32", "fp32", True), ("bf16", "fp32", "bf16", True),
                                                 ("fp32", "bf16", "fp32", False)])
@pytest.mark.parametrize("rows,k", SHAPES + [(2000, 64), (700, 1000)])
def test_norm_gradient(grad, x, gain, carried, rows, k):
    g = gen(rows, k, 1)
    dy, s, w = randn(g, rows, k).to(DT[grad]), (3 * randn(g, rows, k)).to(DT[x]), (1 + 0.3 * randn(g, k)).to(DT[gain])
    c = randn(g, rows, k).to(DT[x]) if carried else None
    dx, size, dw, wsize = norm_gradient(dy, s, w, 1e-5, c)
    # sums of k / 256 and a tree in the two means; a dozen roundings beside them; of the rows' sum, each row's h and as many additions as rows
    tol, wtol = size * E * (2 * (k / 256 + 16) + 16), wsize * E * (rows + (k / 256 + 16) + 16)
    a, aw = sb.rms_norm_backward(dy.cuda(), s.cuda(), w.cuda(), 1e-5, c.cuda() if carried else None)
    assert a.dtype == DT[x] and aw.dtype == DT[gain] and aw.shape == (k,)
    within(a, dx, tol + dx.abs() * HALF[x])
    within(aw, dw, wtol + dw.abs() * HALF[gain])
    b, bw = sb.rms_norm_backward(strided(dy, 3), strided(s, 8), w.cuda(), 1e-5, strided(c, 5) if carried else None, dtype=torch.float32)
    within(b, dx, tol + dx.abs() * E)
    within(bw, dw, wtol + dw.abs() * HALF[gain])
    again = sb.rms_norm_backward(dy.cuda(), s.cuda(), w.cuda(), 1e-5, c.cuda() if carried else None)
    assert torch.equal(again[0], a) and torch.equal(again[1], aw)


@gpu
def test_norm_gradient_by_differences():
    """<c, y(s + h d) - y(s - h d)> / 2 h against <dx, d>.  y is of degree 0 in s: along d its third derivative is below 15 |gain| (|d| / |s|)^3 a row (Euclidean), so the quotient is off by
    h^2 / 6 times |c| that, and by the two calls' errors over 2 h."""
    g = gen(5)
    rows, k, h = 6, 128, 2.0 ** -6
    s, c, d, w = randn(g, rows, k), randn(g, rows, k), randn(g, rows, k), 1 + 0.3 * randn(g, k)
    y = lambda t: sb.rms_norm(t.cuda(), w.cuda(), 1e-6).cpu().double()
    up, down = s + h * d, s - h * d
    step = (up.double() - down.double()) / (2 * h)
    quotient = (c.double() * (y(up) - y(down))).sum(1) / (2 * h)
    dx, dw = sb.rms_norm_backward(c.cuda(), s.cuda(), w.cuda(), 1e-6)
    norm = lambda t: t.double().norm(dim=1)
    third = 15 * math.sqrt(k) * w.abs().max().double() * (norm(step) / norm(s)) ** 3
    calls = (c.double().abs() * (norm_error(y(up), k) + norm_error(y(down), k))).sum(1) / (2 * h)
    assert ((quotient - (dx.cpu().double() * step).sum(1)).abs() <= h * h / 6 * norm(c) * third + calls + 1e-6 * norm(c) * norm(step)).all()
    # linear in the gain
    e = randn(g, k)
    moved = sb.rms_norm(s.cuda(), e.cuda(), 1e-6).cpu().double()
    assert abs(float((c.double() * moved).sum() - (dw.cpu().double() * e.double()).sum())) <= 64 * E * float((c.double() * moved).abs().sum() * 2 + 1)


@gpu
@pytest.mark.parametrize("x,res", [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp32", None)])
def test_norm_autograd(x, res):
    """Both outputs used, one of them, or the other; the same numbers as by hand; refusals."""
    g = gen(11)
    rows, k = 37, 200
    a = randn(g, rows, k).to(DT[x]).cuda().requires_grad_()
    r = randn(g, rows, k).to(DT[res]).cuda().requires_grad_() if res else None
    w = (1 + 0.1 * randn(g, k)).to(DT[x]).cuda().requires_grad_()
    cy, cs = randn(g, rows, k).cuda(), randn(g, rows, k).cuda()
    wide = torch.float32 if "fp32" in (x, res) else torch.bfloat16
    for use_y, use_s in ((1, 1), (1, 0), (0, 1)) if res else ((1, 0),):
        for t in (a, r, w):
            if t is not None:
                t.grad = None
        got = sb.rms_norm(a, w, 1e-5, r, torch.float32)
        y, s = got if res else (got, None)
        with torch.no_grad():
            plain = sb.rms_norm(a, w, 1e-5, r, torch.float32)
        assert torch.equal(y, plain[0] if res else plain) and y.requires_grad
        ((y * cy).sum() * use_y + ((s * cs.to(s.dtype)).sum() * use_s if use_s else 0)).backward() if use_y else (s * cs.to(s.dtype)).sum().backward()
        if use_y:
            dx, dw = sb.rms_norm_backward(cy, s.detach() if res else a.detach(), w.detach(), 1e-5, cs.to(s.dtype) if use_s else None, wide)
        else:
            dx, dw = cs.to(s.dtype), torch.zeros_like(w)
        assert torch.equal(a.grad, dx.to(DT[x])) and torch.equal(w.grad, dw)
        if res:
            assert torch.equal(r.grad, dx.to(DT[res]))
    sb.rms_norm(a, w, 1e-5, r)[0].sum().backward()
    with pytest.raises(ValueError):
        sb.rms_norm(a, w, 1e-5, r, torch.int8)
    if res:
        with pytest.raises(ValueError):
            sb.rms_norm(a, w, 1e-5, r, sum_out=r.detach())


@gpu
def test_norm_of_no_rows():
    w = torch.ones(64, device="cuda")
    assert sb.rms_norm(torch.zeros(0, 64, device="cuda"), w).shape == (0, 64)
    codes, scale, s = sb.rms_norm(torch.zeros(0, 64, device="cuda"), w, residual=torch.zeros(0, 64, device="cuda"), dtype=torch.int8, group=32)
    assert codes.shape == s.shape == (0, 64) and scale.shape == (0, 2)
    dx, dw = sb.rms_norm_backward(torch.zeros(0, 64, device="cuda"), torch.zeros(0, 64, device="cuda"), w)
    assert dx.shape == (0, 64) and not dw.any()


# ------------------------------------------------------------------------------------------------ distillation
def target(ids, values, id_map, lse, T, V):
    """(entries' ids in the student, p, ln p) in 64 bits"""
    has = ids.long().clone()
    if id_map is not None:
        ok = (has >= 0) & (has < len(id_map))
        has = torch.where(ok, id_map.long()[has.clamp(0, len(id_map) - 1)], torch.full_like(has, -1))
    has = torch.where((has >= 0) & (has < V) & (values != -math.inf), has, torch.full_like(has, -1))
    v = torch.where(has >= 0, values.double(), torch.full_like(values.double(), -math.inf)) / T
    ln_p = v - lse.double()[:, None] if lse is not None else torch.log_softmax(v, 1)
    ln_p = torch.where(has >= 0, ln_p, torch.full_like(ln_p, -math.inf))
    return has, ln_p.exp(), ln_p


def distilled(z, ids, values, id_map, lse, T, kind, grad):
    """(loss, its tolerance, gradient, its tolerance) in 64 bits, of 32-bit arithmetic"""
    rows, V = z.shape
    has, p, ln_p = target(ids, values, id_map, lse, T, V)
    zd = z.double()
    m = zd.amax(1, keepdim=True)
    arg = (zd - m) / T
    ln_q = torch.log_softmax(zd / T, 1)
    q = ln_q.exp()
    at = torch.where(has >= 0, ln_q.gather(1, has.clamp_min(0)), torch.zeros_like(ln_p))
    term = p * ((ln_p if kind == "kl" else 0.0) - at)
    term = torch.where(p > 0, term, torch.zeros_like(term))
    none = ~(has >= 0).any(1)
    mass = p.sum(1)
    loss = term.sum(1).masked_fill(none, 0.0)
    log_s = torch.logsumexp(arg, 1)
    # an entry's own p: its argument's roundings, exp's, the normaliser's; then the terms; and what the sum of V exponentials has (each argument's rounding counts by its q)
    v_arg = torch.where(has >= 0, (values.double() - torch.where(has >= 0, values.double(), torch.full_like(values.double(), -math.inf)).amax(1, keepdim=True)).abs() / T, torch.zeros_like(p))
    if lse is not None:
        v_arg = torch.where(has >= 0, values.double().abs() / T + lse.double().abs()[:, None], torch.zeros_like(p))
    p_off = p * E * (4 * v_arg + ids.shape[1] / 16 + 48)
    finite = lambda t: torch.where(t.isfinite(), t, torch.zeros_like(t))
    s_off = E * (finite(q * arg.abs()).sum(1) * 4 + V / 128 + 48)
    size = finite((ln_p.abs() if kind == "kl" else 0.0) + at.abs() + log_s.abs()[:, None])
    tol = (p_off * (size + 1)).sum(1) + (p * E * 8 * (size + finite(v_arg))).sum(1) + mass * (s_off + 4 * E * log_s.abs())
    dense = torch.zeros_like(zd).scatter_add_(1, has.clamp_min(0), p)
    dense_off = torch.zeros_like(zd).scatter_add_(1, has.clamp_min(0), p_off + p * 4 * E)
    w = (grad.double() if grad is not None else torch.ones(rows, dtype=torch.float64))[:, None] / T
    dz = (w * (q * mass[:, None] - dense)).masked_fill(none[:, None], 0.0)
    # relative errors hold for normal numbers: exponentials below 2^-126 may become 0 (the largest is 1, so S >= 1), and bf16 results below it are multiples of 2^-133
    dtol = 2.0 ** -133 + w.abs() * mass[:, None] * 2.0 ** -126 + w.abs() * (finite(q * (E * (4 * arg.abs() + 16) + s_off[:, None])) * mass[:, None] + q * p_off.sum(1, keepdim=True) + dense_off)
    return loss, tol, dz, dtol


def entries(g, rows, V, K, Vt, share=0.0):
    """ids (with repetitions), descending values, a map that leaves ids out"""
    ids = torch.randint(0, Vt or V, (rows, K), generator=g)
    ids[torch.rand(rows, K, generator=g) < share] = -1
    values = (randn(g, rows, K) * 3).sort(1, descending=True).values
    id_map = None
    if Vt:
        id_map = torch.full((Vt,), -1, dtype=torch.int32)
        id_map[torch.randperm(Vt, generator=g)[:V].sort().values] = torch.arange(V, dtype=torch.int32)
    return ids, values, id_map


DISTILL = [(1, 1, 1, 0, 1.0), (3, 5, 9, 0, 1.0), (61, 1024, 16, 4096, 1.0), (7, 1000, 7, 0, 2.0), (5, 32000, 64, 128256, 1.0), (4, 10007, 33, 20000, 0.7), (2, 128256, 16, 0, 3.0), (300, 250, 5, 0, 1.0),
           (9, 50257, 200, 0, 1.0), (2, 4097, 1024, 5000, 1.0), (40, 32001, 3, 0, 0.25), (200, 8192, 4, 9000, 10.0),
           (3, 600001, 9, 0, 1.0), (320, 4100, 1024, 0, 1.0)]


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["kl", "ce"])
@pytest.mark.parametrize("rows,V,K,Vt,T", DISTILL)
def test_distillation(dtype, kind, rows, V, K, Vt, T):
    """Loss and gradient, apart and at once; ids several times in a row, ids that the student lacks, rows without an entry; strided, off their alignment, in place."""
    g = gen(rows, V, K)
    z = (3 * randn(g, rows, V)).to(DT[dtype])
    ids, values, id_map = entries(g, rows, V, K, Vt, 0.2)
    if rows > 2:
        ids[1] = -1
    weight = torch.rand(rows, generator=g)
    loss, tol, dz, dtol = distilled(z, ids, values, id_map, None, T, kind, weight)
    kw = dict(id_map=None if id_map is None else id_map.cuda(), temperature=T)
    i, v = ids.cuda(), values.cuda()
    a, stats = sb.distill_loss(z.cuda(), i, v, kind=kind, want_stats=True, **kw)
    within(a, loss, tol)
    assert torch.equal(a, sb.distill_loss(z.cuda(), i.int(), v, kind=kind, **kw))
    b, db = sb.distill_loss_and_grad(weight.cuda(), z.cuda(), i, v, kind=kind, **kw)
    within(b, loss, tol)
    within(db, dz, dtol + dz.abs() * HALF[dtype])
    d = sb.distill_loss_backward(weight.cuda(), z.cuda(), stats, i, v, **kw)
    within(d, dz, dtol + dz.abs() * HALF[dtype])
    for out, more in (("fp32", 3), ("bf16", 8), (dtype, 5)):
        room = torch.full((rows, V + 2 * more), 5.0, dtype=DT[out], device="cuda")
        c, dc = sb.distill_loss_and_grad(weight.cuda(), strided(z, more), i, v, kind=kind, out=room[:, more: more + V], **kw)
        within(c, loss, tol)
        within(dc, dz, dtol + dz.abs() * HALF[out])
        assert (room[:, :more] == 5).all() and (room[:, more + V:] == 5).all()
        e = sb.distill_loss_backward(weight.cuda(), strided(z, 7), stats, i, v, dtype=DT[out], **kw)
        within(e, dz, dtol + dz.abs() * HALF[out])
    over = z.cuda()
    c, dc = sb.distill_loss_and_grad(weight.cuda(), over, i, v, kind=kind, out=over, **kw)
    assert dc is over and torch.equal(over, db) and torch.equal(c, b)
    over = z.cuda()
    assert torch.equal(sb.distill_loss_backward(weight.cuda(), over, stats, i, v, out=over, **kw), d)
    wide = sb.distill_loss_and_grad(None, z.cuda()[:1].expand(rows, V), i, v, kind=kind, **kw)          # one row of logits for all
    want = distilled(z[:1].expand(rows, V), ids, values, id_map, None, T, kind, None)
    within(wide[0], want[0], want[1])
    within(wide[1], want[2], want[3] + want[2].abs() * HALF[dtype])


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_distillation_with_the_teachers_normaliser(dtype):
    """Probabilities that do not add up to one, in bf16 and fp32."""
    g = gen(8)
    rows, V, K, T = 21, 3001, 20, 1.5
    z, full = randn(g, rows, V), (4 * randn(g, rows, V)).to(DT[dtype])
    values, ids = full.float().topk(K, 1)
    values = values.to(DT[dtype])
    lse = torch.logsumexp(full.double() / T, 1).float()
    loss, tol, dz, dtol = distilled(z, ids, values, None, lse, T, "kl", None)
    got, d = sb.distill_loss_and_grad(None, z.cuda(), ids.cuda(), values.cuda(), values_lse=lse.cuda(), temperature=T)
    within(got, loss, tol)
    within(d, dz, dtol + dz.abs() * E)
    assert (target(ids, values, None, lse, T, V)[1].sum(1) < 0.99).all()


@gpu
@pytest.mark.parametrize("V", [1000, 1001, 32000, 70001])
@pytest.mark.parametrize("mode", ["both", "apart"])
def test_distillation_of_masked_and_odd_logits(V, mode):
    """Logits of -inf and of the type's lowest value, rows of them alone, infinities, NaN, large ones; teacher's values of -inf, +inf and NaN."""
    g = gen(V)
    z = randn(g, 14, V)
    low = torch.finfo(torch.float32).min
    z[0, V // 2:] = -math.inf
    z[1, 10:] = low
    z[2] = low
    z[3] = -math.inf
    z[4, V - 1] = math.inf
    z[5, V - 2] = math.nan
    z[6] = z[6] * 1e30
    z[7, : V - 1] = -math.inf
    ids, values = torch.arange(5).repeat(14, 1), randn(g, 14, 5)
    ids[6] = z[6].argmax()                              # the others' ln q are below -1e29: five times the same entry
    ids[7, :] = V - 1
    values[8, 2] = -math.inf
    values[9, 1] = math.inf
    values[10, 1] = math.nan
    values[11] = -math.inf
    z[12, 3] = -math.inf                                 # an entry that the student rules out
    z[13] = math.nan
    ids[13] = -1                                         # and a row that does not count
    zc, i, v = z.cuda(), ids.cuda(), values.cuda()
    if mode == "both":
        loss, dz = sb.distill_loss_and_grad(None, zc, i, v)
    else:
        loss, stats = sb.distill_loss(zc, i, v, want_stats=True)
        dz = sb.distill_loss_backward(None, zc, stats, i, v)
    want, tol, dwant, dtol = distilled(z, ids, values, None, None, 1.0, "kl", None)
    rows = [0, 1, 2, 6, 7, 8]
    within(loss[rows], want[rows], tol[rows] + 1e-6)
    # row 1: exponents of 3e38 leave no tolerance by size; what is masked has exactly no part
    dtol[1, 10:] = 0
    within(dz[rows], dwant[rows], dtol[rows].nan_to_num(0.0) + 1e-7)
    for r in (3, 4, 5, 9, 10):
        assert loss[r].isnan() and dz[r].isnan().all(), r
    for r in (11, 13):
        assert loss[r] == 0 and not dz[r].any()
    assert loss[12] == math.inf and dz[12].isfinite().all() and dz[12, 3] < 0
    within(dz[12: 13], dwant[12: 13], dtol[12: 13].nan_to_num(0.0) + 1e-7)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [1000, 1001])
def test_masked_and_odd_logits_in_many_rows(V, dtype):
    """As above, where rows are many: each kind of row is what it is by itself."""
    g = gen(V, 2)
    z = randn(g, 8, V)
    z[0, V // 2:] = -math.inf
    z[1, 10:] = torch.finfo(torch.bfloat16).min
    z[2] = -math.inf
    z[3, V - 1] = math.inf
    z[4, V - 2] = math.nan
    z[5, : V - 1] = -math.inf
    z[6] = math.nan
    ids, values = torch.arange(5).repeat(8, 1), randn(g, 8, 5)
    ids[5], ids[6] = V - 1, -1
    z = z.to(DT[dtype])
    for off in (0, 1):
        few = sb.distill_loss(strided(z, off), ids.cuda(), values.cuda(), want_stats=True)
        many = sb.distill_loss(strided(z.repeat(50, 1), off), ids.repeat(50, 1).cuda(), values.repeat(50, 1).cuda(), want_stats=True)
        for a, b in zip(few, many):
            assert torch.allclose(a.repeat(50, *[1] * (a.dim() - 1)), b, rtol=1e-5, atol=1e-6, equal_nan=True)
    want, tol, _, _ = distilled(z, ids, values, None, None, 1.0, "kl", None)
    within(few[0][[0, 1, 5, 7]], want[[0, 1, 5, 7]], tol[[0, 1, 5, 7]] + 1e-6)
    assert few[0][[2, 3, 4]].isnan().all() and few[0][6] == 0


@gpu
def test_distillation_bad_ids_and_no_rows():
    z, v = torch.randn(3, 100, device="cuda"), torch.zeros(3, 2, device="cuda")
    for bad, site, id_map in ((100, 65, None), (-2, 65, None), (1 << 40, 65, None), (5, 65, torch.zeros(5, dtype=torch.int32)), (4, 66, torch.tensor([0, 1, 2, 3, 100], dtype=torch.int32)),
                              (4, 66, torch.tensor([0, 1, 2, 3, -7], dtype=torch.int32))):
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        ids = torch.tensor([[1, 2], [3, bad], [0, -1]], device="cuda")
        id_map = None if id_map is None else id_map.cuda()
        loss, dz = sb.distill_loss_and_grad(None, z, ids, v, id_map=id_map, status=status)
        alone = torch.tensor([[1, 2], [3, -1], [0, -1]], device="cuda")
        want, dwant = sb.distill_loss_and_grad(None, z, alone, v, id_map=id_map)
        assert torch.equal(loss, want) and torch.equal(dz, dwant) and status.tolist()[:3] == [2, site, 1]
    none = torch.zeros(0, 4, dtype=torch.int64, device="cuda")
    loss, dz = sb.distill_loss_and_grad(None, z[:0], none, v[:0].expand(0, 2).new_zeros(0, 4))
    assert loss.shape == (0,) and dz.shape == (0, 100)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_distillation_autograd_and_differences(dtype):
    """A weighted mean's gradient is that by hand.  Differences: along d with |d| <= 1 the loss's third derivative is below T^-3 (a third central moment of d under q), so the quotient is off by
    h^2 / 6 times that and by the two calls' errors over 2 h."""
    g = gen(2)
    rows, V, K, T, h = 9, 500, 12, 1.5, 2.0 ** -5
    z = randn(g, rows, V).to(DT[dtype])
    ids, values, _ = entries(g, rows, V, K, 0, 0.1)
    weight = torch.rand(rows, generator=g).cuda()
    i, v, leaf = ids.cuda(), values.cuda(), z.cuda().requires_grad_()
    loss = sb.distill_loss(leaf, i, v, temperature=T)
    assert loss.requires_grad and torch.equal(loss, sb.distill_loss(z.cuda(), i, v, temperature=T))
    (loss * weight).sum().backward()
    plain, stats = sb.distill_loss(z.cuda(), i, v, temperature=T, want_stats=True)
    assert torch.equal(leaf.grad, sb.distill_loss_backward(weight, z.cuda(), stats, i, v, temperature=T))
    leaf.grad = None
    sb.distill_loss(leaf, i, v, temperature=T, want_stats=True)[0].sum().backward()                     # an expanded gradient
    assert torch.equal(leaf.grad, sb.distill_loss_backward(None, z.cuda(), stats, i, v, temperature=T))
    if dtype == "fp32":
        d = torch.rand(rows, V, generator=g) * 2 - 1
        up, down = z + h * d, z - h * d
        step = (up.double() - down.double()) / (2 * h)
        f = lambda t: sb.distill_loss(t.cuda(), i, v, temperature=T).cpu().double()
        tol = distilled(up, ids, values, None, None, T, "kl", None)[1] + distilled(down, ids, values, None, None, T, "kl", None)[1]
        off = (f(up) - f(down)) / (2 * h) - (leaf.grad.cpu().double() * step).sum(1)
        assert (off.abs() <= h * h / 6 / T ** 3 * 1.01 + tol / (2 * h) + 64 * E).all()
    with pytest.raises(ValueError):
        sb.distill_loss(z.cuda(), i, v.requires_grad_())


# ------------------------------------------------------------------------------------------------ together, streams, graphs
@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_training_step_together(dtype):
    """Lookup, a norm of the sum with features, a projection, a norm, the LM head over the draft's vocabulary, the loss: gradients of every leaf against the same chain in 64 bits."""
    g = gen(21)
    T, V, k, Vt, Vd, K = 190, 600, 128, 600, 250, 12
    dt = DT[dtype]
    leaves = {"embed": randn(g, V, k), "feat": randn(g, T, k), "g1": 1 + 0.1 * randn(g, k), "w": randn(g, k, k) / k ** 0.5, "g2": 1 + 0.1 * randn(g, k), "head": randn(g, Vd, k) / k ** 0.5}
    leaves = {n: t.to(dt) for n, t in leaves.items()}
    ids = torch.randint(-1, V, (T,), generator=g)
    tid, values, id_map = entries(g, T, Vd, K, Vt, 0.1)
    tid[ids < 0] = -1

    def chain(p, lookup_, norm, loss_):
        x = lookup_(p["embed"])
        h, s = norm(x, p["g1"], p["feat"])
        y, _ = norm(h @ p["w"].T, p["g2"], s)
        return loss_(y @ p["head"].T).sum() / T

    dev = {n: t.cuda().requires_grad_() for n, t in leaves.items()}
    got = chain(dev, lambda w: sb.embedding(ids.cuda(), w), lambda x, w, r: sb.rms_norm(x, w, 1e-5, r), lambda z: sb.distill_loss(z, tid.cuda(), values.cuda(), id_map=id_map.cuda()))
    got.backward()

    ref = {n: t.double().requires_grad_() for n, t in leaves.items()}
    has, p, ln_p = target(tid, values, id_map, None, 1.0, Vd)

    def loss64(z):
        ln_q = torch.log_softmax(z, 1).gather(1, has.clamp_min(0))
        return torch.where(p > 0, p * (ln_p.nan_to_num(0.0, neginf=0.0) - ln_q), torch.zeros_like(p)).sum(1)

    def norm64(x, w, r):
        s = x + r
        return s / (s.square().mean(1, keepdim=True) + 1e-5).sqrt() * w, s
    want = chain(ref, lambda w: torch.where((ids >= 0)[:, None], w[ids.clamp_min(0)], torch.zeros(1, dtype=torch.float64)), norm64, loss64)
    want.backward()
    # a chain of ten roundings of 2^-9 in the mean (bf16; none of them correlated), the LM head's 128 products in the same type; fp32: sums of up to 600
    bound = 0.03 if dtype == "bf16" else 1e-5
    assert abs(got.item() - want.item()) <= bound * abs(want.item())
    for n in leaves:
        a, b = dev[n].grad.cpu().double(), ref[n].grad
        assert (a - b).norm() <= bound * b.norm(), n
    assert not dev["embed"].grad[torch.bincount(ids[ids >= 0], minlength=V).cuda() == 0].any()


@gpu
def test_on_another_stream_and_in_a_graph():
    """Calls on a side stream, and a captured sequence of all of them replayed on new inputs, twice: the same bits as calls one by one."""
    g = gen(4)
    T, V, k, Vd, K = 150, 300, 256, 700, 8
    ids, w, gain = torch.randint(0, V, (T,), generator=g).cuda(), randn(g, V, k).bfloat16().cuda(), torch.ones(k, device="cuda")
    res, z = randn(g, T, k).bfloat16().cuda(), randn(g, T, Vd).cuda()
    tid, values = torch.randint(0, Vd, (T, K), generator=g).cuda(), randn(g, T, K).cuda()

    def all_of_them():
        x = sb.embedding(ids, w, 2.0)
        y, s = sb.rms_norm(x, gain, 1e-5, res)
        codes, scale = sb.rms_norm(s, gain, 1e-5, dtype=torch.float8_e4m3fn, group=64)
        dx, dw = sb.rms_norm_backward(y, s, gain, 1e-5, x)
        loss, dz = sb.distill_loss_and_grad(None, z, tid, values)
        part, stats = sb.distill_loss(z, tid, values, want_stats=True)
        return [x, y, s, codes.float(), scale, dx, dw, loss, dz, part, sb.distill_loss_backward(None, z, stats, tid, values), sb.embedding_backward(dx, ids, V)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = all_of_them()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(there, all_of_them()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = all_of_them()
    for seed in (5, 6):
        h = gen(seed)
        ids.copy_(torch.randint(0, V, (T,), generator=h))
        res.copy_(randn(h, T, k))
        z.copy_(randn(h, T, Vd))
        tid.copy_(torch.randint(0, Vd, (T, K), generator=h))
        graph.replay()
        for a, b in zip(kept, all_of_them()):
            assert torch.equal(a, b)


@gpu
def test_the_decoding_loop_refuses_ids_that_the_table_lacks():
    from paper_2503_01840_b200 import synth
    from paper_2503_01840_b200.kv8_decode import CachedDecoder
    cfg = synth.ModelCfg("K", "bf16", 1, 512, 4, 2, 128, 1408, 2048, 1024, (0, 0, 0), 1e4, batch=1, tree_depth=2, tree_topk=2, tree_nodes=4, seed=3)
    dec = CachedDecoder(cfg, synth.make_target_weights(cfg, "cuda"), 1, 24, "bf16")
    for bad in ([1, 2048], [-1, 5]):
        with pytest.raises(ValueError):
            dec.prefill([torch.tensor(bad)])
    dec.prefill([torch.tensor([0, 2047])])


@gpu
def test_two_streams_at_once():
    """Calls that overlap on the GPU share nothing."""
    g = gen(9)
    z, ids, v = randn(g, 3000, 32000).cuda(), torch.randint(0, 32000, (3000, 20), generator=g).cuda(), randn(g, 3000, 20).cuda()
    x, w, tok = randn(g, 6000, 4096).bfloat16().cuda(), torch.ones(4096, device="cuda"), torch.randint(0, 30000, (6000,), generator=g).cuda()
    a = lambda: [*sb.distill_loss_and_grad(None, z, ids, v), sb.embedding_backward(x, tok, 30000)]
    b = lambda: [*sb.rms_norm_backward(x, x, w), sb.embedding_backward(x, tok.flip(0), 30000), *sb.rms_norm(x, w, residual=x, dtype=torch.int8)]
    want = a(), b()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for s, f in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append(f())
    torch.cuda.synchronize()
    for one, other in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(one, other))


@gpu
def test_a_training_step_in_a_graph():
    """Forward, backward through autograd and the leaves' gradients, captured after a warm-up whose graph is gone; replayed on other inputs as the same step without."""
    g = gen(14)
    T, V, k, Vd, K = 90, 400, 256, 500, 6
    leaves = [randn(g, V, k).cuda().requires_grad_(), torch.ones(k, device="cuda").requires_grad_(), (randn(g, Vd, k) / 16).cuda().requires_grad_()]
    ids, tid, values = torch.randint(0, V, (T,), generator=g).cuda(), torch.randint(0, Vd, (T, K), generator=g).cuda(), randn(g, T, K).cuda()

    def step():
        x = sb.embedding(ids, leaves[0])
        y, _ = sb.rms_norm(x, leaves[1], residual=x * 0.5)
        loss = sb.distill_loss(y @ leaves[2].T, tid, values).mean()
        loss.backward()
        return loss.detach()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
            for t in leaves:
                t.grad = None
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = step()
    kept = [t.grad for t in leaves]
    for seed in (3, 4):
        h = gen(seed)
        ids.copy_(torch.randint(0, V, (T,), generator=h))
        tid.copy_(torch.randint(0, Vd, (T, K), generator=h))
        values.copy_(randn(h, T, K))
        graph.replay()
        replayed = [loss.clone()] + [t.clone() for t in kept]
        for t in leaves:
            t.grad = None
        plain = [step()] + [t.grad for t in leaves]
        assert all(torch.allclose(p, q, rtol=1e-5, atol=1e-7) for p, q in zip(replayed, plain))      # the products are another library's, which may choose by the stream


@gpu
def test_offsets_that_pass_32_bits():
    """The last rows of tensors of more than 2^31 elements: the same bits as by themselves."""
    g = gen(6)
    n, k = 530000, 4096
    big = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    last = randn(g, 40, k).bfloat16().cuda()
    big[-40:] = last
    assert big.numel() > 1 << 31
    ids = torch.arange(n - 40, n, device="cuda")
    assert torch.equal(sb.embedding(ids, big), last)
    w = torch.ones(k, device="cuda")
    y, s = sb.rms_norm(big, w, 1e-5, residual=big)
    y1, s1 = sb.rms_norm(last, w, 1e-5, residual=last)
    assert torch.equal(y[-40:], y1) and torch.equal(s[-40:], s1)
    del s
    dx = sb.rms_norm_backward(big, y, w, 1e-5)[0]
    assert torch.equal(dx[-40:], sb.rms_norm_backward(last, y1, w, 1e-5)[0])
    del y, dx
    out = sb.embedding_backward(last, ids, n)
    assert torch.equal(out[-40:], last) and not out[: n - 40].any()
    tokens = torch.full((n,), -1, device="cuda")
    tokens[-40:] = torch.arange(40, device="cuda")
    assert torch.equal(sb.embedding_backward(big, tokens, 40), last)
    del out, tokens
    z = big.view(-1)[: 67000 * 32400].view(67000, 32400)
    assert z.numel() > 1 << 31
    z[-5:] = randn(g, 5, 32400).bfloat16().cuda()
    tid, values = torch.full((67000, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(67000, 3, device="cuda")
    tid[-5:] = torch.randint(0, 32400, (5, 3), generator=g).int().cuda()
    loss, stats = sb.distill_loss(z, tid, values, want_stats=True)
    one, dz = sb.distill_loss_and_grad(None, z, tid, values)
    few, dfew = sb.distill_loss_and_grad(None, z[-5:].clone(), tid[-5:].clone(), values[-5:].clone())
    # the few rows go by more and smaller slices, so their sums are added in another order
    assert torch.allclose(one[-5:], few, rtol=1e-5) and torch.allclose(loss[-5:], few, rtol=1e-5) and not loss[:-5].any() and not one[:-5].any()
    assert torch.allclose(dz[-5:].float(), dfew.float(), rtol=2.0 ** -7, atol=0) and not dz[:-5].any()
    assert torch.allclose(sb.distill_loss_backward(None, z, stats, tid, values)[-5:].float(), dfew.float(), rtol=2.0 ** -7, atol=0)


@gpu
def test_what_is_written_in_place_is_known_to_autograd():
    """A graph that saved a tensor does not go back through it once a call has written over it."""
    x = torch.randn(4, 32, device="cuda").requires_grad_()
    w, z = torch.ones(32, device="cuda"), torch.randn(4, 32, device="cuda")
    ids, v = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.zeros(4, 1, device="cuda")
    for over in (lambda t: sb.rms_norm(z, w, residual=t, sum_out=t), lambda t: sb.distill_loss_and_grad(None, t, ids, v, out=t), lambda t: sb.embedding(ids[:, 0], z, out=t),
                 lambda t: sb.embedding_backward(z, ids[:, 0], 4, out=t, accumulate=True)):
        y = x * 2
        total = (y * y).sum()
        with torch.no_grad():
            over(y.detach())
        with pytest.raises(RuntimeError):
            total.backward()


@gpu
def test_a_first_call_may_be_captured():
    """In a process of its own: nothing has been launched before, and the larger kernels' shared memory has to be asked for."""
    import subprocess
    import sys
    code = """
import torch
from paper_2503_01840_b200 import binding as sb
g = torch.Generator(device="cuda").manual_seed(1)
z = torch.randn(600, 40000, generator=g, device="cuda")
x, w = torch.randn(300, 8192, generator=g, device="cuda"), torch.ones(8192, device="cuda")
ids, v = torch.randint(0, 40000, (600, 5), generator=g, device="cuda"), torch.randn(600, 5, generator=g, device="cuda")
few = ids[:300, 0].contiguous() % 100
sb._marshal()
def run():
    y, s = sb.rms_norm(x, w, residual=x)
    loss, dz = sb.distill_loss_and_grad(None, z, ids, v)
    plain, stats = sb.distill_loss(z, ids, v, want_stats=True)
    return [y, s, loss, dz, plain, stats, *sb.rms_norm_backward(y, s, w, grad_sum=x), sb.embedding_backward(x, few, 100), sb.distill_loss_backward(None, z, stats, ids, v)]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    kept = run()
graph.replay()
assert all(torch.equal(a, b) for a, b in zip(kept, run()))
"""
    subprocess.run([sys.executable, "-c", code], check=True, timeout=300)


# ------------------------------------------------------------------------------------------------ refusals
def rows_struct(p=4096, stride=64, kind=0):
    return sb._Rows(p, stride, kind)


def test_entry_points_refuse_what_they_cannot_do():
    """Before anything is launched: no GPU is needed."""
    L, ref = sb.lib(), C.byref
    p, bad = 4096, -1
    r = rows_struct
    emb = dict(w=r(), vocab=10, dim=64, bits=32, ids=p, tokens=3, scale=1.0, out=r())
    def embedding(**kw):
        a = {**emb, **kw}
        return L.spec_embedding(a["w"] and ref(a["w"]), a["vocab"], a["dim"], a["bits"], a["ids"], a["tokens"], a["scale"], a["out"] and ref(a["out"]), None, None)
    for kw, rc in ((dict(w=None), -2), (dict(out=None), -2), (dict(ids=None), -2), (dict(w=r(None)), -2), (dict(vocab=0), bad), (dict(dim=0), bad), (dict(bits=16), bad), (dict(tokens=-1), bad),
                   (dict(scale=math.inf), bad), (dict(scale=math.nan), bad), (dict(out=r(stride=63)), bad), (dict(out=r(kind=2)), bad), (dict(w=r(p=4097)), bad), (dict(ids=4098), bad),
                   (dict(bits=64, ids=4100), bad), (dict(dim=(1 << 22) + 1, out=r(stride=1 << 23)), -8), (dict(tokens=(1 << 30) + 1), -8), (dict(tokens=0, w=None, out=None, ids=None), 0)):
        assert embedding(**kw) == rc, kw
    back = dict(g=r(), bits=32, ids=p, tokens=3, vocab=10, dim=64, scale=1.0, acc=0, out=r(), scratch=p, n=1 << 30)
    def backward(**kw):
        a = {**back, **kw}
        return L.spec_embedding_backward(a["g"] and ref(a["g"]), a["bits"], a["ids"], a["tokens"], a["vocab"], a["dim"], a["scale"], a["acc"], a["out"] and ref(a["out"]), a["scratch"], a["n"], None, None)
    need = L.spec_embedding_backward_scratch_bytes(3, 10, 64)
    for kw, rc in ((dict(g=None), -2), (dict(out=None), -2), (dict(scratch=None), -2), (dict(ids=None), -2), (dict(n=need - 1), -3), (dict(scratch=p + 16), -3), (dict(out=r(stride=63)), bad),
                   (dict(g=r(kind=3)), bad), (dict(vocab=0), bad), (dict(scale=math.nan), bad), (dict(tokens=0, acc=1, g=None, scratch=None), 0)):
        assert backward(**kw) == rc, kw
    assert L.spec_embedding_backward_scratch_bytes(-1, 10, 64) == 0 and need > 0
    norm = dict(x=r(), res=None, gt=0, gain=p, eps=1e-5, sum=None, y=r(), scale=None, group=0, rows=3, dim=64)
    def rms(**kw):
        a = {**norm, **kw}
        o = lambda n: a[n] and ref(a[n])
        return L.spec_rms_norm(o("x"), o("res"), a["gt"], a["gain"], a["eps"], o("sum"), o("y"), a["scale"], a["group"], a["rows"], a["dim"], None)
    for kw, rc in ((dict(x=None), -2), (dict(y=None), -2), (dict(gain=None), -2), (dict(y=r(kind=2)), -2), (dict(y=r(kind=3), scale=p, group=8), bad), (dict(group=-16), bad), (dict(eps=-1.0), bad),
                   (dict(eps=math.nan), bad), (dict(gt=2), bad), (dict(gain=p + 2), bad), (dict(res=r()), -2), (dict(sum=r()), bad), (dict(res=r(), sum=r(kind=1)), bad),
                   (dict(res=r(), sum=r(stride=63)), bad), (dict(res=r(p=8192, stride=96), sum=r(p=8192, stride=64)), bad), (dict(x=r(kind=1), res=r(p=8192), sum=r()), bad), (dict(x=r(kind=2)), bad),
                   (dict(y=r(kind=4)), bad), (dict(dim=0), bad), (dict(rows=-1), bad), (dict(dim=(1 << 22) + 1), -8), (dict(rows=0, x=None, y=None), 0)):
        assert rms(**kw) == rc, kw
    grad = dict(g=r(), x=r(), gt=0, gain=p, eps=1e-5, c=None, dx=r(p=8192), dw=p, scratch=p, n=1 << 30, rows=3, dim=64)
    def rms_back(**kw):
        a = {**grad, **kw}
        o = lambda n: a[n] and ref(a[n])
        return L.spec_rms_norm_backward(o("g"), o("x"), a["gt"], a["gain"], a["eps"], o("c"), o("dx"), a["dw"], a["scratch"], a["n"], a["rows"], a["dim"], None)
    need = L.spec_rms_norm_backward_scratch_bytes(3, 64)
    for kw, rc in ((dict(g=None), -2), (dict(x=None), -2), (dict(dx=None), -2), (dict(dw=None), -2), (dict(gain=None), -2), (dict(scratch=None), -2), (dict(n=need - 1), -3), (dict(scratch=p + 8), -3),
                   (dict(dx=r(p=8192, stride=10)), bad), (dict(dx=r(kind=1)), bad), (dict(c=r(p=8192, stride=65)), bad), (dict(eps=math.inf), bad)):
        assert rms_back(**kw) == rc, kw
    teach = dict(ids=p, values=p, lse=None, id_map=None, id_bits=32, values_dtype=0, id_map_n=0, K=4)
    dist = dict(z=r(stride=100), rows=3, vocab=100, T=1.0, grad=None, loss=p, stats=None, dz=r(p=8192, stride=100))
    def distill(**kw):
        t = sb._Teacher(**{**teach, **{k: v for k, v in kw.items() if k in teach}})
        a = {**dist, **kw}
        return L.spec_distill(a["z"] and ref(a["z"]), a["rows"], a["vocab"], None if kw.get("no_teacher") else ref(t), a["T"], 1, a["grad"], a["loss"], a["stats"], a["dz"] and ref(a["dz"]), None, None)
    for kw, rc in ((dict(z=None), -2), (dict(ids=None), -2), (dict(values=None), -2), (dict(no_teacher=1), -2), (dict(loss=None), -2), (dict(loss=None, dz=None, stats=p), -2), (dict(K=0), bad), (dict(K=1025), -8),
                   (dict(T=0.0), bad), (dict(T=1e5), bad), (dict(T=math.nan), bad), (dict(T=-1.0), bad), (dict(id_bits=8), bad), (dict(values_dtype=2), bad), (dict(id_map=p), bad), (dict(vocab=0), bad),
                   (dict(rows=-1), bad), (dict(dz=r(p=8192, stride=99)), bad), (dict(dz=r(stride=100, kind=1)), bad), (dict(z=r(stride=100, kind=2)), bad), (dict(stats=p + 4), bad), (dict(grad=p + 2), bad),
                   (dict(rows=0, z=None, dz=None), 0)):
        assert distill(**kw) == rc, kw


def test_the_binding_refuses_tensors_off_the_gpu_and_odd_arguments():
    w, ids, x, g = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64), torch.zeros(3, 8), torch.ones(8)
    for call in (lambda: sb.embedding(ids, w), lambda: sb.embedding_backward(x, ids, 4), lambda: sb.rms_norm(x, g), lambda: sb.rms_norm_backward(x, x, g),
                 lambda: sb.distill_loss(x, ids[:, None], x[:, :1]), lambda: sb.distill_loss(x, ids[:, None], x[:, :1], kind="js")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        sb.embedding([1, 2], w)


@gpu
def test_the_binding_refuses():
    c = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    w, ids, x, g, i2, v2 = c(4, 8), c(3, dtype=torch.int64), c(3, 8), c(8), c(3, 2, dtype=torch.int32), c(3, 2)
    i = torch.int64
    for error, call in ((ValueError, lambda: sb.embedding(ids.float(), w)), (ValueError, lambda: sb.embedding(ids[None], w)), (TypeError, lambda: sb.embedding(ids, w.half())), (ValueError, lambda: sb.embedding(ids, w.T)),
                        (TypeError, lambda: sb.embedding(ids, w, dtype=torch.float16)), (ValueError, lambda: sb.embedding(ids, w, out=c(3, 7))), (TypeError, lambda: sb.embedding(ids, w, "a")),
                        (ValueError, lambda: sb.embedding(ids, w, out=c(3, 8, dtype=torch.bfloat16), dtype=torch.float32)), (sb.SpecError, lambda: sb.embedding(ids, w, math.inf)),
                        (ValueError, lambda: sb.embedding(ids[:2][:, None].expand(2, 3)[:, 0], w.T)), (ValueError, lambda: sb.embedding_backward(x, ids[:2], 4)), (ValueError, lambda: sb.embedding_backward(x, ids, 0)),
                        (ValueError, lambda: sb.embedding_backward(x, ids, 4, accumulate=True)), (ValueError, lambda: sb.embedding_backward(x, ids, 4, out=c(5, 8))),
                        (sb.SpecError, lambda: sb.embedding_backward(x, ids, 4, out=c(1, 8).expand(4, 8))), (ValueError, lambda: sb.embedding(c(6, dtype=i)[::2], w)),
                        (ValueError, lambda: sb.rms_norm(x[0], g)), (ValueError, lambda: sb.rms_norm(x, c(7))), (TypeError, lambda: sb.rms_norm(x.half(), g)), (ValueError, lambda: sb.rms_norm(x, g, residual=c(3, 7))),
                        (ValueError, lambda: sb.rms_norm(x, g, sum_out=x)), (ValueError, lambda: sb.rms_norm(x, g, residual=x, sum_out=c(3, 8, dtype=torch.bfloat16))), (ValueError, lambda: sb.rms_norm(x, g, group=8)),
                        (TypeError, lambda: sb.rms_norm(x, g, dtype=torch.float8_e5m2)), (sb.SpecError, lambda: sb.rms_norm(x, g, -1.0)), (TypeError, lambda: sb.rms_norm(x, g, "a")),
                        (ValueError, lambda: sb.rms_norm_backward(x, c(2, 8), g)), (ValueError, lambda: sb.rms_norm_backward(x, x, g, grad_sum=c(3, 7))), (TypeError, lambda: sb.rms_norm_backward(x, x, g, dtype=torch.int8)),
                        (ValueError, lambda: sb.distill_loss(x, i2[:2], v2)), (ValueError, lambda: sb.distill_loss(x, i2, v2[:, :1])), (ValueError, lambda: sb.distill_loss(x, i2.float(), v2)),
                        (ValueError, lambda: sb.distill_loss(x, i2, v2, kind="mse")), (ValueError, lambda: sb.distill_loss(x, i2, v2, id_map=ids)), (ValueError, lambda: sb.distill_loss(x, i2, v2, values_lse=c(2))),
                        (sb.SpecError, lambda: sb.distill_loss(x, i2, v2, temperature=0.0)), (sb.SpecError, lambda: sb.distill_loss(x, i2[:, :0], v2[:, :0])), (TypeError, lambda: sb.distill_loss(x.half(), i2, v2)),
                        (ValueError, lambda: sb.distill_loss_backward(c(2), x, v2, i2, v2)), (ValueError, lambda: sb.distill_loss_backward(None, x, c(3, 1), i2, v2)),
                        (ValueError, lambda: sb.distill_loss_and_grad(None, x, i2, v2, out=c(3, 7))), (ValueError, lambda: sb.embedding(ids, w, status=c(4)))):
        with pytest.raises(error):
            call()
