"""The plans that the operators around the layers take for many rows, against 64 bits: blocks that take several rows in turn, rows that are looked at before they are read, outputs in an
input's place."""
import ctypes as C

import pytest
import torch

import test_layer_operators as layers
from paper_2503_01840_b200 import binding as sb
from test_layer_operators import DT, E, HALF, gen, randn, within

pytestmark = pytest.mark.gpu


# More rows than 148 SMs have blocks: at most 16 an SM of narrow rows, 12 of 1024 columns, 4 of 4096, 2 of 8192, 1 of 16384
@pytest.mark.parametrize("x,res,gain,out", layers.TYPES)
@pytest.mark.parametrize("rows,k", [(7000, 264), (4001, 1000), (2000, 2048), (1900, 4096), (901, 8192), (460, 16384), (450, 10000), (5000, 248), (700, 1002)])
def test_norm_of_more_rows_than_blocks(x, res, gain, out, rows, k):
    g = gen(rows, k)
    xs, w = randn(g, rows, k).to(DT[x]), (1 + 0.3 * randn(g, k)).to(DT[gain])
    rs = (20 * randn(g, rows, k)).to(DT[res]) if res else None
    s, y = layers.normed(xs, rs, w, 1e-5)
    got = sb.rms_norm(xs.cuda(), w.cuda(), 1e-5, rs.cuda() if res else None, DT[out])
    a, total = got if res else (got, None)
    within(a, y, layers.norm_error(y, k) + y.abs() * HALF[out])
    if not res:
        return
    within(total, s, s.abs() * (E + HALF[res]))
    into = rs.cuda()                                     # rows behind the one that is written are under way
    b, t = sb.rms_norm(xs.cuda(), w.cuda(), 1e-5, into, DT[out], sum_out=into)
    assert t is into and torch.equal(b, a) and torch.equal(into, total)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("x,res", [("bf16", "bf16"), ("fp32", None), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,k,group", [(7000, 264, 32), (4001, 1000, 0), (1900, 4096, 128), (1900, 4096, 0), (901, 8192, 0), (901, 8192, 256), (460, 16384, 0), (450, 10000, 64)])
def test_norm_in_8_bits_of_more_rows_than_blocks(fmt, x, res, rows, k, group):
    """Every row has a size of its own, so that a maximum of the row before, or after, would show in its scale."""
    g = gen(rows, k, group)
    top = 448.0 if fmt == "e4m3" else 127.0
    xs, w = randn(g, rows, k).to(DT[x]), (1 + 0.3 * randn(g, k)).to(torch.bfloat16)
    rs = randn(g, rows, k).to(DT[res]) if res else None
    big = torch.randint(0, k, (rows,), generator=g)
    xs[torch.arange(rows), big] = (10.0 ** (3 * torch.rand(rows, generator=g))).to(DT[x])
    s, y = layers.normed(xs, rs, w, 1e-5)
    n = group or k
    groups = -(-k // n)
    amax = torch.nn.functional.pad(y.abs(), (0, groups * n - k)).view(rows, groups, n).amax(2)
    scale = (amax / top).clamp_min(layers.FLOOR)
    got = sb.rms_norm(xs.cuda(), w.cuda(), 1e-5, rs.cuda() if res else None, DT[fmt], group)
    rel = layers.norm_error(torch.ones(1, dtype=torch.float64), k)
    within(got[1], scale, scale * (rel + 3 * E))
    wide = scale.repeat_interleave(n, 1)[:, :k]
    value = got[0].cpu().double() * got[1].cpu().double().repeat_interleave(n, 1)[:, :k]
    # half a step, as a scale that is off shifts it, of which the norm's own error is a part
    step = torch.maximum(y.abs() * 2.0 ** -4, wide * 2.0 ** -10) if fmt == "e4m3" else wide * 0.5
    within(value, y, step * (1 + 2.0 ** -10) + y.abs() * (rel + 8 * E) * 8)
    if res:
        within(got[2], s, s.abs() * (E + HALF[res]))


@pytest.mark.parametrize("grad,x,gain,carried", [("bf16", "bf16", "bf16", True), ("bf16", "bf16", "bf16", False), ("fp32", "fp32", "fp32", True), ("bf16", "fp32", "bf16", True),
                                                 ("fp32", "bf16", "fp32", False)])
@pytest.mark.parametrize("rows,k", [(5000, 256), (3001, 1000), (1500, 2048), (1000, 4096), (500, 8192), (3000, 1002), (400, 20001)])
def test_norm_gradient_of_more_rows_than_blocks(grad, x, gain, carried, rows, k):
    """The gain's gradient is the sum of what each block has of its rows; the kernel for any width, too."""
    g = gen(rows, k, 1)
    dy, s, w = randn(g, rows, k).to(DT[grad]), (3 * randn(g, rows, k)).to(DT[x]), (1 + 0.3 * randn(g, k)).to(DT[gain])
    c = randn(g, rows, k).to(DT[x]) if carried else None
    dx, size, dw, wsize = layers.norm_gradient(dy, s, w, 1e-5, c)
    # as for fewer rows: sums of k / 256 and a tree in the two means, a dozen roundings beside them; of the rows' sum, each row's h and as many additions as rows
    tol, wtol = size * E * (2 * (k / 256 + 16) + 16), wsize * E * (rows + (k / 256 + 16) + 16)
    a, aw = sb.rms_norm_backward(dy.cuda(), s.cuda(), w.cuda(), 1e-5, c.cuda() if carried else None)
    within(a, dx, tol + dx.abs() * HALF[x])
    within(aw, dw, wtol + dw.abs() * HALF[gain])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,k", [(1000, 4096), (500, 8192), (3001, 1000), (3000, 1002), (400, 20001), (9, 136)])
def test_norm_gradient_in_an_inputs_place(dtype, rows, k):
    """dx over the gradient, over what was normed, over what is carried: the same bits as apart from them, also where the rows that a block takes next are under way."""
    g = gen(rows, k, 2)
    L, ref = sb.lib(), C.byref
    kind = 0 if dtype == "fp32" else 1
    dy, s, c, w = randn(g, rows, k).to(DT[dtype]), randn(g, rows, k).to(DT[dtype]), randn(g, rows, k).to(DT[dtype]), (1 + 0.3 * randn(g, k)).to(DT[dtype]).cuda()
    want = sb.rms_norm_backward(dy.cuda(), s.cuda(), w, 1e-5, c.cuda())
    n = L.spec_rms_norm_backward_scratch_bytes(rows, k)
    for over in range(3):
        t = [dy.cuda(), s.cuda(), c.cuda()]
        r = [sb._Rows(x.data_ptr(), k, kind) for x in t]
        dw, scratch = torch.empty_like(w), torch.empty(n, dtype=torch.uint8, device="cuda")
        rc = L.spec_rms_norm_backward(ref(r[0]), ref(r[1]), kind, w.data_ptr(), 1e-5, ref(r[2]), ref(r[over]), dw.data_ptr(), scratch.data_ptr(), n, rows, k,
                                      torch.cuda.current_stream().cuda_stream)
        assert rc == 0 and torch.equal(t[over], want[0]) and torch.equal(dw, want[1]), over


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["kl", "ce"])
@pytest.mark.parametrize("rows,V,K,Vt,T", [(1500, 1024, 16, 4096, 1.0), (700, 8009, 33, 20000, 0.7), (400, 32000, 64, 0, 1.0), (330, 50257, 7, 0, 1.0), (170, 128256, 16, 0, 2.0),
                                           (90, 128256, 200, 200000, 1.0)])
def test_distillation_of_many_rows(dtype, kind, rows, V, K, Vt, T):
    """More CTAs than are on the GPU at a time, one a row and in clusters: rows are read only if one of their ids counts, and the ids of later ones are fetched ahead."""
    g = gen(rows, V, K)
    z = (3 * randn(g, rows, V)).to(DT[dtype])
    ids, values, id_map = layers.entries(g, rows, V, K, Vt, 0.2)
    empty = torch.rand(rows, generator=g) < 0.3
    empty[[0, rows - 1]] = torch.tensor([True, False])
    ids[empty] = -1
    z[empty] = float("nan")                              # what is not looked at
    weight = torch.rand(rows, generator=g)
    loss, tol, dz, dtol = layers.distilled(z.masked_fill(empty[:, None], 0.0), ids, values, id_map, None, T, kind, weight)
    kw = dict(id_map=None if id_map is None else id_map.cuda(), temperature=T)
    zc, i, v = z.cuda(), ids.cuda(), values.cuda()
    a, stats = sb.distill_loss(zc, i, v, kind=kind, want_stats=True, **kw)
    within(a, loss, tol)
    b, db = sb.distill_loss_and_grad(weight.cuda(), zc, i, v, kind=kind, **kw)
    within(b, loss, tol)
    within(db, dz, dtol + dz.abs() * HALF[dtype])
    d = sb.distill_loss_backward(weight.cuda(), zc, stats, i, v, **kw)
    within(d, dz, dtol + dz.abs() * HALF[dtype])
    c, dc = sb.distill_loss_and_grad(weight.cuda(), zc, i, v, kind=kind, out=torch.empty(rows, V + 5, device="cuda")[:, 3: 3 + V], **kw)      # off their alignment
    within(c, loss, tol)
    within(dc, dz, dtol + dz.abs() * E)
    over = z.cuda()
    c, dc = sb.distill_loss_and_grad(weight.cuda(), over, i, v, kind=kind, out=over, **kw)
    assert dc is over and torch.equal(over, db) and torch.equal(c, b)
