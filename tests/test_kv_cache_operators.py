"""Rotary positions and their gradient, and writing and reading a paged cache in bf16, fp32, e4m3 or int8, against plain forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2503_01840_b200 import binding as sb

gpu = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}
FLOOR = 2.0 ** -120


def turned(x, pos, freq, layout, mscale, sign=1.0):
    """x float64 [T][H][hd] on the CPU, pair by pair"""
    y, n = x.clone(), len(freq)
    ang = pos.double()[:, None] * freq
    c, s = (ang.cos() * mscale)[:, None], (sign * ang.sin() * mscale)[:, None]
    ia = torch.arange(n) if layout == "half" else 2 * torch.arange(n)
    ib = ia + (n if layout == "half" else 1)
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def turn_error(x, freq, layout, mscale):
    """Most that 32-bit arithmetic may be off by: two products and a sum (2^-24 each of at most |a| + |b|), cosine and sine off by 2^-22
    (the reduced angle's rounding, pi 2^-24, and the functions' last places)."""
    n, e = len(freq), torch.zeros_like(x)
    ia = torch.arange(n) if layout == "half" else 2 * torch.arange(n)
    ib = ia + (n if layout == "half" else 1)
    e[..., ia] = e[..., ib] = (x[..., ia].abs() + x[..., ib].abs()) * mscale * 2.0 ** -21
    return e


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,H,hd,rot,layout", [(1, 1, 2, 2, "half"), (1, 40, 128, 128, "half"), (3, 40, 128, 128, "interleaved"), (129, 5, 64, 32, "half"),
                                               (70, 7, 80, 80, "half"), (33, 3, 80, 20, "interleaved"), (17, 2, 256, 256, "half"), (5, 9, 256, 128, "interleaved"),
                                               (12, 4, 128, 0, "half"), (8, 2, 37, 30, "half"), (600, 3, 128, 64, "half"), (41, 2, 48, 16, "half"), (9, 3, 96, 96, "half"),
                                               (9, 3, 64, 24, "interleaved"), (31, 2, 16, 16, "interleaved")])
def test_rotary_and_gradient(dtype, T, H, hd, rot, layout):
    """Views of a wider projection, in place, positions to 10^6 and below zero, the gradient as the transposed matrix and by differences."""
    g = torch.Generator().manual_seed(T * hd)
    wide = torch.randn(T, H + 2, hd + (8 if hd % 16 == 0 else 3), generator=g).to(DT[dtype])
    pos = torch.randint(-1000, 1000000, (T,), generator=g, dtype=torch.int32)
    freq, _ = sb.rope_frequencies(rot, 1e4, device="cpu") if rot else (torch.zeros(0, dtype=torch.float64), 1.0)
    mscale = 1.1386
    x = wide[:, 1:1 + H, :hd]
    want = turned(x.double(), pos, freq, layout, mscale)
    tol = turn_error(x.double(), freq, layout, mscale) + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
    dev = wide.cuda()
    xd = dev[:, 1:1 + H, :hd]
    got = sb.rotary(xd, pos.cuda(), freq.cuda(), layout=layout, mscale=mscale)
    assert got.is_contiguous() and ((got.cpu().double() - want).abs() <= tol).all()
    grad = torch.randn(T, H, hd, generator=g).to(DT[dtype])
    back = sb.rotary_backward(grad.cuda(), pos.cuda(), freq.cuda(), layout=layout, mscale=mscale)
    want_b = turned(grad.double(), pos, freq, layout, mscale, -1.0)
    tol_b = turn_error(grad.double(), freq, layout, mscale) + (want_b.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
    assert ((back.cpu().double() - want_b).abs() <= tol_b).all()
    # by differences: the map is linear, so <grad, f(x + d) - f(x)> is <gradient, d> up to the errors of the three calls
    d = torch.randn(T, H, hd, generator=g).to(DT[dtype])
    moved = sb.rotary((x + d).cuda(), pos.cuda(), freq.cuda(), layout=layout, mscale=mscale).cpu().double()
    step = (x + d).double() - x.double()
    off = (grad.double() * (moved - got.cpu().double())).sum() - (back.cpu().double() * step).sum()
    most = (grad.double().abs() * (turn_error((x + d).double(), freq, layout, mscale) + tol + moved.abs() * 2.0 ** -8)).sum() + (tol_b * step.abs()).sum()
    assert off.abs() <= most
    # in place: the same bits, nothing beside it touched
    sb.rotary(xd, pos.cuda(), freq.cuda(), layout=layout, mscale=mscale, out=xd)
    assert torch.equal(xd, got)
    rest = torch.ones_like(wide, dtype=torch.bool)
    rest[:, 1:1 + H, :hd] = False
    assert torch.equal(dev.cpu()[rest], wide[rest])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_autograd_takes_the_gradient(dtype, layout):
    """Of a view of a projection, through a sum (whose gradient is expanded), with a second pass over the same x, and of the gradient itself; the same bits as
    rotary_backward's.  No graph where none is wanted."""
    T, H, hd = 33, 3, 64
    g = torch.Generator().manual_seed(7)
    wide = torch.randn(T, H + 1, hd, generator=g).to(DT[dtype]).cuda().requires_grad_()
    pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32).cuda()
    freq = sb.rope_frequencies(hd // 2, 1e4)[0]
    w = torch.randn(T, H, hd, generator=g).to(DT[dtype]).cuda()
    kw = dict(layout=layout, mscale=1.25)
    y = sb.rotary(wide[:, :H], pos, freq, **kw)
    with torch.no_grad():
        plain = sb.rotary(wide[:, :H], pos, freq, **kw)
    assert y.requires_grad and not plain.requires_grad and torch.equal(y, plain) and not sb.rotary(wide.detach(), pos, freq, **kw).requires_grad
    (y * w).sum().backward()
    want = sb.rotary_backward(w, pos, freq, **kw)
    assert torch.equal(wide.grad[:, :H], want) and not wide.grad[:, H:].any()
    wide.grad = None
    sb.rotary(wide[:, :H], pos, freq, **kw).sum().backward()
    assert torch.equal(wide.grad[:, :H], sb.rotary_backward(torch.ones_like(w), pos, freq, **kw))
    x, v = wide.detach()[:, :H].clone().requires_grad_(), w.clone().requires_grad_()
    (gx,) = torch.autograd.grad(sb.rotary(x, pos, freq, **kw), x, v, create_graph=True)
    (gv,) = torch.autograd.grad((gx * x.detach()).sum(), v)
    assert torch.equal(gx, sb.rotary_backward(v.detach(), pos, freq, **kw)) and torch.equal(gv, sb.rotary(x.detach(), pos, freq, **kw))
    (gb,) = torch.autograd.grad(sb.rotary_backward(x, pos, freq, **kw), x, w)
    assert torch.equal(gb, sb.rotary(w, pos, freq, **kw))
    with pytest.raises(ValueError):
        sb.rotary(x, pos, freq, out=torch.empty_like(w), **kw)
    with pytest.raises(ValueError):
        sb.rotary(w, pos, freq, out=x, **kw)
    with torch.no_grad():
        assert torch.equal(sb.rotary(x, pos, freq, out=torch.empty_like(w), **kw), sb.rotary(x, pos, freq, **kw))


def test_frequencies():
    """The kinds of scaling at their ends: fast pairs kept, the slowest divided by the factor, everything between the two."""
    base, one = sb.rope_frequencies(128, 5e5, device="cpu")
    assert one == 1.0 and torch.allclose(base, torch.tensor([5e5 ** (-i / 64) for i in range(64)], dtype=torch.float64), rtol=1e-14, atol=0)
    lin, _ = sb.rope_frequencies(128, 5e5, "linear", 4.0, device="cpu")
    assert torch.equal(lin, base / 4)
    ntk, _ = sb.rope_frequencies(128, 5e5, "ntk", 4.0, device="cpu")
    assert ntk[0] == 1.0 and abs(float(ntk[-1] / base[-1]) - 0.25) < 1e-12
    turns = 8192 * base / (2 * math.pi)
    wav, _ = sb.rope_frequencies(128, 5e5, "wavelength", 8.0, device="cpu")
    assert torch.equal(wav[turns >= 4], base[turns >= 4]) and torch.equal(wav[turns <= 1], base[turns <= 1] / 8)
    rot, m = sb.rope_frequencies(128, 5e5, "rotations", 8.0, 8192, 1.0, 32.0, device="cpu")
    assert abs(m - (0.1 * math.log(8) + 1)) < 1e-12 and torch.equal(rot[turns > 32], base[turns > 32]) and torch.allclose(rot[turns < 0.8], base[turns < 0.8] / 8, rtol=1e-14)
    for f in (wav, rot):
        assert ((f <= base) & (f >= base / 8 * (1 - 1e-12))).all() and (f[1:] < f[:-1]).all()
    for bad in (dict(scaling="cubic"), dict(rot_dim=7), dict(factor=0.5), dict(scaling="ntk", rot_dim=2)):
        with pytest.raises(ValueError):
            sb.rope_frequencies(**{"rot_dim": 64, "theta": 1e4, "device": "cpu", **bad})


@pytest.mark.parametrize("rot,theta,factor,trained", [(128, 5e5, 8.0, 8192), (64, 1e4, 4.0, 4096), (80, 1e6, 2.5, 32768)])
def test_frequencies_between_their_ends(rot, theta, factor, trained):
    """The by-parts scalings pair by pair, with the bounds that they have unless others are given."""
    wav, one = sb.rope_frequencies(rot, theta, "wavelength", factor, trained, device="cpu")
    rotations, m = sb.rope_frequencies(rot, theta, "rotations", factor, trained, device="cpu")
    assert one == 1.0 and m == pytest.approx(0.1 * math.log(factor) + 1.0, rel=1e-15)
    # the pairs (as real numbers) that turn 32 times and once in the trained context, brought to whole ones outwards
    first, last = ((rot / 2) * math.log(trained / (2 * math.pi * turns), theta) for turns in (32.0, 1.0))
    first, last = max(math.floor(first), 0), min(math.ceil(last), rot - 1)
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        length = 2 * math.pi / f                                         # positions of a turn
        if length < trained / 4:
            want = f
        elif length > trained:
            want = f / factor
        else:
            part = (trained / length - 1.0) / 3.0
            want = (1.0 - part) * f / factor + part * f
        assert float(wav[i]) == pytest.approx(want, rel=1e-12)
        part = min(max((i - first) / (last - first), 0.0), 1.0)
        assert float(rotations[i]) == pytest.approx((1.0 - part) * f + part * f / factor, rel=1e-12)
    assert torch.equal(rotations, sb.rope_frequencies(rot, theta, "rotations", factor, trained, 1.0, 32.0, device="cpu")[0])
    assert torch.equal(wav, sb.rope_frequencies(rot, theta, "wavelength", factor, trained, 1.0, 4.0, device="cpu")[0])


def make_cache(g, fmt, pages, G, ps, hd, seqs, pps):
    """Pools that hold junk, a table of distinct pages"""
    dev = {}
    for x in ("k", "v"):
        if fmt in TOP:
            dev[x + "_pool"] = torch.randint(0, 127, (pages, G, ps, hd), generator=g, dtype=torch.uint8).cuda().view(DT[fmt])
            dev[x + "_scale"] = torch.rand(pages, G, ps, generator=g).cuda()
        else:
            dev[x + "_pool"] = torch.randn(pages, G, ps, hd, generator=g).to(DT[fmt]).cuda()
            dev[x + "_scale"] = None
    dev["page_table"] = torch.randperm(pages, generator=g)[: seqs * pps].view(seqs, pps).to(torch.int32).cuda()
    return dev


def raw(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def code_error(z, fmt):
    """Half a step of the format at z, and 2^-20 of z for the 32-bit scale, reciprocal and product"""
    half = torch.full_like(z, 0.5) if fmt == "int8" else torch.maximum(2.0 ** (torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 4), torch.tensor(2.0 ** -10))
    return half + z.abs() * 2.0 ** -20


SHAPES = [(1, 1, 1, 16, 16, "half", 16, 1), (65, 4, 2, 64, 64, "half", 16, 3), (40, 32, 8, 128, 128, "half", 16, 2), (77, 3, 3, 128, 64, "interleaved", 20, 4),
          (23, 5, 1, 80, 80, "half", 3, 2), (30, 4, 2, 256, 256, "interleaved", 1, 1), (19, 2, 2, 48, 16, "half", 64, 2), (200, 16, 2, 64, 64, "interleaved", 32, 5),
          (33, 8, 4, 256, 128, "half", 16, 2), (50, 0, 4, 128, 0, "half", 16, 2), (12, 2, 1, 32, 32, "half", 7, 1), (21, 6, 3, 240, 240, "half", 5, 2)]


@gpu
@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "e4m3"), ("fp32", "e4m3"), ("bf16", "int8"), ("fp32", "int8")])
@pytest.mark.parametrize("T,H,G,hd,rot,layout,ps,seqs", SHAPES)
def test_append_and_read(dtype, fmt, T, H, G, hd, rot, layout, ps, seqs):
    g = torch.Generator().manual_seed(T * hd + ps)
    pps = -(-2 * T // ps) + 1
    pages = seqs * pps + 2
    cache = make_cache(g, fmt, pages, G, ps, hd, seqs, pps)
    before = {x: raw(cache[x]).clone() for x in ("k_pool", "v_pool")} | {x: cache[x].clone() for x in ("k_scale", "v_scale") if cache[x] is not None}
    gap = 8 if hd % 16 == 0 and T % 2 else 0
    qkv = torch.randn(T, H + 2 * G, hd + gap, generator=g).to(DT[dtype])
    qkv[0, H:] = 0                                                       # a row of zeros
    if T > 2:
        qkv[1, H:, :hd] *= 1e-30 if dtype == "fp32" else 2.0 ** -90      # far below one
        qkv[2, H:, :hd] *= 2.0 ** 70                                     # and above
    seq = torch.randint(-1, seqs, (T,), generator=g, dtype=torch.int32) if T > 1 else torch.zeros(1, dtype=torch.int32)
    kvpos = torch.randperm(pps * ps, generator=g)[:T].to(torch.int32)
    pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32)
    freq = sb.rope_frequencies(rot, 5e5, device="cpu")[0] if rot else None
    dev = qkv.cuda()[:, :, :hd]
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    q_out = sb.kv_append(dev[:, H: H + G], dev[:, H + G:], cache["k_pool"], cache["v_pool"], cache["page_table"], seq.cuda(), pos.cuda(),
                         k_scale=cache["k_scale"], v_scale=cache["v_scale"], q=dev[:, :H] if H else None, inv_freq=None if freq is None else freq.cuda(),
                         layout=layout, row_kvpos=kvpos.cuda(), status=status)
    assert not status.any()
    f = torch.zeros(0, dtype=torch.float64) if freq is None else freq
    x = qkv[:, :, :hd].double()
    if H:
        want = turned(x[:, :H], pos, f, layout, 1.0)
        tol = turn_error(x[:, :H], f, layout, 1.0) + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
        assert ((q_out.cpu().double() - want).abs() <= tol).all()
    live = torch.nonzero(seq >= 0).flatten()
    page = cache["page_table"].cpu()[seq[live].long(), (kvpos[live] // ps).long()].long()
    off = (kvpos[live] % ps).long()
    out32 = sb.kv_read(cache["k_pool"], cache["v_pool"], cache["page_table"], seq.cuda(), kvpos.cuda(), k_scale=cache["k_scale"], v_scale=cache["v_scale"],
                       dtype=torch.float32, status=status)
    out16 = sb.kv_read(cache["k_pool"], cache["v_pool"], cache["page_table"], seq.cuda(), kvpos.cuda(), k_scale=cache["k_scale"], v_scale=cache["v_scale"])
    assert not status.any()
    for i, name in enumerate("kv"):
        rows = x[:, H: H + G] if name == "k" else x[:, H + G:]
        err = turn_error(rows, f, layout, 1.0)[live] if name == "k" else torch.zeros_like(rows[live])
        want = (turned(rows, pos, f, layout, 1.0) if name == "k" else rows)[live]
        pool = cache[name + "_pool"].cpu()
        got = raw(pool)[page, :, off]
        if fmt in TOP:
            scale = (want.abs().amax(-1) / TOP[fmt]).clamp_min(FLOOR)
            have = cache[name + "_scale"].cpu()[page, :, off].double()
            assert ((have - scale).abs() <= scale * 2.0 ** -22 + err.amax(-1) / TOP[fmt]).all()
            z = want / have[..., None]
            codes = got.view(DT[fmt]).double()
            assert ((codes - z).abs() <= code_error(z, fmt) + err / have[..., None]).all()
            value = codes * have[..., None]
        else:
            value = got.double()
            assert ((value - want).abs() <= err + (want.abs() * 2.0 ** -8 if fmt == "bf16" else 0)).all()
        # read back: one product, rounded to 32 bits and from there to the output's type; rows of no sequence are zero
        assert torch.equal(out32[i].cpu()[live], value.float()) and torch.equal(out16[i].cpu()[live], value.float().to(torch.bfloat16))
        dead = torch.ones(T, dtype=torch.bool)
        dead[live] = False
        assert not out32[i].cpu()[dead].any() and not out16[i].cpu()[dead].any()
        # nothing else is written
        was = before[name + "_pool"].clone()
        was[page.cuda(), :, off.cuda()] = got.cuda()
        assert torch.equal(raw(cache[name + "_pool"]), was)
        if fmt in TOP:
            was = before[name + "_scale"].clone()
            was[page.cuda(), :, off.cuda()] = have.float().cuda()
            assert torch.equal(cache[name + "_scale"], was)


@gpu
@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("bf16", "int8"), ("fp32", "fp32")])
def test_long_prompt(dtype, fmt):
    """Blocks of several tokens and several rounds of heads, and reading back by blocks of several rows: as the definition, token by token."""
    T, H, G, hd, ps = 3001, 8, 4, 128, 16
    g = torch.Generator().manual_seed(8)
    cache = make_cache(g, fmt, 200, G, ps, hd, 1, 190)
    qkv = torch.randn(T, H + 2 * G, hd, generator=g).to(DT[dtype])
    freq, _ = sb.rope_frequencies(hd, 5e5, device="cpu")
    seq, pos = torch.zeros(T, dtype=torch.int32).cuda(), torch.arange(T, dtype=torch.int32).cuda()
    dev = qkv.cuda()
    sc = {"k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
    args = cache["k_pool"], cache["v_pool"], cache["page_table"], seq, pos
    q = sb.kv_append(dev[:, H: H + G], dev[:, H + G:], *args, **sc, q=dev[:, :H], inv_freq=freq.cuda())
    k, v = sb.kv_read(*args, **sc, dtype=torch.float32)
    x = qkv.double()
    want = turned(x[:, : H + G], pos.cpu(), freq, "half", 1.0)
    err = turn_error(x[:, : H + G], freq, "half", 1.0)
    assert ((q.cpu().double() - want[:, :H]).abs() <= err[:, :H] + (want[:, :H].abs() * 2.0 ** -8 if dtype == "bf16" else 0)).all()
    for got, rows, e in ((k, want[:, H:], err[:, H:]), (v, x[:, H + G:], 0.0)):
        if fmt in TOP:
            scale = (rows.abs().amax(-1, keepdim=True) / TOP[fmt])
            e = e + code_error(rows / scale, fmt) * scale * (1 + 2.0 ** -20)
        assert ((got.cpu().double() - rows).abs() <= e + rows.abs() * 2.0 ** -20).all()


@gpu
def test_many_tokens_of_few_heads():
    """Blocks of sixteen tokens with a few heads each, both types, and blocks that a token's heads do not fill."""
    for T, H, hd, dtype, layout in ((20003, 5, 64, "fp32", "half"), (30001, 3, 64, "bf16", "interleaved"), (901, 1, 128, "bf16", "half"), (9000, 1, 16, "fp32", "half")):
        g = torch.Generator().manual_seed(T)
        x = torch.randn(T, H, hd, generator=g).to(DT[dtype])
        pos = torch.randint(0, 200000, (T,), generator=g, dtype=torch.int32)
        freq, _ = sb.rope_frequencies(hd, 1e4, device="cpu")
        want = turned(x.double(), pos, freq, layout, 1.0)
        got = sb.rotary(x.cuda(), pos.cuda(), freq.cuda(), layout=layout)
        assert ((got.cpu().double() - want).abs() <= turn_error(x.double(), freq, layout, 1.0) + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)).all()


@gpu
@pytest.mark.parametrize("ts,hs", [(1 << 26, 64), ((1 << 26) + 8, 64), (128, 1 << 18), (64, (1 << 18) + 8)])
def test_long_strides(ts, hs):
    """Token and head strides at both sides of what 32-bit offsets in a block allow."""
    g = torch.Generator(device="cuda").manual_seed(3)
    T, H, hd = (17, 2, 64) if ts > 1 << 20 else (2, 40, 64)
    buf = torch.zeros((T - 1) * ts + (H - 1) * hs + hd, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((T, H, hd), (ts, hs, 1))
    x.copy_(torch.randn(T, H, hd, generator=g, device="cuda"))
    pos = torch.arange(1000, 1000 + T, dtype=torch.int32, device="cuda")
    freq, _ = sb.rope_frequencies(hd, 1e4)
    want = sb.rotary(x.contiguous(), pos, freq)
    assert torch.equal(sb.rotary(x, pos, freq), want)
    out = torch.zeros_like(buf).as_strided((T, H, hd), (ts, hs, 1))
    assert torch.equal(sb.rotary(x, pos, freq, out=out), want)


@gpu
@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("bf16", "bf16"), ("fp32", "int8"), ("fp32", "fp32")])
@pytest.mark.parametrize("shift", [1, 4])
def test_heads_off_their_alignment(dtype, fmt, shift):
    """Tensors that start `shift` elements into their allocation give what aligned ones give: the same bits for values, the codes of rotated keys
    within what the two kernels' roundings may differ by."""
    T, H, G, hd, ps = 19, 4, 2, 128, 16
    g = torch.Generator().manual_seed(shift)
    qkv = torch.randn(T, H + 2 * G, hd, generator=g).to(DT[dtype])
    freq, _ = sb.rope_frequencies(hd, 1e4)
    pos, seq = torch.arange(T, dtype=torch.int32).cuda(), torch.zeros(T, dtype=torch.int32).cuda()
    buf = torch.zeros(qkv.numel() + shift, dtype=DT[dtype], device="cuda")
    off = buf[shift:].view(qkv.shape)
    off.copy_(qkv)
    outs = []
    for x in (qkv.cuda(), off):
        cache = make_cache(torch.Generator().manual_seed(1), fmt, 6, G, ps, hd, 1, 4)
        sc = {"k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
        args = cache["k_pool"], cache["v_pool"], cache["page_table"], seq, pos
        q = sb.kv_append(x[:, H: H + G], x[:, H + G:], *args, **sc, q=x[:, :H], inv_freq=freq)
        outs.append((q, sb.rotary(x[:, :H], pos, freq), *sb.kv_read(*args, **sc, dtype=torch.float32)))
    (q0, r0, k0, v0), (q1, r1, k1, v1) = outs
    assert torch.equal(v0, v1) and torch.equal(q0, r0) and torch.equal(q1, r1)
    err = turn_error(qkv[:, :H].double(), freq.cpu(), "half", 1.0).cuda()
    assert ((q0.double() - q1.double()).abs() <= 2 * err + (q0.double().abs() * 2.0 ** -7 if dtype == "bf16" else 0)).all()
    top = k0.abs().amax(-1, keepdim=True).double()
    step = (k0.double().abs() * 2.0 ** -3 + top / 448 * 2.0 ** -8) if fmt == "e4m3" else top / 127 if fmt == "int8" else k0.double().abs() * (2.0 ** -7 if fmt == "bf16" else 0)
    assert ((k0.double() - k1.double()).abs() <= step * 1.001 + 2 * turn_error(qkv[:, H: H + G].double(), freq.cpu(), "half", 1.0).cuda()).all()


def test_tensors_that_are_not_on_the_gpu_are_refused():
    """The C++ part of the binding loads and checks without a device."""
    x, pos = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32)
    freq, _ = sb.rope_frequencies(64, 1e4, device="cpu")
    pool, table = torch.zeros(4, 2, 16, 64), torch.zeros(1, 4, dtype=torch.int32)
    for call in (lambda: sb.rotary(x, pos, freq), lambda: sb.rotary_backward(x, pos, freq), lambda: sb.kv_append(x[:, :2], x[:, :2], pool, pool, table, pos, pos),
                 lambda: sb.kv_read(pool, pool, table, pos, pos), lambda: sb.decode_attention(x, pool, pool, table, pos)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        sb.rotary(None, pos, freq)
    with pytest.raises(TypeError):
        sb.decode_attention(x, pool.half(), pool.half(), table, pos)


@gpu
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hd", [64, 80, 128])
def test_rows_with_infinities_and_nan_read_back_as_nan(fmt, hd):
    g = torch.Generator().manual_seed(3)
    cache = make_cache(g, fmt, 4, 2, 16, hd, 1, 2)
    k = torch.randn(6, 2, hd, generator=g)
    k[1, 0, 5], k[2, 1, 7], k[3, 0, 0] = float("inf"), float("nan"), -float("inf")
    seq, pos = torch.zeros(6, dtype=torch.int32).cuda(), torch.arange(6, dtype=torch.int32).cuda()
    args = cache["k_pool"], cache["v_pool"], cache["page_table"], seq, pos
    sb.kv_append(k.cuda(), k.cuda(), *args, k_scale=cache["k_scale"], v_scale=cache["v_scale"])
    for out in sb.kv_read(*args, k_scale=cache["k_scale"], v_scale=cache["v_scale"], dtype=torch.float32):
        bad = torch.isnan(out).cpu()
        want = torch.zeros(6, 2, hd, dtype=torch.bool)
        want[1, 0], want[2, 1], want[3, 0] = True, True, True
        assert torch.equal(bad, want)


@gpu
def test_out_of_range_rows_are_left_out_and_recorded():
    g = torch.Generator().manual_seed(4)
    for seq, pos, page, site in ((2, 0, 0, 60), (0, 32, 0, 60), (0, -1, 0, 60), (0, 3, 9, 61), (0, 3, -1, 61)):
        cache = make_cache(g, "e4m3", 9, 2, 16, 64, 2, 2)
        if page:
            cache["page_table"][0, 0] = page
        before = raw(cache["k_pool"]).clone()
        k = torch.randn(3, 2, 64, generator=g).cuda()
        rows = torch.tensor([-1, seq, -1], dtype=torch.int32).cuda()
        at = torch.full((3,), pos, dtype=torch.int32).cuda()
        args = cache["k_pool"], cache["v_pool"], cache["page_table"], rows, at
        for call in (lambda st: sb.kv_append(k, k, *args, k_scale=cache["k_scale"], v_scale=cache["v_scale"], status=st),
                     lambda st: sb.kv_read(*args, k_scale=cache["k_scale"], v_scale=cache["v_scale"], status=st)):
            status = torch.zeros(4, dtype=torch.int32, device="cuda")
            out = call(status)
            s = status.tolist()
            assert s[:3] == [2, site, 1], s
            assert torch.equal(raw(cache["k_pool"]), before)
            if out is not None:
                assert not out[0].any() and not out[1].any()
            call(None)


@gpu
def test_empty_calls():
    cache = make_cache(torch.Generator().manual_seed(1), "int8", 4, 2, 16, 64, 2, 2)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    freq, _ = sb.rope_frequencies(64, 1e4)
    assert sb.rotary(torch.zeros(0, 4, 64, device="cuda"), none, freq).shape == (0, 4, 64)
    k = torch.zeros(0, 2, 64, device="cuda")
    q = sb.kv_append(k, k, cache["k_pool"], cache["v_pool"], cache["page_table"], none, none, k_scale=cache["k_scale"], v_scale=cache["v_scale"],
                     q=torch.zeros(0, 6, 64, device="cuda"), inv_freq=freq)
    assert q.shape == (0, 6, 64)
    ko, vo = sb.kv_read(cache["k_pool"], cache["v_pool"], cache["page_table"], none, none, k_scale=cache["k_scale"], v_scale=cache["v_scale"])
    assert ko.shape == vo.shape == (0, 2, 64)


@gpu
def test_refusals():
    cache = make_cache(torch.Generator().manual_seed(1), "int8", 4, 2, 16, 64, 2, 2)
    args = lambda **kw: [{**cache, **kw}[n] for n in ("k_pool", "v_pool", "page_table")]
    sc = {"k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = torch.zeros(1, 2, 64, device="cuda")
    freq, _ = sb.rope_frequencies(64, 1e4)
    for bad in (dict(row_seq=one.long()), dict(row_seq=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(row_pos=one.cpu()), dict(k=k[..., :32]),
                dict(v=k.bfloat16()), dict(k_scale=None), dict(k_scale=cache["k_scale"][:2]), dict(v_pool=cache["v_pool"][:2]),
                dict(page_table=cache["page_table"].long()), dict(q=torch.zeros(2, 4, 64, device="cuda")), dict(inv_freq=freq.float()), dict(layout="both", inv_freq=freq),
                dict(k=torch.zeros(1, 64, 2, device="cuda").transpose(1, 2)), dict(status=one)):
        call = {"k": k, "v": k, "k_pool": cache["k_pool"], "v_pool": cache["v_pool"], "page_table": cache["page_table"], "row_seq": one, "row_pos": one, **sc, **bad}
        with pytest.raises(ValueError):
            sb.kv_append(**call)
    with pytest.raises(sb.SpecError) as e:                               # an fp32 cache holds no bf16 keys
        c = make_cache(torch.Generator().manual_seed(1), "fp32", 4, 2, 16, 64, 2, 2)
        sb.kv_append(k.bfloat16(), k.bfloat16(), c["k_pool"], c["v_pool"], c["page_table"], one, one)
    assert e.value.code == -1
    with pytest.raises(sb.SpecError) as e:                               # more rotated dimensions than a head has
        sb.kv_append(k, k, *args(), one, one, **sc, inv_freq=sb.rope_frequencies(66, 1e4)[0])
    assert e.value.code == -1
    with pytest.raises(sb.SpecError) as e:                               # head sizes of a cache are multiples of 16
        c = make_cache(torch.Generator().manual_seed(1), "fp32", 4, 2, 16, 40, 2, 2)
        sb.kv_append(k[..., :40].contiguous(), k[..., :40].contiguous(), c["k_pool"], c["v_pool"], c["page_table"], one, one)
    assert e.value.code == -8
    with pytest.raises(TypeError):
        sb.kv_read(cache["k_pool"].to(torch.int16), cache["v_pool"].to(torch.int16), cache["page_table"], one, one)
    with pytest.raises(TypeError):
        sb.kv_read(*args(), one, one, **sc, dtype=torch.float16)
    x = torch.zeros(4, 2, 64, device="cuda")
    four = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(positions=one), dict(inv_freq=None), dict(out=x[:, :1]), dict(out=x.bfloat16()), dict(layout="")):
        with pytest.raises(ValueError):
            sb.rotary(**{"x": x, "positions": four, "inv_freq": freq, **bad})
    with pytest.raises(sb.SpecError):
        sb.rotary(torch.zeros(4, 1, 512, device="cuda"), four, freq)
    with pytest.raises(TypeError):
        sb.rotary(x.half(), four, freq)


def test_c_refusals_without_a_device():
    """Argument checks of the C entry points come before anything touches the device."""
    import ctypes as C
    L = sb.lib()
    rope = sb._Rope(16, 64, 0, 1.0)
    good = dict(k=256, v=256, k_scale=None, v_scale=None, page_table=256, n_seq=1, pages_per_seq=1, page_size=16, num_pages=4, n_kv_heads=2, head_dim=64, format=1)
    cache = lambda **kw: C.byref(sb._KvCache(*[{**good, **kw}[n] for n, _ in sb._KvCache._fields_]))
    append = lambda c, dtype=1, tokens=1, k=256, r=None: L.spec_kv_append(dtype, None, 0, 0, None, 0, k, 128, 64, 256, 128, 64, 256, 256, None, tokens, r, c, None, None)
    assert append(cache(), tokens=0) == 0 and append(cache(), tokens=-1) == -1 and append(cache(), dtype=0) == -1 and append(cache(), dtype=5) == -1
    assert append(cache(k=None)) == -2 and append(cache(format=2)) == -2 and append(cache(format=9)) == -1 and append(cache(page_size=0)) == -1
    assert append(cache(head_dim=24)) == -8 and append(cache(head_dim=272)) == -8 and append(cache(k=264)) == -1 and append(cache(), k=None) == -2
    assert append(cache(num_pages=1 << 30)) == -8 and append(cache(pages_per_seq=1 << 30)) == -8 and append(None) == -2 and append(cache(), k=257) == -1
    assert append(cache(), r=C.byref(sb._Rope(16, 66, 0, 1.0))) == -1 and append(cache(), r=C.byref(sb._Rope(16, 63, 0, 1.0))) == -1
    assert append(cache(), r=C.byref(sb._Rope(None, 64, 0, 1.0))) == -2 and append(cache(), r=C.byref(sb._Rope(16, 64, 2, 1.0))) == -1
    turn = lambda x=256, out=512, ts=128, dtype=1, hd=64, r=rope: L.spec_rotary(dtype, x, 128, 64, out, ts, 64, 256, 1, 2, hd, C.byref(r) if r else None, 0, None)
    assert turn(x=None) == -2 and turn(r=None) == -2 and turn(hd=272) == -8 and turn(hd=0) == -1 and turn(dtype=2) == -1 and turn(out=256, ts=256) == -1
    read = lambda c, rows=1, dtype=1, out=512: L.spec_kv_read(c, 256, 256, rows, dtype, out, 512, None, None)
    assert read(cache(), rows=0) == 0 and read(cache(), rows=-1) == -1 and read(cache(), dtype=2) == -1 and read(cache(), out=None) == -2 and read(cache(), out=520) == -1
    n = L.spec_decode_attention_workspace_bytes()
    attend = lambda c, dtype=1, batch=1, heads=4, scale=0.0, q=256, ts=256, ws=256, nb=n: L.spec_decode_attention(dtype, q, ts, c, 256, batch, heads, scale, 512, None, ws, nb, None, None)
    assert attend(cache(), batch=0) == 0 and attend(cache(), batch=2) == -1 and attend(cache(), heads=3) == -1 and attend(cache(), scale=math.inf) == -1
    assert attend(cache(), scale=math.nan) == -1 and attend(cache(), q=None) == -2 and attend(cache(), q=258) == -1 and attend(cache(), ts=257) == -1
    assert attend(cache(), ws=None) == -2 and attend(cache(), ws=264) == -3 and attend(cache(), nb=n - 1) == -3 and attend(cache(n_seq=9000), batch=9000) == -8
    assert attend(cache(), dtype=0) == -1


@gpu
def test_tensors_of_another_gpu_are_refused(monkeypatch):
    """Each tensor of a call by turns; torch's fake tensors stand for those of a second GPU (they have its device and no memory, and it need not be there)."""
    from torch._subclasses import fake_tensor
    monkeypatch.setattr(fake_tensor, "init_gpu_context", lambda device: None)
    fake = fake_tensor.FakeTensorMode()

    def away(t):
        with fake:
            return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda:1")

    cache = make_cache(torch.Generator().manual_seed(1), "int8", 4, 2, 16, 64, 2, 2)
    x, k, pos = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    freq, _ = sb.rope_frequencies(64, 1e4)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    seq = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    calls = ((sb.rotary, dict(x=x, positions=pos, inv_freq=freq, out=torch.empty_like(x))),
             (sb.rotary_backward, dict(grad=x, positions=pos, inv_freq=freq, out=torch.empty_like(x))),
             (sb.kv_append, dict(cache, k=k, v=k.clone(), row_seq=seq, row_pos=pos, row_kvpos=pos.clone(), q=x, inv_freq=freq, status=status)),
             (sb.kv_read, dict(cache, row_seq=seq, row_kvpos=pos, status=status)),
             (sb.decode_attention, dict(cache, q=x, lengths=pos, out=torch.empty_like(x), workspace=sb.decode_workspace(), status=status)))
    for f, good in calls:
        f(**good)
        for name, t in good.items():
            with pytest.raises(ValueError):
                f(**{**good, name: away(t)})
        f(**good)
    assert not status.any()


@gpu
def test_more_than_an_int_counts_is_refused():
    """Tokens and heads are handed on in 32 bits.  (Expanded tensors: they have one element's memory, and no output is made for them.)"""
    cache = make_cache(torch.Generator().manual_seed(1), "int8", 4, 2, 16, 64, 2, 2)
    freq, _ = sb.rope_frequencies(64, 1e4)
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.zeros(1, 1, 64, device="cuda")
    many = (1 << 32) + 1
    for wide in (x.expand(1, many, 64), x.expand(many, 1, 64)):
        with pytest.raises(ValueError, match="2\\^31"):
            sb.rotary(wide, one, freq)
        with pytest.raises(ValueError, match="2\\^31"):
            sb.kv_append(x.expand(1, 2, 64), x.expand(1, 2, 64), cache["k_pool"], cache["v_pool"], cache["page_table"], one, one, cache["k_scale"], cache["v_scale"], q=wide)
        with pytest.raises(ValueError, match="2\\^31"):
            sb.decode_attention(wide, cache["k_pool"], cache["v_pool"], cache["page_table"], one, cache["k_scale"], cache["v_scale"])
    with pytest.raises(ValueError, match="2\\^31"):
        sb.kv_read(cache["k_pool"], cache["v_pool"], cache["page_table"], one.expand(many), one.expand(many), cache["k_scale"], cache["v_scale"])
