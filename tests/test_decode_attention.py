"""Attention of one new token per sequence over a paged cache in bf16, fp32, e4m3 or int8, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2503_01840_b200 import binding as sb

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}


def pools(g, fmt, pages, G, ps, hd, spread=0.0):
    """Random pools; spread: the scales of tokens differ by up to 2^spread either way."""
    out = {}
    for x in ("k", "v"):
        t = torch.randn(pages, G, ps, hd, generator=g, device="cuda")
        if spread:
            t *= 2.0 ** ((torch.rand(pages, G, ps, 1, generator=g, device="cuda") * 2 - 1) * (spread if x == "v" else 1.0))
        if fmt in TOP:
            s = (t.abs().amax(-1) / TOP[fmt]).clamp_min(2.0 ** -120)
            y = t / s[..., None]
            out[x + "_pool"], out[x + "_scale"] = (y.round().clamp(-127, 127) if fmt == "int8" else y.clamp(-448, 448)).to(DT[fmt]), s
        else:
            out[x + "_pool"], out[x + "_scale"] = t.to(DT[fmt]), None
    return out


def u8(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def spoil(cache, table, lens, ps):
    """NaN wherever no sequence has a position"""
    pages = cache["k_pool"].shape[0]
    used = torch.zeros(pages * ps, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        used[table[b].long()[at // ps] * ps + at % ps] = True
    free = ~used.view(pages, ps)
    for x in ("k", "v"):
        fmt = cache[x + "_pool"].dtype
        view = u8(cache[x + "_pool"]).transpose(1, 2)
        view[free] = 0x7F if fmt == torch.float8_e4m3fn else 0x80 if fmt == torch.int8 else math.nan
        if cache[x + "_scale"] is not None:
            cache[x + "_scale"].transpose(1, 2)[free] = math.nan


def definition(q, cache, table, lens, ps, scale):
    """(out, lse, sum p |v|) in 64 bits"""
    B, H, hd = q.shape
    G = cache["k_pool"].shape[1]
    out, mag = torch.zeros(2, B, H, hd, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n == 0:
            continue
        at = torch.arange(n, device="cuda")
        page, off = table[b].long()[at // ps], at % ps
        k, v = (u8(cache[x])[page, :, off].view(cache[x].dtype).double() for x in ("k_pool", "v_pool"))
        if cache["k_scale"] is not None:
            k, v = k * cache["k_scale"][page, :, off].double()[..., None], v * cache["v_scale"][page, :, off].double()[..., None]
        k, v = (t.repeat_interleave(H // G, 1) for t in (k, v))
        s = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
        lse[b] = torch.logsumexp(s, -1)
        p = (s - lse[b][:, None]).exp()
        out[b], mag[b] = torch.einsum("hn,nhd->hd", p, v), torch.einsum("hn,nhd->hd", p, v.abs())
    return out, lse, mag


def check(q, cache, table, lens, ps, scale=None, **kw):
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = (q, cache["k_pool"], cache["v_pool"], table, length)
    out, lse = sb.decode_attention(*args, k_scale=cache["k_scale"], v_scale=cache["v_scale"], scale=scale, want_lse=True, status=status, **kw)
    want, want_lse, mag = definition(q, cache, table, lens, ps, scale if scale is not None else q.shape[-1] ** -0.5)
    assert not status.any()
    # Scores are sums of up to 256 fp32 terms with rounding errors of random sign, 2^-24 of terms that add up to some tens: 5e-5 is ten
    # times what that gives, and a score of s is rounded to 2^-24 s a few times besides.  bf16 queries: probabilities rounded
    # by 2^-8 at most, and the output by as much.
    bf16 = q.dtype == torch.bfloat16
    empty = torch.tensor([n == 0 for n in lens], device="cuda")
    high = want_lse[~empty].abs().max().item() * 2.0 ** -21 if not empty.all() else 0.0
    tol = mag * (2.0 ** -7 if bf16 else 0.0) + (mag + 1e-30) * (5e-5 + high)
    assert ((out.double() - want).abs() <= tol).all(), ((out.double() - want).abs() / (mag + 1e-30)).max()
    assert not out[empty].any() and (lse[empty] == -math.inf).all()
    assert ((lse - want_lse)[~empty].abs() <= 5e-5 + 1e-6 * want_lse[~empty].abs()).all()
    if not empty.all():
        rel = ((out.double() - want).norm() / want.norm()).item()
        # 1.66e-3 from the output's rounding and 1.13e-3 from the probabilities': over few rows no more than their worst, 2^-8 each
        assert rel < ((2.5e-3 if q[~empty].shape[0] * q.shape[1] >= 64 else 2.0 ** -7) if bf16 else 1e-5 + high), rel
    again, lse2 = sb.decode_attention(*args, k_scale=cache["k_scale"], v_scale=cache["v_scale"], scale=scale, want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    return out, lse


def table_for(g, lens, ps, extra=2):
    """Distinct pages in random order; entries that no position reaches are no pages at all"""
    need = [-(-n // ps) for n in lens]
    ids = torch.randperm(sum(need) + extra, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(need + [1])), -5, dtype=torch.int32, device="cuda")
    table[:, -1] = 1 << 30
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at: at + n]
        at += n
    return table, sum(need) + extra


KINDS = [("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "int8"), ("fp32", "fp32"), ("fp32", "e4m3"), ("fp32", "int8")]
HEADS = [(32, 8, 128), (5, 5, 128), (4, 2, 64), (16, 2, 64), (8, 2, 256), (6, 2, 48), (10, 2, 80), (16, 1, 128), (24, 1, 64), (3, 3, 16), (18, 2, 240), (7, 1, 128), (17, 1, 256)]
LENS = [([1], 16), ([0], 16), ([0, 5, 0], 16), ([15, 16, 17, 33, 1], 16), ([1000, 3, 0, 257], 20), ([64, 128, 127, 129], 64), ([31, 2, 7], 1), ([90], 3), ([4099], 16)]


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("H,G,hd", HEADS)
def test_against_the_definition(dtype, fmt, H, G, hd):
    for i, (lens, ps) in enumerate(LENS):
        g = torch.Generator(device="cuda").manual_seed(H * hd + i)
        table, pages = table_for(g, lens, ps)
        cache = pools(g, fmt, pages, G, ps, hd)
        spoil(cache, table, lens, ps)
        wide = torch.randn(len(lens), H + 2 * G, hd, generator=g, device="cuda").to(DT[dtype])
        check(wide[:, :H], cache, table, lens, ps)


@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_many_sequences(dtype, fmt):
    """More sequences than CTAs, most of them of a tile or none; and a batch that has one long sequence among short ones."""
    for B, H, G, hd, ps, most, long in ((700, 4, 2, 64, 16, 40, 0), (3000, 2, 1, 64, 4, 3, 0), (37, 8, 2, 128, 16, 30, 9000)):
        g = torch.Generator(device="cuda").manual_seed(B)
        lens = torch.randint(0, most, (B,), generator=g, device="cuda").tolist()
        if long:
            lens[B // 2] = long
        table, pages = table_for(g, lens, ps)
        cache = pools(g, fmt, pages, G, ps, hd)
        q = torch.randn(B, H, hd, generator=g, device="cuda").to(DT[dtype])
        check(q, cache, table, lens, ps)


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("B,H,G,hd,ps,least,most", [(60, 32, 8, 128, 16, 0, 300),        # several (sequence, KV head)s a CTA, dealt out evenly
                                                    (20, 24, 8, 128, 16, 90, 100),       # whole ones, one or two a CTA
                                                    (33, 40, 40, 128, 16, 1, 40),        # many short ones, whole
                                                    (33, 64, 2, 128, 64, 200, 900),      # chunks of heads
                                                    (2, 16, 1, 64, 32, 3000, 5000),      # one of them shared by all CTAs, in two levels of joins
                                                    (3, 4, 1, 256, 16, 2000, 2500)])
def test_ways_of_dealing_out_the_work(dtype, fmt, B, H, G, hd, ps, least, most):
    g = torch.Generator(device="cuda").manual_seed(B * hd)
    lens = torch.randint(least, most + 1, (B,), generator=g, device="cuda").tolist()
    table, pages = table_for(g, lens, ps)
    cache = pools(g, fmt, pages, G, ps, hd)
    spoil(cache, table, lens, ps)
    check(torch.randn(B, H, hd, generator=g, device="cuda").to(DT[dtype]), cache, table, lens, ps)


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("B,H,G,hd", [(24, 16, 1, 128), (12, 28, 2, 128), (3, 128, 8, 128), (23, 15, 1, 64), (11, 66, 2, 128), (5, 80, 5, 256)])
def test_fourteen_and_more_heads_of_a_kv_head(dtype, fmt, B, H, G, hd):
    """All of them walk the cache together, or by chunks; with 22 (sequence, KV head)s and more."""
    g = torch.Generator(device="cuda").manual_seed(B * H)
    lens = torch.randint(0, 500, (B,), generator=g, device="cuda").tolist()
    table, pages = table_for(g, lens, 16)
    cache = pools(g, fmt, pages, G, 16, hd)
    spoil(cache, table, lens, 16)
    check(torch.randn(B, H, hd, generator=g, device="cuda").to(DT[dtype]), cache, table, lens, 16)


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("hd", [128, 80])
def test_scales_queries_and_scores_of_very_different_sizes(dtype, fmt, hd):
    """Values whose scales differ by 2^16 from token to token, queries of 2^-60 and 2^40, a scale of its own, scores that rise with the
    position so that every tile moves the maximum, and a first token that outweighs all others."""
    g = torch.Generator(device="cuda").manual_seed(hd)
    lens, ps = [700, 33, 1], 16
    table, pages = table_for(g, lens, ps)
    cache = pools(g, fmt, pages, 2, ps, hd, spread=8.0)
    q = torch.randn(3, 8, hd, generator=g, device="cuda").to(DT[dtype])
    check(q, cache, table, lens, ps, scale=0.3)
    check(q * 2.0 ** -60, cache, table, lens, ps, scale=2.0 ** 58)
    check(q * 2.0 ** 40, cache, table, lens, ps, scale=2.0 ** -43)
    check(q * 2.0 ** 40, cache, table, lens, ps, scale=-(2.0 ** -43))
    if fmt in TOP:
        ramp = torch.zeros(pages, 2, ps, device="cuda")
        for b, n in enumerate(lens):
            at = torch.arange(n, device="cuda")
            ramp[table[b].long()[at // ps], :, at % ps] = (0.01 * at.float())[:, None]
        flat = dict(cache, k_pool=torch.ones_like(cache["k_pool"], dtype=torch.float32).to(DT[fmt]), k_scale=ramp)
        up = torch.ones_like(q)
        check(up, flat, table, lens, ps, scale=1.0 / hd * 8)             # scores 0, 0.08, 0.16, ...
        check(up, flat, table, lens, ps, scale=-8.0 / hd)
        check(up, flat, table, lens, ps, scale=-800.0 / hd)              # all but the first tokens underflow


@pytest.mark.parametrize("dtype,fmt", KINDS[1:3] + KINDS[4:])
@pytest.mark.parametrize("H,G,hd", [(8, 2, 128), (16, 1, 64), (4, 1, 256), (8, 2, 80)])
@pytest.mark.parametrize("at", [0, 17, 350, 699])
def test_a_value_far_above_the_others_that_hardly_counts(dtype, fmt, H, G, hd, at):
    """One position's values are 2^16 .. 2^40 times the others'.  Half of the heads see its key far below their maximum, so that it is next to nothing of
    their output; for the other half of them it outweighs everything.  Neither may cost the other its bits."""
    g = torch.Generator(device="cuda").manual_seed(at + hd)
    lens, ps = [700, 64], 16
    table, pages = table_for(g, lens, ps)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for power in (16, 24, 40):
        cache = pools(g, fmt, pages, G, ps, hd)
        where = (int(table[0, at // ps]), slice(None), at % ps)
        cache["v_scale"][where] *= 2.0 ** power
        code = torch.full((G, hd), TOP[fmt], device="cuda")
        cache["k_pool"][where] = code.to(DT[fmt])
        cache["k_scale"][where] = 1.0 / TOP[fmt]                         # a key of ones
        q = torch.randn(2, H, hd, generator=g, device="cuda") * 0.5
        # q . ones = -+ 2 power sqrt(hd): a score of that over sqrt(hd), 2^-2.9 power of the others' weight or 2^2.9 power
        q -= q.mean(-1, keepdim=True)
        q[:, 0::2] -= 2.0 * power / hd ** 0.5
        q[:, 1::2] += 2.0 * power / hd ** 0.5
        q = q.to(DT[dtype])
        sc = {"k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
        out, lse = sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, **sc, want_lse=True)
        want, want_lse, mag = definition(q, cache, table, lens, ps, hd ** -0.5)
        # the largest p times scale of each head: as an output over values whose every element is their scale
        largest = torch.zeros(2, H, 1, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            t = torch.arange(n, device="cuda")
            page, off = table[b].long()[t // ps], t % ps
            k = (u8(cache["k_pool"])[page, :, off].view(DT[fmt]).double() * cache["k_scale"][page, :, off].double()[..., None]).repeat_interleave(H // G, 1)
            p = (torch.einsum("hd,nhd->hn", q[b].double(), k) * hd ** -0.5 - want_lse[b][:, None]).exp()
            largest[b, :, 0] = (p * cache["v_scale"][page, :, off].double().repeat_interleave(H // G, 1).T).amax(1)
        # As in check(); and products of a probability and a scale are f16, the largest of a run at 2^6 or more of its 2^-25: no position is off by more than 2^-31 of the
        # largest product times the largest code.  (Where that one's code is 0 the other positions' sum may be below it.)
        high = want_lse.abs().max().item() * 2.0 ** -21
        tol = mag * ((2.0 ** -7 if dtype == "bf16" else 0.0) + 5e-5 + high) + max(lens) * 2.0 ** -31 * largest * TOP[fmt]
        assert ((out.double() - want).abs() <= tol).all(), ((out.double() - want).abs() / tol).max()
        assert ((lse - want_lse).abs() <= 5e-5 + 1e-6 * want_lse.abs()).all()


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "e4m3")])
def test_infinities_and_nan(dtype, fmt):
    """Rows whose scores are all -inf give 0 and -inf; a NaN among the visible positions reaches the heads that see it and no others."""
    g = torch.Generator(device="cuda").manual_seed(9)
    lens, ps, H, G, hd = [300, 40], 16, 4, 2, 128
    table, pages = table_for(g, lens, ps)
    cache = pools(g, fmt, pages, G, ps, hd)
    q = torch.randn(2, H, hd, generator=g, device="cuda").to(DT[dtype])
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    run = lambda: sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, k_scale=cache["k_scale"], v_scale=cache["v_scale"], want_lse=True)
    kf = cache["k_pool"].float()
    kf[..., 5] = -1.0 - kf[..., 5].abs()
    cache["k_pool"] = kf.to(DT[fmt])
    out, lse = run()
    assert torch.isfinite(out).all()
    q[0, 1, 5] = float("inf")
    out2, lse2 = run()
    assert (out2[0, 1] == 0).all() and lse2[0, 1] == -math.inf
    same = torch.ones(2, H, dtype=torch.bool, device="cuda")
    same[0, 1] = False
    assert torch.equal(out2[same], out[same]) and torch.equal(lse2[same], lse[same])
    q[0, 1, 5] = 0.0
    out, lse = run()
    where = (int(table[0, 7]), 1, 3)                                     # position 115 of sequence 0, KV head 1: heads 2 and 3
    if fmt == "e4m3":
        cache["v_scale"][where] = math.nan
    else:
        cache["v_pool"][where][9] = math.nan
    out3, lse3 = run()
    hit = torch.zeros(2, H, hd, dtype=torch.bool, device="cuda")
    hit[0, 2:, 9] = True
    if fmt == "e4m3":
        hit[0, 2:] = True
    assert torch.equal(torch.isnan(out3), hit) and torch.equal(out3[~hit], out[~hit]) and torch.equal(lse3, lse)


def test_offsets_past_32_bits():
    """A pool of more than 2^31 elements, the sequence's pages at its end."""
    G, ps, hd = 8, 16, 256
    pages = (1 << 31) // (G * ps * hd) + 40
    for fmt, dtype in (("int8", "bf16"), ("e4m3", "fp32")):
        g = torch.Generator(device="cuda").manual_seed(2)
        cache = {x: torch.zeros(pages, G, ps, hd, dtype=torch.uint8, device="cuda").view(DT[fmt]) for x in ("k_pool", "v_pool")}
        cache |= {x: torch.zeros(pages, G, ps, device="cuda") for x in ("k_scale", "v_scale")}
        n = 500
        table = (pages - 1 - torch.randperm(-(-n // ps), generator=g, device="cuda")).to(torch.int32)[None]
        k, v = torch.randn(2, n, G, hd, generator=g, device="cuda").to(DT[dtype])
        seq, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
        sc = {"k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
        sb.kv_append(k, v, cache["k_pool"], cache["v_pool"], table, seq, pos, **sc)
        ko, vo = sb.kv_read(cache["k_pool"], cache["v_pool"], table, seq, pos, **sc, dtype=torch.float32)
        assert ((ko - k.float()).norm() / k.float().norm()) < 0.05 and ((vo - v.float()).norm() / v.float().norm()) < 0.05
        check(torch.randn(1, 16, hd, generator=g, device="cuda").to(DT[dtype]), cache, table, [n], ps)


def test_streams_graphs_and_workspaces():
    """A side stream has its own workspace; a captured call takes one of the caller's and replays on changed inputs; results are the same bits."""
    g = torch.Generator(device="cuda").manual_seed(5)
    lens, ps, H, G, hd = [2000, 17, 0, 400], 16, 32, 8, 128
    table, pages = table_for(g, lens, ps)
    cache = pools(g, "e4m3", pages, G, ps, hd)
    q = torch.randn(4, H, hd, generator=g, device="cuda").to(torch.bfloat16)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    sc = {"k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
    out = sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, **sc)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mine = sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, **sc)
    side.synchronize()
    assert torch.equal(mine, out)
    ws, static, held = sb.decode_workspace(), q.clone(), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.decode_attention(static, cache["k_pool"], cache["v_pool"], table, length, **sc, out=held, workspace=ws)
    for s in (1.0, -0.5, 2.0):
        static.copy_(q * s)
        graph.replay()
        assert torch.equal(held, sb.decode_attention(static, cache["k_pool"], cache["v_pool"], table, length, **sc))
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(other, stream=torch.cuda.Stream()):            # a capture of a stream without a workspace has to bring one
        static.add_(0)
        with pytest.raises(ValueError):
            sb.decode_attention(static, cache["k_pool"], cache["v_pool"], table, length, **sc, out=held)
    with pytest.raises(sb.SpecError) as e:
        sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, **sc, workspace=ws[:1024])
    assert e.value.code == -3


def test_captures_do_not_get_a_streams_kept_workspace():
    """Nor on a stream that has one from the calls before: two graphs, or a graph and a call on that stream, would share it.  Two graphs with a
    workspace each replay side by side, beside calls on the stream of their captures."""
    g = torch.Generator(device="cuda").manual_seed(15)
    lens, ps, H, G, hd = [3000, 17, 900], 16, 32, 8, 128
    table, pages = table_for(g, lens, ps)
    cache = pools(g, "e4m3", pages, G, ps, hd)
    qs = [torch.randn(3, H, hd, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3)]
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    run = lambda q, **kw: sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, k_scale=cache["k_scale"], v_scale=cache["v_scale"], **kw)
    want = [run(q) for q in qs]
    warm, beside = torch.cuda.Stream(), torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        run(qs[0])
    warm.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=warm):
        qs[0].add_(0)
        with pytest.raises(ValueError):
            run(qs[0])
    graphs, outs = [], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        outs.append(torch.empty_like(qs[i]))
        ws = sb.decode_workspace()
        torch.cuda.synchronize()
        with torch.cuda.graph(graphs[i], stream=warm):
            for _ in range(8):
                run(qs[i], out=outs[i], workspace=ws)
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(beside):
            graphs[0].replay()
        graphs[1].replay()
        with torch.cuda.stream(warm):
            mine = [run(qs[2]) for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and all(torch.equal(m, want[2]) for m in mine)


def test_lengths_and_pages_out_of_range_are_recorded():
    g = torch.Generator(device="cuda").manual_seed(6)
    lens, ps, H, G, hd = [40, 20], 16, 4, 2, 64
    table, pages = table_for(g, lens, ps)
    cache = pools(g, "e4m3", pages, G, ps, hd)
    q = torch.randn(2, H, hd, generator=g, device="cuda").to(torch.bfloat16)
    table[1] = table[0]
    run = lambda ln, tb: sb.decode_attention(q, cache["k_pool"], cache["v_pool"], tb, torch.tensor(ln, dtype=torch.int32, device="cuda"),
                                             k_scale=cache["k_scale"], v_scale=cache["v_scale"], status=status)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    out = run([40, -3], table)
    assert status.tolist()[:3] == [2, 62, 1] and not out[1].any()
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert torch.equal(run([40, 49], table)[1], run([40, 48], table)[1]) and status.tolist() == [2, 62, 1, 49]
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    broken = table.clone()
    broken[1, 1] = pages
    out = run([40, 32], broken)
    assert status.tolist() == [2, 63, 1, pages]
    # the positions of the page that is none are left out
    assert torch.equal(out[1], run([40, 16], table)[1])


def test_refusals():
    g = torch.Generator(device="cuda").manual_seed(6)
    cache = pools(g, "int8", 4, 2, 16, 64)
    table, n = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    q = torch.zeros(2, 4, 64, device="cuda")
    good = {"q": q, "k_pool": cache["k_pool"], "v_pool": cache["v_pool"], "page_table": table, "lengths": n, "k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}
    sb.decode_attention(**good)
    for bad in (dict(lengths=n.long()), dict(lengths=n[:1]), dict(q=q[..., :32]), dict(q=torch.zeros(2, 64, 4, device="cuda").transpose(1, 2)), dict(out=q[:1]),
                dict(out=q.bfloat16()), dict(k_scale=None), dict(scale=0.0), dict(scale=math.nan), dict(page_table=table.t()), dict(status=n)):
        with pytest.raises(ValueError):
            sb.decode_attention(**{**good, **bad})
    for bad, code in ((dict(q=torch.zeros(2, 3, 64, device="cuda")), -1), (dict(q=torch.zeros(3, 4, 64, device="cuda"), lengths=torch.ones(3, dtype=torch.int32, device="cuda")), -1),
                      (dict(scale=math.inf), -1), (dict(q=torch.zeros(2 * 4 * 64 + 1, device="cuda")[1:].view(2, 4, 64)), -1)):
        with pytest.raises(sb.SpecError) as e:
            sb.decode_attention(**{**good, **bad})
        assert e.value.code == code
    with pytest.raises(TypeError):
        sb.decode_attention(**{**good, "q": q.half()})


def test_a_scale_that_is_zero_in_32_bits_is_refused():
    """The C entry point takes 0 for its default.  The smallest scales that are not 0 count: all scores then are as good as 0."""
    g = torch.Generator(device="cuda").manual_seed(6)
    cache = pools(g, "int8", 4, 2, 16, 64)
    table, n = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2), torch.tensor([20, 32], dtype=torch.int32, device="cuda")
    q = torch.randn(2, 4, 64, generator=g, device="cuda")
    run = lambda scale: sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, n, k_scale=cache["k_scale"], v_scale=cache["v_scale"], scale=scale)
    for scale in (1e-60, -1e-60, 2.0 ** -151):
        with pytest.raises(ValueError):
            run(scale)
    v = cache["v_pool"].float() * cache["v_scale"][..., None]
    for scale in (2.0 ** -149, -1e-40):
        out = run(scale)
        for b in range(2):
            mean = v[table[b].long()].transpose(1, 2).reshape(32, 2, 64)[: int(n[b])].mean(0).repeat_interleave(2, 0)
            # sums of at most 32 values of up to 4 or so, rounded to 22 bits of the products at worst
            assert ((out[b] - mean).abs() <= 1e-5).all()


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("hd", [64, 80, 128, 256])
def test_scores_far_below_zero(dtype, fmt, hd):
    """All scores of a head at -1e29 .. -2e38: where they are equal the output is the mean of the values, where one is higher than the others by a 64th it is that one's value."""
    g = torch.Generator(device="cuda").manual_seed(hd)
    lens, ps, H, G = [77, 16, 1], 16, 4, 2
    table, pages = table_for(g, lens, ps)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = -torch.ones(3, H, hd, device="cuda").to(DT[dtype])
    for size in (1e29, 1e31, 1e35, 2e38):
        for best in (None, 0, 13):
            cache = pools(g, fmt, pages, G, ps, hd)
            k = torch.full((pages, G, ps), size / hd, device="cuda")
            if best is not None:
                for b, n in enumerate(lens):
                    k[int(table[b, min(best, n - 1) // ps]), :, min(best, n - 1) % ps] *= 63 / 64
            if fmt in TOP:
                cache["k_pool"], cache["k_scale"] = torch.ones_like(cache["k_pool"], dtype=torch.float32).to(DT[fmt]), k
            else:
                cache["k_pool"] = k[..., None].expand(-1, -1, -1, hd).contiguous().to(DT[fmt])
            out, lse = sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, length, k_scale=cache["k_scale"], v_scale=cache["v_scale"], scale=1.0, want_lse=True)
            for b, n in enumerate(lens):
                t = torch.arange(n, device="cuda") if best is None else torch.tensor([min(best, n - 1)], device="cuda")
                page, off = table[b].long()[t // ps], t % ps
                v = u8(cache["v_pool"])[page, :, off].view(cache["v_pool"].dtype).double()
                if fmt in TOP:
                    v = v * cache["v_scale"][page, :, off].double()[..., None]
                v = v.repeat_interleave(H // G, 1)
                # weights of 1 / n are exact in every type but for the sum's rounding; bf16 outputs round by 2^-8 at most, products in f16 by 2^-11
                tol = v.abs().mean(0) * ((2.0 ** -8 + 2.0 ** -11 if dtype == "bf16" else 0.0) + 5e-5)
                assert ((out[b].double() - v.mean(0)).abs() <= tol).all(), (size, best, b)
                # the score in its keys' rounding (bf16: 2^-8), sums of equal terms and the turn to powers of two and back
                want = -size * (1.0 if best is None else 63 / 64)
                assert ((lse[b].double() - want).abs() <= size * (2.0 ** -8 if fmt == "bf16" else 1e-5)).all(), (size, best, b)


@pytest.mark.parametrize("dtype,fmt,hd", [("bf16", "e4m3", 64), ("fp32", "int8", 32)])
def test_a_sequence_of_as_many_positions_as_an_int_counts(dtype, fmt, hd):
    """2^31 - 2 of them, in pages that are all the same one: the output of that page alone, and its sum as many times.  (Tensor cores' tiles and plain FMAs'.)"""
    g = torch.Generator(device="cuda").manual_seed(1)
    ps, n = 42966, 49981
    cache = pools(g, fmt, 1, 1, ps, hd)
    table = torch.zeros(1, n, dtype=torch.int32, device="cuda")
    q = torch.randn(1, 4, hd, generator=g, device="cuda").to(DT[dtype])
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    run = lambda m: sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, torch.tensor([m], dtype=torch.int32, device="cuda"), k_scale=cache["k_scale"],
                                        v_scale=cache["v_scale"], want_lse=True, status=status)
    one, lse1 = run(ps)
    out, lse = run(ps * n)
    assert not status.any() and ps * n == 2 ** 31 - 2
    # a lane adds up to 2^18 terms one after the other, each sum rounded by 2^-24; bf16 outputs by 2^-8 twice; relative to sum p |v|, of which no value is above 6
    assert ((lse - lse1) - math.log(n)).abs().max() <= 2.0 ** -6 + 1e-5
    assert ((out.double() - one.double()).abs() <= 6 * 2.0 ** -5 + (2.0 ** -7 * one.double().abs() if dtype == "bf16" else 0)).all()
    assert (out.double() - one.double()).norm() <= 0.05 * one.double().norm()


def test_large_calls_are_refused_by_the_tables_width():
    """2^16 pages of 4096 positions for each of 128 sequences are more than 2^30 tiles, whatever the lengths say; for 32 sequences they are not."""
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = pools(g, "e4m3", 2, 1, 4096, 128)
    table = torch.zeros(1, 1 << 16, dtype=torch.int32, device="cuda").repeat(64, 1)
    q = torch.randn(128, 1, 128, generator=g, device="cuda").to(torch.bfloat16)
    run = lambda b, t: sb.decode_attention(q[:b], cache["k_pool"], cache["v_pool"], t, torch.full((b,), 5, dtype=torch.int32, device="cuda"), k_scale=cache["k_scale"], v_scale=cache["v_scale"])
    with pytest.raises(sb.SpecError) as e:
        run(128, table.repeat(2, 1))
    assert e.value.code == -8
    assert torch.equal(run(32, table[:32]), run(32, table[:32, :1].contiguous()))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("H,G,hd", [(32, 8, 128), (16, 1, 128), (8, 4, 64), (8, 2, 256), (8, 2, 80)])
def test_outputs_in_bf16_lose_little_but_their_own_rounding(fmt, H, G, hd):
    """Keys of which some dimensions are larger than the others, so that few positions count: the error is that of rounding the definition to bf16, but for probabilities of sixteen bits or
    (8-bit caches, times the value's scale) of eleven: 2^-12 of each at most, independent of one another, next to the output's 2^-9 in the mean; a 20th is more than that makes."""
    g = torch.Generator(device="cuda").manual_seed(H + hd)
    B, ps = 24, 16
    lens = torch.randint(1, 1500, (B,), generator=g, device="cuda").tolist()
    table, pages = table_for(g, lens, ps)
    cache = pools(g, fmt, pages, G, ps, hd)
    gain = torch.ones(hd, device="cuda")
    gain[:: max(1, hd // 4)] = 6.0
    if fmt in TOP:
        cache["k_scale"] *= 2.5
    else:
        cache["k_pool"] = (cache["k_pool"].float() * gain).to(DT[fmt])
    q = torch.randn(B, H, hd, generator=g, device="cuda").to(torch.bfloat16)
    out = sb.decode_attention(q, cache["k_pool"], cache["v_pool"], table, torch.tensor(lens, dtype=torch.int32, device="cuda"), k_scale=cache["k_scale"], v_scale=cache["v_scale"])
    want, _, _ = definition(q, cache, table, lens, ps, hd ** -0.5)
    assert (out.double() - want).norm() <= 1.05 * (want.to(torch.bfloat16).double() - want).norm()


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("B,H,G,hd", [(24, 16, 1, 128), (12, 18, 2, 128), (8, 45, 3, 128), (3, 128, 8, 128), (23, 11, 1, 64), (11, 66, 2, 64), (80, 15, 1, 128)])
@pytest.mark.parametrize("least,most", [(0, 100), (3000, 9000)])
def test_many_heads_of_a_kv_head_in_a_wide_table(dtype, fmt, B, H, G, hd, least, most):
    """Short sequences, whose heads go by halves although the table would hold long ones, and long ones, which go as one chunk (or the fewest): odd halves, three chunks, shared and whole segments."""
    if B * G * most > 300000 and fmt == "fp32":
        most = 4000                                      # plain FMAs know no halves
    g = torch.Generator(device="cuda").manual_seed(B * H + most)
    lens = torch.randint(least, most, (B,), generator=g, device="cuda").tolist()
    table, pages = table_for(g, lens, 16)
    table = torch.nn.functional.pad(table, (0, 3000 - table.shape[1]), value=-9)
    cache = pools(g, fmt, pages, G, 16, hd)
    spoil(cache, table, lens, 16)
    check(torch.randn(B, H, hd, generator=g, device="cuda").to(DT[dtype]), cache, table, lens, 16)
