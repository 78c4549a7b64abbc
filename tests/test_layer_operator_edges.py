"""What calls of the operators around the layers have to refuse, keep or say, beside their numbers."""
import pytest
import torch

import test_layer_operators as layers
from paper_2503_01840_b200 import binding as sb

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("grads", [True, False])
def test_forward_mode_tangents_are_refused_not_dropped(grads):
    """A tensor with a tangent, with gradients on or off (which forward mode does not heed): an error, never an output without a tangent, which stands for one of zeros."""
    from torch.autograd import forward_ad as fwd
    x, w, h = torch.randn(4, 32, device="cuda"), torch.ones(32, device="cuda"), torch.randn(4, 2, 16, device="cuda")
    ids, v, pos = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    freq, _ = sb.rope_frequencies(16, 1e4)
    with fwd.dual_level(), torch.set_grad_enabled(grads):
        dual = lambda t: fwd.make_dual(t, torch.ones_like(t))
        for call in (lambda: sb.embedding(pos, dual(x)), lambda: sb.rms_norm(dual(x), w), lambda: sb.rms_norm(x, dual(w)), lambda: sb.rms_norm(x, w, residual=dual(x)),
                     lambda: sb.rms_norm(dual(x), w, dtype=torch.int8), lambda: sb.rms_norm(x, w, residual=dual(x), sum_out=x.clone()), lambda: sb.embedding(pos, dual(x), out=x.clone()),
                     lambda: sb.distill_loss(dual(x), ids, v), lambda: sb.distill_loss(x, ids, dual(v)), lambda: sb.distill_loss(x, ids, v, values_lse=dual(v[:, 0].contiguous())),
                     lambda: sb.rotary(dual(h), pos, freq), lambda: sb.rotary(dual(h), pos, freq, out=h.clone())):
            with pytest.raises((RuntimeError, ValueError)):
                call()
        for call in (lambda: sb.embedding(pos, x), lambda: sb.rms_norm(x, w), lambda: sb.distill_loss(x, ids, v), lambda: sb.rotary(h, pos, freq)):
            assert fwd.unpack_dual(call()).tangent is None      # no tensor has one: the calls go on as outside


def teacher():
    return torch.randn(4, 32, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")


@gpu
def test_an_id_map_without_entries_is_refused():
    """It is no map of ids, and not the absence of one either: ids would be taken for the student's own."""
    z, ids, v = teacher()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    _, stats = sb.distill_loss(z, ids, v, want_stats=True)
    for call in (lambda: sb.distill_loss(z, ids, v, id_map=none), lambda: sb.distill_loss_and_grad(None, z, ids, v, id_map=none),
                 lambda: sb.distill_loss_backward(None, z, stats, ids, v, id_map=none)):
        with pytest.raises(ValueError):
            call()


@gpu
def test_row_values_of_another_shape_are_refused():
    """Two rows of two are not four rows; a dimension of 1 more, or none, is no other shape."""
    z, ids, v = teacher()
    loss, stats = sb.distill_loss(z, ids, v, want_stats=True)
    lse, g = torch.rand(4, device="cuda"), torch.rand(4, device="cuda")
    calls = [lambda x=x: sb.distill_loss(z, ids, v, values_lse=x) for x in (lse.view(2, 2), lse.view(2, 1, 2), lse[:2])]
    calls += [lambda x=x: sb.distill_loss_backward(x, z, stats, ids, v) for x in (g.view(2, 2), g[:3])]
    calls += [lambda x=x: sb.distill_loss_and_grad(x, z, ids, v) for x in (g.view(2, 2), g[:3])]
    calls += [lambda x=x: sb.distill_loss_backward(None, z, x, ids, v) for x in (stats.view(2, 4), stats.view(2, 2, 2), stats.T.contiguous(), stats[:3])]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    for x in (lse[:, None], lse[None], lse[None, :, None]):
        assert torch.equal(sb.distill_loss(z, ids, v, values_lse=x), sb.distill_loss(z, ids, v, values_lse=lse))
    for x, y in ((g[:, None], stats.flatten()), (g[None], stats[None]), (g, stats[:, :, None])):
        assert torch.equal(sb.distill_loss_backward(x, z, y, ids, v), sb.distill_loss_backward(g, z, stats, ids, v))
    row = lambda t: t[:1]
    assert torch.equal(sb.distill_loss_backward(row(g)[None], row(z), row(stats)[0], row(ids), row(v)), sb.distill_loss_backward(g, z, stats, ids, v)[:1])


@gpu
def test_a_flag_that_is_neither_true_nor_false_is_refused():
    """Before anything is written: accumulating is not overwriting."""
    z, ids, _ = teacher()
    out = torch.full((4, 32), 3.0, device="cuda")
    with pytest.raises(RuntimeError):
        sb.embedding_backward(z, ids[:, 0].contiguous(), 4, out=out, accumulate=torch.ones(2))
    assert (out == 3).all()
    again = sb.embedding_backward(z, ids[:, 0].contiguous(), 4, out=out.clone(), accumulate=torch.ones(1))
    assert torch.equal(again, sb.embedding_backward(z, ids[:, 0].contiguous(), 4, out=out, accumulate=True))


def repeated(how, rows, K, V, g):
    """ids that differ in a row but for: the last as the first; the second half as the first; every fifth; all alike; each as the one before it; with holes"""
    ids = (torch.randint(0, V, (rows, 1), generator=g) + 7919 * torch.arange(K)) % V
    at = torch.arange(K)
    place = {"none": at, "one": at.where(at < K - 1, torch.zeros_like(at)), "halves": at % max(1, K // 2), "fifths": at.where(at % 5 > 0, torch.zeros_like(at)), "all": at * 0,
             "pairs": at // 2 * 2, "holes": at % max(1, K // 3)}[how]
    ids = ids[:, place]
    if how == "holes":
        ids[torch.rand(rows, K, generator=g) < 0.3] = -1
    return ids


@gpu
@pytest.mark.parametrize("K", [2, 31, 32, 33, 64, 200, 1024])
@pytest.mark.parametrize("how", ["one", "halves", "fifths", "all", "pairs", "holes"])
def test_repeated_ids_in_the_gradient(how, K):
    """In clusters, slices and the kernel for any vocabulary: against 64 bits, and the same bits where the entries come from a map of many ids to one."""
    g = torch.Generator().manual_seed(K)
    for rows, V in ((7, 8009), (400, 8009), (2, 450001)):
        z, ids, values = 2 * torch.randn(rows, V, generator=g), repeated(how, rows, K, V, g), 2 * torch.randn(rows, K, generator=g)
        loss, tol, want, dtol = layers.distilled(z, ids, values, None, None, 1.0, "kl", None)
        got, dz = sb.distill_loss_and_grad(None, z.cuda(), ids.cuda(), values.cuda())
        layers.within(got, loss, tol)
        layers.within(dz, want, dtol + want.abs() * layers.E)
        # the same through a map: twice as many ids, one behind the other to the same
        twin = torch.where(ids >= 0, ids * 2 + torch.randint(0, 2, ids.shape, generator=g), ids)
        many = torch.arange(V, dtype=torch.int32).repeat_interleave(2).cuda()
        again, dagain = sb.distill_loss_and_grad(None, z.cuda(), twin.cuda(), values.cuda(), id_map=many)
        assert torch.equal(again, got) and torch.equal(dagain, dz)


@gpu
def test_a_repeated_id_does_not_cost_the_square_of_the_entries():
    """Rows of a thousand entries, one of which repeats another's id, all of them, or none: an entry more or less to add up is no reason for many times the time."""
    g = torch.Generator().manual_seed(1)
    rows, V, K = 2000, 32000, 1024
    z, values = torch.randn(rows, V, generator=g).bfloat16().cuda(), torch.randn(rows, K, generator=g).cuda()

    def time_of(how):
        ids = repeated(how, rows, K, V, g).int().cuda()
        best = float("inf")
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            sb.distill_loss_and_grad(None, z, ids, values)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best
    plain = time_of("none")
    for how in ("one", "halves", "all"):
        assert time_of(how) < 4 * plain, how


@gpu
@pytest.mark.parametrize("how", ["none", "halves", "all", "holes"])
@pytest.mark.parametrize("rows", [9, 400])
def test_what_kl_is_where_ids_repeat(how, rows):
    """The sum over the entries as they stand: the divergence of the added-up probabilities from the student's less sum p ln(P / p); "ce" and the gradient are those of the added-up ones."""
    g = torch.Generator().manual_seed(rows)
    V, K = 3001, 24
    z, ids, values = torch.randn(rows, V, generator=g), repeated(how, rows, K, V, g), torch.randn(rows, K, generator=g)
    z[0] = -100.0
    z[0, ids[0].clamp_min(0)] = 100.0                    # a student that is sure of the teacher's entries
    has, p, ln_p = layers.target(ids, values, None, None, 1.0, V)
    dense = torch.zeros(rows, V, dtype=torch.float64).scatter_add_(1, has.clamp_min(0), p)
    ln_q = torch.log_softmax(z.double(), 1)
    merged = torch.where(dense > 0, dense * (dense.clamp_min(1e-300).log() - ln_q), torch.zeros_like(dense)).sum(1)
    less = torch.where(p > 0, p * (dense.gather(1, has.clamp_min(0)).clamp_min(1e-300).log() - ln_p), torch.zeros_like(p)).sum(1)
    assert (merged > -1e-12).all() and (less > -1e-12).all() and (how != "none" or less.abs().max() < 1e-12)
    loss, tol, _, _ = layers.distilled(z, ids, values, None, None, 1.0, "kl", None)
    got, dz = sb.distill_loss_and_grad(None, z.cuda(), ids.cuda(), values.cuda())
    layers.within(got, merged - less, tol)
    layers.within(sb.distill_loss(z.cuda(), ids.cuda(), values.cuda()), merged - less, tol)
    _, tol, _, dtol = layers.distilled(z, ids, values, None, None, 1.0, "ce", None)
    layers.within(sb.distill_loss(z.cuda(), ids.cuda(), values.cuda(), kind="ce"), -(dense * ln_q).sum(1), tol)
    want = ln_q.exp() * dense.sum(1, keepdim=True) - dense
    layers.within(dz, want, dtol + want.abs() * layers.E)
    if how == "all":
        assert got[0] < -1.0                             # below 0: the merged divergence is 0 there
