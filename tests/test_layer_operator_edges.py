"""What calls of the operators around the layers have to refuse, keep or say, beside their numbers."""
import pytest
import torch

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
