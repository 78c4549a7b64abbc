"""The decoding loop over an 8-bit cache against SpecDecoder's plain steps on the same weights."""
import numpy as np
import pytest
import torch

from paper_2503_01840_b200 import binding as sb
from paper_2503_01840_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "int8"])
def test_tokens_and_hidden_states_as_the_decoder_without_a_draft(cache):
    from paper_2503_01840_b200.kv8_decode import CachedDecoder
    cfg = synth.ModelCfg("K", "bf16", 2, 512, 4, 2, 128, 1408, 2048, 1024, (0, 0, 1), 5e5, batch=3, tree_depth=2, tree_topk=2, tree_nodes=4, seed=11)
    w, dw, _, _ = synth.make_structured(cfg, 1.0, device="cuda", residual_scale=1.0)
    d2t = dw["d2t"].cpu()
    prompts = [synth.structured_prompt(cfg, d2t, n, seed=n).numpy() for n in (1, 40, 301)]
    dec = sb.SpecDecoder(cfg, w, dw, batch=3, max_ctx=400)
    mine = CachedDecoder(cfg, w, 3, 400, cache)
    assert np.array_equal(mine.prefill(prompts).cpu().numpy(), dec.prefill(prompts, 64))
    for _ in range(6):
        tokens, hidden = mine.step()
        assert np.array_equal(tokens.cpu().numpy(), dec.plain_step())
        for b in range(3):
            h = torch.from_numpy(dec.debug(sb.DBG_NODE_HIDDEN, b).reshape(-1, cfg.hidden)[0].copy()).cuda()
            want = h * torch.rsqrt(h.square().mean() + cfg.rms_eps) * w["final_norm"].float()
            # bf16 activations of two layers round a few times by 2^-9 in the mean; the cache's rounding (e4m3: 2.6e-2 of a value in the mean)
            # reaches the hidden state through attention outputs that are a part of it
            assert (hidden[b].float() - want).norm() / want.norm() < (0.03 if cache == "e4m3" else 0.01), (cache, b)
    dec.close()


def test_what_the_cache_has_no_room_for_is_refused():
    """Prompts longer than max_ctx or none at all, another number of them than sequences, and the step that would pass max_ctx; what fits is computed as in a larger cache."""
    from paper_2503_01840_b200.kv8_decode import CachedDecoder
    cfg = synth.ModelCfg("K", "bf16", 1, 512, 4, 2, 128, 1408, 2048, 1024, (0, 0, 0), 1e4, batch=2, tree_depth=2, tree_topk=2, tree_nodes=4, seed=3)
    w = synth.make_target_weights(cfg, "cuda")
    small, large = CachedDecoder(cfg, w, 2, 24, "e4m3"), CachedDecoder(cfg, w, 2, 64, "e4m3")
    g = torch.Generator().manual_seed(2)
    ids = lambda n: torch.randint(0, 2048, (n,), generator=g).numpy()
    for bad in ([ids(25), ids(3)], [ids(0), ids(3)], [ids(3)], [ids(3)] * 3):
        with pytest.raises(ValueError):
            small.prefill(bad)
    prompts = [ids(22), ids(7)]
    assert torch.equal(small.prefill(prompts), large.prefill(prompts))
    for _ in range(2):
        assert torch.equal(small.step()[0], large.step()[0])
    for _ in range(2):
        with pytest.raises(ValueError):
            small.step()
    assert small.lengths.tolist() == [24, 9]
    large.step()
    small.prefill([ids(24), ids(24)])
    with pytest.raises(ValueError):
        small.step()
