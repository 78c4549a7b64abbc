"""The decoding loop over an 8-bit cache: weights, prompts and tokens as programs have them."""
import pytest
import torch

from paper_2503_01840_b200 import synth

pytestmark = pytest.mark.gpu


def model(batch):
    cfg = synth.ModelCfg("K", "bf16", 1, 512, 4, 2, 128, 1408, 2048, 1024, (0, 0, 0), 1e4, batch=batch, tree_depth=2, tree_topk=2, tree_nodes=4, seed=3)
    return cfg, synth.make_target_weights(cfg, "cuda")


def prompts(*lengths):
    g = torch.Generator().manual_seed(7)
    return [torch.randint(0, 2048, (n,), generator=g) for n in lengths]


def test_weights_that_need_gradients():
    """A module's parameters, with gradients on: the same tokens and hidden states as without."""
    from paper_2503_01840_b200.kv8_decode import CachedDecoder
    cfg, w = model(2)
    plain = CachedDecoder(cfg, w, 2, 64, "bf16")
    want = [plain.prefill(prompts(9, 20)), *plain.step(), *plain.step()]
    leaf = lambda t: {n: leaf(x) for n, x in t.items()} if isinstance(t, dict) else [leaf(x) for x in t] if isinstance(t, list) else torch.nn.Parameter(t)
    trained = CachedDecoder(cfg, leaf(w), 2, 64, "bf16")
    got = [trained.prefill(prompts(9, 20)), *trained.step(), *trained.step()]
    assert torch.is_grad_enabled()
    for a, b in zip(got, want):
        assert torch.equal(a, b) and not a.requires_grad


def test_a_refused_prompt_leaves_the_sequences_as_they_were():
    """Ids that the table lacks in the second prompt: nothing of the first has been written, and the sequences go on."""
    from paper_2503_01840_b200.kv8_decode import CachedDecoder
    cfg, w = model(2)
    kept, other = CachedDecoder(cfg, w, 2, 64, "bf16"), CachedDecoder(cfg, w, 2, 64, "bf16")
    for dec in (kept, other):
        dec.prefill(prompts(30, 20))
    for bad in (2048, -1):
        with pytest.raises(ValueError):
            kept.prefill([prompts(25, 25)[1], torch.tensor([5, bad, 6])])
    for _ in range(2):
        for a, b in zip(kept.step(), other.step()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("of", [lambda t: t.long(), lambda t: t.to(torch.int16), lambda t: torch.stack([t, t.flip(0)], 1)[:, 0], lambda t: t.cpu()])
def test_tokens_that_a_program_puts_in_the_place_of_the_greedy_ones(of):
    """Of any integer type, a column of a table of them, on the host; prompts too."""
    from paper_2503_01840_b200.kv8_decode import CachedDecoder
    cfg, w = model(2)
    plain, forced = CachedDecoder(cfg, w, 2, 64, "bf16"), CachedDecoder(cfg, w, 2, 64, "bf16")
    tokens = torch.tensor([2047, 3], dtype=torch.int32, device="cuda")
    given = [p.cuda() for p in prompts(9, 20)]
    assert torch.equal(plain.prefill(given), forced.prefill([of(p) for p in given]))
    plain.tokens, forced.tokens = tokens, of(tokens)
    for a, b in zip(plain.step(), forced.step()):
        assert torch.equal(a, b)
