"""The serving loop of speculate.py, which runs the paged store, its attention and the verification of drafts together."""
import pytest
import torch

from paper_2503_24358_amd import speculate, squat

pytestmark = pytest.mark.gpu


def _prompts(model, lengths):
    g = torch.Generator().manual_seed(3)
    return [torch.randint(0, model.vocab, (n,), generator=g) for n in lengths]


@pytest.mark.parametrize("bits,group", [(4, 32), (8, 128), (2, 64)])
def test_drafts_do_not_change_what_a_greedy_target_says(bits, group):
    """Token by token or with drafted tokens, from chunks or single tokens: the same text (the store holds the same codes either way)."""
    model = speculate.Model(vocab=512, seed=5)
    prompts = _prompts(model, (300, 1, 70, 33))
    texts = []
    for drafts in (0, 3, 7):
        engine = speculate.Engine(model, prompts, 24, drafts, bits=bits, group=group, greedy=True)
        texts.append(speculate.generate(engine, 24)[0])
    assert texts[0] == texts[1] == texts[2]


def test_the_cache_holds_what_was_accepted():
    """After some steps a sequence's pages read back as the quantized keys and values of its prompt and its accepted tokens."""
    model = speculate.Model(vocab=256, seed=6)
    prompts = _prompts(model, (45, 20))
    engine = speculate.Engine(model, prompts, 40, 4, page=16, greedy=False)
    texts = [p.tolist() for p in prompts]
    for _ in range(5):
        accepted, out = engine.step()
        for t, a, row in zip(texts, accepted.tolist(), out.tolist()):
            t.extend(row[:a + 1])
    for s, text in enumerate(texts):
        n = int(engine.kv_len[s])
        assert n == len(text) - 1                         # (the newest token is not in the cache yet)
        tokens = torch.tensor(text[:-1], device="cuda")
        _, k, v = model.projections(tokens)
        slots = engine._slots(torch.full((n,), s, device="cuda"), torch.arange(n, device="cuda"))
        got = engine.store.read(slots, torch.float32)
        fresh = squat.PagedStore(-(-n // 16), model.heads, 16, 4, 32)
        order = torch.arange(n, device="cuda")
        fresh.write(k, v, order)
        want = fresh.read(order, torch.float32)
        # (the projections of a batch and of one sequence differ in their last bits, and so may a code beside a border)
        for a, b in zip(got, want):
            assert (a - b).abs().max() <= 0.5 and ((a - b).abs() > 0.02).float().mean() < 0.01


def test_with_an_update_matrix():
    model = speculate.Model(vocab=512, seed=7)
    engine = speculate.Engine(model, _prompts(model, (200, 65)), 12, 3, bits=2, subspace=8)
    texts, steps = speculate.generate(engine, 12)
    assert all(len(t) == 12 and all(0 <= x < 512 for x in t) for t in texts) and steps <= 12
