"""The whole block around a small attention model (examples/speculative_block.py): append, attention of
draft paths, verification, keep, commit (GPU)."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module")
def block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import speculative_block as m
    return m


def prompts_of(B, m, V=500, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, V, (B, m), dtype=torch.int32, device="cuda", generator=g)


def plain_logits(block, target, tokens):
    """The model's logits after every token of one text, with a cache of its own built at once."""
    n = tokens.shape[0]
    fresh = block.Target()
    kv = torch.tensor([n], dtype=torch.int32, device="cuda")
    first = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    width = -(-n // 16)
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None].contiguous()
    return fresh(tokens, block.psd.make_seqs(first, kv, table, n, n, n))


def test_keyed_text_is_the_targets_whatever_is_drafted(block):
    """The text under the key is the same with a good and a poor drafter and any number of drafts a block; every
    token is the one the plain model's logits give in its context."""
    target = block.Target()
    prompts = prompts_of(5, 6)
    good = block.good_drafter(target)
    poor = torch.randn(good.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    texts, rates = [], []
    for drafter, gamma in ((good, 4), (poor, 4), (good, 7), (good, 1)):
        text, rate = block.keyed(target, drafter, prompts, 60, gamma=gamma)
        print("[block] keyed", gamma, rate, flush=True)
        texts.append(text)
        rates.append(rate)
    for text in texts[1:]:
        assert torch.equal(text, texts[0])
    assert rates[0] > rates[1] + 0.2, rates  # the good drafter's paths are really followed
    # plain decoding: the same race on the logits of the text so far, one position at a time
    psd = block.psd
    params = psd.make_params(7, 500, 4, 6, 1.0, 1.0, dtype=torch.float32)
    ws = psd.new_workspace(params, 1, 1)
    for b in range(2):
        text = texts[0][b]
        logits = plain_logits(block, target, text)
        for t in range(6, 60):
            rows = logits[t - 1].expand(1, 2, 500).contiguous()
            out = psd.verify(params, ws, text[None, t - 6:t].contiguous(), torch.tensor([t], device="cuda"), rows,
                             draft_tokens=torch.zeros((1, 4, 1), dtype=torch.int32, device="cuda"))
            assert int(out["out_tokens"][0, 0]) == int(text[t]), (b, t)


def test_given_numbers_follow_the_target(block):
    """Texts from given random numbers: every token had a probability, a good drafter commits more, and the
    same numbers give the same text."""
    target = block.Target()
    prompts = prompts_of(6, 3)
    good = block.good_drafter(target)
    poor = torch.randn(good.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    a, rate = block.given(target, good, prompts, 50, seed=3)
    b, _ = block.given(target, good, prompts, 50, seed=3)
    _, worse = block.given(target, poor, prompts, 50, seed=3)
    print("[block] given", rate, worse, flush=True)
    assert torch.equal(a, b)
    assert rate > worse
    assert bool(((a >= 0) & (a < 500)).all())


def test_example_runs(block, capsys):
    block.main()
    out = capsys.readouterr().out
    assert "same text: True" in out and "given random numbers" in out
