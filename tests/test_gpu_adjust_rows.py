"""Adjusted logits in the forms that many rows take (GPU): several rows a workgroup, read ahead of one another, with drafts
counted and taken back, in long and short stretches of the vocabulary.  Bounds as in test_gpu_adjust.py."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import serving4_ref as ref4  # noqa: E402
from test_gpu_serving import BF16, F32, HALF, ULP  # noqa: E402

# B, K, gamma, V: which form each takes is checked by test_adjust_cut.py
SHAPES = [(800, 2, 2, 1000), (110, 4, 4, 1003), (130, 3, 4, 20011), (64, 4, 4, 100003)]


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


def bits(t):
    return t.view(torch.int16 if t.dtype == BF16 else torch.int32)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("in_place", [False, True], ids=["beside", "in_place"])
@pytest.mark.parametrize("mask", [0, 1, 2], ids=["no_mask", "mask", "mask_a_row"])
@pytest.mark.parametrize("B,K,gamma,V", SHAPES)
def test_rows(psd, B, K, gamma, V, mask, in_place, dtype):
    print("[adjust rows]", B, K, gamma, V, mask, in_place, dtype, flush=True)
    S, words = gamma + 1, -(-V // 32)
    g = torch.Generator().manual_seed(V + mask)
    dev = torch.Generator(device="cuda").manual_seed(V)
    logits = (torch.randn((B, K, S, V), generator=dev, device="cuda") * 3).to(dtype)
    order = torch.randperm(V, generator=g).to(torch.int32)
    in_text, in_drafts, in_bias = order[:40], order[30:90], order[85:100]  # drafts that the text lacks, biases of neither
    in_text[0], in_bias[0] = V - 1, V - 2  # the end that fills no piece
    pick = lambda of, *n: of[torch.randint(0, len(of), n, generator=g)]  # noqa: E731
    drafts = pick(in_drafts, B, K, gamma)
    again = torch.rand((B, K, gamma), generator=g) < 0.4
    drafts = torch.where(again, drafts[:, :1, :1], drafts).contiguous()  # the same ones along a path and on several
    x = dict(text=pick(in_text, B, 70), length=torch.randint(0, 71, (B,), generator=g), drafts=drafts,
             rho=0.7 + torch.rand(B, generator=g), presence=torch.randn(B, generator=g), frequency=torch.randn(B, generator=g) * 0.3,
             bias_tokens=pick(in_bias, B, 5), bias=torch.randn((B, 5), generator=g))
    if mask:
        shape = (B, words) if mask == 1 else (B, K, S, words)
        w = torch.randint(-(1 << 31), 1 << 31, shape, generator=dev, device="cuda")
        choice = torch.rand(shape, generator=dev, device="cuda")
        allowed = torch.where(choice < 0.3, 0, torch.where(choice < 0.6, -1, w)).to(torch.int32)
    names = dict(text="text", length="length", drafts="draft_tokens", rho="repetition", presence="presence", frequency="frequency",
                 bias_tokens="bias_tokens", bias="bias")
    kw = {names[n]: t.cuda() for n, t in x.items()}
    if mask:
        kw["allowed"] = allowed
    given = logits.clone()
    out = psd.adjust_logits(psd.make_params(0, V, K, 0, dtype=dtype), given, out=given if in_place else None, **kw)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(bits(given), bits(logits))
    # tokens that nothing names, of every row: as they were, or gone
    still = torch.ones(V, dtype=torch.bool, device="cuda")
    still[torch.cat((in_text, in_drafts, in_bias)).long().cuda()] = False
    want = logits
    if mask:
        may = ((allowed.unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).flatten(-2)[..., :V] > 0
        want = torch.where(may if mask == 2 else may[:, None, None], logits, float("-inf"))
    assert bool(((bits(out) == bits(want)) | ~still).all())
    # the rows of some sequences, the first and the last among them, in 64 bits
    some = sorted({0, 1, B // 3, B // 2, B - 2, B - 1})
    at = torch.tensor(some)
    few = {n: t[at] for n, t in x.items()}
    if mask:
        few["allowed"] = allowed[at.cuda()].cpu()
    exact, size = ref4.adjust(logits[at.cuda()].cpu(), **few)
    got = out[at.cuda()].cpu().double()
    gone = exact == float("-inf")
    assert torch.equal(got == float("-inf"), gone)
    tol = (5 + 5) * ULP * size + HALF[dtype] * exact.abs()
    off = (got - exact).abs()
    assert bool((off <= tol)[~gone].all()), (float((off - tol)[~gone].max()), ((off > tol) & ~gone).nonzero()[:3].tolist())
