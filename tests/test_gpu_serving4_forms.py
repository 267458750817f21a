"""Attention over a cache held in 4 bits in every form that the plan can choose: each kernel, head size and tile, with stretches
that end where sequences end and others, whole sequences and joined ones (GPU).  Lengths are ragged, unused places NaN groups; some
sequences of each call are compared with 64 bits, within the bounds of test_gpu_serving4.py."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import serving4_ref as ref4  # noqa: E402
from test_gpu_serving import BF16, F32, ULP, path_mask  # noqa: E402
from test_gpu_serving4 import attention_bounds  # noqa: E402

P = 16
# dtype, query heads, key/value heads, head size, sequences, new tokens, cached tokens of the longest; a call of each form, which
# test_attention4_forms.py checks
FORMS = [
(F32, 16, 16, 40, 33, 1, 10),
    (F32, 8, 1, 40, 300, 1, 141),
    (F32, 2, 2, 40, 2, 1, 10),
    (F32, 4, 1, 40, 2, 1, 1593),
    (F32, 4, 1, 40, 130, 9, 30),
    (F32, 8, 1, 40, 8, 130, 140),
    (F32, 8, 1, 40, 2, 3, 14),
    (F32, 4, 1, 40, 2, 8, 1518),
    (F32, 4, 4, 80, 130, 1, 9),
    (F32, 8, 1, 72, 2, 130, 8164),
    (F32, 4, 1, 80, 2, 1, 9),
    (F32, 4, 1, 72, 2, 3, 670),
    (F32, 2, 2, 192, 130, 1, 10),
    (F32, 4, 1, 192, 3, 130, 1667),
    (F32, 2, 2, 200, 2, 1, 12),
    (F32, 8, 1, 200, 2, 1, 435),
    (BF16, 16, 16, 40, 33, 1, 9),
    (BF16, 4, 1, 40, 300, 1, 143),
    (BF16, 4, 1, 40, 2, 1, 9),
    (BF16, 16, 4, 40, 5, 2, 2409),
    (BF16, 4, 1, 40, 300, 5, 13),
    (BF16, 4, 1, 40, 300, 5, 245),
    (BF16, 8, 1, 40, 2, 3, 24),
    (BF16, 16, 4, 40, 17, 5, 4156),
    (BF16, 2, 2, 72, 300, 1, 9),
    (BF16, 4, 1, 80, 300, 1, 136),
    (BF16, 2, 2, 80, 2, 1, 9),
    (BF16, 4, 4, 128, 2, 5, 1516),
    (BF16, 4, 1, 72, 300, 5, 13),
    (BF16, 4, 1, 72, 300, 5, 164),
    (BF16, 4, 1, 72, 2, 5, 20),
    (BF16, 32, 8, 96, 16, 8, 1515),
    (BF16, 2, 2, 192, 130, 1, 9),
    (BF16, 12, 4, 192, 65, 1, 129),
    (BF16, 2, 2, 200, 2, 2, 10),
    (BF16, 4, 1, 192, 2, 4, 814),
    (BF16, 4, 4, 192, 300, 17, 113),
    (BF16, 2, 2, 192, 65, 17, 1099),
    (BF16, 28, 4, 200, 33, 3, 1000),
    (BF16, 12, 4, 192, 16, 8, 3404),
    (BF16, 28, 4, 40, 65, 5, 19),
    (BF16, 4, 4, 40, 2, 2, 1541),
    (BF16, 4, 1, 40, 2, 9, 46),
    (BF16, 4, 1, 40, 2, 9, 371),
    (BF16, 32, 8, 72, 33, 9, 17),
    (BF16, 12, 4, 72, 2, 2, 1600),
    (BF16, 4, 1, 72, 2, 9, 19),
    (BF16, 4, 1, 72, 2, 9, 277),
    (BF16, 4, 1, 192, 2, 5, 18),
    (BF16, 8, 1, 200, 2, 3, 338),
]
# drafted blocks as they are served, with and without their paths' masks; single tokens over long caches; windows
BLOCKS = [(BF16, 32, 8, 128, 64, 17, 300, 4, 0), (BF16, 32, 8, 128, 64, 17, 300, 0, 0), (BF16, 32, 8, 80, 64, 17, 260, 4, 0),
          (BF16, 32, 8, 80, 64, 17, 260, 0, 0), (BF16, 16, 4, 256, 64, 5, 900, 0, 0), (BF16, 16, 4, 256, 64, 5, 900, 4, 0),
          (BF16, 16, 4, 256, 16, 5, 2100, 0, 0), (BF16, 32, 8, 128, 16, 1, 8000, 0, 0), (BF16, 32, 8, 128, 16, 17, 2048, 4, 0),
          (BF16, 32, 8, 128, 64, 5, 700, 0, 0), (BF16, 32, 8, 64, 64, 5, 700, 4, 0), (BF16, 32, 8, 128, 48, 1, 5000, 0, 1000),
          (F32, 32, 8, 128, 16, 17, 700, 4, 0), (F32, 32, 8, 64, 16, 17, 700, 4, 0), (F32, 16, 4, 256, 16, 5, 900, 4, 0)]


def lengths(B, n, kv):
    """New and cached tokens of each sequence: the longest every other, one new token less every fifth."""
    return [(n - (b % 5 == 1 and n > 1), kv if b % 2 == 0 else n + (37 * b + 11) % (kv - n + 1)) for b in range(B)]


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


class Shape:
    def __init__(self, D):
        self.D = D


def check(psd, dtype, H, G, D, B, n, kv, gamma=0, window=0):
    print("[attention4 form]", dtype, H, G, D, B, n, kv, gamma, window, flush=True)
    lens = lengths(B, n, kv)
    groups = -(-D // 32)
    start = [0]
    for new, _ in lens:
        start.append(start[-1] + new)
    T, width = start[-1], -(-kv // P) + 1
    pages = B * width + 2
    g = torch.Generator(device="cuda").manual_seed(B * 1000 + kv)
    table = torch.randperm(pages, generator=g, device="cuda")[:B * width].view(B, width)
    cached = torch.tensor([x for _, x in lens], device="cuda")
    held = (torch.arange(width * P, device="cuda") < cached[:, None]).view(B, width, P)
    there = torch.zeros((pages, P), dtype=torch.bool, device="cuda")
    there[table.flatten()] = held.flatten(0, 1)

    def pool(width, low, high):
        return torch.randint(low, high, (pages, G, P, width), generator=g, device="cuda", dtype=torch.uint8).transpose(1, 2)

    codes = [pool(16 * groups, 0, 256) for _ in range(2)]
    scales = [pool(groups, 123, 128) for _ in range(2)]
    for s in scales:
        s[~there] = 255
    q = torch.randn((T, H, D), generator=g, device="cuda").to(dtype)
    out, lse = torch.full((T + 3, H, D), 7.0, dtype=dtype, device="cuda"), torch.full((T + 3, H), 7.0, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = psd.make_cache4(*codes, *scales, D, dtype=dtype)
    seqs = psd.make_seqs(ints(start), ints([x for _, x in lens]), table.to(torch.int32), T, n, kv)
    mask = None
    if gamma:  # a root and its paths; a sequence with a token less has a shorter last path
        paths = path_mask(-(-(n - 1) // gamma), gamma)
        mask = ints([paths[i] for new, _ in lens for i in range(new)])
    ws = psd.new_attention_workspace(cache, seqs, H)
    call = lambda: psd.attention(cache, seqs, q, ws, window=window, mask=mask, out=out, want_lse=True, lse=lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out[:T]).all()) and bool(torch.isfinite(lse[:T]).all()), "a place that no row sees was used"
    assert bool((out[T:] == 7.0).all()) and bool((lse[T:] == 7.0).all())
    once = out.clone(), lse.clone()
    call()
    torch.cuda.synchronize()
    assert torch.equal(out, once[0]) and torch.equal(lse, once[1])
    for b in sorted({0, 1, B // 2, B - 2, B - 1} & set(range(B))):
        new, have = lens[b]
        at = torch.arange(have, device="cuda")
        page, place = table[b, at // P], at % P
        k, v = (ref4.decode(c[page, place].cpu(), s[page, place].cpu(), D) for c, s in zip(codes, scales))
        rows = q[start[b]:start[b + 1]].cpu().double().view(new, G, H // G, D)
        pos, own = torch.arange(have), have - new + torch.arange(new)
        sees = pos <= own[:, None]
        if window:
            sees &= pos > own[:, None] - window
        if gamma:
            bits = torch.tensor([[paths[i][j // 32] >> (j % 32) & 1 for j in range(new)] for i in range(new)], dtype=torch.bool)
            sees = torch.cat((torch.ones((new, have - new), dtype=torch.bool), bits), 1)
        product = lambda a, b: torch.einsum("nghd,cgd->nghc", a, b) * D ** -0.5  # noqa: E731
        hidden = ~sees[:, None, None]
        score = product(rows, k).masked_fill(hidden, -math.inf)
        size = float(product(rows.abs(), k.abs()).masked_fill(hidden, 0).max())
        want_lse = torch.logsumexp(score, -1)
        p = torch.exp(score - want_lse[..., None])
        want, spread = (torch.einsum("nghc,cgd->nghd", p, x).reshape(new, H, D) for x in (v, v.abs()))
        tol, lse_tol = attention_bounds(Shape(D), want, spread, size, float(v.abs().max()), have, dtype)
        got, got_lse = out[start[b]:start[b + 1]].cpu().double(), lse[start[b]:start[b + 1]].cpu().double()
        off = (got - want).abs()
        assert bool((off <= tol).all()), (b, float((off - tol).max()), (off > tol).nonzero()[:3].tolist())
        want_lse = want_lse.reshape(new, H)
        assert float(((got_lse - want_lse).abs() - ULP * want_lse.abs()).max()) <= lse_tol, b


@pytest.mark.parametrize("i", range(len(FORMS)), ids=["-".join(str(x).replace("torch.", "") for x in f) for f in FORMS])
def test_forms(psd, i):
    check(psd, *FORMS[i])


@pytest.mark.parametrize("i", range(len(BLOCKS)), ids=["-".join(str(x).replace("torch.", "") for x in f) for f in BLOCKS])
def test_blocks(psd, i):
    check(psd, *BLOCKS[i])
