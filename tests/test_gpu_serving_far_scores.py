"""Attention with finite scores so large that one rounding of a score is a factor of more than float32 holds in a
weight (GPU): the row's highest scores take everything, in each of the kernels.

Queries and keys have equal elements of 8 significant bits, so their products and sums are exact in float32 for head
sizes up to 256 and equal scores are equal bits.  Two that differ do so by more than one part in 2^8, far above the
rounding of the scale.  So every output is the mean of the highest-scoring tokens' values, within the rounding of their
equal weights and of the result, and lse the highest score plus the logarithm of their number."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import serving_ref as ref  # noqa: E402
from test_gpu_serving import HALF, ULP, attention_bounds  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
FAR = 1 << 22


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


def check(psd, lens, H, G, D, dtype, scale, window=0, mask=None, max_kv=None, lo=1e4, hi=3e4, seed=1):
    print("[far scores]", lens, H, G, D, dtype, scale, window, max_kv, flush=True)
    s = ref.Sequences(lens, G, D, 16, dtype, seed=seed)
    g = torch.Generator().manual_seed(seed)

    def level(*shape):
        return (lo + (hi - lo) * torch.rand(shape, generator=g)).to(BF16).to(dtype)

    there = ~torch.isnan(s.k.float())
    s.k = torch.where(there, level(*s.k.shape[:-1], 1).expand(s.k.shape), s.k)
    q = level(s.rows, H, 1).expand(s.rows, H, D).contiguous()
    q[torch.rand((s.rows, H), generator=g) < 0.3] *= -1.0  # the lowest key wins
    cache, seqs, dk, dv = s.handles(psd, None, max_kv)
    dmask = None if mask is None else torch.tensor(mask, dtype=torch.int32, device="cuda")
    o = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, H), scale=scale, window=window, mask=dmask,
                      want_lse=True)
    torch.cuda.synchronize()
    want, lse, spread, size, vmax = ref.attention(s, q, scale, window, mask)
    kv = max(k for _, k in lens)
    got, got_lse = o["out"].cpu().double(), o["lse"].cpu().double()
    assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(got_lse).all())
    # where neighbouring scores are not yet far apart, the roundings of scale and score move the weights
    score = 8 * ULP * size if size < 2.0 ** 13 else 0.0
    tol = HALF[dtype] * want.abs() + (2 * score + (kv + 8) * ULP) * vmax
    if dtype == BF16:
        tol = tol + HALF[BF16] * spread
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())
    # the scale times log2 e, the product with it and the way back to natural logarithms round once each
    assert bool(((got_lse - lse).abs() <= 6 * ULP * lse.abs() + score + (kv + 8) * ULP).all())
    return size


@pytest.mark.parametrize("max_kv", [None, FAR], ids=["near", "far"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_far_scores(psd, D, dtype, max_kv):
    size = 0.0
    for scale in (D ** -0.5, -(D ** -0.5), 1.0):
        size = max(size, check(psd, [(1, 500), (5, 300), (70, 300), (150, 150)], 8, 2, D, dtype, scale, max_kv=max_kv))
    assert size > 2.0 ** 31  # half a unit in the last place is a factor of 2^64 and more


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 20, 70, 200])
def test_far_scores_in_parts(psd, n, dtype):
    check(psd, [(n, 2900)], 4, 1, 128, dtype, 128 ** -0.5, seed=2)
    check(psd, [(n, 2900)], 4, 1, 128, dtype, 128 ** -0.5, window=1500, seed=3)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_far_scores_under_masks(psd, dtype):
    see = [[(1 << (i % 31)) | 1, i] for i in range(40)]
    check(psd, [(40, 300)], 8, 2, 128, dtype, 128 ** -0.5, mask=see, seed=4)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("exponent", range(8, 40, 4))
def test_from_near_to_far(psd, exponent, dtype):
    """Scores of about 2^8 to 2^36, the sizes among which the kernels change how they take the maximum out."""
    size = 2.0 ** exponent
    check(psd, [(70, 300), (2, 400)], 8, 2, 128, dtype, size / (128 * 16384.0 * 16384.0), lo=16384.0, hi=32768.0, seed=exponent)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("value,scale", [(1e38, 0.125), (1e36, 16.0)])
@pytest.mark.parametrize("max_kv", [None, FAR], ids=["near", "far"])
@pytest.mark.parametrize("n", [3, 70])
def test_scores_past_float32(psd, n, max_kv, value, scale, dtype):
    """A score that is infinite in float32, before or with the scale, makes its row NaN; other rows stay as they are."""
    s = ref.Sequences([(n, 300)], 1, 64, 16, dtype, seed=5)
    s.k = s.k.abs()
    q = torch.randn((n, 4, 64), generator=s.gen).to(dtype)
    q[n - 2, 2] = 0
    want, lse, spread, size, vmax = ref.attention(s, q, scale)
    tol, _ = attention_bounds(s, want, spread, size, vmax, 300, dtype)
    q[n - 2, 2] = value
    cache, seqs, dk, dv = s.handles(psd, None, max_kv)
    got = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4), scale=scale)["out"].cpu().double()
    assert bool(torch.isnan(got[n - 2, 2]).all())
    others = torch.ones((n, 4), dtype=torch.bool)
    others[n - 2, 2] = False
    assert bool(((got - want).abs() <= tol)[others].all())
