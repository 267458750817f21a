"""Attention of few bfloat16 rows whose host bound of cached tokens is far above the lengths: the kernel for long
caches then divides short ones, whole sequences and parts of them (GPU).  Bounds as in test_gpu_serving.py."""
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
from test_gpu_serving import SHAPES, check_attention, path_mask  # noqa: E402

BF16 = torch.bfloat16
FAR = 1 << 22


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_shapes(psd, shape):
    check_attention(psd, **SHAPES[shape], dtype=BF16, max_kv=FAR)


@pytest.mark.parametrize("n,H,G,D,kv", [(1, 4, 1, 128, 5000), (5, 4, 1, 128, 3001), (1, 16, 8, 128, 4097), (11, 4, 1, 64, 2500),
                                        (15, 4, 2, 128, 2700), (31, 4, 2, 80, 2300), (1, 8, 2, 256, 2999), (35, 4, 4, 200, 1400)])
def test_one_long_sequence_in_parts(psd, n, H, G, D, kv):
    check_attention(psd, [(n, kv)], H, G, D, 24, BF16, max_kv=FAR)


def test_unlike_sequences(psd):
    check_attention(psd, [(1, 3000), (2, 5), (1, 700), (0, 900), (2, 2), (1, 2500), (1, 1)], 8, 2, 128, 16, BF16, max_kv=FAR)
    check_attention(psd, [(16, 1500), (3, 1200), (16, 16), (1, 1)], 4, 1, 128, 64, BF16, max_kv=FAR)
    check_attention(psd, [(3, 40 * b + 3) for b in range(70)], 8, 4, 64, 16, BF16, max_kv=FAR)


def test_windows_and_paths(psd):
    check_attention(psd, [(4, 3000), (2, 2900)], 8, 2, 64, 16, BF16, window=1500, max_kv=FAR)
    check_attention(psd, [(4, 3000), (2, 2900)], 8, 2, 64, 16, BF16, window=1 << 21, max_kv=FAR)
    check_attention(psd, [(7, 2000), (7, 7)], 8, 2, 128, 32, BF16, mask=path_mask(2, 3) * 2, max_kv=FAR)
    check_attention(psd, [(13, 1800), (13, 90)], 8, 2, 64, 32, BF16, mask=path_mask(3, 4) * 2, max_kv=FAR)


@pytest.mark.parametrize("n,H,D", [(2, 4, 64), (6, 8, 128), (3, 4, 256)])
def test_unseen_values(psd, n, H, D):
    """NaN in the last token's key and value, and behind the window; a row that sees them shows it."""
    s = ref.Sequences([(n, 3000), (n, 70)], 2, D, 16, BF16, seed=3)
    q = torch.randn((2 * n, H, D), generator=s.gen).to(BF16)
    want, *_ = ref.attention(s, q, D ** -0.5, 2500)
    for b, pos, value in ((0, 2999, math.nan), (0, 3000 - n - 2500 - 3, math.inf), (1, 69, math.inf)):
        page, place = s.place(b, pos)
        s.k[page, place] = value
        s.v[page, place] = value
    cache, seqs, dk, dv = s.handles(psd, None, FAR)
    got = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, H), window=2500)["out"].cpu().double()
    for rows in (slice(0, n - 1), slice(n, 2 * n - 1)):
        assert float((got[rows] - want[rows]).abs().max()) < 0.03
    assert not bool(torch.isfinite(got[n - 1]).any()) and not bool(torch.isfinite(got[2 * n - 1]).any())


@pytest.mark.parametrize("kv", [90, 3000])
def test_rows_of_nan_scores_alone(psd, kv):
    s = ref.Sequences([(2, kv), (3, 2)], 1, 64, 16, BF16, seed=4)
    q = torch.randn((s.rows, 4, 64), generator=s.gen).to(BF16)
    want, *_ = ref.attention(s, q, 0.125)
    q[0, 1, 5] = math.nan
    cache, seqs, dk, dv = s.handles(psd, None, FAR)
    o = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4), scale=0.125, want_lse=True)
    out, lse = o["out"].cpu().double(), o["lse"].cpu().double()
    assert bool(torch.isnan(out[0, 1]).all()) and math.isnan(float(lse[0, 1]))
    others = torch.ones((s.rows, 4), dtype=torch.bool)
    others[0, 1] = False
    assert float((out - want)[others].abs().max()) < 0.03
    assert bool((lse[2] == -math.inf).all()) and bool((out[2] == 0).all())


def test_same_bits_every_time(psd):
    """Who finishes a part first does not change its sum."""
    s = ref.Sequences([(1, 6000), (1, 300), (2, 4000)], 2, 128, 64, BF16, seed=7)
    q = torch.randn((s.rows, 8, 128), generator=s.gen).to(BF16).cuda()
    cache, seqs, dk, dv = s.handles(psd, None, FAR)
    ws = psd.new_attention_workspace(cache, seqs, 8)
    first = psd.attention(cache, seqs, q, ws)["out"].clone()
    for _ in range(20):
        assert bool(torch.equal(psd.attention(cache, seqs, q, ws)["out"], first))
