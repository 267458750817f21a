"""Attention of prompts among single tokens: sequences with far fewer row tiles than the longest, whose missing
tiles lie inside a workgroup's work (GPU).  Bounds as in test_gpu_serving.py."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

from test_gpu_serving import check_attention, path_mask  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
def test_one_prompt(psd, D, dtype):
    check_attention(psd, [(1, 300), (160, 200)] + [(1, 200 + 30 * b) for b in range(8)], 16, 4, D, 16, dtype)


def test_prompts_between_empty_sequences(psd):
    check_attention(psd, [(90, 400), (0, 300), (1, 90), (0, 0), (2, 700), (130, 130), (1, 1)], 32, 8, 128, 16, F32)
    check_attention(psd, [(90, 400), (0, 300), (1, 90), (2, 700)], 32, 8, 64, 16, F32, window=150)
    check_attention(psd, [(33, 400), (1, 200), (33, 33)], 8, 2, 96, 16, F32, mask=path_mask(8, 4) + [[1, 0]] + path_mask(8, 4))


def test_two_tiles_of_large_heads(psd):
    check_attention(psd, [(16, 900), (1, 700), (3, 8), (12, 600)], 16, 4, 256, 16, BF16, max_kv=1 << 20)
    check_attention(psd, [(60, 400), (3, 400), (1, 1)], 4, 4, 192, 16, BF16, max_kv=1 << 20)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_bounds_far_above_the_lengths(psd, dtype):
    check_attention(psd, [(5, 300), (1, 40), (1, 900)], 32, 8, 128, 16, dtype, max_new=400)
    check_attention(psd, [(3, 300), (2, 40), (1, 900)], 8, 8, 64, 16, dtype, max_new=1000, max_kv=1 << 20)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("most", [1 << 16, (1 << 31) - 1])
def test_any_bound_of_new_tokens(psd, most, dtype):
    """A bound above the call's rows is that of its rows: the work is done, and no index passes 32 bits."""
    check_attention(psd, [(5, 300), (1, 40)], 8, 2, 64, 16, dtype, max_new=most)
    check_attention(psd, [(3, 100), (70, 80)], 64, 1, 128, 16, dtype, max_new=most)
