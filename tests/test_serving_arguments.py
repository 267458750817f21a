"""Bounds, strides and buffers that a call over the paged cache is given: what is accepted means what it says, what
cannot be meant is refused before anything is launched (no GPU)."""
import pytest

torch = pytest.importorskip("torch")

from test_serving_abi import structs  # noqa: E402


@pytest.fixture(scope="module")
def psd():
    from paper_2609_21858_amd import psd as m
    return m


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("H,G,D", [(128, 1, 128), (32, 8, 128), (8, 8, 64), (64, 8, 256)])
def test_far_bound_of_new_tokens(psd, H, G, D, dtype):
    """No sequence has more new tokens than the call has rows: a bound above asks for the same workspace."""
    want = None
    for most in (20, 21, 1 << 20, (1 << 31) - 1):
        c, s, _, _ = structs(psd, c__heads=G, c__head_dim=D, c__dtype=dtype, c__stride_head=D, c__stride_token=G * D,
                             c__stride_page=16 * G * D, s__max_new=most)
        n = psd.attention_workspace_bytes(c, s, H)
        assert want is None or n == want, most
        want = n
