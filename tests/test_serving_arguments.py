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


class Calls:
    """Stands for the library: records the calls, launches nothing."""

    def __init__(self):
        self.seen = []

    def psd_kv_keep(self, *args):
        self.seen.append(args)
        return 0


def small_call(psd, B=3):
    pool = torch.zeros((8, 16, 2, 64), dtype=torch.bfloat16)
    start, kv = torch.arange(B + 1, dtype=torch.int32), torch.full((B,), 9, dtype=torch.int32)
    seqs = psd.make_seqs(start, kv, torch.zeros((B, 2), dtype=torch.int32), B, 1, 32)
    return psd.make_cache(pool, pool.clone()), seqs, start, kv


def test_rows_of_the_page_table(psd):
    start, kv = torch.arange(4, dtype=torch.int32), torch.full((3,), 9, dtype=torch.int32)
    one = torch.zeros((1, 5), dtype=torch.int32)
    wide = torch.zeros((3, 9), dtype=torch.int32)
    overlapping = torch.zeros(30, dtype=torch.int32).as_strided((3, 5), (4, 1))
    for bad in (one.expand(3, -1), one[:, :1].expand(3, 1), overlapping):
        with pytest.raises(psd.PsdError) as e:
            psd.make_seqs(start, kv, bad, 3, 1, 32)
        assert e.value.status == psd.PSD_E_ARG
    assert psd.make_seqs(start, kv, wide[:, 2:7], 3, 1, 32).table_stride == 9
    assert psd.make_seqs(start, kv, torch.zeros(30, dtype=torch.int32).as_strided((3, 5), (5, 1)), 3, 1, 32).table_stride == 5
    for single in (one, one.expand(1, -1), torch.zeros(9, dtype=torch.int32).as_strided((1, 5), (0, 1))):
        assert psd.make_seqs(start[:2], kv[:1], single, 1, 1, 32).table_stride == 5


def test_rows_of_kept_indices(psd, monkeypatch):
    """One path's indices, the same for every sequence: an expanded tensor has one row in memory, not B."""
    cache, seqs, start, kv = small_call(psd)
    calls = Calls()
    monkeypatch.setattr(psd, "_lib", calls)
    monkeypatch.setattr(psd, "_stream", lambda stream=None: None)
    n_keep = torch.ones(3, dtype=torch.int32)
    path = torch.arange(5, dtype=torch.int32)
    for bad in (path.expand(3, -1), path[:1].expand(3, 1), torch.zeros(30, dtype=torch.int32).as_strided((3, 5), (3, 1))):
        with pytest.raises(psd.PsdError) as e:
            psd.kv_keep(cache, seqs, bad, n_keep)
        assert e.value.status == psd.PSD_E_ARG and not calls.seen
    for good, stride in ((path.expand(3, -1).contiguous(), 5), (torch.zeros((3, 8), dtype=torch.int32)[:, 1:6], 8)):
        psd.kv_keep(cache, seqs, good, n_keep)
        assert calls.seen.pop()[3:5] == (stride, 5)
    one_cache, one_seqs, _, _ = small_call(psd, 1)
    psd.kv_keep(one_cache, one_seqs, path.expand(1, -1), n_keep[:1])
    assert calls.seen.pop()[3:5] == (5, 5)


def test_new_lengths_share_no_memory_with_what_is_read(psd):
    """kv_out is written by one workgroup while others read the lengths, row starts and kept indices."""
    from test_serving_abi import keep

    base = 1 << 20
    parts = structs(psd, s__kv_len=base, s__new_start=base + 4096)  # four sequences
    for out in (base, base - 12, base + 12, base + 4096, base + 4096 + 16, base + 8192, base + 8192 + 12, base + 12288,
                base + 12288 + 4 * 19):
        assert keep(psd, *parts, idx=base + 12288, n=base + 8192, out=out) == psd.PSD_E_ARG, out - base
        assert b"kv_out" in psd.lib().psd_last_error()
