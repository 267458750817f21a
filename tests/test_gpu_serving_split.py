"""Attention whose work is divided over workgroups: many sequences, very unlike ones, long caches in parts,
and that the division changes nothing from call to call (GPU).  Bounds as in test_gpu_serving.py."""
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
from test_gpu_serving import check_attention, path_mask  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


@TYPES
def test_more_sequences_than_threads(psd, dtype):
    """700 sequences, some without new tokens or without any, and one that is far longer than the others."""
    g = torch.Generator().manual_seed(9)
    lens = []
    for b in range(700):
        n = int(torch.randint(0, 4, (1,), generator=g))
        lens.append((n, n + int(torch.randint(0, 40, (1,), generator=g))))
    lens[600] = (3, 2000)
    check_attention(psd, lens, 4, 2, 64, 16, dtype, print_name="700")


@TYPES
def test_a_head_of_its_own_for_each_query(psd, dtype):
    check_attention(psd, [(1, 20 * b + 1) for b in range(40)], 16, 16, 64, 16, dtype)


@TYPES
@pytest.mark.parametrize("n,H,G,D,kv", [(1, 4, 1, 128, 5000), (5, 4, 1, 128, 3001), (1, 16, 8, 128, 4097), (11, 4, 1, 64, 2500),
                                        (40, 4, 1, 128, 2700), (130, 2, 2, 64, 2300), (1, 8, 2, 256, 2999), (35, 4, 2, 200, 1400)])
def test_one_long_sequence_in_parts(psd, n, H, G, D, kv, dtype):
    check_attention(psd, [(n, kv)], H, G, D, 24, dtype)


@TYPES
def test_unlike_sequences(psd, dtype):
    """Cuts inside sequences, whole short ones between them, rows of several sizes."""
    check_attention(psd, [(1, 3000), (2, 5), (1, 700), (0, 900), (2, 2), (1, 2500), (1, 1)], 8, 2, 128, 16, dtype)
    check_attention(psd, [(40, 1500), (3, 1200), (40, 40), (1, 1)], 4, 1, 128, 64, dtype)


@TYPES
def test_windows_and_paths_in_parts(psd, dtype):
    check_attention(psd, [(4, 3000), (2, 2900)], 8, 2, 64, 16, dtype, window=1500)
    check_attention(psd, [(60, 2600)], 4, 1, 128, 16, dtype, window=1100)
    check_attention(psd, [(17, 2000), (17, 17)], 8, 2, 128, 32, dtype, mask=path_mask(4, 4) * 2)
    check_attention(psd, [(33, 1800)], 8, 2, 64, 32, dtype, mask=path_mask(4, 8))


@TYPES
@pytest.mark.parametrize("n", [2, 70])
def test_unseen_values_in_parts(psd, n, dtype):
    """NaN in the last token's key and value, and behind the window, in a cache that is cut."""
    s = ref.Sequences([(n, 3000)], 1, 64, 16, dtype, seed=3)
    q = torch.randn((n, 4, 64), generator=s.gen).to(dtype)
    want, *_ = ref.attention(s, q, 0.125, 2500)
    for pos, value in ((2999, math.nan), (3000 - n - 2500 - 3, math.inf)):
        page, place = s.place(0, pos)
        s.k[page, place] = value
        s.v[page, place] = value
    cache, seqs, dk, dv = s.handles(psd)
    got = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4), window=2500)["out"].cpu().double()
    assert bool(torch.isfinite(got[:-1]).all()) and not bool(torch.isfinite(got[-1]).any())
    assert float((got[:-1] - want[:-1]).abs().max()) < (0.01 if dtype == BF16 else 1e-4)


@TYPES
@pytest.mark.parametrize("n,kv", [(2, 90), (2, 3000), (70, 90), (70, 3000)])
def test_rows_of_nan_scores_alone(psd, n, kv, dtype):
    """A NaN query makes every score of its row NaN: so are its output and lse, whole or in parts, and the
    other rows stay as they are.  (A row that sees nothing stays zeros.)"""
    s = ref.Sequences([(n, kv), (3, 2)], 1, 64, 16, dtype, seed=4)
    q = torch.randn((s.rows, 4, 64), generator=s.gen).to(dtype)
    want, want_lse, *_ = ref.attention(s, q, 0.125)
    q[n - 2, 1, 5] = math.nan
    cache, seqs, dk, dv = s.handles(psd)
    o = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4), scale=0.125, want_lse=True)
    out, lse = o["out"].cpu().double(), o["lse"].cpu().double()
    assert bool(torch.isnan(out[n - 2, 1]).all()) and math.isnan(float(lse[n - 2, 1]))
    others = torch.ones((s.rows, 4), dtype=torch.bool)
    others[n - 2, 1] = False
    assert float((out - want)[others].abs().max()) < (0.03 if dtype == BF16 else 1e-4)
    assert bool(torch.equal(lse[others] == -math.inf, want_lse[others] == -math.inf))
    assert bool((lse[n] == -math.inf).all()) and bool((out[n] == 0).all())


@TYPES
def test_same_bits_every_time(psd, dtype):
    """Who finishes a part first does not change its sum, and one workspace serves calls of other shapes."""
    g = torch.Generator(device="cuda").manual_seed(1)
    ws = None
    runs = []
    for lens, H in (([(1, 6000), (1, 300), (2, 4000)], 8), ([(40, 3000)], 8), ([(1, 6000), (1, 300), (2, 4000)], 8)):
        s = ref.Sequences(lens, 2, 128, 64, dtype, seed=7)
        q = torch.randn((s.rows, H, 128), generator=s.gen).to(dtype).cuda()
        cache, seqs, dk, dv = s.handles(psd)
        need = psd.attention_workspace_bytes(cache, seqs, H)
        if ws is None:
            ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        assert need <= ws.numel()
        first = psd.attention(cache, seqs, q, ws, want_lse=True)
        for _ in range(6):
            torch.randn((1 << 20,), device="cuda", generator=g)
            again = psd.attention(cache, seqs, q, ws, want_lse=True)
            assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])
        runs.append(first)
    assert torch.equal(runs[0]["out"], runs[2]["out"])


@TYPES
@pytest.mark.parametrize("interleaved,R", [(False, 64), (True, 64), (False, 20), (False, 0)])
def test_append_of_many_rows(psd, interleaved, R, dtype):
    """A wave a row from some number of rows on: the same bits as the rows in smaller calls."""
    n, H, G, D, P = 2500, 4, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((n, H + 2 * G, D), device="cuda", generator=g).to(dtype)
    w = torch.randn((2, D), device="cuda", generator=g).to(dtype)
    angle = torch.rand((n, max(R // 2, 1)), device="cuda", generator=g) * 6
    cos, sin = (angle.cos(), angle.sin()) if R else (None, None)
    width = -(-n // P)
    table = torch.randperm(width, device="cuda", generator=g).to(torch.int32)[None].contiguous()
    pools, queries = [], []
    for cut in (n, 1000):
        k = torch.zeros((width, P, G, D), dtype=dtype, device="cuda")
        v = torch.zeros_like(k)
        out = torch.empty((n, H, D), dtype=dtype, device="cuda")
        for at in range(0, n, cut):
            rows = min(cut, n - at)
            seqs = psd.make_seqs(torch.tensor([0, rows], dtype=torch.int32).cuda(),
                                 torch.tensor([at + rows], dtype=torch.int32).cuda(), table, rows, rows, n)
            part = x[at:at + rows]
            psd.kv_append(psd.make_cache(k, v), seqs, part[:, H:H + G], part[:, H + G:], q=part[:, :H], q_out=out[at:at + rows],
                          cos=cos, sin=sin, interleaved=interleaved, q_norm=w[0], k_norm=w[1])
        pools += [k, v]
        queries.append(out)
    torch.cuda.synchronize()
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3]) and torch.equal(queries[0], queries[1])
    seq = table[0].long()
    assert torch.equal(pools[1][seq].reshape(-1, G, D)[:n], x[:, H + G:])


@pytest.mark.parametrize("rows,kv", [(40, 2000), (70, 4000), (600, 5000), (2048, 6000)])
def test_workspace_of_windowed_calls(psd, rows, kv):
    """A window's parts stay inside the workspace that the bounds without it ask for."""
    H, G, D, P = 8, 2, 128, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    width = -(-kv // P)
    k = torch.randn((width, P, G, D), device="cuda", generator=g).to(BF16)
    cache = psd.make_cache(k, k.clone())
    table = torch.arange(width, device="cuda", dtype=torch.int32)[None].contiguous()
    seqs = psd.make_seqs(torch.tensor([0, rows], dtype=torch.int32).cuda(), torch.tensor([kv], dtype=torch.int32).cuda(), table,
                         rows, rows, kv)
    q = torch.randn((rows, H, D), device="cuda", generator=g).to(BF16)
    need = psd.attention_workspace_bytes(cache, seqs, H)
    whole = torch.zeros(need + (1 << 20), dtype=torch.uint8, device="cuda")
    whole[need:] = 0x5A
    roomy = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    for window in (1, 64, 300, 1000, 1900, 3000, 1 << 30, (1 << 31) - 1):
        a = psd.attention(cache, seqs, q, whole[:need] if need else None, window=window)["out"]
        b = psd.attention(cache, seqs, q, roomy, window=window)["out"]
        assert bool((whole[need:] == 0x5A).all()), window
        assert float((a.float() - b.float()).abs().max()) < 0.05 and bool(torch.isfinite(a.float()).all()), window
    # a window wider than the cache is none
    assert float((psd.attention(cache, seqs, q, roomy)["out"].float() - b.float()).abs().max()) < 0.05


@TYPES
@pytest.mark.parametrize("rows", [2, 90])
def test_lengths_that_no_call_can_have(psd, rows, dtype):
    """Lengths outside every bound are cut: such a sequence's rows see nothing or the bounded cache, the others are
    what they are."""
    s = ref.Sequences([(rows, 100), (rows, 150), (rows, 120)], 2, 64, 16, dtype)
    q = torch.randn((3 * rows, 4, 64), generator=s.gen).to(dtype)
    want, *_ = ref.attention(s, q, 0.125)
    cache, seqs, dk, dv = s.handles(psd)
    ws = psd.new_attention_workspace(cache, seqs, 4)
    starts, kv_len, table = seqs.tensors
    for bad in (-1, -(1 << 31), (1 << 31) - 1, 0):
        kv = kv_len.clone()
        kv[1] = bad
        odd = psd.make_seqs(starts, kv, table, 3 * rows, rows, 150)
        for window, mask in ((0, None), (40, None), ((1 << 31) - 1, None), (0, torch.zeros((3 * rows, 1), dtype=torch.int32, device="cuda"))):
            got = psd.attention(cache, odd, q.cuda(), ws, scale=0.125, window=window, mask=mask)["out"].cpu().double()
            if bad <= 0:
                assert bool((got[rows:2 * rows] == 0).all())
            if window != 40 and mask is None:
                tol = 0.03 if dtype == BF16 else 1e-4
                assert float((got[:rows] - want[:rows]).abs().max()) < tol
                assert float((got[2 * rows:] - want[2 * rows:]).abs().max()) < tol
    # starts past the rows and out of order: the rows that are there are those of sequences that hold them
    odd = psd.make_seqs(torch.tensor([0, rows, 1 << 30, (1 << 31) - 1], dtype=torch.int32).cuda(), kv_len, table, 3 * rows, rows, 150)
    got = psd.attention(cache, odd, q.cuda(), ws, scale=0.125)["out"].cpu().double()
    assert float((got[:rows] - want[:rows]).abs().max()) < (0.03 if dtype == BF16 else 1e-4)
    k = torch.zeros((3 * rows, 2, 64), dtype=dtype, device="cuda")
    psd.kv_append(cache, odd, k, k)
    psd.kv_keep(cache, odd, torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
