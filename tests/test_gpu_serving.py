"""The paged cache, its attention and the verification from given random numbers against plain
64-bit implementations (GPU).

Unused places of every pool hold NaN, so a read past a sequence's end shows.  Bounds are those
of the arithmetic: float32 sums of n products err by at most n 2^-24 of the sum of their
magnitudes, bfloat16 results (8 significant bits) round by 2^-8 of themselves at most, and
bfloat16 attention also rounds each softmax weight by 2^-8 at most."""
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

BF16, F32 = torch.bfloat16, torch.float32
ULP = 2.0 ** -24
HALF = {BF16: 2.0 ** -8 * 1.01, F32: 2.0 ** -24 * 1.01}  # unit roundoffs (8 and 24 significant bits)


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


# ---------------------------------------------------------------- attention

def attention_bounds(seqs, out, spread, size, vmax, kv, dtype):
    """Largest errors of out and lse: scores err by (D + 4) ulp of their magnitude, exponentials and their
    sums by (kv + 8) ulp, and bfloat16 weights and results by half a bfloat16 ulp each."""
    score = (seqs.D + 4) * ULP * size
    rel = 2 * score + (kv + 8) * ULP
    tol = rel * vmax + HALF[dtype] * out.abs()
    if dtype == BF16:
        tol = tol + HALF[BF16] * spread
    return tol, score + (kv + 8) * ULP


def check_attention(psd, lens, H, G, D, P, dtype, window=0, mask=None, heads_first=False, seed=1, scale=None, in_place=False,
                    strided=False, max_new=None, max_kv=None, poke=None, print_name=""):
    print("[attention]", print_name, lens[:4], len(lens), H, G, D, P, dtype, window, flush=True)
    s = ref.Sequences(lens, G, D, P, dtype, seed=seed, heads_first=heads_first)
    T = s.rows
    q = torch.randn((T, H, D), generator=s.gen).to(dtype)
    if poke:
        poke(s, q)
    cache, seqs, dk, dv = s.handles(psd, max_new, max_kv)
    scale = D ** -0.5 if scale is None else scale
    ws = psd.new_attention_workspace(cache, seqs, H)
    dq = q.cuda()
    if strided:
        wide = torch.full((T, H + 3, D + 8), math.nan, dtype=dtype, device="cuda")
        wide[:, 1:H + 1, :D] = dq
        dq = wide[:, 1:H + 1, :D]
    out = dq if in_place else torch.full((T, H, D), 7.0, dtype=dtype, device="cuda")
    dmask = None if mask is None else torch.tensor([[w - (1 << 32) if w >= 1 << 31 else w for w in r] for r in mask],
                                                   dtype=torch.int32, device="cuda")
    o = psd.attention(cache, seqs, dq, ws, scale=scale, window=window, mask=dmask, out=out, want_lse=True)
    torch.cuda.synchronize()
    want, lse, spread, size, vmax = ref.attention(s, q, scale, window, mask)
    kv = max(kv for _, kv in lens)
    tol, lse_tol = attention_bounds(s, want, spread, size, vmax, kv, dtype)
    n = s.new_start[-1]
    got, got_lse = o["out"].cpu().double()[:n], o["lse"].cpu().double()[:n]
    want, lse, tol = want[:n], lse[:n], tol[:n]
    assert bool(torch.isfinite(got).all()), "a place that no row sees was used"
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), (float(((got - want).abs() - tol).max()), bad.nonzero()[:3].tolist())
    empty = lse == -math.inf
    assert bool(torch.equal(got_lse == -math.inf, empty))
    assert bool((got[empty] == 0).all())
    d = (got_lse - lse)[~empty].abs()
    assert not d.numel() or float((d - lse_tol - ULP * lse[~empty].abs()).max()) <= 0, float(d.max())
    return o


SHAPES = [
    # one new token, lengths from one to several tiles, pages that end inside one
    dict(lens=[(1, 1), (1, 2), (1, 16), (1, 17), (1, 31), (1, 32), (1, 33), (1, 63), (1, 64), (1, 65), (1, 200)], H=8, G=2, D=128, P=16),
    dict(lens=[(1, 700), (1, 3), (1, 129)], H=4, G=4, D=64, P=5),
    dict(lens=[(1, 1030)], H=16, G=1, D=128, P=64),
    # a block's rows
    dict(lens=[(5, 300), (5, 5), (3, 77), (1, 64)], H=32, G=8, D=128, P=16),
    dict(lens=[(9, 140), (2, 9)], H=7, G=1, D=80, P=24),
    dict(lens=[(17, 400)], H=12, G=4, D=96, P=100),
    # sizes that nobody padded, and the largest heads
    dict(lens=[(4, 90), (1, 1)], H=6, G=2, D=8, P=1),
    dict(lens=[(3, 150)], H=10, G=2, D=72, P=7),
    dict(lens=[(2, 190), (33, 40)], H=4, G=2, D=256, P=32),
    dict(lens=[(6, 100)], H=5, G=1, D=200, P=3),
    # a prompt, its chunk behind a cache, ragged lengths, an empty sequence between
    dict(lens=[(130, 130), (0, 50), (67, 300), (1, 1), (0, 0), (100, 131)], H=8, G=2, D=128, P=16),
    dict(lens=[(257, 400)], H=4, G=4, D=64, P=64),
    dict(lens=[(150, 777)], H=3, G=1, D=128, P=33),
    dict(lens=[(200, 260)], H=2, G=2, D=256, P=16),
    dict(lens=[(140, 300)], H=4, G=2, D=112, P=16),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", range(len(SHAPES)))
def test_attention_shapes(psd, n, dtype):
    check_attention(psd, **SHAPES[n], dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 5000])
def test_attention_windows(psd, window, dtype):
    check_attention(psd, [(1, 300), (5, 333), (40, 200), (1, 1)], 8, 2, 128, 16, dtype, window=window)
    check_attention(psd, [(150, 400)], 4, 2, 64, 24, dtype, window=window)


def path_mask(K, gamma):
    n = 1 + K * gamma
    rows = []
    for i in range(n):
        k, d = divmod(i - 1, gamma) if i else (0, -1)
        see = [0] + [1 + k * gamma + j for j in range(d + 1)]
        rows.append([sum(1 << (j % 32) for j in see if j // 32 == w) for w in range(-(-n // 32))])
    return rows


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("K,gamma,kv", [(1, 1, 2), (2, 4, 9), (4, 4, 300), (8, 8, 500), (16, 8, 129), (5, 7, 97)])
def test_attention_paths(psd, K, gamma, kv, dtype):
    n = 1 + K * gamma
    check_attention(psd, [(n, kv), (n, n + 40)], 8, 2, 128, 16, dtype, mask=path_mask(K, gamma) * 2)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_masks_that_leave_rows_empty(psd, dtype):
    """Random bits, rows of zeros, and bits past the words' end; sequences without a prefix."""
    g = torch.Generator().manual_seed(5)
    lens = [(70, 70), (40, 41), (3, 3)]
    mask = [[int(x) for x in torch.randint(0, 1 << 32, (2,), generator=g)] for _ in range(113)]
    for t in (0, 5, 69, 70, 111, 112):
        mask[t] = [0, 0]
    o = check_attention(psd, lens, 6, 2, 64, 16, dtype, mask=mask)
    assert float(o["lse"][5].max()) == -math.inf and float(o["out"][5].abs().max()) == 0.0


def test_attention_more_new_tokens_than_cached(psd):
    """kv_len below n_b: the first new tokens have no position and see nothing."""
    s = ref.Sequences([(6, 4)], 2, 64, 16, F32)
    cache, seqs, dk, dv = s.handles(psd, max_new=6)
    q = torch.randn((6, 4, 64), generator=s.gen)
    o = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4), want_lse=True)
    torch.cuda.synchronize()
    want, lse, *_ = ref.attention(s, q, 64 ** -0.5)
    assert bool((o["lse"][:2] == -math.inf).all()) and bool((o["out"][:2] == 0).all())
    assert float((o["out"].cpu().double() - want).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 40, 150])
def test_attention_unseen_values_change_nothing(psd, rows, dtype):
    """NaN and infinities in keys and values of later tokens, and of tokens behind the window."""
    def poke(s, q):
        page, place = s.place(0, s.lens[0][1] - 1)
        s.k[page, place] = math.nan
        s.v[page, place] = math.inf
        page, place = s.place(0, s.lens[0][1] - 2)
        s.v[page, place, :, ::3] = math.nan
        page, place = s.place(0, s.lens[0][1] - rows - 61)
        s.v[page, place] = -math.inf
        s.k[page, place] = math.inf

    D, H, G, W = 64, 4, 2, 60
    s = ref.Sequences([(rows, 300)], G, D, 16, dtype, seed=3)
    q = torch.randn((rows, H, D), generator=s.gen).to(dtype)
    want, *_ = ref.attention(s, q, D ** -0.5, W)
    poke(s, q)
    cache, seqs, dk, dv = s.handles(psd)
    got = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, H), window=W)["out"].cpu().double()
    assert bool(torch.isfinite(got[:-2]).all())
    assert float((got[:-2] - want[:-2]).abs().max()) < (0.03 if dtype == BF16 else 1e-4)
    assert not bool(torch.isfinite(got[-1]).any())          # it sees both
    assert not bool(torch.isfinite(got[-2][:, ::3]).any())   # it sees the NaN values


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_layouts(psd, dtype):
    """Heads before places in memory, views with gaps, and the output written over the queries."""
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 64, 16, dtype, heads_first=True)
    check_attention(psd, [(70, 100), (1, 40)], 8, 4, 64, 16, dtype, strided=True)
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 64, 16, dtype, strided=True, in_place=True)
    check_attention(psd, [(90, 333)], 8, 2, 128, 16, dtype, in_place=True)
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 64, 16, dtype, max_new=64, max_kv=3000)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_large_scores(psd, dtype):
    """Scores of several hundred: the running maximum moves far, and one token takes nearly all."""
    check_attention(psd, [(1, 500), (5, 300), (130, 300)], 8, 2, 128, 16, dtype, scale=4.0)
    check_attention(psd, [(1, 500), (70, 300)], 8, 2, 128, 16, dtype, scale=-1.0)
    check_attention(psd, [(3, 100)], 4, 2, 64, 16, dtype, scale=0.0)


def test_attention_pages_outside_the_pool(psd):
    s = ref.Sequences([(2, 100)], 2, 64, 16, F32)
    bad = int(s.table[0, 2])
    q = torch.randn((2, 4, 64), generator=s.gen)
    want, *_ = ref.attention(s, q, 0.125, bad_pages=(bad,))
    for wrong in (-1, s.pages, 1 << 30, -(1 << 31)):
        table = s.table.clone()
        table[0, 2] = wrong
        dk, dv = s.k.cuda(), s.v.cuda()
        cache = psd.make_cache(dk, dv)
        seqs = psd.make_seqs(torch.tensor([0, 2], dtype=torch.int32).cuda(), torch.tensor([100], dtype=torch.int32).cuda(),
                             table.cuda(), 2, 2, 100)
        o = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4), scale=0.125)
        assert float((o["out"].cpu().double() - want).abs().max()) < 1e-5, wrong


def test_attention_lengths_past_the_bounds(psd):
    """Rows and positions past the host's bounds are not touched."""
    s = ref.Sequences([(4, 40), (4, 60)], 2, 64, 16, F32)
    cache, seqs, dk, dv = s.handles(psd)
    small = psd.make_seqs(*seqs.tensors, 6, 2, 50)
    q = torch.randn((8, 4, 64), generator=s.gen).cuda()
    out = torch.full((8, 4, 64), 7.0, device="cuda")
    psd.attention(cache, small, q, psd.new_attention_workspace(cache, small, 4), out=out)
    torch.cuda.synchronize()
    assert bool((out[2:4] == 7).all()) and bool((out[6:] == 7).all())
    assert bool(torch.isfinite(out).all())


def test_attention_offsets_past_32_bits(psd):
    """Pages 2^30 elements apart (a pool of 6.4 GB each): offsets need more than 32 bits."""
    G, D, P = 1, 64, 16
    lens = [(2, 40)]
    s = ref.Sequences(lens, G, D, P, BF16, spare=0, width_extra=0)
    step = 1 << 30
    pools = []
    for t in (s.k, s.v):
        flat = torch.empty(2 * step + P * G * D, dtype=BF16, device="cuda")
        view = flat.as_strided((3, P, G, D), (step, G * D, D, 1))
        view.copy_(t)
        pools.append(view)
    cache = psd.make_cache(*pools)
    seqs = psd.make_seqs(torch.tensor([0, 2], dtype=torch.int32).cuda(), torch.tensor([40], dtype=torch.int32).cuda(),
                         s.table.cuda(), 2, 2, 40)
    q = torch.randn((2, 4, D), generator=s.gen).to(BF16)
    o = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4))
    want, *_ = ref.attention(s, q, D ** -0.5)
    assert float((o["out"].cpu().double() - want).abs().max()) < 0.02
    # the last token's key and value go to the far page
    k = torch.ones((2, 1, D), dtype=BF16, device="cuda")
    psd.kv_append(cache, seqs, k, 2 * k)
    torch.cuda.synchronize()
    page, place = s.place(0, 39)
    assert bool((pools[0][page, place] == 1).all()) and bool((pools[1][page, place] == 2).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_long_cache(psd, dtype):
    """A cache long enough to be split over many workgroups, against torch in float64."""
    H, G, D, P, kv, n = 8, 2, 128, 64, 20011, 3
    g = torch.Generator(device="cuda").manual_seed(4)
    width = -(-kv // P)
    k = torch.randn((width, P, G, D), device="cuda", generator=g).to(dtype)
    v = torch.randn((width, P, G, D), device="cuda", generator=g).to(dtype)
    table = torch.randperm(width, device="cuda", generator=g).to(torch.int32)[None].contiguous()
    q = torch.randn((n, H, D), device="cuda", generator=g).to(dtype)
    cache = psd.make_cache(k, v)
    seqs = psd.make_seqs(torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([kv], dtype=torch.int32).cuda(), table,
                         n, n, kv)
    o = psd.attention(cache, seqs, q, psd.new_attention_workspace(cache, seqs, H), want_lse=True)
    kk = k[table[0].long()].reshape(-1, G, D)[:kv].double()
    vv = v[table[0].long()].reshape(-1, G, D)[:kv].double()
    for h in range(H):
        x = q[:, h].double() @ kk[:, h // 4].t() * D ** -0.5
        x.masked_fill_(torch.arange(kv, device="cuda") > torch.arange(kv - n, kv, device="cuda")[:, None], -math.inf)
        want = torch.softmax(x, -1) @ vv[:, h // 4]
        # weights of about 1 / kv each: the output is about kv^-1/2, its errors 2^-9 of that
        tol = 4 * 2.0 ** -9 * kv ** -0.5 if dtype == BF16 else 200 * ULP
        assert float((o["out"][:, h].double() - want).abs().max()) < 5 * tol
        assert float((o["lse"][:, h].double() - torch.logsumexp(x, -1)).abs().max()) < 300 * ULP * 10


# ---------------------------------------------------------------- append

APPENDS = [
    dict(lens=[(1, 1)], H=4, G=2, D=128, P=16, R=128),
    dict(lens=[(1, 30), (1, 17), (1, 16)], H=32, G=8, D=128, P=16, R=128),
    dict(lens=[(5, 40), (0, 9), (3, 3)], H=8, G=2, D=64, P=7, R=64),
    dict(lens=[(9, 20)], H=6, G=3, D=80, P=24, R=40),
    dict(lens=[(4, 11)], H=5, G=1, D=72, P=1, R=26),
    dict(lens=[(3, 8), (2, 2)], H=2, G=2, D=256, P=16, R=256),
    dict(lens=[(70, 90)], H=3, G=3, D=96, P=32, R=0),
    dict(lens=[(2, 5)], H=12, G=4, D=8, P=4, R=6),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n", range(len(APPENDS)))
def test_append(psd, n, interleaved, norm, dtype):
    c = APPENDS[n]
    check_append(psd, **c, interleaved=interleaved, norm=norm, dtype=dtype, heads_first=n % 2 == 1, in_place=n % 3 == 2)


def check_append(psd, lens, H, G, D, P, R, interleaved, norm, dtype, heads_first=False, in_place=False, positions=None,
                 with_q=True):
    print("[append]", lens, H, G, D, P, R, interleaved, norm, dtype, flush=True)
    eps = 1e-5
    s = ref.Sequences(lens, G, D, P, dtype, seed=2, heads_first=heads_first)
    T = s.rows
    qkv = torch.randn((T, H + 2 * G, D), generator=s.gen).to(dtype)
    w = (1 + 0.2 * torch.randn((2, D), generator=s.gen)).to(dtype) if norm else None
    table_rows = 200
    angle = torch.rand((table_rows, max(R // 2, 1)), generator=s.gen) * 6.28
    cos, sin = (angle.cos(), angle.sin()) if R else (None, None)
    cache, seqs, dk, dv = s.handles(psd)
    d = qkv.cuda()
    q, k, v = d[:, :H], d[:, H:H + G], d[:, H + G:]
    got = psd.kv_append(cache, seqs, k, v, q=q if with_q else None, q_out=q if in_place and with_q else None,
                        cos=cos.cuda() if R else None, sin=sin.cuda() if R else None, interleaved=interleaved,
                        positions=None if positions is None else positions.cuda(), q_norm=w[0].cuda() if norm else None,
                        k_norm=w[1].cuda() if norm else None, eps=eps)
    torch.cuda.synchronize()
    want_k, want_v = s.k.double(), s.v.double()
    tol_k = torch.zeros_like(want_k)
    for b in range(s.B):
        for i in range(lens[b][0]):
            t, c = s.new_start[b] + i, s.first(b) + i
            p = c if positions is None else int(positions[t])
            cc, ss = (cos[p].double(), sin[p].double()) if R else (None, None)
            heads = [(qkv[t, :H], 0), (qkv[t, H:H + G], 1)]
            for x, which in heads:
                y, size = ref.norm_rotate(x.double(), w[which].double() if norm else None, eps, cc, ss, interleaved)
                # norm: a mean of D squares, a root, two products; rotation: two products and a sum
                tol = HALF[dtype] * y.abs() + (D / 2 + 12) * ULP * size if norm else HALF[dtype] * y.abs() + 4 * ULP * size
                if which == 0 and with_q:
                    assert bool(((got[t].cpu().double() - y).abs() <= tol).all()), (t, float(((got[t].cpu().double() - y).abs() - tol).max()))
                elif which == 1:
                    page, place = s.place(b, c)
                    want_k[page, place], tol_k[page, place] = y, tol
            page, place = s.place(b, c)
            want_v[page, place] = qkv[t, H + G:].double()
    for g_, w_, tol in ((dk, want_k, tol_k), (dv, want_v, torch.zeros_like(want_v))):
        g_ = g_.cpu().double()
        assert bool(torch.equal(torch.isnan(g_), torch.isnan(w_))), "a place of another token was written"
        assert bool((torch.nan_to_num(g_ - w_).abs() <= tol).all())


def test_append_positions_and_no_queries(psd):
    pos = torch.tensor([7, 8, 8, 9, 9, 3], dtype=torch.int32)
    check_append(psd, [(5, 12), (1, 4)], 4, 2, 64, 16, 64, False, True, BF16, positions=pos)
    check_append(psd, [(5, 12), (1, 4)], 4, 2, 64, 16, 64, True, False, F32, positions=pos, with_q=False)


def test_append_places_that_do_not_exist(psd):
    """No position below 0, no page outside the pool, no place past the table: nothing else is written, and a
    rotation position outside the tables gives NaN."""
    s = ref.Sequences([(4, 2), (3, 50)], 2, 64, 16, F32)
    s.table[1, 3] = s.pages
    cache, seqs, dk, dv = s.handles(psd)
    before = dk.clone()
    k = torch.randn((7, 2, 64), device="cuda")
    psd.kv_append(cache, seqs, k, k)
    torch.cuda.synchronize()
    changed = (torch.nan_to_num(dk, 9.0) != torch.nan_to_num(before, 9.0)).any(-1).any(-1).nonzero().tolist()
    want = sorted([list(s.place(0, 0)), list(s.place(0, 1)), list(s.place(1, 47))])
    assert sorted(changed) == want
    cos = torch.ones((10, 32), device="cuda")
    q = psd.kv_append(cache, seqs, k, k, q=k, cos=cos, sin=cos, positions=torch.tensor([0, 10, -1, 9, 2, 3, 4], dtype=torch.int32).cuda())
    nan = torch.isnan(q).all(-1).all(-1).tolist()
    assert nan == [False, True, True, False, False, False, False]


# ---------------------------------------------------------------- keep

@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("layers", [None, 3])
def test_keep(psd, layers, heads_first, dtype):
    lens = [(17, 40), (17, 17), (9, 30), (1, 5), (0, 6), (33, 40)]
    keeps = [[0, 9, 10, 11, 12], [0, 1, 2], [1, 2, 3, 4, 5, 6, 7, 8], [0], [], [0, 2, 3, 5, 8, 13, 21, 32]]
    s = ref.Sequences(lens, 2, 64, 7, dtype, layers=layers, heads_first=heads_first)
    cache, seqs, dk, dv = s.handles(psd)
    width = 8
    keep = torch.full((6, width + 2), 77, dtype=torch.int32)
    for b, x in enumerate(keeps):
        keep[b, :len(x)] = torch.tensor(x, dtype=torch.int32)
    n_keep = torch.tensor([5, 3, 8, 9, 4, 8], dtype=torch.int32)  # past the new tokens: cut
    got = psd.kv_keep(cache, seqs, keep.cuda()[:, :width], n_keep.cuda())
    torch.cuda.synchronize()
    assert got.tolist() == [s.first(b) + min(int(n_keep[b]), lens[b][0], width) for b in range(6)]
    for t, d in ((s.k, dk), (s.v, dv)):
        want = t.clone()
        for b, x in enumerate(keeps):
            for i, j in enumerate(x):
                src, dst = s.place(b, s.first(b) + j), s.place(b, s.first(b) + i)
                want[..., dst[0], dst[1], :, :] = t[..., src[0], src[1], :, :]
        d = d.cpu()
        assert bool(torch.equal(torch.nan_to_num(d, 55.0), torch.nan_to_num(want, 55.0)))


# ---------------------------------------------------------------- verification from given random numbers

def logits(g, B, n, V, dtype, peak):
    z = torch.randn((B, n, V), generator=g) * 2.0 - peak * torch.log(1 + torch.rand((B, n, V), generator=g) * (V - 1))
    return z.to(dtype)


def check_given(psd, B, gamma, V, dtype, T=(1.0, 1.0), seed=0, n_drafts=None, edit=None, tau=0.7, ties=False):
    print("[given]", B, gamma, V, dtype, T, flush=True)
    g = torch.Generator().manual_seed(seed)
    target = logits(g, B, gamma + 1, V, dtype, 1.0)
    draft = (target[:, :gamma].float() + tau * torch.randn((B, gamma, V), generator=g)).to(dtype)
    e = torch.empty((B, V)).exponential_(generator=g).clamp_(min=1e-30)
    x = (draft.float() / T[1] - torch.empty((B, gamma, V)).exponential_(generator=g).log()).argmax(-1).to(torch.int32)
    u = torch.rand((B, gamma), generator=g)
    if edit:
        edit(target, draft, x, u, e)
    params = psd.make_params(0, V, 1, 0, T[0], T[1], dtype=dtype)
    ws = psd.new_verify_given_workspace(params, B, gamma)
    ws.fill_(0xAB)  # needs no clearing
    nd = None if n_drafts is None else torch.tensor(n_drafts, dtype=torch.int32)
    want, length, p_lse, q_lse, near = ref.verify_given(target, draft, x, u, e, T[0], T[1], nd)
    dev = [t.cuda() for t in (target, draft, x, u, e)]
    for _ in range(2):
        o = psd.verify_given(params, ws, *dev, n_drafts=None if nd is None else nd.cuda(), want_lse=True)
        torch.cuda.synchronize()
        for b in range(B):
            if ties or near[b] > 1e-5:  # decisions further apart than float32 errs
                assert o["out_tokens"][b].tolist() == want[b].tolist(), (b, near[b])
                assert int(o["out_len"][b]) == int(length[b])
        for got, lse in ((o["target_lse"], p_lse), (o["draft_lse"], q_lse)):
            got = got.cpu().double()
            assert bool(torch.equal(got == -math.inf, lse == -math.inf))
            ok = torch.isfinite(lse)
            assert not ok.any() or float(((got - lse)[ok].abs() / lse[ok].abs().clamp(min=1.0)).max()) < 1e-6
    assert ties or sum(n > 1e-5 for n in near) >= 0.9 * B
    return o, length


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,gamma,V", [(1, 1, 1), (3, 2, 2), (2, 4, 7), (5, 3, 1000), (64, 1, 33), (2, 32, 777), (7, 4, 50257),
                                       (1, 4, 128256), (300, 2, 65)])
def test_given(psd, B, gamma, V, dtype):
    o, length = check_given(psd, B, gamma, V, dtype)
    if B >= 64:
        assert len(set(length.tolist())) > 1


@pytest.mark.parametrize("T", [(0.7, 0.7), (0.05, 2.0), (3.0, 0.2)])
def test_given_temperatures(psd, T):
    check_given(psd, 16, 4, 3001, F32, T=T, seed=3)
    check_given(psd, 16, 4, 3001, BF16, T=T, seed=4)


def test_given_ragged_drafts(psd):
    check_given(psd, 8, 5, 999, BF16, n_drafts=[0, 1, 5, 3, -2, 9, 4, 2], tau=0.1)


def test_given_same_rows_accept_all(psd):
    def edit(target, draft, x, u, e):
        draft.copy_(target[:, :4])
        x.copy_((draft.float() - torch.log(torch.empty_like(draft, dtype=F32).exponential_(generator=torch.Generator().manual_seed(1))))
                .argmax(-1))
        u.mul_(0.999)
    o, length = check_given(psd, 6, 4, 500, F32, edit=edit)
    assert length.tolist() == [5] * 6


def test_given_masked_and_empty_rows(psd):
    """-inf logits, rows without a finite logit, drafts outside the vocabulary, drafts of probability 0."""
    def edit(target, draft, x, u, e):
        target[0, 1] = -math.inf                     # no target: refused there, nothing to emit
        draft[1, 0] = -math.inf                      # no drafter: accepted wherever p > 0
        x[2, 0] = 400
        x[3, 1] = -1
        target[4, :, ::2] = -math.inf
        x[4, 0] = 2                                  # p = 0: refused, u = 0 included
        u[4, 0] = 0.0
        draft[5, 0, :] = -math.inf
        draft[5, 0, 7] = 3.0
        x[5, 0] = 7
        target[6, 0, :] = -math.inf
        target[6, 0, 9] = 1.0                        # one token has all of p
        target[7] = -math.inf
    o, length = check_given(psd, 8, 3, 400, F32, edit=edit, seed=8)
    tokens = o["out_tokens"].tolist()
    assert tokens[7][0] == -1 and int(length[7]) == 1
    assert int(length[2]) == 1 and int(length[4]) == 1


def test_given_ties_go_to_the_lowest_token(psd):
    def edit(target, draft, x, u, e):
        target.zero_()
        draft.zero_()
        u.fill_(0.5)
        e.fill_(1.0)
        e[:, 300:] = 0.5
    o, length = check_given(psd, 2, 2, 5000, F32, edit=edit, ties=True)
    assert o["out_tokens"][:, 2].tolist() == [300, 300]


def test_given_follows_the_target(psd):
    """The first emitted token over many sequences follows p whatever the drafter: chi-square at 6 sigma."""
    V, B = 12, 60000
    g = torch.Generator(device="cuda").manual_seed(11)
    p_row, q_row = torch.randn(V, device="cuda", generator=g), torch.randn(V, device="cuda", generator=g)
    target = p_row.expand(B, 2, V).contiguous()
    draft = q_row.expand(B, 1, V).contiguous()
    x = torch.multinomial(torch.softmax(q_row, 0), B, replacement=True, generator=g).to(torch.int32)[:, None].contiguous()
    params = psd.make_params(0, V, 1, 0, dtype=F32)
    e = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    u = torch.rand((B, 1), device="cuda", generator=g)
    o = psd.verify_given(params, psd.new_verify_given_workspace(params, B, 1), target, draft, x, u, e)
    count = torch.bincount(o["out_tokens"][:, 0].long(), minlength=V).double()
    want = torch.softmax(p_row.double(), 0) * B
    chi = float(((count - want) ** 2 / want).sum())
    assert chi < (V - 1) + 6 * (2 * (V - 1)) ** 0.5, chi


# ---------------------------------------------------------------- streams and graphs

def test_other_stream_and_graph(psd):
    """The whole block on a stream of its own, captured: replays follow lengths that change on the device."""
    H, G, D, P, B = 8, 2, 64, 16, 3
    s = ref.Sequences([(5, 60), (5, 33), (5, 5)], G, D, P, BF16)
    cache, seqs, dk, dv = s.handles(psd, max_kv=80)
    kv_len = seqs.tensors[1]
    q = torch.randn((15, H, D), generator=s.gen).to(BF16)
    dq = q.cuda()
    ws = psd.new_attention_workspace(cache, seqs, H)
    out = torch.empty((15, H, D), dtype=BF16, device="cuda")
    keep = torch.tensor([[0, 2, 4]] * B, dtype=torch.int32, device="cuda")
    n_keep = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    kv_out = torch.empty(B, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()

    def block():
        qq = psd.kv_append(cache, seqs, dq[:, :G], dq[:, G:2 * G], q=dq, stream=stream, q_out=out)
        psd.attention(cache, seqs, qq, ws, out=out, stream=stream)
        psd.kv_keep(cache, seqs, keep, n_keep, kv_out=kv_out, stream=stream)

    torch.cuda.synchronize()
    block()
    torch.cuda.synchronize()
    eager = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        block()
    for lens in ([60, 33, 5], [61, 30, 7], [60, 33, 5], [70, 5, 9]):
        dk.copy_(torch.randn(dk.shape, generator=torch.Generator().manual_seed(1)).to(BF16))
        dv.copy_(torch.randn(dk.shape, generator=torch.Generator().manual_seed(2)).to(BF16))
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        start_k, start_v = dk.clone(), dv.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, got_k, got_kv = out.clone(), dk.clone(), kv_out.tolist()
        dk.copy_(start_k)
        dv.copy_(start_v)
        torch.cuda.synchronize()
        block()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_k, dk) and got_kv == kv_out.tolist()
        assert got_kv == [lens[0] - 4, lens[1] - 3, lens[2] - 2]
    assert not torch.equal(eager, out)
