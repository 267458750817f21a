"""The operators over a cache held in 4 bits against plain 64-bit implementations (GPU).

Unused places of every pool are NaN groups, so a read past a sequence's end shows.  Bounds are those of the arithmetic
(see test_gpu_serving.py): a code's products with bfloat16 terms are exact, so bfloat16 rows have the same bounds as
over a bfloat16 cache, and float32 rows, three terms each, those of sums of three times as many products.  Codes are
decided in 64 bits and have to be the definition's."""
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
import serving_ref as ref  # noqa: E402
from test_gpu_serving import BF16, F32, HALF, SHAPES, ULP, path_mask  # noqa: E402


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


# ---------------------------------------------------------------- append

def rope_tables(n, R, seed=3):
    g = torch.Generator().manual_seed(seed)
    angle = torch.rand((n, max(R // 2, 1)), generator=g, dtype=torch.float64) * 6.3
    return angle.cos().float()[:, :R // 2].contiguous(), angle.sin().float()[:, :R // 2].contiguous()


def same(x, y):
    return bool(((x == y) | (x.isnan() & y.isnan())).all())


def check_append(psd, lens, H, G, D, P, dtype, R=0, norm=False, interleaved=False, heads_first=True, positions=None, poke=None,
                 seed=5, stream=None):
    print("[append4]", lens[:4], len(lens), H, G, D, P, dtype, R, norm, interleaved, flush=True)
    s = ref4.Sequences4(lens, G, D, P, dtype, seed=seed, heads_first=heads_first)
    T, g = s.rows, s.gen
    qkv = torch.randn((T, (H + 2 * G) * D), generator=g).to(dtype)
    if poke:
        poke(qkv, H, G, D)
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split((H * D, G * D, G * D), 1))
    dev = qkv.cuda()
    dq, dk, dv = (t.unflatten(1, (-1, D)) for t in dev.split((H * D, G * D, G * D), 1))
    cache, seqs, pools = s.handles(psd)
    before = [p.cpu() for p in pools]
    n_pos = max(kv for _, kv in lens) + 2
    cos, sin = rope_tables(n_pos, R) if R else (None, None)
    wq, wk = ((1 + 0.2 * torch.randn(D, generator=g)).to(dtype) for _ in range(2)) if norm else (None, None)
    held = [torch.full((T, G, D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    kw = dict(q=dq, cos=None if cos is None else cos.cuda(), sin=None if sin is None else sin.cuda(), interleaved=interleaved,
              q_norm=None if wq is None else wq.cuda(), k_norm=None if wk is None else wk.cuda(), eps=1e-6,
              positions=None if positions is None else positions.cuda(), k_held=held[0], v_held=held[1])
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    q_out = psd.kv_append(cache, seqs, dk, dv, stream=stream, **kw)
    torch.cuda.synchronize()
    after = [p.cpu() for p in pools]
    kh, vh = (h.cpu().double() for h in held)
    eps = float(torch.tensor(1e-6))
    expect = [p.clone() for p in before]
    near = []
    for b in range(s.B):
        for i in range(s.lens[b][0]):
            t, pos = s.new_start[b] + i, s.first(b) + i
            rp = pos if positions is None else int(positions[t])
            c, sn = (None, None) if not R else (cos[rp].double(), sin[rp].double())
            kk, _ = ref.norm_rotate(k[t].double(), None if wk is None else wk.double(), eps, c, sn, interleaved)
            qq, size = ref.norm_rotate(q[t].double(), None if wq is None else wq.double(), eps, c, sn, interleaved)
            # 64-bit arithmetic leaves a few 2^-53 of what was added up: codes that near to a border may be either
            codes, scales, close = ref4.encode(kk, near=1e-12, computed=D if norm else R)
            vcodes, vscales = ref4.encode(v[t].double())
            assert same(vh[t], ref4.decode(vcodes, vscales, D)), ("v_held", b, i)
            want = ref4.decode(codes, scales, D)
            sure = ~close.repeat_interleave(32, -1)[:, :D]
            assert same(kh[t][sure], want[sure]), ("k_held", b, i)
            got_q = q_out[t].cpu().double()
            fine = torch.isfinite(qq)
            tol = (D + 8) * ULP * size + HALF[dtype] * qq.abs()
            assert bool(((got_q - qq).abs() <= tol)[fine].all()), ("q", b, i, float(((got_q - qq).abs() - tol)[fine].max()))
            if pos < 0:
                continue
            page, place = s.place(b, pos)
            for pool, x in zip(expect, (codes, vcodes, scales, vscales)):
                pool[page, place] = x
            near.append((page, place, close))
    for page, place, close in near:
        for j in (0, 2):
            n = 16 if j == 0 else 1
            at = close.repeat_interleave(n, -1)
            expect[j][page, place] = torch.where(at, after[j][page, place], expect[j][page, place])
    for name, e, x in zip(("k", "v", "k_scale", "v_scale"), expect, after):
        assert torch.equal(e, x), (name, (e != x).nonzero()[:4].tolist())
    assert sum(int(c.sum()) for _, _, c in near) < 3


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,R,interleaved", [(128, 128, False), (128, 64, True), (64, 0, False), (80, 40, False), (96, 96, True),
                                             (256, 128, False), (8, 8, False), (40, 12, False), (200, 200, True), (72, 0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_append_shapes(psd, D, R, interleaved, norm, dtype):
    check_append(psd, [(1, 1), (3, 40), (0, 7), (5, 5), (2, 18)], 6, 2, D, 16, dtype, R=R, norm=norm, interleaved=interleaved)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_append_layouts_and_many_rows(psd, dtype):
    check_append(psd, [(3, 20), (2, 9)], 3, 3, 128, 5, dtype, R=128, heads_first=False)
    check_append(psd, [(2, 20)], 40, 40, 64, 7, dtype, R=64, norm=True)           # more heads than a wave's groups
    check_append(psd, [(1100, 1200), (3, 3)], 2, 1, 64, 64, dtype, R=32, norm=True)  # a wave a row
    positions = torch.tensor([4, 0, 5, 5, 1], dtype=torch.int32)
    check_append(psd, [(3, 20), (2, 9)], 4, 2, 96, 8, dtype, R=64, positions=positions)
    check_append(psd, [(3, 20), (2, 9)], 4, 2, 96, 8, dtype, R=64, stream=torch.cuda.Stream())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_append_borders(psd, dtype):
    """Ties between two codes and two scales, zeros, numbers at both ends of float32, infinities and NaN."""
    def poke(qkv, H, G, D):
        rows = qkv.view(qkv.shape[0], -1, 32)
        ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.5, 0.0, -0.0,
                             7.0, -7.0, 4.5, 5.5, 0.2, -0.1, 2.0, 3.0, 1.0, 0.5, 1.5, 4.0, 0.0, 6.9])
        first, n = H * D // 32, G * D // 32
        for j, scale in enumerate([1.0, 2.0 ** -126, 2.0 ** 100, 2.0 ** 125, 2.0 ** -100, 0.0, 2.0 ** -130]):
            rows[0, first + j] = (ties * scale).to(qkv.dtype)
        rows[1, first] = (ties * 0.5).to(qkv.dtype)
        rows[1, first + 1, 3] = 7.03125                       # the least bfloat16 above 7
        rows[1, first + 2, 5] = math.inf
        rows[1, first + 3, 31] = math.nan
        rows[1, first + 4, 0] = -math.inf
        rows[1, first + 5] = torch.finfo(qkv.dtype).max
        rows[1, first + 6] = -torch.finfo(qkv.dtype).max / 3
        rows[1, first + 7] = 2.0 ** -133
        rows[:, first + n:first + 2 * n] = rows[:, first:first + n]  # values as keys
    check_append(psd, [(2, 20)], 4, 4, 64, 16, dtype, poke=poke)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_append_tokens_without_a_place(psd, dtype):
    """Positions before 0, pages outside the pool and rows past the last sequence: nothing is written there."""
    check_append(psd, [(6, 4), (2, 30)], 2, 2, 64, 16, dtype, R=64, positions=torch.arange(8, dtype=torch.int32))
    s = ref4.Sequences4([(3, 40)], 2, 64, 16, dtype)
    s.table[0, 2] = -1
    cache, seqs, pools = s.handles(psd)
    seqs.rows = 5
    k, v = (torch.randn((5, 2, 64), generator=s.gen).to(dtype).cuda() for _ in range(2))
    held = torch.full((5, 2, 64), 3.0, dtype=dtype, device="cuda")
    psd.kv_append(cache, seqs, k, v, k_held=held)
    torch.cuda.synchronize()
    for p, was in zip(pools, (s.kc, s.vc, s.ks, s.vs)):
        assert torch.equal(p.cpu(), was)
    assert bool((held[3:] == 3.0).all()) and not bool((held[:3] == 3.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,R,rows", [(128, 64, 3), (80, 40, 3), (64, 64, 1100)])
def test_append_held_in_place(psd, D, R, rows, dtype):
    """The held values written over the keys and values that they come from, the queries over themselves."""
    got = []
    for in_place in (False, True):
        s = ref4.Sequences4([(rows, rows + 9), (2, 11)], 2, D, 16, dtype)
        g = torch.Generator().manual_seed(8)
        q, k, v = (torch.randn((s.rows, n, D), generator=g).to(dtype).cuda() for n in (6, 2, 2))
        cache, seqs, pools = s.handles(psd)
        cos, sin = (x.cuda() for x in rope_tables(rows + 20, R))
        outs = (q, k, v) if in_place else tuple(torch.empty_like(x) for x in (q, k, v))
        psd.kv_append(cache, seqs, k, v, q=q, q_out=outs[0], cos=cos, sin=sin, k_held=outs[1], v_held=outs[2])
        torch.cuda.synchronize()
        got.append([x.cpu() for x in outs] + [p.cpu() for p in pools])
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- attention

def attention_bounds(s, out, spread, size, vmax, kv, dtype):
    terms = 1 if dtype == BF16 else 3
    score = (terms * s.D + 4) * ULP * size
    rel = 2 * score + (terms * kv + 8) * ULP
    tol = rel * vmax + HALF[dtype] * out.abs()
    if dtype == BF16:
        tol = tol + HALF[BF16] * spread
    return tol, score + (terms * kv + 8) * ULP


def check_attention(psd, lens, H, G, D, P, dtype, window=0, mask=None, heads_first=True, seed=1, scale=None, in_place=False,
                    strided=False, max_new=None, max_kv=None, poke=None, stream=None, ws=None, bad_pages=()):
    print("[attention4]", lens[:4], len(lens), H, G, D, P, dtype, window, flush=True)
    s = ref4.Sequences4(lens, G, D, P, dtype, seed=seed, heads_first=heads_first)
    T = s.rows
    q = torch.randn((T, H, D), generator=s.gen).to(dtype)
    if poke:
        poke(s, q)
    cache, seqs, _ = s.handles(psd, max_new, max_kv)
    scale = D ** -0.5 if scale is None else scale
    ws = psd.new_attention_workspace(cache, seqs, H) if ws is None else ws
    dq = q.cuda()
    if strided:
        wide = torch.full((T, H + 3, D + 8), math.nan, dtype=dtype, device="cuda")
        wide[:, 1:H + 1, :D] = dq
        dq = wide[:, 1:H + 1, :D]
    out = dq if in_place else torch.full((T, H, D), 7.0, dtype=dtype, device="cuda")
    dmask = None if mask is None else torch.tensor([[w - (1 << 32) if w >= 1 << 31 else w for w in r] for r in mask],
                                                   dtype=torch.int32, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    o = psd.attention(cache, seqs, dq, ws, scale=scale, window=window, mask=dmask, out=out, want_lse=True, stream=stream)
    torch.cuda.synchronize()
    want, lse, spread, size, vmax = ref.attention(s, q, scale, window, mask, bad_pages)
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


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", range(len(SHAPES)))
def test_attention_shapes(psd, n, dtype):
    check_attention(psd, **SHAPES[n], dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 192])
def test_attention_more_short_sequences_than_workgroups(psd, D, dtype):
    """Sequences below a stretch's least length, some without rows, more of them than threads."""
    check_attention(psd, [(1, 5)] * 40, 16, 16, D, 16, dtype)
    check_attention(psd, [(b % 3, b % 3 + 7 * b % 140) for b in range(36)], 32, 16, D, 16, dtype)
    check_attention(psd, [(1, 1 + b % 9) for b in range(260)] + [(2, 300)], 4, 2, D, 16, dtype)
    check_attention(psd, [(9, 9 + 11 * b % 130) for b in range(34)], 48, 16, D, 16, dtype)  # 27 rows


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 5000])
def test_attention_windows(psd, window, dtype):
    check_attention(psd, [(1, 300), (5, 333), (40, 200), (1, 1)], 8, 2, 128, 16, dtype, window=window)
    check_attention(psd, [(150, 400)], 4, 2, 64, 24, dtype, window=window)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("K,gamma,kv", [(1, 1, 2), (2, 4, 9), (4, 4, 300), (8, 8, 500), (5, 7, 97)])
def test_attention_paths(psd, K, gamma, kv, dtype):
    n = 1 + K * gamma
    check_attention(psd, [(n, kv), (n, n + 40)], 8, 2, 128, 16, dtype, mask=path_mask(K, gamma) * 2)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_masks_that_leave_rows_empty(psd, dtype):
    g = torch.Generator().manual_seed(5)
    lens = [(70, 70), (40, 41), (3, 3)]
    mask = [[int(x) for x in torch.randint(0, 1 << 32, (2,), generator=g)] for _ in range(113)]
    for t in (0, 5, 69, 70, 111, 112):
        mask[t] = [0, 0]
    o = check_attention(psd, lens, 6, 2, 64, 16, dtype, mask=mask)
    assert float(o["lse"][5].max()) == -math.inf and float(o["out"][5].abs().max()) == 0.0
    check_attention(psd, [(6, 4)], 4, 2, 64, 16, dtype)  # rows before position 0 see nothing


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,D", [(3, 64), (3, 256), (9, 128), (40, 64), (150, 64), (150, 200)])
def test_attention_unseen_values_change_nothing(psd, rows, D, dtype):
    """NaN groups in keys and values of later tokens, and of tokens behind the window."""
    H, G, W = 4, 2, 60
    s = ref4.Sequences4([(rows, 300)], G, D, 16, dtype, seed=3)
    q = torch.randn((rows, H, D), generator=s.gen).to(dtype)
    want, _, spread, size, vmax = ref.attention(s, q, D ** -0.5, W)
    tol, _ = attention_bounds(s, want, spread, size, vmax, 300, dtype)
    kv = s.lens[0][1]
    page, place = s.place(0, kv - 1)
    s.ks[page, place] = 255
    page, place = s.place(0, kv - 2)
    s.vs[page, place, :, 0] = 255
    page, place = s.place(0, kv - rows - 61)
    s.ks[page, place] = 255
    s.vs[page, place] = 255
    cache, seqs, _ = s.handles(psd)
    got = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, H), window=W)["out"].cpu().double()
    assert bool(torch.isfinite(got[:-2]).all())
    assert bool(((got - want).abs() <= tol)[:-2].all())
    assert not bool(torch.isfinite(got[-1]).any())          # it sees the NaN key
    assert not bool(torch.isfinite(got[-2][:, :32]).any())  # it sees the NaN group,
    if D > 32:
        assert bool(((got - want).abs() <= tol)[-2][:, 32:].all())  # and the others' values as they are


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_layouts(psd, dtype):
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 64, 16, dtype, heads_first=False)
    check_attention(psd, [(70, 100), (1, 40)], 8, 4, 64, 16, dtype, strided=True, heads_first=False)
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 64, 16, dtype, strided=True, in_place=True)
    check_attention(psd, [(90, 333)], 8, 2, 128, 16, dtype, in_place=True)
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 64, 16, dtype, max_new=64, max_kv=3000)
    check_attention(psd, [(5, 100), (1, 40)], 8, 4, 96, 16, dtype, stream=torch.cuda.Stream())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_attention_pages_outside_the_pool(psd, dtype):
    """Cached tokens on such a page are seen by no row."""
    for rows, H, G, D in ((1, 4, 2, 128), (4, 4, 1, 64), (120, 2, 1, 128)):
        bad = []

        def poke(s, q):
            bad[:] = [s.pages + 3, -5]
            s.table[0, 3], s.table[0, 9] = bad

        check_attention(psd, [(rows, 400)], H, G, D, 16, dtype, poke=poke, bad_pages=bad)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,H,G,D", [([(1, 5000)], 4, 1, 128), ([(1, 9000), (1, 40), (1, 3000)], 8, 2, 64),
                                        ([(5, 6000), (5, 5)], 8, 1, 128), ([(2, 4000)], 2, 2, 256), ([(9, 3000)], 4, 1, 80)])
def test_attention_work_that_is_cut(psd, lens, H, G, D, dtype):
    """Sequences that many workgroups share, in a workspace that several calls use one after the other."""
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    a = check_attention(psd, lens, H, G, D, 16, dtype, ws=ws)
    b = check_attention(psd, lens, H, G, D, 16, dtype, ws=ws)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_attention_large_scores(psd):
    """Scales that push scores far out, and queries of very different sizes in one row (float32: all terms count)."""
    for rows in (2, 100):
        check_attention(psd, [(rows, 200)], 4, 2, 64, 16, BF16, scale=30.0)

    def poke(s, q):
        q *= 10.0 ** torch.linspace(-6, 2, q.shape[-1])
    check_attention(psd, [(3, 200)], 4, 2, 128, 16, F32, poke=poke)
    check_attention(psd, [(3, 200)], 4, 2, 128, 16, F32, scale=-2.0)


def test_attention_far_offsets(psd):
    """Pools whose pages lie past 2^32 bytes of codes."""
    D, G, P = 64, 1, 16
    s = ref4.Sequences4([(2, 60), (1, 33)], G, D, P, BF16)
    q = torch.randn((3, 4, D), generator=s.gen).to(BF16)
    want, _, spread, size, vmax = ref.attention(s, q, D ** -0.5)
    tol, _ = attention_bounds(s, want, spread, size, vmax, 60, BF16)
    stride = 5 * 10 ** 9 // s.pages // 16 * 16

    def far(t, width):
        big = torch.empty((stride * (s.pages - 1) + P * G * width,), dtype=torch.uint8, device="cuda")
        view = big.as_strided((s.pages, P, G, width), (stride, G * width, width, 1))
        view.copy_(t)
        return view
    pools = [far(t, w) for t, w in ((s.kc, 32), (s.vc, 32), (s.ks, 2), (s.vs, 2))]
    cache = psd.make_cache4(*pools, D)
    _, seqs, _ = s.handles(psd)
    got = psd.attention(cache, seqs, q.cuda(), psd.new_attention_workspace(cache, seqs, 4))["out"].cpu().double()
    assert bool(((got - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 5, 80])
def test_captured_calls_follow_the_lengths(psd, rows, dtype):
    """Append and attention in one graph, replayed with other lengths: each replay is the eager call's result."""
    H, G, D, P, B = 8, 2, 128, 16, 3
    width = 40
    cache = psd.new_cache4(B * width, P, G, D, dtype=dtype)
    table = torch.randperm(B * width, device="cuda").to(torch.int32).view(B, width)
    start = (torch.arange(B + 1, device="cuda") * rows).to(torch.int32)
    kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    seqs = psd.make_seqs(start, kv_len, table, B * rows, rows, width * P)
    ws = psd.new_attention_workspace(cache, seqs, H)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((B * rows, (H + 2 * G) * D), device="cuda", dtype=dtype)
    q, k, v = (t.unflatten(1, (-1, D)) for t in x.split((H * D, G * D, G * D), 1))
    out, lse = torch.empty((B * rows, H, D), device="cuda", dtype=dtype), torch.empty((B * rows, H), device="cuda")

    def step():
        psd.kv_append(cache, seqs, k, v)
        psd.attention(cache, seqs, q, ws, out=out, want_lse=True, lse=lse)

    def fill(n):
        kv_len.copy_(torch.tensor([n, min(n + 37, width * P), rows], dtype=torch.int32))
        x.normal_(generator=g)

    fill(rows)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in (rows, rows + 90, 600, rows + 3, 300):
        fill(n)
        step()
        eager = out.clone(), lse.clone()
        out.fill_(5.0)
        lse.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), n


# ---------------------------------------------------------------- keep

@pytest.mark.parametrize("D,G,P,layers,heads_first", [(128, 8, 16, 3, True), (80, 2, 5, 1, False), (256, 3, 64, 2, True), (8, 1, 1, 4, True)])
def test_keep(psd, D, G, P, layers, heads_first):
    lens = [(9, 30), (5, 5), (0, 12), (9, 9), (70, 100)]
    s = ref4.Sequences4(lens, G, D, P, BF16, layers=layers, heads_first=heads_first)
    cache, seqs, pools = s.handles(psd)
    width = 66
    keep = torch.full((5, width), 1000, dtype=torch.int32)
    rows = [[0, 5, 6, 8], [1, 3], [], list(range(9)), list(range(1, 66))]
    for b, row in enumerate(rows):
        keep[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    n_keep = torch.tensor([len(r) for r in rows], dtype=torch.int32)
    kv = psd.kv_keep(cache, seqs, keep.cuda(), n_keep.cuda())
    torch.cuda.synchronize()
    want = [t.clone() for t in (s.kc, s.vc, s.ks, s.vs)]
    for b, row in enumerate(rows):
        for i, x in enumerate(row):
            (pf, cf), (pt, ct) = s.place(b, s.first(b) + x), s.place(b, s.first(b) + i)
            for w, was in zip(want, (s.kc, s.vc, s.ks, s.vs)):
                w[:, pt, ct] = was[:, pf, cf]
    for p, w in zip(pools, want):
        assert torch.equal(p.cpu(), w)
    assert kv.tolist() == [s.first(b) + len(r) for b, r in enumerate(rows)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,R,interleaved", [(64, 64, False), (64, 64, True), (96, 24, False), (256, 256, False)])
def test_append_next_to_borders(psd, D, R, interleaved, dtype):
    """Turned keys that are no floats and whose nearest float is a border between two codes, or two scales: the code is that of
    the key itself, which a sum of a border and a far smaller product has exactly in 64 bits."""
    half, n_pos = R // 2, 6
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    cos = torch.ones((n_pos, half))
    sin = torch.tensor([2.0 ** -28, -(2.0 ** -28), 2.0 ** -40, -(2.0 ** -40), 2.0 ** -28, -(2.0 ** -28)])[:, None].expand(-1, half).contiguous()
    k = torch.zeros((n_pos, 2, D))
    r = torch.arange(half)
    a, b = (2 * r, 2 * r + 1) if interleaved else (r, r + half)
    for t in range(n_pos):
        for h in range(2):
            k[t, h, a] = borders[(r + t) % 7] * torch.where(r % 2 > 0, -1.0, 1.0)
            k[t, h, b] = torch.where(r % 3 > 0, 1.0, -1.0)
            k[t, h, a[::8]] = 6.0 if t < 4 else 7.0  # the group's scale, and next to the border of two
    k[:, 1, R:] = 2.5  # (not turned: a tie)
    k[4:, 1] *= 2.0 ** 120
    k = k.to(dtype)
    exact = torch.stack([ref.norm_rotate(k[t].double(), None, 0.0, cos[t].double(), sin[t].double(), interleaved)[0] for t in range(n_pos)])
    codes, scales = ref4.encode(exact)
    rounded = ref4.encode(exact.float().double())
    assert all(bool((rounded[0][t] != codes[t]).any()) for t in range(n_pos)), "these keys tell nothing"
    assert bool((rounded[1] != scales).any())
    s = ref4.Sequences4([(n_pos, n_pos)], 2, D, 16, dtype)
    cache, seqs, pools = s.handles(psd)
    held = torch.empty((n_pos, 2, D), dtype=dtype, device="cuda")
    psd.kv_append(cache, seqs, k.cuda(), k.cuda(), cos=cos.cuda(), sin=sin.cuda(), interleaved=interleaved, k_held=held)
    torch.cuda.synchronize()
    page = int(s.table[0, 0])
    assert torch.equal(pools[0][page, :n_pos].cpu(), codes) and torch.equal(pools[2][page, :n_pos].cpu(), scales)
    assert torch.equal(held.cpu().double(), ref4.decode(codes, scales, D))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows,kv", [(1, 1), (1, 64), (5, 5), (40, 40), (130, 64)])
def test_attention_reads_every_scale_byte(psd, rows, kv, D, dtype):
    """Every scale byte that is defined and all 16 codes, a scale to a sequence: rows that weigh all tokens alike have the first's
    values over their number, and where a row sees one token alone, one product is its lse; 255 is NaN, whatever the code.  In
    blocks that rows see whole and in others."""
    n, P, B = D // 32, 64, 256
    table = torch.randperm(B, generator=torch.Generator().manual_seed(D + kv)).to(torch.int32).view(B, 1)
    at = table[:, 0].long()
    start = torch.arange(B + 1, dtype=torch.int32) * rows
    seqs = psd.make_seqs(start.cuda(), torch.full((B,), kv, dtype=torch.int32).cuda(), table.cuda(), B * rows, rows, kv)
    every = torch.arange(256, dtype=torch.uint8)[:, None].expand(-1, n)

    def first(codes, scales):
        """Pools whose first tokens hold these codes and scales, the others zeros."""
        c, s = torch.zeros((B, P, 1, 16 * n), dtype=torch.uint8), torch.full((B, P, 1, n), 127, dtype=torch.uint8)
        c[at, 0, 0], s[at, 0, 0] = codes, scales
        return c.cuda(), s.cuda()

    def attend(keys, values, q):
        cache = psd.make_cache4(keys[0], values[0], keys[1], values[1], D, dtype=dtype)
        o = psd.attention(cache, seqs, q.to(dtype).cuda(), psd.new_attention_workspace(cache, seqs, 1), scale=1.0, want_lse=True)
        return o["out"].cpu().double().view(B, rows, D), o["lse"].cpu().double().view(B, rows)

    zeros = first(torch.zeros(16 * n, dtype=torch.uint8), torch.full((n,), 127, dtype=torch.uint8))
    q = torch.zeros((B * rows, 1, D))
    code = (torch.arange(D) % 16).to(torch.uint8)
    out, _ = attend(zeros, first(code[0::2] + 16 * code[1::2], every), q)
    value = torch.tensor(ref4.LEVELS + [-x for x in ref4.LEVELS], dtype=torch.float64)[code.long()] * 2.0 ** (torch.arange(256).double() - 127)[:, None]
    # one rounding, of which 2^-133 (bfloat16) or 2^-149 may be the least step, and the quotient's
    step = 2.0 ** -133 if dtype == BF16 else 2.0 ** -149
    for i in range(rows):
        seen = kv - rows + i + 1
        if seen > 0:
            want = value[:253] / seen
            off = (out[:253, i] - want).abs()
            assert bool((off <= (HALF[dtype] + 4 * ULP) * want.abs() + step).all()), (i, (off / want.abs().clamp(min=step)).max())
            assert not bool(torch.isfinite(out[255, i]).any()), (i, out[255, i, :16].tolist())
    if kv == rows:
        q[:, 0, D // 2 + 1] = 1
        for c in range(16):
            _, lse = attend(first(torch.full((16 * n,), 17 * c, dtype=torch.uint8), every), zeros, q)
            want = (ref4.LEVELS[c & 7] * (-1 if c & 8 else 1)) * 2.0 ** (torch.arange(253).double() - 127)
            off, fine = (lse[:253, 0] - want).abs(), want.abs() * 1.45 < 2.0 ** 128  # (in units of ln 2)
            assert bool((off <= 4 * ULP * want.abs() + 2.0 ** -148)[fine].all()), (c, float((off / want.abs())[fine].max()))
            assert bool(torch.isnan(lse[255, 0])), (c, float(lse[255, 0]))
