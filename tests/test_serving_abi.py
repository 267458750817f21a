"""Refusals of the paged cache's operators and of the verification from given random numbers: every
invalid argument returns its status before anything is launched (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

FAKE = 4096  # a non-NULL, 256-aligned dummy address: never dereferenced by rejected calls
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def psd():
    from paper_2609_21858_amd import psd as m
    return m


def structs(psd, **edit):
    c = psd.Cache(FAKE, FAKE, psd.PSD_BF16, 8, 128, 16, 100, 1, 0, 16 * 8 * 128, 8 * 128, 128)
    s = psd.Seqs(4, 20, 5, 4096, 256, 256, FAKE, FAKE, FAKE)
    r = psd.Rows(FAKE, 32 * 128, 128)
    t = psd.Rotation(128, 0, 4096, FAKE, FAKE, None, FAKE, FAKE, 1e-6)
    for name, value in edit.items():
        which, field = name.split("__")
        setattr({"c": c, "s": s, "r": r, "t": t}[which], field, value)
    return c, s, r, t


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(psd, c, s, r, t, k="r", q="r", q_out="r", H=32):
    pick = lambda x: ref(r) if x == "r" else None  # noqa: E731
    return psd.lib().psd_kv_append(ref(c), ref(s), ref(t), pick(k), ref(r), pick(q), pick(q_out), H, None)


def attend(psd, c, s, r, t=None, H=32, scale=0.1, window=0, mask=None, words=0, q="r", ws=FAKE, n=1 << 40):
    return psd.lib().psd_attention(ref(c), ref(s), ref(r) if q == "r" else None, H, scale, window, mask, words, ref(r), None,
                                   ws, n, None)


def keep(psd, c, s, r=None, t=None, idx=FAKE, stride=5, width=5, n=FAKE, out=FAKE + 256):
    return psd.lib().psd_kv_keep(ref(c), ref(s), idx, stride, width, n, out, None)


CACHE_AND_SEQS = [("c__k", None), ("c__v", None), ("c__k", FAKE + 8), ("c__dtype", 2), ("c__dtype", -1), ("c__heads", 0),
                  ("c__heads", 1025), ("c__head_dim", 0), ("c__head_dim", 12), ("c__head_dim", 264), ("c__page_tokens", 0),
                  ("c__page_tokens", 65537), ("c__pages", 0), ("c__layers", 0), ("c__stride_page", 4), ("c__stride_token", -128),
                  ("c__stride_head", 129), ("s__batch", 0), ("s__batch", (1 << 19) + 1), ("s__rows", 0),
                  ("s__rows", (1 << 23) + 1), ("s__max_new", 0), ("s__max_kv", 0), ("s__max_kv", (1 << 30) + 1),
                  ("s__table_width", 0), ("s__table_stride", 255), ("s__new_start", None), ("s__kv_len", None), ("s__table", None)]


@pytest.mark.parametrize("field,value", CACHE_AND_SEQS)
def test_bad_cache_and_sequences(psd, field, value):
    parts = structs(psd, **{field: value})
    for call in (append, attend, keep):
        assert call(psd, *parts) == psd.PSD_E_ARG, call.__name__
        assert psd.lib().psd_last_error()


def test_null_structs(psd):
    c, s, r, t = structs(psd)
    for call in (append, attend, keep):
        assert call(psd, None, s, r, t) == psd.PSD_E_ARG
        assert call(psd, c, None, r, t) == psd.PSD_E_ARG
    assert append(psd, c, s, r, None) == psd.PSD_E_ARG


@pytest.mark.parametrize("field,value", [("t__rotary", -2), ("t__rotary", 3), ("t__rotary", 130), ("t__cos", None), ("t__sin", None),
                                         ("t__positions_max", 0), ("t__eps", -1.0), ("t__eps", NAN), ("t__eps", INF),
                                         ("t__q_norm", FAKE + 2), ("t__k_norm", FAKE + 8), ("r__data", None),
                                         ("r__data", FAKE + 4), ("r__stride_row", 100), ("r__stride_head", -8)])
def test_append_refusals(psd, field, value):
    assert append(psd, *structs(psd, **{field: value})) == psd.PSD_E_ARG


def test_append_queries(psd):
    parts = structs(psd)
    assert append(psd, *parts, k=None) == psd.PSD_E_ARG
    assert append(psd, *parts, q=None) == psd.PSD_E_ARG      # q_out without q
    assert append(psd, *parts, q_out=None) == psd.PSD_E_ARG
    for H in (0, 12, 2048, -8):
        assert append(psd, *parts, H=H) == psd.PSD_E_ARG


def test_attention_refusals(psd):
    parts = structs(psd)
    for bad in (dict(H=0), dict(H=12), dict(H=2048), dict(scale=NAN), dict(scale=INF), dict(window=-1), dict(mask=FAKE, words=0),
                dict(mask=FAKE, words=1, window=5), dict(q=None)):
        assert attend(psd, *parts, **bad) == psd.PSD_E_ARG, bad
    assert attend(psd, *structs(psd, r__stride_row=9)) == psd.PSD_E_ARG
    need = psd.lib().psd_attention_workspace_bytes(ref(parts[0]), ref(parts[1]), 32)
    assert need != ctypes.c_size_t(-1).value
    if need:
        for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
            assert attend(psd, *parts, **bad) == psd.PSD_E_WORKSPACE, bad


def test_attention_workspace_of_invalid_arguments(psd):
    for field, value in (("c__heads", 0), ("s__max_kv", 0), ("s__batch", 0)):
        c, s, r, t = structs(psd, **{field: value})
        assert psd.lib().psd_attention_workspace_bytes(ref(c), ref(s), 32) == ctypes.c_size_t(-1).value
        with pytest.raises(psd.PsdError):
            psd.attention_workspace_bytes(c, s, 32)
    c, s, r, t = structs(psd, c__k=None, s__table=None)  # sizing reads no pointer
    assert psd.attention_workspace_bytes(c, s, 32) >= 0


def test_keep_refusals(psd):
    parts = structs(psd)
    for bad in (dict(idx=None), dict(n=None), dict(width=0), dict(stride=4), dict(out=FAKE)):  # FAKE is kv_len itself
        assert keep(psd, *parts, **bad) == psd.PSD_E_ARG, bad
    assert keep(psd, *structs(psd, c__layers=2, c__stride_layer=3)) == psd.PSD_E_ARG


def given(psd, params, B=4, gamma=3, n=None, ws=FAKE, **null):
    p = {k: None if null.get(k) == "null" else FAKE for k in ("target", "draft", "tokens", "u", "e", "out", "len")}
    if n is None:
        n = psd.verify_given_workspace_bytes(params, B, gamma)
    return psd.lib().psd_verify_given(ctypes.byref(params), B, gamma, p["target"], p["draft"], p["tokens"], None, p["u"], p["e"],
                                      p["out"], p["len"], None, None, ws, n, None)


@pytest.mark.parametrize("field,value", [("vocab", 0), ("vocab", (1 << 19) + 1), ("num_drafts", 0), ("num_drafts", 2), ("top_k", 5),
                                         ("temp_target", 0.0), ("temp_draft", NAN), ("dtype", 3)])
def test_given_bad_params(psd, field, value):
    p = psd.make_params(0, 1000, 1, 0)
    setattr(p, field, value)
    assert given(psd, p, n=1 << 30) == psd.PSD_E_ARG
    assert psd.verify_given_workspace_bytes(p, 4, 3) == 0
    with pytest.raises(psd.PsdError):
        psd.new_verify_given_workspace(p, 4, 3, device="cpu")


def test_given_bad_arguments(psd):
    p = psd.make_params(0, 1000, 1, 0)
    for B, gamma in ((0, 3), (4, 0), (4, 33), (1 << 19, 32)):
        assert given(psd, p, B=B, gamma=gamma, n=1 << 40) == psd.PSD_E_ARG
        assert psd.verify_given_workspace_bytes(p, B, gamma) == 0
    for name in ("target", "draft", "tokens", "u", "e", "out", "len"):
        assert given(psd, p, **{name: "null"}) == psd.PSD_E_ARG, name
    assert given(psd, p, ws=None) == psd.PSD_E_WORKSPACE
    assert given(psd, p, ws=FAKE + 128) == psd.PSD_E_WORKSPACE
    assert given(psd, p, n=psd.verify_given_workspace_bytes(p, 4, 3) - 1) == psd.PSD_E_WORKSPACE


def test_binding_refuses_layouts(psd):
    """Shapes, types and strides that the pointers cannot say are refused by the binding."""
    k = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    cache = psd.make_cache(k, k.clone())
    assert (cache.pages, cache.page_tokens, cache.heads, cache.head_dim, cache.layers) == (4, 16, 2, 64, 1)
    five = torch.zeros((3, 4, 16, 2, 64), dtype=torch.float32)
    assert psd.make_cache(five, five.clone()).layers == 3
    start, kv, table = (torch.zeros(n, dtype=torch.int32) for n in ((3,), (2,), (2, 5)))
    seqs = psd.make_seqs(start, kv, table, 4, 2, 64)
    rows = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(psd.PsdError):
        psd.make_cache(k, k.transpose(1, 2))
    with pytest.raises(psd.PsdError):
        psd.make_cache(k.half(), k.half())
    with pytest.raises(psd.PsdError):
        psd.make_cache(k.transpose(2, 3), k.transpose(2, 3))
    for bad in (lambda: psd.make_seqs(start.long(), kv, table, 4, 2, 64), lambda: psd.make_seqs(start[:2], kv, table, 4, 2, 64),
                lambda: psd.make_seqs(start, kv, table.t(), 4, 2, 64)):
        with pytest.raises(psd.PsdError):
            bad()
    for bad in (dict(k=rows[:3]), dict(k=rows.float()), dict(k=rows[:, :1]), dict(v=rows[..., :32]), dict(q=rows.float()),
                dict(cos=torch.zeros((4, 32))), dict(cos=torch.zeros((4, 32)).half(), sin=torch.zeros((4, 32)).half()),
                dict(q_norm=torch.zeros(64)), dict(k_norm=torch.zeros(32, dtype=torch.bfloat16)),
                dict(positions=torch.zeros(3, dtype=torch.int32)), dict(positions=torch.zeros(4))):
        with pytest.raises(psd.PsdError):
            psd.kv_append(cache, seqs, **{**dict(k=rows, v=rows), **bad})
    for bad in (dict(q=rows.float()), dict(q=rows[:2]), dict(mask=torch.zeros((4, 1))), dict(mask=torch.zeros((2, 1), dtype=torch.int32)),
                dict(out=rows[:, :1])):
        with pytest.raises(psd.PsdError):
            psd.attention(cache, seqs, **{**dict(q=rows, ws=None), **bad})
    with pytest.raises(psd.PsdError):
        psd.kv_keep(cache, seqs, torch.zeros((2, 3)), kv)
    with pytest.raises(psd.PsdError):
        psd.kv_keep(cache, seqs, torch.zeros((3, 3), dtype=torch.int32), kv)
