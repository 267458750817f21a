"""Refusals of the operators over a cache held in 4 bits, of the reservation and of the adjusted logits: every invalid
argument returns its status before anything is launched (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

FAKE = 1 << 20  # a non-NULL, 256-aligned dummy address: never dereferenced by rejected calls
STEP = 1 << 16  # between dummy arrays
NAN, INF = float("nan"), float("inf")
NEW = ("psd_kv_append4", "psd_attention4", "psd_attention4_workspace_bytes", "psd_kv_keep4", "psd_kv_reserve", "psd_adjust_logits")


@pytest.fixture(scope="module")
def psd():
    from paper_2609_21858_amd import psd as m
    return m


def test_exports(psd):
    for name in NEW:
        assert hasattr(psd.lib(), name) and name in psd.EXPORTS


def structs(psd, **edit):
    c = psd.Cache4(FAKE, FAKE, FAKE, FAKE, psd.PSD_BF16, 8, 128, 16, 100, 1, 0, 16 * 8 * 64, 64, 16 * 64, 0, 16 * 8 * 4, 4, 16 * 4)
    s = psd.Seqs(4, 20, 5, 4096, 256, 256, FAKE, FAKE, FAKE)
    r = psd.Rows(FAKE, 32 * 128, 128)
    t = psd.Rotation(128, 0, 4096, FAKE, FAKE, None, FAKE, FAKE, 1e-6)
    for name, value in edit.items():
        which, field = name.split("__")
        setattr({"c": c, "s": s, "r": r, "t": t}[which], field, value)
    return c, s, r, t


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(psd, c, s, r, t, k="r", q="r", q_out="r", H=32, held=None):
    pick = lambda x: ref(r) if x == "r" else None  # noqa: E731
    return psd.lib().psd_kv_append4(ref(c), ref(s), ref(t), pick(k), ref(r), pick(q), pick(q_out), H, ref(held), None, None)


def attend(psd, c, s, r, t=None, H=32, scale=0.1, window=0, mask=None, words=0, q="r", ws=FAKE, n=1 << 40):
    return psd.lib().psd_attention4(ref(c), ref(s), ref(r) if q == "r" else None, H, scale, window, mask, words, ref(r), None,
                                    ws, n, None)


def keep(psd, c, s, r=None, t=None, idx=FAKE, stride=5, width=5, n=FAKE, out=FAKE + STEP):
    return psd.lib().psd_kv_keep4(ref(c), ref(s), idx, stride, width, n, out, None)


CACHE_AND_SEQS = [("c__k", None), ("c__v", None), ("c__k_scale", None), ("c__v_scale", None), ("c__k", FAKE + 8), ("c__dtype", 2),
                  ("c__heads", 0), ("c__heads", 1025), ("c__head_dim", 0), ("c__head_dim", 12), ("c__head_dim", 264),
                  ("c__page_tokens", 0), ("c__page_tokens", 65537), ("c__pages", 0), ("c__layers", 0), ("c__stride_page", 8),
                  ("c__stride_token", -64), ("c__stride_head", 72), ("c__scale_page", -1), ("c__scale_token", 1 << 44),
                  ("c__scale_head", -4), ("s__batch", 0), ("s__batch", (1 << 19) + 1), ("s__rows", 0), ("s__rows", (1 << 23) + 1),
                  ("s__max_new", 0), ("s__max_kv", 0), ("s__max_kv", (1 << 30) + 1), ("s__table_width", 0), ("s__table_stride", 255),
                  ("s__new_start", None), ("s__kv_len", None), ("s__table", None)]


@pytest.mark.parametrize("field,value", CACHE_AND_SEQS)
def test_bad_cache_and_sequences(psd, field, value):
    parts = structs(psd, **{field: value})
    for call in (append, attend, keep):
        assert call(psd, *parts) == psd.PSD_E_ARG, call.__name__
        assert psd.lib().psd_last_error()


def test_layers(psd):
    for field, value in (("c__stride_layer", 24), ("c__scale_layer", -1)):
        assert keep(psd, *structs(psd, c__layers=2, **{field: value})) == psd.PSD_E_ARG


def test_null_structs(psd):
    c, s, r, t = structs(psd)
    for call in (append, attend, keep):
        assert call(psd, None, s, r, t) == psd.PSD_E_ARG
        assert call(psd, c, None, r, t) == psd.PSD_E_ARG
    assert append(psd, c, s, r, None) == psd.PSD_E_ARG


@pytest.mark.parametrize("field,value", [("t__rotary", -2), ("t__rotary", 3), ("t__rotary", 130), ("t__cos", None),
                                         ("t__positions_max", 0), ("t__eps", -1.0), ("t__eps", NAN), ("t__q_norm", FAKE + 2),
                                         ("r__data", None), ("r__data", FAKE + 4), ("r__stride_row", 100), ("r__stride_head", -8)])
def test_append_refusals(psd, field, value):
    assert append(psd, *structs(psd, **{field: value})) == psd.PSD_E_ARG


def test_append_rows(psd):
    parts = structs(psd)
    for bad in (dict(k=None), dict(q=None), dict(q_out=None), dict(H=12), dict(H=0), dict(held=psd.Rows(None, 1024, 128)),
                dict(held=psd.Rows(FAKE + 2, 1024, 128)), dict(held=psd.Rows(FAKE, 1023, 128))):
        assert append(psd, *parts, **bad) == psd.PSD_E_ARG, bad


def test_attention_refusals(psd):
    parts = structs(psd)
    for bad in (dict(H=0), dict(H=12), dict(H=2048), dict(scale=NAN), dict(scale=INF), dict(window=-1), dict(mask=FAKE, words=0),
                dict(mask=FAKE, words=1, window=5), dict(q=None)):
        assert attend(psd, *parts, **bad) == psd.PSD_E_ARG, bad
    need = psd.lib().psd_attention4_workspace_bytes(ref(parts[0]), ref(parts[1]), 32)
    assert 0 < need < 1 << 30
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
        assert attend(psd, *parts, **bad) == psd.PSD_E_WORKSPACE, bad
    for field, value in (("c__heads", 0), ("s__max_kv", 0), ("c__scale_page", -1)):
        c, s, _, _ = structs(psd, **{field: value})
        with pytest.raises(psd.PsdError):
            psd.attention_workspace_bytes(c, s, 32)
    c, s, _, _ = structs(psd, c__k=None, c__k_scale=None, s__table=None)  # sizing reads no pointer
    assert psd.attention_workspace_bytes(c, s, 32) == need


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("H,G,D", [(128, 1, 128), (32, 8, 128), (8, 8, 64), (64, 8, 256), (1024, 1024, 8)])
def test_workspace_of_far_bounds(psd, H, G, D, dtype):
    """No sequence has more new tokens than the call has rows, and the slots of all workgroups fit what is asked for."""
    want = None
    for most in (20, 21, 1 << 20, (1 << 31) - 1):
        c, s, _, _ = structs(psd, c__heads=G, c__head_dim=D, c__dtype=dtype, s__max_new=most, s__max_kv=1 << 20)
        n = psd.attention_workspace_bytes(c, s, H)
        assert want is None or n == want, most
        want = n


def test_keep_refusals(psd):
    parts = structs(psd)
    for bad in (dict(idx=None), dict(n=None), dict(width=0), dict(stride=4), dict(out=FAKE), dict(out=FAKE + 8)):
        assert keep(psd, *parts, **bad) == psd.PSD_E_ARG, bad


# ---------------------------------------------------------------- reservation

ARRAYS = ("n_new", "kv_have", "held", "table", "new_start", "kv_len", "granted", "row_seq", "positions", "slots")


def reserve(psd, pages=None, seqs=None, null=(), **edit):
    p = psd.Pages(16, 100, FAKE, FAKE + STEP)
    s = psd.Seqs(4, 20, 5, 4096, 256, 256, None, None, None)
    r = psd.Reservation(*(FAKE + (2 + i) * STEP for i in range(len(ARRAYS))))
    for name in null:
        setattr(r, name, None)
    for name, value in edit.items():
        which, field = name.split("__")
        setattr({"p": p, "s": s, "r": r}[which], field, value)
    pick = {"pages": p, "seqs": s, "r": r}
    if pages == "none":
        pick["pages"] = None
    if seqs == "none":
        pick["seqs"] = None
    return psd.lib().psd_kv_reserve(ref(pick["pages"]), ref(pick["seqs"]), ref(pick["r"]), None)


@pytest.mark.parametrize("field,value", [("p__page_tokens", 0), ("p__page_tokens", 65537), ("p__pages", 0), ("p__ring", None),
                                         ("p__state", None), ("s__batch", 0), ("s__rows", 0), ("s__max_new", 0), ("s__max_kv", 0),
                                         ("s__table_width", 0), ("s__table_stride", 255), ("r__slots", FAKE + 40 * STEP + 4)])
def test_reserve_refusals(psd, field, value):
    assert reserve(psd, **{field: value}) == psd.PSD_E_ARG
    assert psd.lib().psd_last_error()


def test_reserve_null(psd):
    assert reserve(psd, pages="none") == psd.PSD_E_ARG
    assert reserve(psd, seqs="none") == psd.PSD_E_ARG
    for name in ARRAYS[:6]:
        assert reserve(psd, null=(name,)) == psd.PSD_E_ARG, name


def test_reserve_shares_no_memory(psd):
    """What one workgroup writes while others read, or write besides, is in no other array."""
    at = {name: FAKE + (2 + i) * STEP for i, name in enumerate(ARRAYS)}
    for out in ARRAYS[2:]:
        for other in ARRAYS:
            if other != out:
                value = at[other] if out == "slots" else at[other] + 4
                assert reserve(psd, **{"r__" + out: value}) == psd.PSD_E_ARG, (out, other)
        assert reserve(psd, **{"r__" + out: FAKE}) == psd.PSD_E_ARG            # the ring
        assert reserve(psd, **{"r__" + out: FAKE + STEP + 8}) == psd.PSD_E_ARG  # the state
    assert reserve(psd, p__state=FAKE + 4 * 99) == psd.PSD_E_ARG


# ---------------------------------------------------------------- adjusted logits

def adjust(psd, params, B=4, rows=5, depth0=0, logits=FAKE, out=1 << 32, none=False, **edit):
    a = psd.Adjustments(FAKE, 100, 100, FAKE, None, FAKE, 4, FAKE, FAKE, FAKE, FAKE, FAKE, 8, FAKE, 32, 0)
    for name, value in edit.items():
        setattr(a, name, value)
    return psd.lib().psd_adjust_logits(ctypes.byref(params), None if none else ctypes.byref(a), B, rows, depth0, logits, out, None)


@pytest.mark.parametrize("bad", [dict(B=0), dict(B=(1 << 19) + 1), dict(rows=0), dict(rows=34), dict(rows=6), dict(depth0=-1),
                                 dict(depth0=1), dict(logits=None), dict(out=None), dict(none=True), dict(length=None), dict(text_max=-1),
                                 dict(text_max=1 << 20, text_stride=1 << 20), dict(text_stride=99), dict(gamma=0), dict(gamma=33),
                                 dict(bias_width=-1), dict(bias_width=1025), dict(bias=None), dict(bias_tokens=None),
                                 dict(allowed_seq=-1), dict(allowed_row=-1), dict(logits=FAKE + 1), dict(out=FAKE + 2),
                                 dict(out=FAKE + 4 * 5 * 1000 * 2 - 2), dict(B=1 << 19, rows=33, gamma=32)])
def test_adjust_refusals(psd, bad):
    assert adjust(psd, psd.make_params(0, 1000, 1, 0), **bad) == psd.PSD_E_ARG
    assert psd.lib().psd_last_error()


@pytest.mark.parametrize("field,value", [("vocab", 0), ("vocab", (1 << 19) + 1), ("num_drafts", 0), ("num_drafts", 33), ("dtype", 3)])
def test_adjust_bad_params(psd, field, value):
    p = psd.make_params(0, 1000, 1, 0)
    setattr(p, field, value)
    assert adjust(psd, p) == psd.PSD_E_ARG


# ---------------------------------------------------------------- the binding

def test_binding_of_caches(psd):
    k, s = torch.zeros((4, 16, 2, 48), dtype=torch.uint8), torch.zeros((4, 16, 2, 3), dtype=torch.uint8)
    c = psd.make_cache4(k, k.clone(), s, s.clone(), 80)
    assert (c.pages, c.page_tokens, c.heads, c.head_dim, c.layers, c.dtype) == (4, 16, 2, 80, 1, psd.PSD_BF16)
    assert (c.stride_page, c.stride_token, c.stride_head) == (16 * 2 * 48, 96, 48) and (c.scale_page, c.scale_token, c.scale_head) == (96, 6, 3)
    for bad in ((k, k.transpose(1, 2), s, s, 80), (k, k, s, s, 64), (k, k, s, s, 128), (k.int(), k.int(), s, s, 80), (k, k, s[:3], s[:3], 80),
                (k[0], k[0], s[0], s[0], 80), (k[..., ::2], k[..., ::2], s, s, 40), (k, k, s.float(), s.float(), 80)):
        with pytest.raises(psd.PsdError) as e:
            psd.make_cache4(*bad)
        assert e.value.status == psd.PSD_E_ARG
    with pytest.raises(psd.PsdError):
        psd.make_cache4(k, k, s, s, 80, dtype=torch.float16)
    new = psd.new_cache4(5, 16, 2, 80, layers=3, dtype=torch.float32, device="cpu")
    assert new.layers == 3 and new.stride_token == 48 and new.stride_head == 16 * 48 and new.scale_token == 3
    one = psd.cache4_layer(new, 2)
    assert one.layers == 1 and one.k == new.k + 2 * new.stride_layer and one.v_scale == new.v_scale + 2 * new.scale_layer
    assert one.dtype == psd.PSD_F32
    for bad in ((new, 3), (new, -1), (c, 0)):
        with pytest.raises(psd.PsdError):
            psd.cache4_layer(*bad)


def test_binding_of_rows(psd):
    cache = psd.new_cache4(4, 16, 2, 64, device="cpu")
    start, kv, table = (torch.zeros(n, dtype=torch.int32) for n in ((3,), (2,), (2, 5)))
    seqs = psd.make_seqs(start, kv, table, 4, 2, 64)
    rows = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    for bad in (dict(k=rows[:3]), dict(k=rows.float()), dict(v=rows[..., :32]), dict(q=rows.float()), dict(k_held=rows[:2]),
                dict(v_held=rows.float())):
        with pytest.raises(psd.PsdError):
            psd.kv_append(cache, seqs, **{**dict(k=rows, v=rows), **bad})
    with pytest.raises(psd.PsdError):  # a cache in 16 bits holds what it is given
        k = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
        psd.kv_append(psd.make_cache(k, k.clone()), seqs, rows, rows, k_held=rows)
    for bad in (dict(q=rows.float()), dict(q=rows[:2]), dict(out=rows[:, :1])):
        with pytest.raises(psd.PsdError):
            psd.attention(cache, seqs, **{**dict(q=rows, ws=None), **bad})


def test_binding_of_reservations(psd):
    pages = psd.new_pages(10, 16, device="cpu")
    assert pages.tensors[0].tolist() == list(range(10)) and pages.tensors[1].tolist() == [0, 10, 0, 0]
    ints = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    for bad in ((ints(10).long(), ints(4)), (ints(10), ints(3)), (ints(10), ints(4).float())):
        with pytest.raises(psd.PsdError):
            psd.make_pages(*bad, 16)
    seqs = psd.make_seqs(ints(3), ints(2), ints(2, 5), 4, 2, 64)
    good = dict(n_new=ints(2), kv_have=ints(2), held=ints(2))
    for bad in (dict(n_new=ints(3)), dict(kv_have=ints(2).long()), dict(held=ints(4)[::2]), dict(granted=ints(3)),
                dict(out={"slots": ints(4)}), dict(out={"row_seq": ints(5)}), dict(out={"positions": ints(8)[::2]})):
        with pytest.raises(psd.PsdError):
            psd.kv_reserve(pages, seqs, **{**good, **bad})


def test_binding_of_adjustments(psd):
    p = psd.make_params(0, 100, 2, 0)
    z = torch.zeros((3, 2, 4, 100), dtype=torch.bfloat16)
    ints = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    text = dict(text=ints(3, 9), length=torch.zeros(3, dtype=torch.int64))
    for bad in (dict(logits=z.float()), dict(logits=z[:, :1]), dict(logits=z[..., :99]), dict(logits=z.transpose(1, 2)), dict(logits=z[:, 0]),
                dict(out=z.float()), dict(out=z[:2]), dict(text=ints(3, 9)), dict(text, length=torch.zeros(3)), dict(text, text=ints(2, 9)),
                dict(text, text=ints(1, 9).expand(3, 9)), dict(text, text_from=ints(3)), dict(draft_tokens=ints(3, 4)),
                dict(draft_tokens=ints(3, 2, 3).long()), dict(draft_tokens=ints(3, 2, 6)[..., ::2]), dict(repetition=torch.zeros(2)),
                dict(presence=torch.zeros(3).double()), dict(frequency=torch.zeros((3, 1))), dict(bias_tokens=ints(3, 5)),
                dict(bias_tokens=ints(3, 5), bias=torch.zeros((3, 4))), dict(bias_tokens=ints(3, 5), bias=torch.zeros((3, 5)).double()),
                dict(allowed=ints(3, 3)), dict(allowed=ints(3, 2, 4, 3)), dict(allowed=ints(3, 2, 3, 4)), dict(allowed=ints(3, 4).long())):
        with pytest.raises(psd.PsdError) as e:
            psd.adjust_logits(p, **{**dict(logits=z), **bad})
        assert e.value.status == psd.PSD_E_ARG, sorted(bad)


def test_binding_of_host_memory(psd):
    """Tensors in host memory, which would fault the GPU, are refused by every call."""
    ints = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    cache = psd.new_cache4(4, 16, 2, 64, device="cpu")
    seqs = psd.make_seqs(ints(3), ints(2), ints(2, 5), 4, 2, 64)
    rows = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    z = torch.zeros((2, 1, 3, 50))
    for call in (lambda: psd.kv_append(cache, seqs, rows, rows), lambda: psd.attention(cache, seqs, rows, None),
                 lambda: psd.kv_keep(cache, seqs, ints(2, 3), ints(2)),
                 lambda: psd.kv_reserve(psd.new_pages(4, 16, device="cpu"), seqs, ints(2), ints(2), ints(2)),
                 lambda: psd.adjust_logits(psd.make_params(0, 50, 1, 0, dtype=torch.float32), z)):
        with pytest.raises(psd.PsdError) as e:
            call()
        assert "host memory" in str(e.value)
