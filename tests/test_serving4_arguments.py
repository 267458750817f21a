"""The device of every tensor that a call over a cache held in 4 bits, a reservation or an adjustment of logits is given (no
GPU): tensors in host memory say that they are on a device, and the library only records the calls."""
import pytest

torch = pytest.importorskip("torch")

BF16 = torch.bfloat16


class On0(torch.Tensor):
    def get_device(self):
        return 0


class On1(torch.Tensor):
    def get_device(self):
        return 1


class Calls:
    """Stands for the library: records the calls, launches nothing."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        if not name.startswith("psd_"):
            raise AttributeError(name)
        return lambda *args: self.seen.append(name) or 0


@pytest.fixture
def calls(psd, monkeypatch):
    c = Calls()
    monkeypatch.setattr(psd, "_lib", c)
    monkeypatch.setattr(psd, "_stream", lambda stream=None: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return c


@pytest.fixture(scope="module")
def psd():
    from paper_2609_21858_amd import psd as m
    return m


def ints(*n):
    return torch.zeros(n, dtype=torch.int32)


# what each call is given: structures by their tensors, and its own tensors, the main one first
CACHE = dict(k=(4, 16, 2, 32), v=(4, 16, 2, 32), k_scale=(4, 16, 2, 2), v_scale=(4, 16, 2, 2))
CACHE = {n: torch.zeros(s, dtype=torch.uint8) for n, s in CACHE.items()}
SEQS = dict(new_start=ints(3), kv_len=ints(2), table=ints(2, 5))
PAGES = dict(ring=ints(10), state=ints(4))
ROWS = torch.zeros((4, 2, 64), dtype=BF16)
TURN = torch.zeros((9, 32))

OWN = {
    "kv_append": dict(k=ROWS, v=ROWS, q=ROWS, q_out=ROWS, cos=TURN, sin=TURN, positions=ints(4), q_norm=ROWS[0, 0], k_norm=ROWS[0, 0],
                      k_held=ROWS, v_held=ROWS),
    "attention": dict(q=ROWS, ws=torch.zeros(256, dtype=torch.uint8), mask=ints(4, 1), out=ROWS, lse=torch.zeros((4, 2))),
    "kv_keep": dict(keep=ints(2, 3), n_keep=ints(2), kv_out=ints(2)),
    "kv_reserve": dict(n_new=ints(2), kv_have=ints(2), held=ints(2), granted=ints(2), row_seq=ints(4), positions=ints(4),
                       slots=torch.zeros(4, dtype=torch.int64)),
    "adjust_logits": dict(logits=torch.zeros((3, 2, 4, 100)), out=torch.zeros((3, 2, 4, 100)), text=ints(3, 9),
                          length=torch.zeros(3, dtype=torch.int64), text_from=torch.zeros(3, dtype=torch.int64), draft_tokens=ints(3, 2, 3),
                          repetition=torch.ones(3), presence=torch.ones(3), frequency=torch.ones(3), bias_tokens=ints(3, 5),
                          bias=torch.ones((3, 5)), allowed=ints(3, 4)),
}
STRUCTS = {"kv_append": (CACHE, SEQS), "attention": (CACHE, SEQS), "kv_keep": (CACHE, SEQS), "kv_reserve": (PAGES, SEQS), "adjust_logits": ()}


def run(psd, name, elsewhere=None, kind=torch.Tensor):
    """The call with all tensors on device 0, but for the one named `elsewhere`."""
    def on(tensors):
        return {n: t.clone().as_subclass(kind if n == elsewhere else On0) for n, t in tensors.items()}

    made = []
    for s in STRUCTS[name]:
        t = on(s)
        made.append(psd.make_cache4(**t, head_dim=64) if s is CACHE else psd.make_seqs(**t, rows=4, max_new=2, max_kv=64) if s is SEQS
                    else psd.make_pages(**t, page_tokens=16))
    own = on(OWN[name])
    if name == "attention":
        own["want_lse"] = True
    if name == "kv_reserve":
        own["out"] = {n: own.pop(n) for n in ("row_seq", "positions", "slots")}
    if name == "adjust_logits":
        made.append(psd.make_params(0, 100, 2, 0, dtype=torch.float32))
    return getattr(psd, name)(*made, **own)


@pytest.mark.parametrize("name", list(OWN))
def test_tensors_on_one_device_are_taken(psd, calls, name):
    run(psd, name)
    assert len(calls.seen) == 1


@pytest.mark.parametrize("kind", [torch.Tensor, On1], ids=["host", "other"])
@pytest.mark.parametrize("name,tensor", [(n, t) for n in OWN for t in [*OWN[n], *(x for s in STRUCTS[n] for x in s)]])
def test_a_tensor_elsewhere_is_refused(psd, calls, name, tensor, kind):
    with pytest.raises(psd.PsdError) as e:
        run(psd, name, tensor, kind)
    assert e.value.status == psd.PSD_E_ARG and not calls.seen


def test_structures_without_their_make_function(psd, calls):
    """They hold addresses alone: nothing to compare."""
    keep, n_keep, kv_out = (t.as_subclass(On0) for t in (ints(2, 3), ints(2), ints(2)))
    cache = psd.Cache4(256, 256, 256, 256, psd.PSD_BF16, 2, 64, 16, 4, 1, 0, 1024, 64, 32, 0, 64, 4, 2)
    psd.kv_keep(cache, psd.Seqs(2, 4, 2, 64, 5, 5, 256, 256, 256), keep, n_keep, kv_out)
    assert calls.seen == ["psd_kv_keep4"]


def test_no_sequences_with_masks(psd):
    """A batch of nothing is refused as any other bad batch, whatever its masks."""
    with pytest.raises(psd.PsdError) as e:
        psd.adjust_logits(psd.make_params(0, 100, 2, 0, dtype=torch.float32), torch.zeros((0, 2, 4, 100)), allowed=ints(0, 2, 4, 4))
    assert e.value.status == psd.PSD_E_ARG
