"""Places for a call's tokens against the plain definition (GPU)."""
import os
import random
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import serving4_ref as ref4  # noqa: E402


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """The same sequences in the plain form and on the device."""

    def __init__(self, psd, B, pages, P, width, rows, max_new, max_kv, seed=0, stride=0):
        order = list(range(pages))
        random.Random(seed).shuffle(order)
        first = seed * 7 % pages
        self.plain = ref4.Pool(pages, P, B, width, order, first)
        self.psd, self.B, self.rows, self.max_new, self.max_kv = psd, B, rows, max_new, max_kv
        self.pages = psd.make_pages(ints(self.plain.ring), ints([first, pages, 0, 0]), P)
        wide = torch.full((B, stride or width), -1, dtype=torch.int32, device="cuda")
        self.table = wide[:, :width]
        self.start, self.kv, self.held = ints([7] * (B + 1)), ints([7] * B), ints([0] * B)
        self.seqs = psd.make_seqs(self.start, self.kv, self.table, rows, max_new, max_kv)

    def call(self, n_new, have, **kw):
        o = self.psd.kv_reserve(self.pages, self.seqs, ints(n_new), ints(have), self.held, **kw)
        torch.cuda.synchronize()
        self.check(o, n_new, have)
        return o

    def check(self, o, n_new, have):
        granted, start, kv, seq, pos, slot = self.plain.reserve(n_new, have, self.rows, self.max_new, self.max_kv)
        assert o["granted"].tolist() == granted
        assert self.start.tolist() == start and self.kv.tolist() == kv
        if "slots" in o:
            assert o["row_seq"].tolist() == seq and o["positions"].tolist() == pos and o["slots"].tolist() == slot
        assert self.held.tolist() == self.plain.held
        assert self.table.tolist() == self.plain.table
        ring, state = (t.tolist() for t in self.pages.tensors)
        assert state == [self.plain.first, len(self.plain.free), 0, 0]
        n = len(ring)
        assert [ring[(state[0] + i) % n] for i in range(state[1])] == self.plain.free
        # every page is free or held, once
        pages = self.plain.free + [p for row in self.plain.table for p in row if p >= 0]
        assert sorted(pages) == list(range(n))


@pytest.mark.parametrize("B,pages,P,width,rows,max_new,max_kv", [
    (1, 5, 16, 4, 64, 64, 64), (7, 40, 16, 9, 300, 100, 140), (64, 300, 8, 12, 600, 40, 96), (3, 20, 1, 12, 30, 12, 12),
    (600, 900, 24, 5, 3000, 60, 110), (1500, 4000, 100, 3, 20000, 250, 300), (33, 100, 7, 30, 4000, 200, 200)])
def test_serving_steps(psd, B, pages, P, width, rows, max_new, max_kv):
    """Sequences that start, grow, shrink after a block, wait for pages or rows, and end."""
    rng = random.Random(B * 100 + P)
    both = Both(psd, B, pages, P, width, rows, max_new, max_kv, seed=B, stride=width + 3)
    have = [0] * B
    for step in range(8):
        print("[reserve]", B, pages, P, step, flush=True)
        many = rng.random() < 0.5
        n_new = [rng.choice([0, 1, 5, rng.randint(0, max_new + 2), -3]) if many or rng.random() < 0.3 else 1 for _ in range(B)]
        both.call(n_new, have, rows_out=step != 5)
        kv = both.kv.tolist()
        # what stays: everything, a part of the block, or nothing (the request has ended)
        have = [rng.choice([kv[b], kv[b], rng.randint(min(have[b], kv[b]), kv[b]), 0]) for b in range(B)]


def test_nothing_asked_and_everything_refused(psd):
    both = Both(psd, 5, 6, 16, 4, 20, 32, 64)
    both.call([0] * 5, [0] * 5)
    both.call([33, 65, 20, 1, 0], [0] * 5)       # too long, too long, all rows, none left
    both.call([1, 1, 1, 1, 1], [0, 0, 20, 0, 0])
    both.call([16, 0, 1, 1, 1], [1, 1, 20, 1, 1])  # the first takes the last page


def test_a_sequence_without_pages_holds_back_those_behind_it(psd):
    both = Both(psd, 4, 5, 16, 8, 200, 100, 128)
    o = both.call([16, 80, 16, 0], [0] * 4)
    assert o["granted"].tolist() == [16, 0, 0, 0]
    o = both.call([1, 64, 0, 0], [15, 0, 0, 0])  # the first needs none
    assert o["granted"].tolist() == [1, 64, 0, 0]
    o = both.call([0, 0, 40, 0], [16, 0, 0, 0])  # pages that come back serve the next call
    assert o["granted"].tolist() == [0, 0, 0, 0]
    o = both.call([0, 0, 40, 0], [16, 0, 0, 0])
    assert o["granted"].tolist() == [0, 0, 40, 0]


def test_lengths_outside_their_bounds(psd):
    """A kv_have below 0 counts as 0, one above the table as what the table holds; counters nobody left are cut."""
    both = Both(psd, 3, 30, 16, 4, 100, 64, 1000)
    both.call([10, 10, 60], [-5, 0, 0])
    both.call([1, 0, 5], [9, 4, 5000])
    o = psd.kv_reserve(psd.make_pages(ints([3, 1, 2]), ints([99, 99, 0, 0]), 16), both.seqs, ints([5, 0, 0]), ints([0, 0, 0]),
                       ints([0, 0, 0]))
    torch.cuda.synchronize()
    assert o["granted"].tolist() == [5, 0, 0] and 0 <= int(both.table[0, 0]) < 4


def test_captured_and_replayed_on_another_stream(psd):
    """One graph of reserve and trim, replayed with other requests: the plain form's pages each time."""
    B, P = 20, 16
    both = Both(psd, B, 200, P, 20, 2600, 130, 320, seed=3)
    n_new, have, none = ints([0] * B), ints([0] * B), ints([0] * B)
    out = {}

    def step():
        out.update(psd.kv_reserve(both.pages, both.seqs, n_new, have, both.held))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    both.check(out, [0] * B, [0] * B)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = random.Random(1)
    h = [0] * B
    for i in range(6):
        n = [rng.randint(0, 130) for _ in range(B)]
        n_new.copy_(ints(n))
        have.copy_(ints(h))
        graph.replay()
        torch.cuda.synchronize()
        both.check(out, n, h)
        h = [rng.randint(0, x) for x in both.kv.tolist()]
    assert none.tolist() == [0] * B


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "graph"])
def test_reserve_and_trim_back_to_back_on_another_stream(psd, captured):
    """A reservation and the trim of what does not stay, on one ring and table with nothing of the host in between, several
    workgroups each; as a graph replayed on a stream of its own.  Both calls are the plain form's every time."""
    B, P, width, rows = 200, 16, 20, 20000
    order = list(range(1500))
    random.Random(8).shuffle(order)
    plain = ref4.Pool(1500, P, B, width, order, 700)
    pages = psd.make_pages(ints(plain.ring), ints([700, 1500, 0, 0]), P)
    table, held = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), ints([0] * B)
    (start, kv), (start2, kv2) = ((ints([7] * (B + 1)), ints([7] * B)) for _ in range(2))
    seqs, after = psd.make_seqs(start, kv, table, rows, 130, 320), psd.make_seqs(start2, kv2, table, rows, 130, 320)
    n_new, have, stay, kept, none = (ints([0] * B) for _ in range(5))
    out, trimmed = {}, {}

    def step():
        out.update(psd.kv_reserve(pages, seqs, n_new, have, held, out=out))
        torch.minimum(kv, stay, out=kept)
        trimmed.update(psd.kv_reserve(pages, after, none, kept, held, out=trimmed))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()  # (nothing asked)
    torch.cuda.synchronize()
    plain.reserve([0] * B, [0] * B, rows, 130, 320)
    graph = torch.cuda.CUDAGraph()
    if captured:
        with torch.cuda.graph(graph):
            step()
    rng = random.Random(5)
    h = [0] * B
    for i in range(8):
        n = [rng.randint(0, 130) for _ in range(B)]
        st = [rng.choice([0, x + rng.randint(0, 130), 400]) for x in h]
        for t, x in ((n_new, n), (have, h), (stay, st)):
            t.copy_(ints(x))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay() if captured else step()
        torch.cuda.synchronize()
        granted, first, lens, seq, pos, slot = plain.reserve(n, h, rows, 130, 320)
        assert out["granted"].tolist() == granted and start.tolist() == first and kv.tolist() == lens
        assert out["row_seq"].tolist() == seq and out["positions"].tolist() == pos and out["slots"].tolist() == slot
        h = [min(a, b) for a, b in zip(lens, st)]
        assert kept.tolist() == h
        granted, first, lens, seq, pos, slot = plain.reserve([0] * B, h, rows, 130, 320)
        assert trimmed["granted"].tolist() == granted == [0] * B and start2.tolist() == first and kv2.tolist() == lens == h
        assert held.tolist() == plain.held and table.tolist() == plain.table
        ring, state = (t.tolist() for t in pages.tensors)
        assert state == [plain.first, len(plain.free), 0, 0]
        assert [ring[(state[0] + j) % 1500] for j in range(state[1])] == plain.free
