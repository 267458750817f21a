"""Steps of a server as they are run together: reserve, append, attend, adjust, verify, keep, over a cache held in 4 bits, each
against its plain implementation on the state that the others left (GPU); and the example's loop."""
import math
import os
import random
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "examples"))
sys.path.insert(0, os.path.join(ROOT, "tests"))

import serving4_ref as ref4  # noqa: E402
import serving_ref as ref  # noqa: E402
from test_gpu_serving import BF16, F32, HALF, ULP  # noqa: E402
from test_gpu_serving4 import attention_bounds  # noqa: E402


@pytest.fixture(scope="module")
def block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import speculative_block as m
    return m


class State:
    """What ref.attention reads, of the pools as they are."""

    def __init__(self, pools, table, start, kv, G, D, P):
        kc, vc, ks, vs = (p.cpu() for p in pools)
        self.k, self.v = ref4.decode(kc, ks, D), ref4.decode(vc, vs, D)
        self.table, self.new_start, self.G, self.D, self.P = table.cpu(), start, G, D, P
        self.lens = [(start[b + 1] - start[b], kv[b]) for b in range(len(kv))]
        self.B = len(kv)

    place = ref.Sequences.place


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_serving_steps(block, dtype):
    psd = block.psd
    B, H, G, D, P, V, gamma, width, blocks = 6, 4, 2, 80, 8, 900, 3, 12, 5
    rng, g = random.Random(4), torch.Generator().manual_seed(4)
    cache = psd.new_cache4(40, P, G, D, dtype=dtype)  # fewer pages than all of them want
    pages, plain = psd.new_pages(40, P), ref4.Pool(40, P, B, width)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    start, kv, held = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, B, B))
    rows, max_new = B * 30, 30
    seqs = psd.make_seqs(start, kv, table, rows, max_new, width * P)
    ws = psd.new_attention_workspace(cache, seqs, H)
    params = psd.make_params(0, V, 1, 0, 0.9, 1.1, dtype=dtype)
    vws = psd.new_verify_given_workspace(params, B, gamma)
    text = torch.randint(0, V, (B, 100), generator=g, dtype=torch.int32)
    have = [0] * B
    for step in range(blocks):
        print("[step]", step, dtype, flush=True)
        # a prompt of its own length first, then the root and its drafts; a sequence ends now and then
        have = [0 if rng.random() < 0.1 else h for h in have]
        n_new = [gamma + 1 if h else rng.randint(gamma + 1, max_new) for h in have]
        o = psd.kv_reserve(pages, seqs, torch.tensor(n_new, dtype=torch.int32, device="cuda"),
                           torch.tensor(have, dtype=torch.int32, device="cuda"), held)
        torch.cuda.synchronize()
        granted, first, lens, seq, pos, slot = plain.reserve(n_new, have, rows, max_new, width * P)
        assert o["granted"].tolist() == granted and start.tolist() == first and kv.tolist() == lens and o["slots"].tolist() == slot
        assert o["positions"].tolist() == pos and o["row_seq"].tolist() == seq and table.tolist() == plain.table
        T = first[-1]
        q, k, v = ((torch.randn((rows, n, D), generator=g) * (1 + step)).to(dtype) for n in (H, G, G))
        psd.kv_append(cache, seqs, k.cuda(), v.cuda())
        torch.cuda.synchronize()
        pools = [cache.tensors[i] for i in (0, 1, 2, 3)]
        for t in range(T):  # each token's codes are where its slot says
            page, place = divmod(slot[t], P)
            for j, x in ((0, k), (1, v)):
                codes, scales = ref4.encode(x[t].double())
                assert torch.equal(pools[j][page, place].cpu(), codes) and torch.equal(pools[2 + j][page, place].cpu(), scales)
        a = psd.attention(cache, seqs, q.cuda(), ws, want_lse=True)
        torch.cuda.synchronize()
        s = State(pools, table, first, lens, G, D, P)
        want, lse, spread, size, vmax = ref.attention(s, q, D ** -0.5)
        tol, lse_tol = attention_bounds(s, want, spread, size, vmax, max(lens), dtype)
        assert bool(((a["out"].cpu().double() - want).abs() <= tol)[:T].all())
        assert float((a["lse"].cpu().double() - lse)[:T].abs().max()) <= lse_tol + ULP * float(lse[:T].abs().max())
        # the last gamma + 1 rows of each sequence are a block's logits (of those granted; the others' rows are made up)
        last = torch.tensor([[max(0, first[b + 1] - gamma - 1 + i) for i in range(gamma + 1)] for b in range(B)])
        logits = (a["out"].float().cpu()[last].reshape(B, gamma + 1, H * D) @ torch.randn((H * D, V), generator=g)).to(dtype)
        drafts = torch.randint(0, V, (B, gamma), generator=g, dtype=torch.int32)
        length = torch.tensor([rng.randint(0, 100) for _ in range(B)])
        presence, frequency = torch.rand(B, generator=g) * 2, torch.rand(B, generator=g)
        rho = 1 + torch.rand(B, generator=g)
        z = psd.adjust_logits(params, logits.cuda(), text=text.cuda(), length=length.cuda(), draft_tokens=drafts[:, None].cuda().contiguous(),
                              repetition=rho.cuda(), presence=presence.cuda(), frequency=frequency.cuda())
        torch.cuda.synchronize()
        wz, zsize = ref4.adjust(logits[:, None], text, length, drafts=drafts[:, None], rho=rho, presence=presence, frequency=frequency)
        zc = z.cpu()
        assert bool(((zc.double() - wz[:, 0]).abs() <= 5 * ULP * zsize[:, 0] + HALF[dtype] * wz[:, 0].abs()).all())
        rows_d = torch.randn((B, gamma, V), generator=g).to(dtype)
        u, e = torch.rand((B, gamma), generator=g), torch.empty((B, V)).exponential_(generator=g).clamp_(min=1e-30)
        out = psd.verify_given(params, vws, z, rows_d.cuda(), drafts.cuda(), u.cuda(), e.cuda())
        tokens, n_out, _, _, near = ref.verify_given(zc, rows_d, drafts, u, e, 0.9, 1.1)
        for b in range(B):
            if near[b] > 1e-5:
                assert out["out_tokens"][b].tolist() == tokens[b].tolist() and int(out["out_len"][b]) == int(n_out[b])
        # keep what was accepted: here any ascending choice of the new tokens
        keep = [sorted(rng.sample(range(n), rng.randint(1, n))) if n else [] for n in granted]
        index = torch.full((B, max_new), 99, dtype=torch.int32)
        for b, row in enumerate(keep):
            index[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
        before = [p.cpu().clone() for p in pools]
        kept = psd.kv_keep(cache, seqs, index.cuda(), torch.tensor([len(r) for r in keep], dtype=torch.int32).cuda())
        torch.cuda.synchronize()
        expect = [p.clone() for p in before]
        for b, row in enumerate(keep):
            for i, x in enumerate(row):
                (pf, cf), (pt, ct) = s.place(b, have[b] + x), s.place(b, have[b] + i)
                for w, was in zip(expect, before):
                    w[pt, ct] = was[pf, cf]
        assert all(torch.equal(p.cpu(), w) for p, w in zip(pools, expect))
        have = [h + len(r) for h, r in zip(have, keep)]
        assert kept.tolist() == have
        assert bool(torch.isfinite(torch.stack([ref4.decode(p, q_, D)[table[b, 0].cpu()] for b in range(B) if granted[b]
                                                for p, q_ in ((expect[0], expect[2]),)])).all())


def test_example_over_4_bits(block):
    """The loop over a cache in 4 bits: same numbers, same text; every token had a probability; and a presence penalty that
    outweighs every logit leaves no token twice, in the text or within a block."""
    g = torch.Generator(device="cuda").manual_seed(1)
    prompts = torch.randperm(500, device="cuda", generator=g)[:6 * 3].to(torch.int32).view(6, 3)
    target = block.Target(bits=4)
    good = block.good_drafter(target)
    a, rate = block.given(target, good, prompts, 60, seed=3)
    b, _ = block.given(block.Target(bits=4), good, prompts, 60, seed=3)
    assert torch.equal(a, b) and bool(((a >= 0) & (a < 500)).all()) and rate >= 1.0
    c, rate = block.given(target, good, prompts, 60, seed=3, presence=1e4)
    assert all(len(set(row)) == 60 for row in c.tolist()) and math.isfinite(rate)
    assert not all(len(set(row)) == 60 for row in a.tolist())
    d, _ = block.keyed(target, good, prompts, 40)
    assert bool(((d >= 0) & (d < 500)).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_captured_steps(block, dtype):
    """The whole step in one graph, replayed with other requests, rows and random numbers: state and outputs are those of
    the same calls made one by one (which test_serving_steps compares with their plain forms)."""
    psd = block.psd
    B, H, G, D, P, V, gamma, width, pages = 5, 4, 2, 80, 8, 900, 3, 12, 36
    max_new, rows = 20, B * 20
    params = psd.make_params(0, V, 1, 0, 0.9, 1.1, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(6)
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    normal = lambda *n: torch.randn(n, generator=g, device="cuda").to(dtype)  # noqa: E731

    class Server:
        def __init__(self):
            self.cache, self.pages = psd.new_cache4(pages, P, G, D, dtype=dtype), psd.new_pages(pages, P)
            self.table, self.held = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), ints(B)
            self.seqs = psd.make_seqs(ints(B + 1), ints(B), self.table, rows, max_new, width * P)
            self.ws, self.vws = psd.new_attention_workspace(self.cache, self.seqs, H), psd.new_verify_given_workspace(params, B, gamma)
            self.n_new, self.have, self.kept = ints(B), ints(B), ints(B)
            self.q, self.k, self.v = (torch.zeros((rows, n, D), dtype=dtype, device="cuda") for n in (H, G, G))
            self.weights = torch.zeros((gamma + 1, V), dtype=torch.float32, device="cuda")
            self.text, self.length = ints(B, 100), torch.zeros(B, dtype=torch.int64, device="cuda")
            self.drafts, self.draft_rows = ints(B, gamma), torch.zeros((B, gamma, V), dtype=dtype, device="cuda")
            self.u, self.e = torch.zeros((B, gamma), device="cuda"), torch.ones((B, V), device="cuda")
            self.presence = torch.ones(B, device="cuda")
            self.last = torch.arange(gamma + 1, device="cuda")
            self.index = torch.arange(max_new, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
            self.places, self.out, self.attended, self.z = {}, {}, {}, None

        def step(self):
            self.places.update(psd.kv_reserve(self.pages, self.seqs, self.n_new, self.have, self.held, out=self.places))
            psd.kv_append(self.cache, self.seqs, self.k, self.v)
            self.attended.update(psd.attention(self.cache, self.seqs, self.q, self.ws, out=self.attended.get("out"), want_lse=True,
                                               lse=self.attended.get("lse")))
            start = self.seqs.tensors[0]
            at = (start[1:, None] - gamma - 1 + self.last).clamp(min=0)
            logits = (self.attended["out"].float()[at][:, :, 0, :1] * self.weights).to(dtype)  # (no library product in a graph)
            self.z = psd.adjust_logits(params, logits, text=self.text, length=self.length, draft_tokens=self.drafts[:, None],
                                       presence=self.presence, out=logits)
            self.out.update(psd.verify_given(params, self.vws, self.z, self.draft_rows, self.drafts, self.u, self.e, out=self.out))
            n = torch.minimum(self.out["out_len"], self.places["granted"])
            psd.kv_keep(self.cache, self.seqs, self.index, n, kv_out=self.kept)

        def fill(self, of):
            for name, t in of.items():
                getattr(self, name).copy_(t)

        def all(self):
            return [*self.cache.tensors, *self.pages.tensors, self.table, self.held, *self.seqs.tensors, self.kept, self.z,
                    *self.attended.values(), *self.places.values(), *self.out.values()]

    eager, captured = Server(), Server()
    for s in (eager, captured):
        s.step()  # (nothing asked)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    have = torch.zeros(B, dtype=torch.int32, device="cuda")
    moved = 0
    for i in range(8):
        n_new = torch.where(have > 0, gamma + 1, torch.randint(gamma + 1, max_new + 1, (B,), generator=g, device="cuda")).to(torch.int32)
        of = dict(n_new=n_new, have=have, q=normal(rows, H, D), k=normal(rows, G, D), v=normal(rows, G, D),
                  weights=normal(gamma + 1, V).float(), text=torch.randint(0, V, (B, 100), generator=g, device="cuda"),
                  length=torch.randint(0, 101, (B,), generator=g, device="cuda"),
                  drafts=torch.randint(0, V, (B, gamma), generator=g, device="cuda"), draft_rows=normal(B, gamma, V),
                  u=torch.rand((B, gamma), generator=g, device="cuda"),
                  e=torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30))
        for s in (eager, captured):
            s.fill(of)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        T = int(eager.seqs.tensors[0][-1])
        for a, b in zip(eager.all(), captured.all()):
            assert a.dtype == b.dtype
            if a.shape[:1] == (rows,) and a.dtype in (dtype, torch.float32):  # attention's rows behind the last are left as they were
                a, b = a[:T], b[:T]
            assert torch.equal(a, b), i
        moved += int(eager.kept.sum())
        have = torch.where(torch.rand(B, generator=g, device="cuda") < 0.15, 0, eager.kept).to(torch.int32)
    assert moved > 0
