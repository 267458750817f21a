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
