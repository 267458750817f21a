"""Adjusted logits against the plain definition in 64 bits (GPU).

A float32 chain of a division or product, at most four sums and the biases' errs by (n + 5) 2^-24 of the sizes added up,
n the biases of one token; the result rounds once."""
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
from test_gpu_serving import BF16, F32, HALF, ULP  # noqa: E402


@pytest.fixture(scope="module")
def psd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21858_amd import psd as m
    return m


def inputs(B, K, S, V, dtype, L=50, gamma=None, n_bias=0, mask=None, seed=0, few=40):
    g = torch.Generator().manual_seed(seed)
    x = dict(logits=(torch.randn((B, K, S, V), generator=g) * 3).to(dtype))
    x["logits"][..., V // 3] = -math.inf
    x["logits"][..., V // 2] = 0.0
    pick = torch.randperm(V, generator=g)[:few].to(torch.int32)
    x["text"] = pick[torch.randint(0, len(pick), (B, L), generator=g)]
    x["text"][torch.rand((B, L), generator=g) < 0.1] = -1
    x["text"][torch.rand((B, L), generator=g) < 0.05] = V
    x["length"] = torch.randint(0, L + 1, (B,), generator=g)
    x["length"][0] = L
    gamma = S - 1 if gamma is None else gamma
    if gamma:
        x["drafts"] = pick[torch.randint(0, len(pick), (B, K, gamma), generator=g)]
        x["drafts"][0, 0, 0] = -1
    x["rho"] = 0.7 + torch.rand((B,), generator=g)
    x["presence"] = torch.randn((B,), generator=g)
    x["frequency"] = torch.randn((B,), generator=g) * 0.3
    if n_bias:
        x["bias_tokens"] = pick[torch.randint(0, len(pick), (B, n_bias), generator=g)].clone()
        x["bias_tokens"][0, 0] = V + 5
        x["bias"] = torch.randn((B, n_bias), generator=g)
    if mask:
        shape = (B, -(-V // 32)) if mask == 1 else (B, K, S, -(-V // 32))
        words = torch.randint(-(1 << 31), 1 << 31, shape, generator=g)
        choice = torch.rand(shape, generator=g)
        x["allowed"] = torch.where(choice < 0.3, torch.zeros_like(words), torch.where(choice < 0.6, torch.full_like(words, -1), words)).to(torch.int32)
    return x


NAMES = dict(text="text", length="length", text_from="text_from", drafts="draft_tokens", rho="repetition", presence="presence",
             frequency="frequency", bias_tokens="bias_tokens", bias="bias", allowed="allowed")


def check(psd, x, depth0=0, in_place=False, three=False, stream=None):
    logits = x["logits"]
    B, K, S, V = logits.shape
    dtype = logits.dtype
    print("[adjust]", tuple(logits.shape), dtype, depth0, in_place, sorted(x), flush=True)
    params = psd.make_params(0, V, K, 0, 1.0, 1.0, dtype=dtype)
    dev = logits.cuda()
    if three:
        dev = dev[:, 0]
    kw = {NAMES[n]: t.cuda() for n, t in x.items() if n != "logits"}
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    out = psd.adjust_logits(params, dev, depth0=depth0, out=dev if in_place else None, stream=stream, **kw)
    torch.cuda.synchronize()
    assert out.shape == dev.shape and (out.data_ptr() == dev.data_ptr()) == in_place
    if not in_place:
        assert torch.equal(dev.reshape(-1).view(torch.int16 if dtype == BF16 else torch.int32).cpu(),
                           logits.reshape(-1).view(torch.int16 if dtype == BF16 else torch.int32))
    want, size = ref4.adjust(logits, depth0=depth0, **{n: t for n, t in x.items() if n != "logits"})
    got = out.cpu().double().reshape(want.shape)
    gone = want == -math.inf
    assert torch.equal(got == -math.inf, gone)
    n = x["bias"].shape[1] if "bias" in x else 0
    # size: what was added up, the quotient's own error among it
    tol = (n + 5) * ULP * size + HALF[dtype] * want.abs()
    off = (got - want).abs()
    assert bool((off <= tol)[~gone].all()), (float((off - tol)[~gone].max()), ((off > tol) & ~gone).nonzero()[:3].tolist())
    return out


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 7, 100, 1024, 8192, 8193, 20001])
@pytest.mark.parametrize("in_place", [False, True])
def test_vocabularies(psd, V, in_place, dtype):
    check(psd, inputs(3, 2, 4, V, dtype, n_bias=9, mask=2, few=min(V, 40)), in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("left_out", ["text", "drafts", "rho", "presence", "frequency", "bias", "allowed", "all"])
def test_each_term_alone_left_out(psd, left_out, in_place):
    x = inputs(2, 3, 3, 500, F32, n_bias=5, mask=1)
    gone = {"text": ("text", "length"), "bias": ("bias", "bias_tokens"), "all": tuple(NAMES)}.get(left_out, (left_out,))
    check(psd, {n: t for n, t in x.items() if n not in gone}, in_place=in_place)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows_of_a_block(psd, dtype):
    check(psd, inputs(2, 1, 5, 999, dtype), three=True)
    check(psd, inputs(2, 4, 1, 999, dtype, gamma=6), depth0=6)      # a path's last rows
    check(psd, inputs(2, 4, 2, 999, dtype, gamma=6), depth0=3)
    check(psd, inputs(2, 32, 2, 300, dtype, gamma=32), depth0=31)
    check(psd, inputs(1, 2, 33, 300, dtype, gamma=32))
    check(psd, inputs(2, 2, 3, 999, dtype, mask=1), stream=torch.cuda.Stream())


def test_texts(psd):
    """Lengths of nothing, beyond the text, and counts that start later; one token all the way."""
    x = inputs(4, 1, 2, 300, F32, L=700)
    x["length"] = torch.tensor([0, 700, 5000, -3])
    check(psd, x)
    x["text_from"] = torch.tensor([0, 650, -7, 0])
    check(psd, x)
    x["text_from"] = torch.tensor([900, 700, 699, 1 << 40])
    check(psd, x)
    x = inputs(1, 1, 2, 300, F32, L=20000)
    x["text"][:] = 17
    check(psd, x)
    x["text"] = x["text"][:, :0].contiguous()
    check(psd, x)
    wide = inputs(2, 1, 2, 300, BF16, L=64)
    wide["text"] = torch.cat((wide["text"], wide["text"]), 1)[:, 5:60]
    check(psd, wide)


def test_lengths_past_32_bits_are_bounded(psd):
    """A length whose lower 32 bits are a count of tokens that are not there."""
    x = inputs(4, 1, 2, 300, F32, L=70)
    x["length"] = torch.tensor([-(1 << 32) + 5000, (1 << 32) + 3, -(1 << 63), 1 << 62])
    check(psd, x)
    x["text_from"] = torch.tensor([0, 60, 0, -(1 << 32) + 65])
    check(psd, x)


@pytest.mark.parametrize("n_bias", [1, 300, 1024])
def test_biases_of_one_token_add_up_in_order(psd, n_bias):
    x = inputs(2, 1, 2, 9000, F32, n_bias=n_bias, few=6)
    a = check(psd, x)
    b = check(psd, x)
    assert torch.equal(a, b)


def test_penalties_reach_the_verification(psd):
    """Rows adjusted in place, in a graph with the verification that reads them, replayed with longer texts."""
    B, gamma, V = 4, 3, 2000
    g = torch.Generator(device="cuda").manual_seed(2)
    params = psd.make_params(0, V, 1, 0, 1.0, 1.0, dtype=F32)
    ws = psd.new_verify_given_workspace(params, B, gamma)
    base = torch.randn((B, gamma + 1, V), device="cuda", generator=g) * 3
    rows, drafts = torch.empty_like(base), torch.randn((B, gamma, V), device="cuda", generator=g)
    tokens = torch.randint(0, V, (B, gamma), device="cuda", generator=g, dtype=torch.int32)
    text = torch.randint(0, V, (B, 3000), device="cuda", generator=g, dtype=torch.int32)
    length = torch.zeros(B, dtype=torch.int64, device="cuda")
    allowed = torch.randint(-(1 << 31), 1 << 31, (B, -(-V // 32)), device="cuda", generator=g).to(torch.int32)
    u, e = torch.rand((B, gamma), device="cuda", generator=g), torch.empty((B, V), device="cuda").exponential_(generator=g)
    strong = torch.full((B,), 30.0, device="cuda")
    out = {}

    def step():
        rows.copy_(base)
        psd.adjust_logits(params, rows, text=text, length=length, draft_tokens=tokens, presence=strong, allowed=allowed, out=rows)
        out.update(psd.verify_given(params, ws, rows, drafts, tokens, u, e, want_lse=True, out=out))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in (0, 10, 1000, 3000):
        length.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], got[k]) for k in out)
        want, _ = ref4.adjust(base.cpu()[:, None], text.cpu(), length.cpu(), drafts=tokens.cpu()[:, None], presence=strong.cpu(),
                              allowed=allowed.cpu())
        assert float((torch.logsumexp(want[:, 0], -1) - out["target_lse"].cpu().double()).abs().max()) < 1e-4
        for b in range(B):
            last = int(out["out_tokens"][b, int(out["out_len"][b]) - 1])
            assert int(allowed[b, last // 32]) >> (last % 32) & 1


def test_repetition_divides(psd):
    """Float32 logits with a repetition penalty alone: the float32 quotient and product, to the bit, over all of float32."""
    g = torch.Generator().manual_seed(11)
    V = 5000
    rho = torch.tensor([1.1, 0.7, 3.0, 1.0 / 3, 2.0 ** -126, 2.0 ** 126, 1.9999999, 1.0])
    B = len(rho)
    z = torch.randn((B, 1, 2, V), generator=g)
    z[:, 0, 1] *= 2.0 ** torch.randint(-140, 126, (B, V), generator=g).double().float()
    z[..., :8] = torch.tensor([0.0, math.inf, -math.inf, 2.0 ** -149, -(2.0 ** -149), 3.4028234663852886e38, -3.4028234663852886e38, 1.0])
    text = torch.arange(V, dtype=torch.int32).expand(B, V).contiguous()
    out = psd.adjust_logits(psd.make_params(0, V, 1, 0, dtype=F32), z.cuda(), text=text.cuda(),
                            length=torch.full((B,), V).cuda(), repetition=rho.cuda()).cpu()
    r = rho[:, None, None, None]
    assert torch.equal(out, torch.where(z > 0, z / r, z * r))
