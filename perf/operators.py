"""Measured operators: one block of speculative decoding around the verification.

A serving program runs, block after block: the new tokens' keys and values go into a paged
cache (``kv_append``: norms of queries and keys, position rotation, scatter), the new tokens
attend over the cache (``attention``: causal chunks or K draft paths behind one root), the
drafted tokens are verified from given random numbers (``verify``), and the accepted path's
keys and values are kept (``keep``).

``own`` false: the plain form, elementary torch operations in 32 bits.  ``own`` true: the
framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# Vocabularies, draft lengths, batches, noise and temperatures of the verification are those of
# the repository's configurations; head layouts, pages and cache lengths are generic.
_HEADS = dict(H=32, G=8, D=128, page=16, dtype="bf16")


def _append(name, **more):
    return {**_HEADS, "R": 128, "norm": False, "interleaved": False, **more, "name": name, "op": "append"}


def _attention(name, **more):
    return {**_HEADS, "window": 0, "K": 0, "gamma": 0, "lse": False, **more, "name": name, "op": "attention"}


def _keep(name, **more):
    return {**_HEADS, **more, "name": name, "op": "keep"}


def _verify(name, **more):
    return {**more, "name": name, "op": "verify"}


def listed():
    return [
        # four interactive requests, one new token each: nothing but latency
        _append("append_single_bf16", B=4, new=1, kv=512),
        # a ragged batch of long prompts, queries and keys normed, part of each head rotated
        _append("append_prompts_bf16", B=8, new=2048, kv=2048, norm=True, R=64, page=64),
        # four interactive requests, one new token each
        _attention("attend_single_bf16", B=4, new=1, kv=512),
        # a serving batch with long caches, one new token each
        _attention("attend_long_bf16", B=32, new=1, kv=16384, page=64),
        # the benchmark's draft length: the root and four drafted tokens of 64 sequences
        _attention("attend_block_bf16", B=64, new=5, kv=4096, lse=True),
        # four draft paths behind one root, each row seeing its own path
        _attention("attend_paths_bf16", B=16, new=17, kv=2048, K=4, gamma=4, page=32),
        # a chunk of a long prompt: matrix products bound it
        _attention("attend_prompt_bf16", B=1, new=2048, kv=16384, page=64),
        # float32, a head size, group and page that nobody padded, a sliding window
        _attention("attend_odd_f32", B=6, new=37, kv=1500, H=12, G=4, D=80, page=24, dtype="f32", window=700,
                   lse=True),
        # one request's four layers after a block of two paths
        _keep("keep_single_bf16", B=1, L=4, K=2, gamma=4, kv=100),
        # the benchmark's block in a 32-layer cache
        _keep("keep_block_bf16", B=64, L=32, K=4, gamma=4, kv=100),
        # one interactive request with a toy vocabulary, float32
        _verify("given_tiny_f32", V=1024, gamma=4, B=1, dtype="f32", sigma=2.0, alpha=1.1, tau=0.8, T=1.0),
        # the benchmark's block with one drafter
        _verify("given_headline_bf16", V=128256, gamma=4, B=64, dtype="bf16", sigma=3.0, alpha=1.2, tau=0.5, T=0.7),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "keep", "verify", "attention", "verify"])
    if op == "verify":
        V = rng.choice([_log(rng, 100, 200000), 32000, 50257, 128256, 151936])
        gamma = rng.randint(1, 8)
        dtype = rng.choice(["f32", "bf16"])
        B = _log(rng, 1, max(1, min(64, 128256 * 9 * 64 // (V * (2 * gamma + 1) * (2 if dtype == "f32" else 1)))))
        return dict(op=op, V=V, gamma=gamma, B=B, dtype=dtype, sigma=rng.choice([2.0, 2.5, 3.0]),
                    alpha=rng.choice([1.0, 1.1, 1.2]), tau=round(rng.uniform(0.3, 1.0), 3), T=rng.choice([0.7, 1.0]))
    H, G = rng.choice([(32, 8), (32, 8), (16, 16), (8, 1), (28, 4), (40, 8), (12, 4), (64, 8)])
    D = rng.choice([64, 80, 96, 128, 128, 192, 256])
    page = rng.choice([8, 16, 24, 32, 64, 100, 256])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    base = dict(op=op, H=H, G=G, D=D, page=page, dtype=dtype)
    if op == "append":
        # no more rows and elements than the listed prompts
        most = 8 * 2048 * 48 * 128 // ((H + 2 * G) * D * (2 if dtype == "f32" else 1))
        new = _log(rng, 1, min(4096, most))
        B = _log(rng, 1, max(1, min(64, most // new)))
        return dict(base, B=B, new=new, kv=new + _log(rng, 1, 512), R=rng.choice([0, D // 2, D, D]) // 2 * 2,
                    norm=rng.random() < 0.5, interleaved=rng.random() < 0.5)
    if op == "keep":
        K, gamma = rng.randint(1, 8), rng.randint(1, 8)
        L = _log(rng, 1, 32)
        most = 64 * 32 * 1024 * 25 // (L * G * D * (gamma + 1) * (2 if dtype == "f32" else 1))
        return dict(base, B=_log(rng, 1, max(1, min(64, most // 8))), L=L, K=K, gamma=gamma,
                    kv=1 + K * gamma + _log(rng, 1, 64))
    kind = rng.choice(["single", "block", "paths", "prompt"])
    K, gamma = (rng.randint(1, 8), rng.randint(1, 8)) if kind == "paths" else (0, 0)
    new = {"single": 1, "block": rng.randint(2, 17), "paths": 1 + K * gamma, "prompt": _log(rng, 64, 2048)}[kind]
    kv = new + _log(rng, 1, 8000)
    # no more visible pairs and no more cache than the listed ones
    heavy = (2 if D > 128 else 1) * (8 if dtype == "f32" else 1)
    most = min(32 * 2048 * 15000 // heavy // (H * new * kv), 32 * 10000 * 1024 // (2 if dtype == "f32" else 1) // (kv * G * D))
    if most < 1:
        kv = new + _log(rng, 1, 500)
        most = 1
    return dict(base, B=_log(rng, 1, max(1, min(64, most))), new=new, kv=kv, window=rng.choice([0, 0, _log(rng, 16, 4096)])
                if K == 0 else 0, K=K, gamma=gamma, lse=rng.random() < 0.5)


# ---------------------------------------------------------------- sizes

def _lengths(c):
    """New and cached tokens of each sequence: the first has the most, the others spread below."""
    new, kv = [], []
    for b in range(c["B"]):
        f = (b * 0.6180339887) % 1.0
        n = c["new"] if c.get("K") or c["new"] <= 17 or b == 0 else max(1, int(c["new"] * (1.0 - 0.75 * f)))
        new.append(n)
        kv.append(max(n, int(c["kv"] * (1.0 - 0.75 * f))))
    return new, kv


def _pairs(c):
    """Visible (row, cached token) pairs and cached tokens that some row sees."""
    pairs = seen = 0
    for n, t in zip(*_lengths(c)):
        start = t - n
        if c["K"]:
            pairs += n * start + 1 + c["K"] * sum(2 + s for s in range(c["gamma"]))
            seen += t
        else:
            w = c["window"] or t
            pairs += sum(min(w, start + i + 1) for i in range(n))
            seen += min(t, n + w - 1)
    return pairs, seen


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "verify":
        rows = c["B"] * (2 * c["gamma"] + 1)
        return {"bytes": rows * c["V"] * e + c["B"] * c["V"] * 4, "flops": 4.0 * rows * c["V"]}
    if c["op"] == "append":
        rows = sum(_lengths(c)[0])
        el = rows * (c["H"] + 2 * c["G"]) * c["D"]
        return {"bytes": 2 * el * e + rows * c["R"] * 4, "flops": 8.0 * el}
    if c["op"] == "keep":
        # on average half of the drafts are kept; the first path's stay where they are
        moved = c["B"] * c["gamma"] / 2 * (c["K"] - 1) / c["K"]
        return {"bytes": max(1.0, moved * c["L"] * 2 * c["G"] * c["D"] * e * 2), "flops": 0.0}
    pairs, seen = _pairs(c)
    rows = sum(_lengths(c)[0])
    return {"bytes": 2 * rows * c["H"] * c["D"] * e + 2 * seen * c["G"] * c["D"] * e, "flops": 4.0 * pairs * c["H"] * c["D"]}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _randn(g, *shape, dtype):
    return torch.randn(shape, device=DEV, generator=g, dtype=torch.float32).to(dtype)


def _paged(c, g, layers=None):
    """Pools of shuffled pages, the page table and the sequences' lengths."""
    dt = _DT[c["dtype"]]
    new, kv = _lengths(c)
    P = c["page"]
    width = -(-max(kv) // P)
    pages = c["B"] * width + 3
    table = torch.randperm(pages, device=DEV, generator=g)[:c["B"] * width].reshape(c["B"], width).to(torch.int32)
    lead = () if layers is None else (layers,)
    s = dict(case=c, P=P, table=table.contiguous(), max_new=max(new), max_kv=max(kv), rows=sum(new),
             new_start=torch.tensor([sum(new[:b]) for b in range(c["B"] + 1)], dtype=torch.int32, device=DEV),
             kv_len=torch.tensor(kv, dtype=torch.int32, device=DEV),
             k_pages=torch.empty(lead + (pages, P, c["G"], c["D"]), dtype=dt, device=DEV).normal_(generator=g),
             v_pages=torch.empty(lead + (pages, P, c["G"], c["D"]), dtype=dt, device=DEV).normal_(generator=g))
    if own:
        from paper_2609_21858_amd import psd

        s["seqs"] = psd.make_seqs(s["new_start"], s["kv_len"], s["table"], s["rows"], s["max_new"], s["max_kv"])
        s["cache"] = psd.make_cache(s["k_pages"], s["v_pages"])
    return s


def _path_words(K, gamma):
    """Visibility bits of 1 + K * gamma new tokens: the root, then K paths of gamma tokens; each token sees
    the root, its path's earlier tokens and itself."""
    n = 1 + K * gamma
    words = [[0] * (-(-n // 32)) for _ in range(n)]
    for i in range(n):
        k, s = divmod(i - 1, gamma) if i else (0, -1)
        for j in [0] + [1 + k * gamma + d for d in range(s + 1)]:
            words[i][j // 32] |= 1 << (j % 32)
    return [[w - (1 << 32) if w >= 1 << 31 else w for w in row] for row in words]


def prepare(c, seed):
    g = _gen(seed)
    if c["op"] == "verify":
        B, V, n, dt = c["B"], c["V"], c["gamma"], _DT[c["dtype"]]
        z = torch.randn((B, n + 1, V), device=DEV, generator=g).mul_(c["sigma"])
        rank = torch.rand((B, n + 1, V), device=DEV, generator=g).mul_(V - 1).add_(1.0)
        z -= rank.log_().mul_(c["alpha"])
        d = torch.randn((B, n, V), device=DEV, generator=g).mul_(c["tau"]).add_(z[:, :n])
        # the drafter's own tokens, drawn from its rows
        x = (d / c["T"] - torch.empty_like(d).exponential_(generator=g).log_()).argmax(-1).to(torch.int32)
        s = dict(case=c, target=z.to(dt), draft=d.to(dt), tokens=x.contiguous(),
                 u=torch.rand((B, n), device=DEV, generator=g),
                 clocks=torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30))
        if own:
            from paper_2609_21858_amd import psd

            s["params"] = psd.make_params(0, V, 1, 0, c["T"], c["T"], dtype=dt)
            s["ws"] = psd.new_verify_given_workspace(s["params"], B, n)
        return s
    if c["op"] == "keep":
        c = dict(c, new=1 + c["K"] * c["gamma"])
        s = _paged(c, g, layers=c["L"])
        path = torch.randint(0, c["K"], (c["B"], 1), device=DEV, generator=g)
        taken = torch.randint(0, c["gamma"] + 1, (c["B"],), device=DEV, generator=g)
        depth = torch.arange(c["gamma"] + 1, device=DEV)
        s["keep"] = torch.where(depth > 0, path * c["gamma"] + depth, 0).to(torch.int32).contiguous()
        s["n_keep"] = (taken + 1).to(torch.int32)
        return s
    s = _paged(c, g)
    dt, T = _DT[c["dtype"]], s["rows"]
    if c["op"] == "append":
        qkv = _randn(g, T, (c["H"] + 2 * c["G"]) * c["D"], dtype=dt)  # one projection's output, viewed three ways
        H, G, D = c["H"], c["G"], c["D"]
        s["q"] = qkv[:, :H * D].unflatten(1, (H, D))
        s["k"] = qkv[:, H * D:(H + G) * D].unflatten(1, (G, D))
        s["v"] = qkv[:, (H + G) * D:].unflatten(1, (G, D))
        R = c["R"]
        s["cos"] = s["sin"] = s["q_norm"] = s["k_norm"] = None
        if R:
            freq = 10000.0 ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) * 2 / R)
            angle = torch.arange(s["max_kv"], device=DEV, dtype=torch.float64)[:, None] * freq
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        if c["norm"]:
            s["q_norm"] = (1 + 0.1 * _randn(g, D, dtype=torch.float32)).to(dt)
            s["k_norm"] = (1 + 0.1 * _randn(g, D, dtype=torch.float32)).to(dt)
        s["q_out"] = torch.empty((T, H, D), dtype=dt, device=DEV)
        return s
    s["q"] = _randn(g, T, c["H"], c["D"], dtype=dt)
    s["scale"] = c["D"] ** -0.5
    s["mask"] = None
    if c["K"]:
        words = torch.tensor(_path_words(c["K"], c["gamma"]), dtype=torch.int32, device=DEV)
        s["mask"] = words.repeat(c["B"], 1).contiguous()
    if own:
        from paper_2609_21858_amd import psd

        s["ws"] = psd.new_attention_workspace(s["cache"], s["seqs"], c["H"])
    return s


# ---------------------------------------------------------------- one pass

def _rows(s):
    """Sequence, index among its new tokens and cache position of every packed row."""
    row = torch.arange(s["rows"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["new_start"][1:], row, right=True)
    i = row - s["new_start"][seq]
    new = s["new_start"][1:] - s["new_start"][:-1]
    return seq, i, s["kv_len"][seq] - new[seq] + i


def _slots(s, seq, pos):
    return s["table"][seq, (pos // s["P"]).long()].long() * s["P"] + pos % s["P"]


def _norm_rotate(x, w, cos, sin, interleaved):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    if cos is None:
        return x
    R = 2 * cos.shape[-1]
    cos, sin, head = cos[:, None], sin[:, None], x[..., :R]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :R // 2], head[..., R // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    head = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((head, x[..., R:]), -1)


def _plain_append(s, c):
    seq, _, pos = _rows(s)
    at = _slots(s, seq, pos)
    cos, sin = (None, None) if s["cos"] is None else (s["cos"][pos.long()], s["sin"][pos.long()])
    dt = s["q"].dtype
    q = _norm_rotate(s["q"], s["q_norm"], cos, sin, c["interleaved"]).to(dt)
    s["k_pages"].flatten(0, 1)[at] = _norm_rotate(s["k"], s["k_norm"], cos, sin, c["interleaved"]).to(dt)
    s["v_pages"].flatten(0, 1)[at] = s["v"]
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attention(s, c):
    B, H, G, D = c["B"], c["H"], c["G"], c["D"]
    n, t, h = s["max_new"], s["max_kv"], c["H"] // c["G"]
    seq, i, pos = _rows(s)
    new = s["new_start"][1:] - s["new_start"][:-1]
    j = torch.arange(t, device=DEV)
    at = s["table"][:, j // s["P"]].long() * s["P"] + j % s["P"]
    k = s["k_pages"].flatten(0, 1)[at].permute(0, 2, 3, 1).float().contiguous()      # [B][G][D][t]
    v = s["v_pages"].flatten(0, 1)[at].permute(0, 2, 1, 3).float().contiguous()      # [B][G][t][D]
    r = torch.arange(n, device=DEV)
    q = s["q"][(s["new_start"][:-1, None] + r).clamp(max=s["rows"] - 1).long()].float()
    q = q.view(B, n, G, h, D).permute(0, 2, 1, 3, 4).reshape(B, G, n * h, D)
    score = torch.matmul(q, k).mul_(s["scale"]).view(B, G, n, h, t)
    start = (s["kv_len"] - new)[:, None, None]
    p = start + r[:, None]                                                            # [B][n][1]
    if c["K"]:
        bit = (j - start).clamp(min=0, max=32 * s["mask"].shape[1] - 1)               # [B][1][t]
        words = s["mask"].view(B, n, -1).gather(2, (bit // 32).expand(B, n, t).long())
        see = (j < start) | (((words >> (bit % 32).int()) & 1) > 0)
        see &= j < s["kv_len"][:, None, None]
    else:
        see = j <= p
        if c["window"]:
            see &= j > p - c["window"]
    score.masked_fill_(~see[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(B, G, n * h, t), v).view(B, G, n, h, D) / torch.where(total > 0, total, 1.0)
    o = {"out": out.permute(0, 2, 1, 3, 4).reshape(B, n, H, D)[seq, i.long()].to(s["q"].dtype)}
    if c["lse"]:
        o["lse"] = (top + total.log()).permute(0, 2, 1, 3, 4).reshape(B, n, H)[seq, i.long()]
    return o


def _plain_keep(s, c):
    new = s["new_start"][1:] - s["new_start"][:-1]
    first = s["kv_len"] - new
    depth = torch.arange(s["keep"].shape[1], device=DEV)
    # depths past n_keep keep what is there: they copy a token onto itself
    src = torch.where(depth < s["n_keep"][:, None], s["keep"], depth) + first[:, None]
    dst = depth + first[:, None]
    seq = torch.arange(c["B"], device=DEV)[:, None]
    src, dst = _slots(s, seq, src), _slots(s, seq, dst)
    kf, vf = s["k_pages"].flatten(1, 2), s["v_pages"].flatten(1, 2)
    kf[:, dst] = kf[:, src]
    vf[:, dst] = vf[:, src]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "kv_len": first + s["n_keep"]}


def _softmax(x, T):
    x = x.float()
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = ((x - top) / T).exp_()
    total = w.sum(-1, keepdim=True)
    return w / torch.where(total > 0, total, 1.0), (top / T + total.log())[..., 0]


def _plain_verify(s, c):
    B, n = c["B"], c["gamma"]
    p, p_lse = _softmax(s["target"], c["T"])
    q, q_lse = _softmax(s["draft"], c["T"])
    x = s["tokens"].long()[..., None]
    ok = s["u"] * q.gather(2, x)[..., 0] < p[:, :n].gather(2, x)[..., 0]
    taken = ok.long().cumprod(1).sum(1)
    seq = torch.arange(B, device=DEV)
    last = p[seq, taken]
    rest = (last - torch.where((taken < n)[:, None], q[seq, taken.clamp(max=n - 1)], 0.0)).clamp_(min=0.0)
    rest = torch.where((rest > 0).any(1, keepdim=True), rest, last)
    score = torch.where(rest > 0, s["clocks"] / rest, math.inf)
    token = torch.where((rest > 0).any(1), score.argmin(1), -1).to(torch.int32)
    d = torch.arange(n + 1, device=DEV)
    padded = torch.cat((s["tokens"], s["tokens"][:, :1]), 1)
    out = torch.where(d < taken[:, None], padded, torch.where(d == taken[:, None], token[:, None], -1))
    return {"out_tokens": out.to(torch.int32), "out_len": (taken + 1).to(torch.int32), "target_lse": p_lse,
            "draft_lse": q_lse}


def run(s):
    c = s["case"]
    if not own:
        return {"append": _plain_append, "attention": _plain_attention, "keep": _plain_keep,
                "verify": _plain_verify}[c["op"]](s, c)
    from paper_2609_21858_amd import psd

    if c["op"] == "append":
        q = psd.kv_append(s["cache"], s["seqs"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], cos=s["cos"], sin=s["sin"],
                          interleaved=c["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if c["op"] == "attention":
        return psd.attention(s["cache"], s["seqs"], s["q"], s["ws"], scale=s["scale"], window=c["window"],
                             mask=s["mask"], want_lse=c["lse"])
    if c["op"] == "keep":
        kv_len = psd.kv_keep(s["cache"], s["seqs"], s["keep"], s["n_keep"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "kv_len": kv_len}
    return psd.verify_given(s["params"], s["ws"], s["target"], s["draft"], s["tokens"], s["u"], s["clocks"],
                            want_lse=True)


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _cached(pages, table, page, b, upto):
    """The first `upto` cached tokens of sequence b, page by page."""
    whole = pages[table[b, :-(-upto // page)].long()].double()
    return whole.reshape(-1, *pages.shape[2:])[:upto]


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "verify":
        lse = [torch.logsumexp(s[name].double() / c["T"], -1) for name in ("target", "draft")]
        return {"out_tokens": None, "out_len": None, "target_lse": lse[0], "draft_lse": lse[1]}
    new, kv = _lengths(dict(c, new=1 + c["K"] * c["gamma"]) if c["op"] == "keep" else c)
    P, table = c["page"], s["table"]
    if c["op"] == "keep":
        for b, (n, t) in enumerate(zip(new, kv)):
            where = [divmod(t - n + i, P) for i in range(n)]
            ids = [(int(table[b, page]), place) for page, place in where]
            kept = s["keep"][b, :int(s["n_keep"][b])].tolist()
            for name in ("k_pages", "v_pages"):
                moved = [s[name][:, ids[i][0], ids[i][1]].clone() for i in kept]
                for (page, place), m in zip(ids, moved):
                    s[name][:, page, place] = m
        return {"k_pages": s["k_pages"].double() if s["k_pages"].numel() < 1e9 else None,
                "v_pages": s["v_pages"].double() if s["v_pages"].numel() < 1e9 else None, "kv_len": None}
    first = [sum(new[:b]) for b in range(c["B"])]
    H, G, D = c["H"], c["G"], c["D"]
    if c["op"] == "append":
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        q_all = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        for b, (n, t) in enumerate(zip(new, kv)):
            row = slice(first[b], first[b] + n)
            pos = torch.arange(t - n, t, device=DEV)
            place = (table[b, pos // P].long(), pos % P)
            for name, w, into in (("q", s["q_norm"], None), ("k", s["k_norm"], k_pages)):
                x = s[name][row].double()
                if w is not None:
                    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
                if c["R"]:
                    half = c["R"] // 2
                    first_dims = torch.arange(half, device=DEV)
                    a_at, b_at = (2 * first_dims, 2 * first_dims + 1) if c["interleaved"] else (first_dims, first_dims + half)
                    turn = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]
                    z = torch.complex(x[..., a_at], x[..., b_at]) * turn
                    x[..., a_at], x[..., b_at] = z.real, z.imag
                if into is None:
                    q_all[row] = x
                else:
                    into[place] = x
            v_pages[place] = s["v"][row].double()
        return {"q": q_all, "k_pages": k_pages, "v_pages": v_pages}
    out = torch.zeros((s["rows"], H, D), dtype=torch.float64, device=DEV)
    lse = torch.full((s["rows"], H), -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, t) in enumerate(zip(new, kv)):
        K, V = _cached(s["k_pages"], table, P, b, t), _cached(s["v_pages"], table, P, b, t)
        see = torch.zeros((n, t), dtype=torch.bool, device=DEV)
        if c["K"]:
            see[:, :t - n + 1] = True
            for k in range(c["K"]):
                at = 1 + k * c["gamma"]
                see[at:at + c["gamma"], t - n + at:t - n + at + c["gamma"]] = torch.ones(
                    (c["gamma"], c["gamma"]), dtype=torch.bool, device=DEV).tril()
        else:
            back = torch.arange(t - n, t, device=DEV)[:, None] - torch.arange(t, device=DEV)
            see = (back >= 0) & (back < (c["window"] or t + 1))
        for h in range(H):
            x = s["q"][first[b]:first[b] + n, h].double() @ K[:, h * G // H].t() * s["scale"]
            x = x.masked_fill(~see, -math.inf)
            lse[first[b]:first[b] + n, h] = torch.logsumexp(x, -1)
            out[first[b]:first[b] + n, h] = torch.softmax(x, -1) @ V[:, h * G // H]
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
