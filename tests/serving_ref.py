"""Plain 64-bit implementations of the paged cache's operators and of the verification from given
random numbers, on the CPU, and the inputs of their tests."""
import math

import torch


class Sequences:
    """Sequences with their page table, and pools whose unused places hold NaN."""

    def __init__(self, lens, G, D, P, dtype, seed=0, layers=None, heads_first=False, spare=2, width_extra=1):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.G, self.D, self.P, self.dtype = lens, G, D, P, dtype
        B = len(lens)
        self.B = B
        self.new_start = [0]
        for n, _ in lens:
            self.new_start.append(self.new_start[-1] + n)
        self.rows = max(1, self.new_start[-1])
        width = max(1, max(-(-max(kv, 0) // P) for _, kv in lens)) + width_extra
        self.pages = B * width + spare
        self.table = torch.randperm(self.pages, generator=g)[:B * width].reshape(B, width).to(torch.int32)
        lead = [] if layers is None else [layers]
        shape = lead + [self.pages, P, G, D]
        self.k = torch.full(shape, math.nan, dtype=torch.float32)
        self.v = torch.full(shape, math.nan, dtype=torch.float32)
        for b, (_, kv) in enumerate(lens):
            for c in range(max(kv, 0)):
                page, place = self.place(b, c)
                self.k[..., page, place, :, :] = torch.randn(lead + [G, D], generator=g)
                self.v[..., page, place, :, :] = torch.randn(lead + [G, D], generator=g)
        self.k, self.v = self.k.to(dtype), self.v.to(dtype)
        self.heads_first = heads_first
        self.gen = g

    def place(self, b, c):
        return int(self.table[b, c // self.P]), c % self.P

    def first(self, b):
        n, kv = self.lens[b]
        return kv - n

    def device(self, t):
        """The pool on the GPU; heads before places in memory with heads_first."""
        if self.heads_first:
            return t.transpose(-3, -2).contiguous().cuda().transpose(-3, -2)
        return t.cuda()

    def handles(self, psd, max_new=None, max_kv=None):
        dk, dv = self.device(self.k), self.device(self.v)
        cache = psd.make_cache(dk, dv)
        seqs = psd.make_seqs(torch.tensor(self.new_start, dtype=torch.int32).cuda(),
                             torch.tensor([kv for _, kv in self.lens], dtype=torch.int32).cuda(), self.table.cuda(), self.rows,
                             max_new or max(1, max(n for n, _ in self.lens)), max_kv or max(1, max(kv for _, kv in self.lens)))
        return cache, seqs, dk, dv


def visible(seqs, b, i, window=0, mask=None):
    """Cache positions that new token i of sequence b sees."""
    n, kv = seqs.lens[b]
    first = kv - n
    if mask is not None:
        row = mask[seqs.new_start[b] + i]
        own = [j for j in range(n) if j // 32 < len(row) and int(row[j // 32]) >> (j % 32) & 1]
        return [c for c in range(max(first, 0))] + [first + j for j in own if first + j >= 0]
    c = first + i
    return [j for j in range(max(0, c - window + 1 if window else 0), c + 1)]


def attention(seqs, q, scale, window=0, mask=None, bad_pages=()):
    """out, lse in float64 and per-element error bounds of the kernels (see bounds in the tests)."""
    T, H, D = q.shape
    out = torch.zeros((T, H, D), dtype=torch.float64)
    spread = torch.zeros((T, H, D), dtype=torch.float64)   # sum p |v|
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    size = 0.0                                              # largest scale * sum |q k|
    vmax = 0.0
    h_per = H // seqs.G
    for b in range(seqs.B):
        for i in range(seqs.lens[b][0]):
            t = seqs.new_start[b] + i
            pos = [c for c in visible(seqs, b, i, window, mask) if seqs.place(b, c)[0] not in bad_pages]
            if not pos:
                continue
            pages = torch.tensor([seqs.place(b, c)[0] for c in pos])
            places = torch.tensor([seqs.place(b, c)[1] for c in pos])
            k = seqs.k[pages, places].double()               # [n][G][D]
            v = seqs.v[pages, places].double()
            qq = q[t].double().reshape(seqs.G, h_per, D)
            s = torch.einsum("ghd,ngd->ghn", qq, k) * scale
            size = max(size, float((torch.einsum("ghd,ngd->ghn", qq.abs(), k.abs()) * scale).max()))
            vmax = max(vmax, float(v.abs().max()))
            l = torch.logsumexp(s, -1)
            p = torch.exp(s - l[..., None])
            out[t] = torch.einsum("ghn,ngd->ghd", p, v).reshape(H, D)
            spread[t] = torch.einsum("ghn,ngd->ghd", p, v.abs()).reshape(H, D)
            lse[t] = l.reshape(H)
    return out, lse, spread, size, vmax


def norm_rotate(x, w, eps, cos, sin, interleaved):
    """x [heads][D] float64; also the size of what is added up in each element."""
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    y, size = x.clone(), x.abs().clone()
    if cos is not None:
        half = cos.shape[0]
        for r in range(half):
            a, b = (2 * r, 2 * r + 1) if interleaved else (r, r + half)
            y[:, a] = x[:, a] * cos[r] - x[:, b] * sin[r]
            y[:, b] = x[:, b] * cos[r] + x[:, a] * sin[r]
            size[:, a] = size[:, b] = x[:, a].abs() + x[:, b].abs()
    return y, size


def verify_given(target, draft, tokens, u, e, T_target, T_draft, n_drafts=None):
    """Tokens, lengths, LSEs and, per sequence, the smallest relative distance by which a decision was taken."""
    B, g1, V = target.shape
    g = g1 - 1

    def soft(row, T):
        z = row.double() / T
        top = z.max()
        if top == -math.inf:
            return torch.zeros_like(z), -math.inf
        w = torch.exp(z - top)
        return w / w.sum(), float(top + torch.log(w.sum()))

    out = torch.full((B, g1), -1, dtype=torch.int64)
    length = torch.zeros(B, dtype=torch.int64)
    p_lse, q_lse = torch.zeros((B, g1), dtype=torch.float64), torch.zeros((B, g), dtype=torch.float64)
    near = []
    for b in range(B):
        p = [soft(target[b, s], T_target) for s in range(g1)]
        q = [soft(draft[b, s], T_draft) for s in range(g)]
        p_lse[b] = torch.tensor([x[1] for x in p])
        q_lse[b] = torch.tensor([x[1] for x in q])
        nd = g if n_drafts is None else min(max(int(n_drafts[b]), 0), g)
        gap = math.inf
        n = 0
        while n < nd:
            x = int(tokens[b, n])
            if not 0 <= x < V:
                break
            left, right = float(u[b, n]) * float(q[n][0][x]), float(p[n][0][x])
            if max(left, right) > 0:
                gap = min(gap, abs(left - right) / max(left, right))
            if not left < right:
                break
            out[b, n] = x
            n += 1
        r = p[n][0].clone()
        if n < nd:
            r = (r - q[n][0]).clamp(min=0)
            if not bool((r > 0).any()):
                r = p[n][0].clone()
        length[b] = n + 1
        score = torch.where(r > 0, e[b].double() / r, math.inf)
        if bool((r > 0).any()):
            low = torch.sort(score).values[:2]
            if len(low) > 1 and float(low[1]) < math.inf and float(low[0]) > 0:
                gap = min(gap, float((low[1] - low[0]) / low[1]))
            out[b, n] = int(score.argmin())
        near.append(gap)
    return out, length, p_lse, q_lse, near
