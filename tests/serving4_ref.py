"""Plain 64-bit implementations of the operators over a cache held in 4 bits, of the reservation of places and of the
adjustment of logits, on the CPU, and the inputs of their tests."""
import math

import torch

import serving_ref as ref

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def encode(x, near=None, computed=None):
    """Codes [..., 16 n] and scale bytes [..., n] (uint8) of x [..., D] float64, n = ceil(D / 32).  near: a relative
    distance; the third result then says which groups have one of the first `computed` elements as near to a border of two
    codes (or to one of two scales), so that arithmetic of that precision may take either.  The others are given, not
    computed: borders are theirs exactly."""
    D = x.shape[-1]
    computed = D if computed is None else computed
    n = -(-D // 32)
    g = torch.nn.functional.pad(x, (0, 32 * n - D)).unflatten(-1, (n, 32))
    top = g.abs().amax(-1)
    none = ~torch.isfinite(top) | (top >= 2.0 ** 128)
    m, e = torch.frexp(torch.where(none, 1.0, top))  # top = m 2^e, 0.5 <= m < 1
    # the least k in [-126, 125] with top <= 7 * 2^k, exactly; 125 where there is none
    k = torch.where(top > 0, torch.where(m <= 0.875, e - 3, e - 2), -126).clamp(-126, 125)
    a = torch.where(none[..., None], 0.0, g.abs()) * (2.0 ** -k.double())[..., None]
    borders = torch.tensor([(p + q) / 2 for p, q in zip(LEVELS, LEVELS[1:])], dtype=torch.float64)
    code = torch.where(none[..., None], 0, 8 * torch.signbit(g).long())
    close = torch.zeros(top.shape, dtype=torch.bool)
    given = torch.arange(32 * n).unflatten(0, (n, 32)) >= computed
    for i, border in enumerate(borders):
        # the border belongs to the even code: the lower one if that is even
        code += (a > border) if i % 2 == 0 else (a >= border)
    if near is not None:
        for border in borders.tolist() + [3.5, 7.0]:  # (the scale changes past the last two)
            close |= (((a - border).abs() <= near * border) & ~given).any(-1)
    code = code.flatten(-2)
    out = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), torch.where(none, 255, k + 127).to(torch.uint8)
    return out if near is None else out + (close,)


def decode(codes, scales, D):
    """The values [..., D] (float64) of codes and scale bytes."""
    levels = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)
    x = torch.stack((levels[(codes & 15).long()], levels[(codes >> 4).long()]), -1).flatten(-2)
    scale = torch.where(scales == 255, math.nan, 2.0 ** (scales.double() - 127))
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)[..., :D]


class Sequences4(ref.Sequences):
    """Sequences whose keys and values are held in 4 bits; k and v are what the codes stand for, unused places NaN."""

    def __init__(self, lens, G, D, P, dtype, seed=0, layers=None, heads_first=True, **more):
        super().__init__(lens, G, D, P, torch.float64, seed=seed, layers=layers, heads_first=heads_first, **more)
        self.rows_dtype = dtype
        self.pack()

    def pack(self):
        """Codes of the present k and v; k and v become their values."""
        self.kc, self.ks = encode(self.k)
        self.vc, self.vs = encode(self.v)
        self.k, self.v = decode(self.kc, self.ks, self.D), decode(self.vc, self.vs, self.D)

    def handles(self, psd, max_new=None, max_kv=None):
        pools = [self.device(t) for t in (self.kc, self.vc, self.ks, self.vs)]
        cache = psd.make_cache4(*pools, self.D, dtype=self.rows_dtype)
        seqs = psd.make_seqs(torch.tensor(self.new_start, dtype=torch.int32).cuda(),
                             torch.tensor([kv for _, kv in self.lens], dtype=torch.int32).cuda(), self.table.cuda(), self.rows,
                             max_new or max(1, max(n for n, _ in self.lens)), max_kv or max(1, max(kv for _, kv in self.lens)))
        return cache, seqs, pools


class Pool:
    """Free pages and what sequences hold, as the reservation defines them."""

    def __init__(self, pages, P, B, width, order=None, first=0):
        self.pages, self.P, self.width = pages, P, width
        self.free = list(range(pages)) if order is None else list(order)
        self.first, self.ring = first, [None] * pages
        for i, p in enumerate(self.free):
            self.ring[(first + i) % pages] = p
        self.table = [[-1] * width for _ in range(B)]
        self.held = [0] * B

    def reserve(self, n_new, have, rows, max_new, max_kv):
        """granted, new_start, kv_len, row_seq, positions, slots (rows past the last: -1)."""
        P, B = self.P, len(n_new)
        most = min(max_kv, self.width * P)
        asked = needed = 0
        available = len(self.free)
        granted, taken = [], []
        have = [min(max(h, 0), most) for h in have]
        for b in range(B):
            n = max(n_new[b], 0)
            if n > max_new or have[b] + n > most:
                n = 0
            need = max(-(-(have[b] + n) // P) - self.held[b], 0)
            asked += n
            needed += need
            ok = asked <= rows and (need == 0 or needed <= available)
            granted.append(n if ok else 0)
            taken.append(need if ok else 0)
        back = []
        took = 0
        for b in range(B):
            keep = -(-(have[b] + granted[b]) // P)
            for j in range(keep, self.held[b]):
                back.append(self.table[b][j])
                self.table[b][j] = -1
            held = min(self.held[b], keep)
            if taken[b]:
                held = self.held[b]
                for _ in range(taken[b]):
                    self.table[b][held] = self.free[took]
                    took += 1
                    held += 1
            self.held[b] = held
        for i, p in enumerate(back):
            self.ring[(self.first + len(self.free) + i) % self.pages] = p
        self.first = (self.first + took) % self.pages
        self.free = self.free[took:] + back
        start = [0]
        seq, pos, slot = [], [], []
        for b in range(B):
            for i in range(granted[b]):
                c = have[b] + i
                seq.append(b)
                pos.append(c)
                slot.append(self.table[b][c // P] * P + c % P)
            start.append(len(seq))
        pad = rows - len(seq)
        return (granted, start, [have[b] + granted[b] for b in range(B)], seq + [-1] * pad, pos + [-1] * pad, slot + [-1] * pad)


def adjust(logits, text=None, length=None, text_from=None, drafts=None, depth0=0, rho=None, presence=None, frequency=None,
           bias_tokens=None, bias=None, allowed=None):
    """Adjusted logits in float64 [B][K][S][V], and the size of what is added up in each."""
    B, K, S, V = logits.shape
    out, size = logits.double().clone(), torch.zeros((B, K, S, V), dtype=torch.float64)
    for b in range(B):
        counts = torch.zeros(V, dtype=torch.int64)
        if text is not None:
            at = max(0, int(text_from[b])) if text_from is not None else 0
            for x in text[b, at:max(at, min(int(length[b]), text.shape[1]))].tolist():
                if 0 <= x < V:
                    counts[x] += 1
        r = 1.0 if rho is None else float(rho[b])
        p = 0.0 if presence is None else float(presence[b])
        f = 0.0 if frequency is None else float(frequency[b])
        for k in range(K):
            for s in range(S):
                c = counts.clone()
                if drafts is not None:
                    for x in drafts[b, k, :depth0 + s].tolist():
                        if 0 <= x < V:
                            c[x] += 1
                z = logits[b, k, s].double()
                y = torch.where(z > 0, z / r, z * r)
                size[b, k, s] = torch.where(c > 0, y.abs() + (f * c).abs() + abs(p), z.abs())
                z = torch.where(c > 0, y - (f * c + p), z)
                if bias_tokens is not None:
                    for v, w in zip(bias_tokens[b].tolist(), bias[b].tolist()):
                        if 0 <= v < V:
                            z[v] += w
                            size[b, k, s, v] += abs(w)
                if allowed is not None:
                    words = allowed[b] if allowed.dim() == 2 else allowed[b, k, s]
                    bits = (words.long()[:, None] >> torch.arange(32)) & 1
                    z = torch.where(bits.flatten()[:V] > 0, z, -math.inf)
                out[b, k, s] = z
    return out, size
