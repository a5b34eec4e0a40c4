"""Plain implementations of the operators of a decoding tenant (definitions in include/gacer.h), in 64 bits on the CPU unless the definition
itself says 32, and inputs for their tests.  Nothing here uses the library."""
import numpy as np
import torch

GROUP = 64
SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)


def bf16(x):
    return torch.as_tensor(x, dtype=torch.float32).to(torch.bfloat16).float()


# -- norm and rotation ---------------------------------------------------------------------------------------------------------------
def qknorm_rope(qkv, heads, kv_heads, dim, positions, table, gamma_q, gamma_k, eps, rotary, sections, interleaved):
    x = qkv.double().clone().reshape(*qkv.shape[:2], heads + 2 * kv_heads, dim)
    for lo, hi, gamma in ((0, heads, gamma_q), (heads, heads + kv_heads, gamma_k)):
        if gamma is not None:
            part = x[:, :, lo:hi]
            x[:, :, lo:hi] = part / torch.sqrt((part ** 2).mean(-1, keepdim=True) + eps) * gamma.double()
    y = x.clone()
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    for b in range(qkv.shape[0]):
        for t in range(qkv.shape[1]):
            for i in range(rotary // 2):
                p = int(positions[b, t, axis[i]])
                c, s = (table[p, i].double() if 0 <= p < table.shape[0] else torch.full((2,), float("nan"), dtype=torch.float64))
                f0, f1 = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
                u, v = x[b, t, :heads + kv_heads, f0], x[b, t, :heads + kv_heads, f1]
                y[b, t, :heads + kv_heads, f0] = u * c - v * s
                y[b, t, :heads + kv_heads, f1] = v * c + u * s
    return y.reshape(qkv.shape)


# -- cache ---------------------------------------------------------------------------------------------------------------------------
def quantise(x):
    """float32 [..., D] -> codes uint8 [..., D], scale and minimum float32 [..., D/64], in fp32 as defined."""
    g = x.float().reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = g.min(-1).values, g.max(-1).values
    bad = ~torch.isfinite(g).all(-1)
    scale, low = bf16((hi - lo) * torch.tensor(1 / 15, dtype=torch.float32)), bf16(lo) + 0.0                  # a minimum of zero is stored without a sign
    bad |= ~torch.isfinite(scale) | ~torch.isfinite(low)
    c = torch.round((g - low[..., None]) / scale[..., None]).clamp(0, 15)
    c = torch.where((scale > 0)[..., None] & ~bad[..., None], c, torch.zeros_like(c))
    scale = torch.where(bad, torch.full_like(scale, float("nan")), scale)
    low = torch.where(bad, torch.zeros_like(low), low)
    return c.reshape(x.shape).to(torch.uint8), scale, low


def words(codes):
    """uint8 codes [..., 8 n] -> int32 words [..., n]"""
    c = codes.numpy().astype(np.uint32).reshape(*codes.shape[:-1], -1, 8)
    w = np.zeros(c.shape[:-1], np.uint32)
    for e, s in enumerate(SHIFTS):
        w |= c[..., e] << np.uint32(s)
    return torch.from_numpy(w.view(np.int32))


def codes_of(w):
    w = w.numpy().view(np.uint32)
    return torch.from_numpy(np.stack([(w >> np.uint32(s)) & 15 for s in SHIFTS], -1).reshape(*w.shape[:-1], -1).astype(np.uint8))


def pairs(scale, low):
    s, m = (torch.where(torch.isnan(t), torch.full_like(t, 0x7FC0, dtype=torch.int32), t.to(torch.bfloat16).view(torch.int16).int() & 0xFFFF).numpy().astype(np.uint32)
            for t in (scale, low))
    return torch.from_numpy((s | (m << np.uint32(16))).view(np.int32))


class RefCache:
    """A cache on the CPU in the library's layout."""

    def __init__(self, pages, kv_heads, page, dim, table, fill=None):
        self.k = torch.zeros(pages, kv_heads, page, dim // 2, dtype=torch.uint8)
        self.v = torch.zeros(pages, kv_heads, page // 32, dim, 16, dtype=torch.uint8)
        self.ks = torch.zeros(pages, kv_heads, page, dim // GROUP, dtype=torch.int32)
        self.vs = torch.zeros_like(self.ks)
        self.table, self.page, self.dim, self.kv_heads, self.pages = table, page, dim, kv_heads, pages
        if fill is not None:                               # every token of every page holds something
            g = fill
            for codes in (self.k, self.v):
                codes.copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
            for s in (self.ks, self.vs):
                scale = 0.1 + 0.3 * torch.rand(s.shape, generator=g)
                s.copy_(pairs(scale, -7.5 * scale + 0.3 * torch.randn(s.shape, generator=g)))

    def where(self, b, p):
        i = p // self.page
        if i >= self.table.shape[1]:
            return None
        page = int(self.table[b, i])
        return (page, p % self.page) if 0 <= page < self.pages else None

    def write(self, b, p, k, v):
        """k, v float32 [kv_heads, D] of one token"""
        at = self.where(b, p)
        if at is None:
            return
        page, o = at
        for codes, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            c, s, m = quantise(x)
            scales[page, :, o] = pairs(s, m)
            if codes is self.k:
                codes[page, :, o] = words(c).view(torch.uint8).reshape(self.kv_heads, -1)
            else:
                block = codes[page, :, o // 32].view(torch.int32)              # [kv_heads, D, 4]
                old = codes_of(block)                                          # [kv_heads, D, 32]
                old[:, :, o % 32] = c
                codes[page, :, o // 32] = words(old).view(torch.uint8).reshape(self.kv_heads, self.dim, 16)

    def value(self, b, p, which):
        """float64 [kv_heads, D] of one token, None where there is no page"""
        at = self.where(b, p)
        if at is None:
            return None
        page, o = at
        if which == "k":
            c, s = codes_of(self.k[page, :, o].contiguous().view(torch.int32)), self.ks[page, :, o]
        else:
            c, s = codes_of(self.v[page, :, o // 32].contiguous().view(torch.int32))[:, :, o % 32], self.vs[page, :, o]
        scale = (s.long() << 16).to(torch.int32).view(torch.float32).double()
        low = (s & -65536).view(torch.float32).double()
        return (c.double().reshape(self.kv_heads, -1, GROUP) * scale[..., None] + low[..., None]).reshape(self.kv_heads, self.dim)

    def span(self, b, start, count, tokens):
        s, c = int(start[b]), tokens if count is None else max(0, min(int(count[b]), tokens))
        return (0, 0) if s < 0 or s > self.table.shape[1] * self.page else (s, c)


def attention(cache, qkv, heads, start, count, scale, window):
    """Returns (out, weight): the result, and sum_j p_j |v_j|, which rounding errors are measured by; both float64 [B, S, heads * D]."""
    n, t = qkv.shape[:2]
    d, g = cache.dim, cache.kv_heads
    out, weight = (torch.zeros(n, t, heads, d, dtype=torch.float64) for _ in range(2))
    for b in range(n):
        s, c = cache.span(b, start, count, t)
        keys = {p: (cache.value(b, p, "k"), cache.value(b, p, "v")) for p in range(max(0, s - window + 1) if window else 0, s + c) if cache.where(b, p)}
        for i in range(c):
            seen = [p for p in keys if p <= s + i and (not window or p > s + i - window)]
            if not seen:
                continue
            k, v = (torch.stack([keys[p][j] for p in seen]) for j in range(2))
            for h in range(heads):
                q = qkv[b, i, h * d:(h + 1) * d].double()
                w = torch.softmax(k[:, h // (heads // g)] @ q * scale, 0)
                out[b, i, h] = w @ v[:, h // (heads // g)]
                weight[b, i, h] = w @ v[:, h // (heads // g)].abs()
    return out.reshape(n, t, -1), weight.reshape(n, t, -1)


# -- sampling ------------------------------------------------------------------------------------------------------------------------
def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logp, margin) of one row (float64 weights of the 32-bit parts): margin is how far, relative to the total, the random
    number and the nucleus stay from a line between two tokens; a 32-bit evaluation agrees where it is well above 1e-7."""
    x = x.astype(np.float32).astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, -np.inf, 1.0
    order = np.lexsort((np.arange(x.size), -x))
    if temperature > 0:
        with np.errstate(invalid="ignore", over="ignore"):
            e = np.where(x == top, 1.0, np.exp((x - top) / temperature))
    else:
        e, top_k = (x == top).astype(np.float64), 1
    if not top_p > 0 or not min_p <= 1:
        top_k = 1
    w = np.floor(e * 2.0 ** 31) / 2.0 ** 31
    margin = 1.0
    keep = order[:top_k] if top_k > 0 else order
    if top_p < 1 and top_k != 1:
        cum = np.cumsum(w[keep])
        reach = top_p * cum[-1]
        margin = min(margin, np.abs(cum - reach).min() / cum[-1])
        keep = keep[cum - w[keep] < reach]
    if top_k != 1:
        margin = min(margin, np.abs(e[keep] - min_p).min() if min_p > 0 else 1.0)
        keep = keep[(e[keep] >= min_p) | (keep == order[0])]
    keep = np.sort(keep)
    keep = keep[w[keep] > 0]
    cum = np.cumsum(w[keep])
    goal = u * cum[-1]
    if cum.size > 1:
        margin = min(margin, np.abs(cum[:-1] - goal).min() / cum[-1])
    token = keep[min(int((cum <= goal).sum()), keep.size - 1)]
    logp = (0.0 if x[token] == top else (x[token] - top) / temperature) - np.log(cum[-1])
    return int(token), float(logp), margin
