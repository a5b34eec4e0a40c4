"""What a decoding tenant's operators cost: norms and rotation of queries and keys, a paged cache held in 4 bits (written,
read back and attended over) and sampling, each with its plain form in PyTorch.

``listed()`` are the measured cases, ``draw()`` gives more of the same ranges.  ``run()`` makes one pass: with ``own`` the
calls a user makes of the package, otherwise the plain form.  Sizes: 12 heads of 64 is the framework's encoder tenant, the
other head layouts, lengths and vocabularies are generic.

The cache's layout is the library's public one: keys ``[page][kv head][token][D/2 bytes]``, values
``[page][kv head][block of 32 tokens][feature][16 bytes]``, both in 32-bit words of eight 4-bit codes whose elements
0..7 start at bits 0, 16, 4, 20, 8, 24, 12, 28; scales ``[page][kv head][token][D/64]`` words, bf16 scale in the low half
and bf16 minimum in the high half.  A code c stands for c * scale + minimum.
"""
import math

import torch

own = False

GROUP = 64                                   # features that share a scale
SHIFTS = (0, 16, 4, 20, 8, 24, 12, 28)
# query heads, key/value heads, features per head
LAYOUTS = ((12, 12, 64), (32, 8, 128), (8, 2, 128), (28, 4, 128), (9, 3, 64), (40, 8, 128), (6, 6, 64), (16, 1, 128))


def listed():
    return [
        # one new token of one conversation: a launch's latency
        dict(name="rotary_one_token", op="rotary", dtype="bf16", batch=1, tokens=1, heads=32, kv_heads=8, dim=128, rotary=128, axes=1, interleaved=False),
        # prompts of image and video tokens: three position axes, half of the features rotated
        dict(name="rotary_video_prompts", op="rotary", dtype="bf16", batch=3, tokens=4111, heads=28, kv_heads=4, dim=128, rotary=64, axes=3, interleaved=False),
        # a decoding step of many conversations enters the cache and is read back
        dict(name="cache_step", op="roundtrip", dtype="f32", batch=96, tokens=1, heads=12, kv_heads=12, dim=64, length=1500, page=64),
        # ragged prompts enter the cache at odd places and are read back
        dict(name="cache_prompts", op="roundtrip", dtype="bf16", batch=6, tokens=5001, heads=32, kv_heads=8, dim=128, length=777, page=32),
        # a whole cache read back, to be moved or attended over in full precision
        dict(name="cache_read_back", op="read", dtype="bf16", batch=8, tokens=8192, heads=32, kv_heads=8, dim=128, length=8192, page=64),
        # one conversation of ordinary length, one token: latency
        dict(name="attend_one_short", op="attend", dtype="bf16", batch=1, tokens=1, heads=12, kv_heads=12, dim=64, length=700, page=32, window=0),
        # a decoding step of a full server, ragged lengths
        dict(name="attend_many_ragged", op="attend", dtype="bf16", batch=64, tokens=1, heads=32, kv_heads=8, dim=128, length=8192, page=64, window=0),
        # one token over one very long document
        dict(name="attend_one_long", op="attend", dtype="bf16", batch=1, tokens=1, heads=32, kv_heads=8, dim=128, length=131072, page=256, window=0),
        # a prompt's own attention, all of it new
        dict(name="attend_prompt", op="attend", dtype="bf16", batch=1, tokens=4096, heads=32, kv_heads=8, dim=128, length=0, page=64, window=0),
        # pieces of prompts after a prefix, with a sliding window, in fp32
        dict(name="attend_window_f32", op="attend", dtype="f32", batch=4, tokens=257, heads=12, kv_heads=12, dim=64, length=2100, page=64, window=1024),
        # one answer, the usual filters: latency
        dict(name="sample_one", op="sample", dtype="f32", batch=1, vocab=32000, top_k=50, top_p=0.9, min_p=0.0),
        # a full server over a large vocabulary, nucleus only
        dict(name="sample_many_nucleus", op="sample", dtype="bf16", batch=256, vocab=131072, top_k=0, top_p=0.95, min_p=0.02),
    ]


def _log(rng, lo, hi):
    n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(("rotary", "roundtrip", "read", "attend", "attend", "sample"))
    dtype = rng.choice(("bf16", "f32"))
    h, g, d = rng.choice(LAYOUTS)
    if op == "sample":
        vocab = _log(rng, 1000, 150000)
        return dict(op=op, dtype=dtype, batch=_log(rng, 1, max(1, 2 ** 24 // vocab)), vocab=vocab, top_k=rng.choice((0, 1, _log(rng, 2, 500))),
                    top_p=rng.choice((1.0, round(rng.uniform(0.5, 0.99), 3))), min_p=rng.choice((0.0, round(rng.uniform(0.01, 0.2), 3))))
    batch = _log(rng, 1, 64)
    if op == "rotary":
        return dict(op=op, dtype=dtype, batch=batch, tokens=_log(rng, 1, 5120 // batch), heads=h, kv_heads=g, dim=d,
                    rotary=rng.choice((d, d // 2)), axes=rng.choice((1, 2, 3)), interleaved=rng.choice((False, True)))
    page = rng.choice((32, 64, 128, 256))
    if op in ("roundtrip", "read"):
        tokens = _log(rng, 1, 16384 // batch)
        return dict(op=op, dtype=dtype, batch=batch, tokens=tokens, heads=h, kv_heads=g, dim=d,
                    length=tokens if op == "read" else _log(rng, 1, 2000), page=page)
    tokens = rng.choice((1, 1, _log(rng, 2, 16), _log(rng, 16, 2048)))
    batch = _log(rng, 1, 64 if tokens < 4 else 16 if tokens < 100 else 2)
    length = rng.choice((0, _log(rng, 1, min(65536, 2 ** 18 // batch) if tokens < 100 else 2000)))
    return dict(op=op, dtype=dtype, batch=batch, tokens=tokens, heads=h, kv_heads=g, dim=d, length=length, page=page,
                window=rng.choice((0, 0, _log(rng, 16, 4096))))


# -- what a program has in hand ---------------------------------------------------------------------------------------------

def _spread(case):
    """(tokens cached before the call, new tokens) of each sequence: ragged where there are several, by the case alone."""
    n, length, tokens = case["batch"], case["length"], case["tokens"]
    if case["op"] == "read":
        return [0] * n, [max(1, tokens - tokens * (5 * i % n) // (2 * n)) for i in range(n)]
    start = [length - length * (7 * i % n) // n for i in range(n)]
    return start, [max(1, tokens - tokens * (3 * i % n) // (4 * n)) for i in range(n)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = dict(case, dtype=dtype)
    n = case["batch"]
    if case["op"] == "sample":
        v = case["vocab"]
        logits = 2.5 * normal(n, v)
        logits += 6.0 * (torch.rand((n, v), generator=gen, device="cuda") < 4.0 / v)       # the few words that fit
        logits[:, v - v // 100:] = float("-inf")                                           # padding of the vocabulary
        s["logits"] = logits.to(dtype)
        s["u"] = torch.rand(n, generator=gen, device="cuda")
        s["temperature"] = 0.5 + torch.rand(n, generator=gen, device="cuda")
        s["top_k"] = torch.full((n,), case["top_k"], dtype=torch.int32, device="cuda") if case["top_k"] else None
        s["top_p"] = torch.full((n,), case["top_p"], device="cuda") if case["top_p"] < 1.0 else None
        s["min_p"] = torch.full((n,), case["min_p"], device="cuda") if case["min_p"] > 0.0 else None
        s["tokens_out"] = torch.empty(n, dtype=torch.int32, device="cuda")
        s["logp_out"] = torch.empty(n, device="cuda")
        return s
    h, g, d, t = case["heads"], case["kv_heads"], case["dim"], case["tokens"]
    width = (h + 2 * g) * d
    if case["op"] == "rotary":
        # queries and keys of a product: a few features are much larger than the rest
        s["qkv"] = (normal(n, t, width) * (1.0 + 4.0 * (normal(width).abs() > 2.5))).to(dtype)
        s["out"] = torch.empty_like(s["qkv"])
        s["gamma_q"] = 1.0 + 0.1 * normal(d)
        s["gamma_k"] = 1.0 + 0.1 * normal(d)
        half, reach = case["rotary"] // 2, 8192
        angle = torch.arange(reach, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        s["table"] = torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()      # [position][pair][cos, sin]
        s["positions"] = torch.randint(0, reach, (n, t, case["axes"]), generator=gen, device="cuda", dtype=torch.int32)
        a = case["axes"]
        s["sections"] = [half // a + (i < half % a) for i in range(a)]
        return s
    start, count = _spread(case)
    page = case["page"]
    per = -(-(max(x + y for x, y in zip(start, count))) // page)
    pages = n * per
    s["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    s["count"] = torch.tensor(count, dtype=torch.int32, device="cuda")
    s["page_table"] = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).reshape(n, per)
    for name, shape in (("k", (pages, g, page, d // 2)), ("v", (pages, g, page // 32, d, 16))):
        # codes of bell-shaped values: the sum of two numbers of three bits in each half of a byte
        a, b = (torch.randint(0, 256, shape, generator=gen, device="cuda", dtype=torch.uint8) & 0x77 for _ in range(2))
        s[name + "_codes"] = a + b
        scale = (0.25 + 0.2 * torch.rand((pages, g, page, d // GROUP), generator=gen, device="cuda")).to(torch.bfloat16)
        low = (scale.float() * (-7.0 + 0.5 * normal(pages, g, page, d // GROUP))).to(torch.bfloat16)
        s[name + "_scales"] = torch.stack((scale, low), -1).contiguous().view(torch.int32).squeeze(-1)
    if case["op"] == "read":
        s["out"] = torch.empty((n, t, 2 * g * d), dtype=dtype, device="cuda")
        return s
    s["qkv"] = normal(n, t, width).to(dtype)
    if case["op"] == "roundtrip":
        s["out"] = torch.empty((n, t, 2 * g * d), dtype=dtype, device="cuda")
    else:
        s["out"] = torch.empty((n, t, h * d), dtype=dtype, device="cuda")
        s["scale"] = 1.0 / math.sqrt(d)
    return s


# -- one pass ---------------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    return {"rotary": _rotary, "roundtrip": _roundtrip, "read": _read, "attend": _attend, "sample": _sample}[state["op"]](state)


def _run_own(s):
    if "session" not in s:                   # the loaded operator list: what a program keeps
        from paper_2304_11745_amd import tokens as T
        ops = T.OpList(s["dtype"], s["batch"])
        layout = dict(heads=s["heads"], kv_heads=s["kv_heads"], head_dim=s["dim"]) if s["op"] != "sample" else {}
        if s["op"] == "rotary":
            ops.qknorm_rope(s["qkv"], s["out"], s["positions"], s["table"], gamma_q=s["gamma_q"], gamma_k=s["gamma_k"], eps=1e-6,
                            rotary_dims=s["rotary"], sections=s["sections"], interleaved=s["interleaved"], **layout)
        elif s["op"] == "sample":
            ops.sample(s["logits"], s["tokens_out"], s["u"], logp=s["logp_out"], temperature=s["temperature"], top_k=s["top_k"],
                       top_p=s["top_p"], min_p=s["min_p"])
        else:
            cache = T.Cache(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"], s["page_table"])
            if s["op"] == "roundtrip":
                ops.cache_write(s["qkv"], cache, s["start"], s["count"], **layout)
            if s["op"] in ("roundtrip", "read"):
                ops.cache_read(s["out"], cache, s["start"], s["count"])
            else:
                ops.cache_attention(s["qkv"], s["out"], cache, s["start"], s["count"], scale=s["scale"], window=s["window"], **layout)
        s["session"] = T.TokenSession([ops])
    s["session"].enqueue(0)
    return {"tokens": s["tokens_out"], "logp": s["logp_out"]} if s["op"] == "sample" else s["out"]


def _rotary(s):
    h, g, d, half = s["heads"], s["kv_heads"], s["dim"], s["rotary"] // 2
    n, t = s["batch"], s["tokens"]
    x = s["qkv"].float().reshape(n, t, h + 2 * g, d)
    q, k, v = x[:, :, :h], x[:, :, h:h + g], x[:, :, h + g:]
    q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * s["gamma_q"]
    k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * s["gamma_k"]
    y = torch.cat((q, k), 2)
    axis = torch.repeat_interleave(torch.arange(s["axes"], device="cuda"), torch.tensor(s["sections"], device="cuda"))
    at = s["positions"].long()[:, :, axis]                                                 # [n, t, half]
    cs = s["table"][at, torch.arange(half, device="cuda")]
    c, si = cs[..., 0][:, :, None], cs[..., 1][:, :, None]
    if s["interleaved"]:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack((a * c - b * si, b * c + a * si), -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat((a * c - b * si, b * c + a * si), -1)
    y = torch.cat((turned, y[..., 2 * half:]), -1)
    return torch.cat((y, v), 2).reshape(n, t, -1).to(s["dtype"])


def _quantised(x):
    """x [..., D] as the values its 4-bit codes stand for."""
    y = x.reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    low, scale = lo.to(torch.bfloat16).float(), ((hi - lo) / 15.0).to(torch.bfloat16).float()
    codes = torch.where(scale > 0, torch.round((y - low) / scale).clamp(0, 15), torch.zeros_like(y))
    return (codes * scale + low).reshape(x.shape)


def _valid(s):
    return torch.arange(s["tokens"], device="cuda")[None] < s["count"][:, None]             # [n, t]


def _roundtrip(s):
    h, g, d = s["heads"], s["kv_heads"], s["dim"]
    x = s["qkv"].float()[..., h * d:].reshape(s["batch"], s["tokens"], 2 * g, d)
    y = _quantised(x).reshape(s["batch"], s["tokens"], -1)
    return torch.where(_valid(s)[..., None], y, torch.zeros_like(y)).to(s["dtype"])


def _values(s, name):
    """The cache's keys or values in 32 bits, [n, g, pages * page, D]."""
    shifts = torch.tensor(SHIFTS, device="cuda", dtype=torch.int32)
    at = s["page_table"].long()
    words = s[name + "_codes"][at].view(torch.int32)
    codes = ((words[..., None] >> shifts) & 15).float()
    n, per, g, page = s["batch"], at.shape[1], s["kv_heads"], s["page"]
    if name == "k":
        codes = codes.reshape(n, per, g, page, s["dim"])
    else:
        codes = codes.reshape(n, per, g, page // 32, s["dim"], 32).transpose(-1, -2).reshape(n, per, g, page, s["dim"])
    pair = s[name + "_scales"][at].contiguous().view(torch.bfloat16).float().reshape(n, per, g, page, s["dim"] // GROUP, 2)
    scale, low = (pair[..., i].repeat_interleave(GROUP, -1) for i in range(2))
    return (codes * scale + low).transpose(1, 2).reshape(n, g, per * page, s["dim"])


def _read(s):
    t = s["tokens"]
    y = torch.cat([_values(s, name).transpose(1, 2)[:, :t].reshape(s["batch"], -1, s["kv_heads"] * s["dim"]) for name in ("k", "v")], -1)
    if y.shape[1] < t:
        y = torch.cat((y, y.new_zeros(y.shape[0], t - y.shape[1], y.shape[2])), 1)
    return torch.where(_valid(s)[..., None], y, torch.zeros_like(y)).to(s["dtype"])


def _attend(s):
    h, g, d, n, t = s["heads"], s["kv_heads"], s["dim"], s["batch"], s["tokens"]
    k, v = _values(s, "k"), _values(s, "v")
    q = s["qkv"].float()[..., :h * d].reshape(n, t, g, h // g, d).permute(0, 2, 3, 1, 4).reshape(n, g, (h // g) * t, d)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]
    at = s["start"].long()[:, None] + torch.arange(t, device="cuda")                        # [n, t]
    key = torch.arange(k.shape[2], device="cuda")
    seen = (key <= at[..., None]) & _valid(s)[..., None]                                    # [n, t, keys]
    if s["window"]:
        seen &= key > at[..., None] - s["window"]
    scores = scores.reshape(n, g, h // g, t, -1).masked_fill(~seen[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p.reshape(n, g, (h // g) * t, -1), v).reshape(n, g, h // g, t, d)
    y = torch.where(total > 0, y / total, torch.zeros_like(y))
    return y.permute(0, 3, 1, 2, 4).reshape(n, t, h * d).to(s["dtype"])


def _sample(s):
    # Weights are whole numbers, so that their sums are the same in every order.
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x)
    n, v = x.shape
    top = x.amax(-1, keepdim=True)
    temperature = s["temperature"][:, None]
    part = torch.where(x == top, torch.ones_like(x), torch.exp((x - top) / temperature))
    weight = (part * 2.0 ** 31).to(torch.int64)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    w, rank = weight.gather(1, order), torch.arange(v, device="cuda")[None]
    if s["top_k"] is not None:
        w = torch.where(rank < s["top_k"].long()[:, None], w, torch.zeros_like(w))
    if s["top_p"] is not None:
        cum = w.cumsum(-1)
        reach = s["top_p"].double()[:, None] * cum[:, -1:].double()
        w = torch.where((rank == 0) | ((cum - w).double() < reach), w, torch.zeros_like(w))
    if s["min_p"] is not None:
        w = torch.where((rank == 0) | (part.gather(1, order) >= s["min_p"][:, None]), w, torch.zeros_like(w))
    cum = torch.zeros_like(w).scatter(1, order, w).cumsum(-1)
    total = cum[:, -1:]
    goal = torch.minimum((s["u"].double()[:, None] * total.double()).floor().to(torch.int64), total - 1)
    token = (cum <= goal).sum(-1, keepdim=True)
    picked = x.gather(1, token)
    logp = torch.where(picked == top, torch.zeros_like(top), (picked - top) / temperature) - torch.log(total.float() * 2.0 ** -31)
    return {"tokens": token[:, 0].to(torch.int32), "logp": logp[:, 0]}


# -- the same from the definitions, in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "roundtrip": _exact_roundtrip, "read": _exact_read, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](s)


def _exact_rotary(s):
    h, g, d = s["heads"], s["kv_heads"], s["dim"]
    y = s["qkv"].double().clone().view(s["batch"], s["tokens"], h + 2 * g, d)
    for lo, hi, gamma in ((0, h, s["gamma_q"]), (h, h + g, s["gamma_k"])):
        part = y[:, :, lo:hi]
        y[:, :, lo:hi] = part / ((part ** 2).sum(-1, keepdim=True) / d + 1e-6).sqrt() * gamma.double()
    pair = 0
    before = y.clone()
    for axis, size in enumerate(s["sections"]):
        for _ in range(size):
            cs = s["table"][s["positions"][:, :, axis].long(), pair].double()[:, :, None]
            i, j = (2 * pair, 2 * pair + 1) if s["interleaved"] else (pair, pair + s["rotary"] // 2)
            a, b = before[:, :, :h + g, i], before[:, :, :h + g, j]
            y[:, :, :h + g, i] = a * cs[..., 0] - b * cs[..., 1]
            y[:, :, :h + g, j] = b * cs[..., 0] + a * cs[..., 1]
            pair += 1
    return y.reshape(s["batch"], s["tokens"], -1)


def _exact_roundtrip(s):
    n, t, g, d = s["batch"], s["tokens"], s["kv_heads"], s["dim"]
    out = torch.zeros(n, t, 2 * g * d, dtype=torch.float64, device="cuda")
    for i, c in enumerate(s["count"].tolist()):
        x = s["qkv"][i, :c, s["heads"] * d:].double().reshape(c, 2 * g * d // GROUP, GROUP)
        lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
        low, step = lo.bfloat16().double(), ((hi - lo) / 15).bfloat16().double()
        codes = ((x - low) / step.clamp_min(1e-300)).round().clamp(0, 15) * (step > 0)
        out[i, :c] = (low + step * codes).reshape(c, -1)
    return out


def _exact_item(s, i, name, length):
    """Keys or values of sequence i, [length, g, D]."""
    d, g, page = s["dim"], s["kv_heads"], s["page"]
    at = s["page_table"][i, :-(-length // page)].long()
    raw = s[name + "_codes"][at].long()
    pair = s[name + "_scales"][at]
    scale = (pair << 16).view(torch.float32).double()
    low = (pair & -65536).view(torch.float32).double()
    half = torch.stack((raw & 15, raw >> 4), -1).flatten(-2).unflatten(-1, (-1, 8))       # 4-bit pieces of each word, lowest first
    codes = torch.stack([half[..., b // 4] for b in SHIFTS], -1).flatten(-2).double()
    if name == "v":
        codes = codes.permute(0, 1, 2, 4, 3).reshape(len(at), g, page, d)
    value = codes.unflatten(-1, (-1, GROUP)) * scale[..., None] + low[..., None]
    return value.flatten(-2).transpose(1, 2).reshape(-1, g, d)[:length]


def _exact_read(s):
    n, t, width = s["batch"], s["tokens"], s["kv_heads"] * s["dim"]
    out = torch.zeros(n, t, 2 * width, dtype=torch.float64, device="cuda")
    for i, c in enumerate(s["count"].tolist()):
        out[i, :c, :width] = _exact_item(s, i, "k", c).reshape(c, -1)
        out[i, :c, width:] = _exact_item(s, i, "v", c).reshape(c, -1)
    return out


def _exact_attend(s):
    h, g, d, n, t = s["heads"], s["kv_heads"], s["dim"], s["batch"], s["tokens"]
    out = torch.zeros(n, t, h, d, dtype=torch.float64, device="cuda")
    for i, (b, c) in enumerate(zip(s["start"].tolist(), s["count"].tolist())):
        k, v = (_exact_item(s, i, name, b + c) for name in ("k", "v"))
        q = s["qkv"][i, :c, :h * d].double().reshape(c, h, d)
        at = torch.arange(b, b + c, device="cuda")[:, None]
        key = torch.arange(b + c, device="cuda")[None]
        hidden = (key > at) | ((key <= at - s["window"]) if s["window"] else torch.zeros_like(key, dtype=torch.bool))
        for j in range(h):
            w = (q[:, j] @ k[:, j // (h // g)].T.contiguous() * s["scale"]).masked_fill(hidden, -math.inf).softmax(-1)
            out[i, :c, j] = w @ v[:, j // (h // g)]
    return out.reshape(n, t, h * d)


def _exact_sample(s):
    # None where a row's random number lies so near the line between two words that 32-bit weights may fall on either side of it.
    token, logp = [], []
    for i in range(s["batch"]):
        x = s["logits"][i].double()
        w = ((x - x.max()) / s["temperature"][i].double()).exp()
        keep = torch.argsort(x, descending=True, stable=True)
        if s["top_k"] is not None:
            keep = keep[:int(s["top_k"][i])]
        if s["top_p"] is not None:
            before = w[keep].cumsum(0) - w[keep]
            line = s["top_p"][i].double() * w[keep].sum()
            if (before - line).abs().min() < 2e-7 * line:
                return None
            keep = keep[before < line]
        if s["min_p"] is not None:
            keep = keep[w[keep] >= s["min_p"][i].double()]
        keep = keep.sort().values
        cum = w[keep].cumsum(0)
        goal = s["u"][i].double() * cum[-1]
        if (cum - goal).abs().min() < 2e-7 * cum[-1]:
            return None
        at = int((cum <= goal).sum())
        token.append(int(keep[at]))
        logp.append(float((w[keep[at]] / cum[-1]).log()))
    return {"tokens": torch.tensor(token, dtype=torch.int32), "logp": torch.tensor(logp, dtype=torch.float64)}


# -- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    n = case["batch"]
    if case["op"] == "sample":
        return {"bytes": n * (case["vocab"] * e + 24), "flops": n * case["vocab"] * 4}
    h, g, d, t = case["heads"], case["kv_heads"], case["dim"], case["tokens"]
    if case["op"] == "rotary":
        return {"bytes": n * t * (2 * (h + 2 * g) * d * e + 4 * case["axes"]) + min(n * t, 8192) * case["rotary"] * 4, "flops": n * t * (h + g) * d * 8}
    start, count = _spread(case)
    token = 2 * g * (d // 2 + 4 * d // GROUP)              # keys and values of one token in the cache
    if case["op"] == "read":
        return {"bytes": sum(count) * token + n * t * 2 * g * d * e, "flops": sum(count) * 4 * g * d}
    if case["op"] == "roundtrip":
        return {"bytes": sum(count) * (2 * g * d * e + 2 * token) + n * t * 2 * g * d * e, "flops": sum(count) * 12 * g * d}
    window, pairs, keys = case["window"], 0, 0
    for b, c in zip(start, count):
        full = max(0, min(c, window - b)) if window else c  # queries that see every key before them
        pairs += full * b + full * (full + 1) // 2 + (c - full) * window
        keys += min(b + c, window + c - 1) if window else b + c
    return {"bytes": keys * token + sum(count) * h * d * e + n * t * h * d * e, "flops": 4 * pairs * h * d}
