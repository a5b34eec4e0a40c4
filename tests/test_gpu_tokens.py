"""Operators of a decoding tenant on the GPU against plain implementations in 64 bits (tests/tokens_ref.py).

Tolerances.  A bf16 result is one rounding (half a unit in the last place, 2^-8 of it at most) of an fp32 value.  Norm and rotation: some
twenty fp32 roundings, 2^-19 of the pair's size.  Codes, scales and minima are defined in fp32: equal bits.  Attention: a score is a sum
of D products of a query of unit size with at most 16 (a code below 32 times its scale, minima included), whose partial sums grow as sqrt(D);
64 roundings of that, 2^-24 each, move a score by 64 2^-24 alpha sqrt(D) 16, and a weight by twice that relatively; the sums over keys add
2^-20, and bf16 weights of bf16 tenants 2^-8.  All of it is relative to sum_j p_j |v_j| (with half of the codes' range added: 16 scales),
which the reference returns.  Tokens: equal, where the reference's margin says that 32 bits decide."""
import ctypes as C

import numpy as np
import pytest
import torch

import tokens_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def session(build, dtype, batch):
    from paper_2304_11745_amd import tokens as T
    ops = T.OpList(DT[dtype], batch)
    build(ops)
    return T.TokenSession([ops])


def dev(t):
    return None if t is None else t.cuda().contiguous()


def on_gpu(ref):
    from paper_2304_11745_amd import tokens as T
    return T.Cache(dev(ref.k), dev(ref.v), dev(ref.ks), dev(ref.vs), dev(ref.table))


# -- norm and rotation ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,tokens,heads,kv,dim,rotary,sections,interleaved,norms,in_place", [
    (1, 1, 4, 4, 64, 64, [32], False, "qk", False),
    (2, 7, 6, 2, 128, 128, [64], True, "qk", True),
    (3, 5, 9, 3, 64, 32, [6, 10], False, "q", False),          # sections that end inside a lane's four pairs
    (1, 33, 5, 1, 128, 96, [15, 17, 16], True, "k", True),
    (2, 3, 7, 7, 96, 48, [24], False, "qk", False),            # heads that fill three quarters of their lanes
    (1, 2, 3, 3, 8, 0, [0], False, "qk", False),               # the smallest head, nothing rotated
    (1, 3, 2, 1, 512, 512, [100, 100, 56], False, "", False),
    (2, 2, 2, 2, 16, 16, [0, 8], False, "qk", True),           # an axis without pairs
    (700, 9, 3, 3, 40, 32, [16], False, "qk", False),          # more workgroups than the small form takes
])
def test_norm_and_rotation(dtype, batch, tokens, heads, kv, dim, rotary, sections, interleaved, norms, in_place):
    g = gen(dim + tokens)
    big = batch > 100
    qkv = (3 * torch.randn(batch, tokens, (heads + 2 * kv) * dim, generator=g)).to(DT[dtype])
    qkv[0, 0, :dim] = 0                                        # a head of zeros: its norm is eps alone
    gq = 1 + 0.2 * torch.randn(dim, generator=g) if "q" in norms else None
    gk = 1 + 0.2 * torch.randn(dim, generator=g) if "k" in norms else None
    reach = 50
    angle = torch.rand(reach, max(1, rotary // 2), generator=g) * 6.28
    table = torch.stack((angle.cos(), angle.sin()), -1)[:, :rotary // 2]
    positions = torch.randint(0, reach, (batch, tokens, len(sections)), generator=g, dtype=torch.int32)
    if rotary:
        positions[0, -1, 0] = reach                            # out of the table
        positions[-1, 0, -1] = -1
    x = dev(qkv)
    out = x if in_place else torch.full_like(x, 7.0)
    s = session(lambda o: o.qknorm_rope(x, out, dev(positions) if rotary else None, dev(table) if rotary else None, heads=heads, kv_heads=kv, head_dim=dim,
                                        gamma_q=dev(gq), gamma_k=dev(gk), eps=1e-5, rotary_dims=rotary, sections=sections, interleaved=interleaved), dtype, batch)
    s.enqueue()
    torch.cuda.synchronize()
    got = out.cpu()
    if big:                                                    # the reference is slow: the ends and some between
        pick = [0, 1, 350, 698, 699]
        qkv, positions, got = qkv[pick], positions[pick], got[pick]
    want = R.qknorm_rope(qkv, heads, kv, dim, positions, table, gq, gk, 1e-5, rotary, sections, interleaved)
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad)
    split = (heads + kv) * dim
    assert torch.equal(got[..., split:], qkv[..., split:])
    size = want[..., :split].nan_to_num().abs().amax()
    err = (got.double() - want).nan_to_num().abs()[..., :split]
    assert (err <= (2.0 ** -8 if dtype == "bf16" else 0) * want[..., :split].nan_to_num().abs() + 2.0 ** -19 * size).all()
    s.close()


# -- cache ---------------------------------------------------------------------------------------------------------------------------
def awkward_values(g, *shape):
    """keys and values with what a quantiser can get wrong: constant groups, huge and tiny ones, infinities, NaN"""
    x = torch.randn(*shape, generator=g)
    flat = x.reshape(-1, R.GROUP)
    n = flat.shape[0]
    kinds = torch.randint(0, 12, (n,), generator=g)
    flat[kinds == 0] = 1.5
    flat[kinds == 1] = 0.0
    flat[kinds == 2] *= 1e30
    flat[kinds == 3] *= 1e-30
    flat[kinds == 4] += 100.0
    flat[(kinds == 5).nonzero()[:2, 0], 3] = float("inf")
    flat[(kinds == 6).nonzero()[:2, 0], 60] = float("nan")
    flat[(kinds == 7).nonzero()[:2, 0], 0] = float("-inf")
    flat[kinds == 8] *= 1e-44
    return x


CACHES = [  # page, dim, heads, kv, tokens, starts, counts
    (32, 64, 4, 4, 1, [0, 31, 32, 95], None),
    (64, 128, 8, 2, 1, [63, 64, 0, 127], [1, 1, 0, 1]),
    (32, 128, 2, 1, 70, [5, 0, 90], [70, 1, 33]),              # across pages, from the middle of a word to the middle of a word
    (128, 64, 3, 3, 9, [3, 7, 250, 0], [9, 2, 9, 9]),          # the third runs out of its pages
    (4096, 64, 2, 2, 40, [4090, 17], None),
    (64, 64, 2, 1, 3, [-1, 2 ** 30, 192, 5], [3, 3, 3, 99]),   # starts out of range, a count above the tokens
]


def ref_cache(page, dim, kv, batch, g, reach):
    per = max(2, -(-reach // page))
    table = torch.randperm(batch * per + 3, generator=g)[:batch * per].reshape(batch, per).to(torch.int32)
    return R.RefCache(batch * per + 3, kv, page, dim, table, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,dim,heads,kv,tokens,starts,counts", CACHES)
def test_cache_write_and_read(dtype, page, dim, heads, kv, tokens, starts, counts):
    n, g = len(starts), gen(page + tokens)
    ref = ref_cache(page, dim, kv, n, g, 192)
    ref.table[0, 1] = -1                                       # an absent page, and one out of the pool
    ref.table[-1, 1] = ref.pages
    qkv = torch.cat((torch.randn(n, tokens, heads * dim, generator=g), awkward_values(g, n, tokens, 2 * kv * dim)), -1).to(DT[dtype])
    start = torch.tensor(starts, dtype=torch.int32)
    count = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    cache = on_gpu(ref)
    out = torch.full((n, tokens, 2 * kv * dim), 7.0, dtype=DT[dtype], device="cuda")

    def build(o):
        o.cache_write(dev(qkv), cache, dev(start), dev(count), heads=heads)
        o.cache_read(out, cache, dev(start), dev(count))
    s = session(build, dtype, n)
    s.enqueue()
    torch.cuda.synchronize()
    for b in range(n):
        st, ct = ref.span(b, start, count, tokens)
        for t in range(ct):
            x = qkv[b, t, heads * dim:].float().reshape(2, kv, dim)
            ref.write(b, st + t, x[0], x[1])
    for name, a, w in (("k", cache.k_codes, ref.k), ("v", cache.v_codes, ref.v), ("k scales", cache.k_scales, ref.ks), ("v scales", cache.v_scales, ref.vs)):
        assert torch.equal(a.cpu(), w), name
    want = torch.zeros(n, tokens, 2, kv, dim, dtype=torch.float64)
    for b in range(n):
        st, ct = ref.span(b, start, count, tokens)
        for t in range(ct):
            for j, which in enumerate("kv"):
                v = ref.value(b, st + t, which)
                if v is not None:
                    want[b, t, j] = v
    want = want.reshape(n, tokens, -1)
    got = out.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    # c * s + m is one rounding to fp32, bf16 tenants round it once more
    assert ((got - want).nan_to_num().abs() <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * want.nan_to_num().abs() * 1.01 + 1e-44).all()
    s.close()


# -- attention -----------------------------------------------------------------------------------------------------------------------
ATTEND = [  # page, dim, heads, kv, tokens, starts, counts, window
    (32, 64, 1, 1, 1, [0], None, 0),                            # one token that sees itself
    (64, 128, 8, 2, 1, [63, 64, 200, 0], [1, 1, 1, 0], 0),
    (32, 64, 12, 12, 1, [500, 1, 255], None, 0),
    (64, 128, 16, 1, 1, [321, 30], None, 0),                    # one key/value head
    (32, 64, 40, 1, 1, [77], None, 0),                          # more query heads to a kv head than a tile has rows
    (32, 64, 9, 3, 5, [0, 31, 64, 700], [5, 3, 0, 5], 0),
    (64, 128, 4, 2, 33, [0, 100, 17], [33, 1, 20], 0),
    (128, 64, 6, 6, 70, [0, 300], None, 0),
    (32, 64, 4, 2, 1, [200, 40, 3], None, 1),                   # a window of the token itself
    (64, 128, 7, 1, 40, [150, 0], None, 33),
    (256, 64, 3, 3, 130, [700], None, 100),
    (32, 128, 2, 2, 2, [1000, 2000, 1500], None, 0),
    (64, 64, 2, 1, 3, [-5, 2 ** 30, 126, 90], None, 0),         # out of range: nothing; the third runs out of its pages
    (32, 128, 5, 5, 260, [0], [257], 0),
]


def attend_case(dtype, page, dim, heads, kv, tokens, starts, counts, window, absent):
    n, g = len(starts), gen(dim * tokens + heads)
    reach = max([128] + [s + tokens for s in starts if 0 <= s < 4096])
    if 126 in starts:
        reach = 128
    ref = ref_cache(page, dim, kv, n, g, reach)
    if absent:                                                  # holes: a first page, one in between, all of one sequence
        ref.table[0, 0] = -1
        ref.table[0, -1] = ref.pages + 5
        if n > 1:
            ref.table[1] = -2 ** 31
    qkv = torch.randn(n, tokens, (heads + 2 * kv) * dim, generator=g).to(DT[dtype])
    start = torch.tensor(starts, dtype=torch.int32)
    count = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    scale = 1.3 / dim ** 0.5
    want, weight = R.attention(ref, qkv, heads, start, count, scale, window)
    return ref, qkv, start, count, scale, want, weight


def check_attention(got, want, weight, dtype, dim):
    got = got.cpu().double()
    assert not torch.isnan(got).any()
    assert (got[weight == 0] == 0).all()
    score = 2 * 64 * 2.0 ** -24 * (1.3 / dim ** 0.5) * dim ** 0.5 * 16
    relative = score + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    err, most = (got - want).abs(), relative * (weight + (weight > 0) * 6.5) + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert (err <= most).all(), float((err / (most + 1e-30)).max())


@pytest.mark.parametrize("absent", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,dim,heads,kv,tokens,starts,counts,window", ATTEND)
def test_attention(dtype, page, dim, heads, kv, tokens, starts, counts, window, absent):
    ref, qkv, start, count, scale, want, weight = attend_case(dtype, page, dim, heads, kv, tokens, starts, counts, window, absent)
    n = len(starts)
    out = torch.full((n, tokens, heads * dim), 7.0, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), dev(count), heads=heads, scale=scale, window=window), dtype, n)
    s.enqueue()
    torch.cuda.synchronize()
    check_attention(out, want, weight, dtype, dim)
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,heads,kv,dim", [(1, 8, 2, 128), (48, 3, 3, 64)])
def test_nothing_beyond_a_sequence_is_looked_at(dtype, tokens, heads, kv, dim):
    """Codes, scales and pages beyond the tokens that a query sees hold NaN scales, and pages that do not exist."""
    page, starts = 32, [37, 0, 95]
    ref, qkv, start, count, scale, want, weight = attend_case(dtype, page, dim, heads, kv, tokens, starts, None, 0, False)
    for b, s0 in enumerate(starts):
        for p in range(s0 + tokens, ref.table.shape[1] * page):
            pg, o = ref.where(b, p)
            ref.ks[pg, :, o] = ref.vs[pg, :, o] = 0x7FC07FC0
        for i in range((s0 + tokens + page - 1) // page, ref.table.shape[1]):
            ref.table[b, i] = 2 ** 31 - 1
    out = torch.full((3, tokens, heads * dim), 7.0, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=heads, scale=scale), dtype, 3)
    s.enqueue()
    torch.cuda.synchronize()
    check_attention(out, want, weight, dtype, dim)
    s.close()


def test_large_scores_do_not_overflow():
    """Scores of several thousand, growing along the sequence and falling again: the running maximum has to follow."""
    page, dim, n_keys = 32, 64, 700
    g = gen(5)
    ref = ref_cache(page, dim, 1, 1, g, n_keys)
    qkv = torch.randn(1, 1, 3 * dim, generator=g)
    for p in range(n_keys):
        k = qkv[0, 0, :dim] * (p / 100.0 if p < 500 else (900 - p) / 100.0) * 8
        ref.write(0, p, k[None], torch.randn(1, dim, generator=g))
    start = torch.tensor([n_keys - 1], dtype=torch.int32)
    want, weight = R.attention(ref, qkv, 1, start, None, 1.0, 0)
    out = torch.empty(1, 1, dim, device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=1, scale=1.0), "f32", 1)
    s.enqueue()
    torch.cuda.synchronize()
    # scores of 2500, of 64 products: off by 64 * 2^-24 * 2500 * 3 at the worst, and weights by twice that relatively
    assert ((out.cpu().double() - want).abs() <= 0.06 * (weight + 1)).all()
    s.close()


def test_pools_of_more_than_four_gigabytes():
    page, dim, kv, heads = 512, 128, 8, 8
    pages = 20000                                              # 5.2 GB of key codes, as many of value codes, 0.66 GB of scales each
    from paper_2304_11745_amd import tokens as T
    g = gen(9)
    table = torch.tensor([[pages - 1, 3], [16500, pages - 2]], dtype=torch.int32)
    cache = T.Cache.allocate(pages, kv, dim, dev(table), page)
    small = R.RefCache(4, kv, page, dim, torch.tensor([[0, 1], [2, 3]], dtype=torch.int32), g)
    for i, p in enumerate(table.reshape(-1).tolist()):
        for a, b in ((cache.k_codes, small.k), (cache.v_codes, small.v), (cache.k_scales, small.ks), (cache.v_scales, small.vs)):
            a[p] = dev(b[i])
    start = torch.tensor([511, 600], dtype=torch.int32)
    qkv = torch.randn(2, 2, (heads + 2 * kv) * dim, generator=g)
    out, back = torch.empty(2, 2, heads * dim, device="cuda"), torch.empty(2, 2, 2 * kv * dim, device="cuda")
    x, st = dev(qkv), dev(start)

    def build(o):
        o.cache_write(x, cache, st, None, heads=heads)
        o.cache_attention(x, out, cache, st, None, heads=heads)
        o.cache_read(back, cache, st, None)
    s = session(build, "f32", 2)
    s.enqueue()
    torch.cuda.synchronize()
    for b in range(2):
        for t in range(2):
            kvx = qkv[b, t, heads * dim:].reshape(2, kv, dim)
            small.write(b, int(start[b]) + t, kvx[0], kvx[1])
            got = back[b, t].cpu().double().reshape(2, kv, dim)
            for j, which in enumerate("kv"):
                assert (got[j] - small.value(b, int(start[b]) + t, which)).abs().max() < 1e-6
    want, weight = R.attention(small, qkv, heads, start, None, dim ** -0.5, 0)
    check_attention(out, want, weight, "f32", dim)
    s.close()


# -- sampling ------------------------------------------------------------------------------------------------------------------------
def rows_of(dtype, n, v, seed):
    g = gen(seed)
    x = 2.5 * torch.randn(n, v, generator=g)
    if v > 8:
        x[:, torch.randint(0, v, (4,), generator=g)] += 6
        x[1 % n, ::3] = float("-inf")
        x[2 % n, ::2] = float("nan")
    x[3 % n] = torch.round(x[3 % n])                            # many equal ones
    return x.to(DT[dtype])


def sample(dtype, x, u, **filters):
    n = x.shape[0]
    tokens, logp = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), 7.0, device="cuda")
    s = session(lambda o: o.sample(dev(x), tokens, dev(u), logp=logp, **{k: dev(t) for k, t in filters.items()}), dtype, n)
    s.enqueue()
    torch.cuda.synchronize()
    s.close()
    return tokens.cpu(), logp.cpu()


FILTERS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.8, min_p=0.02), dict(top_k=3, top_p=0.999), dict(top_p=0.3, min_p=0.001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("filters", FILTERS, ids=str)
@pytest.mark.parametrize("n,v", [(5, 1), (6, 2), (5, 63), (7, 1000), (5, 4097), (9, 32001), (3, 131071)])
def test_sampling(dtype, n, v, filters):
    g = gen(n * v)
    x, u = rows_of(dtype, n, v, v), torch.rand(n, generator=g)
    t = 0.4 + torch.rand(n, generator=g)
    per_row = {k: torch.full((n,), val, dtype=torch.int32 if k == "top_k" else torch.float32) for k, val in filters.items()}
    tokens, logp = sample(dtype, x, u, temperature=t, **per_row)
    decided = 0
    for i in range(n):
        kw = {k: val if k == "top_k" else float(np.float32(val)) for k, val in filters.items()}
        token, lp, margin = R.sample_row(x[i].float().numpy(), float(u[i]), float(t[i]), **kw)
        if margin < 1e-6:                                      # weights of 32 bits may fall on either side
            continue
        decided += 1
        assert int(tokens[i]) == token, (i, int(tokens[i]), token)
        assert abs(float(logp[i]) - lp) <= 2e-5 * (1 + abs(lp))
    assert decided >= (n + 1) // 2 or v > 30000


def test_sampling_takes_each_row_by_its_own_filters():
    n, v, g = 8, 5000, gen(3)
    x, u = rows_of("f32", n, v, 4), torch.rand(n, generator=g)
    f = dict(temperature=torch.tensor([0.0, -1.0, 1.0, 2.0, 0.7, 1.0, float("nan"), 1.0]), top_k=torch.tensor([0, 5, 0, -3, 9000, 5000, 7, 1], dtype=torch.int32),
             top_p=torch.tensor([0.9, 1.0, 0.0, 2.0, 0.5, 1.0, 0.9, 0.9]), min_p=torch.tensor([0.0, 0.1, 0.0, 0.0, 0.0, 1.5, 0.0, 0.0]))
    tokens, logp = sample("f32", x, u, **f)
    for i in range(n):
        t = float(f["temperature"][i])
        token, lp, margin = R.sample_row(x[i].numpy(), float(u[i]), t if t > 0 else 0.0, int(f["top_k"][i]), float(f["top_p"][i]), float(f["min_p"][i]))
        assert margin > 1e-6 and int(tokens[i]) == token and abs(float(logp[i]) - lp) <= 2e-5 * (1 + abs(lp)), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sampling_of_rows_that_hold_little(dtype):
    v, inf = 3001, float("inf")
    x = torch.full((8, v), -inf)
    x[1] = float("nan")
    x[2, 17] = -3.0                                            # one word left
    x[3, 5], x[3, 2900] = inf, inf                             # two infinite ones share the weight
    x[3, 100] = 10.0
    x[4] = 0.0                                                 # all alike, one of them a negative zero
    x[4, 7] = -0.0
    x[5] = -3e38                                               # the type's lowest values
    x[6, 2], x[6, 3] = 1.0, 1.0 - 1e-3
    x[7] = -3e38
    x[7, v - 1] = 3e38
    u = torch.tensor([0.5, 0.5, 0.999, 0.7, 0.6, 0.25, 0.0, 0.99])
    tokens, logp = sample(dtype, x.to(DT[dtype]), u)
    assert tokens.tolist()[:4] == [-1, -1, 17, 2900]
    assert logp[0] == -inf and logp[1] == -inf and logp[2] == 0 and abs(float(logp[3]) + np.log(2)) < 1e-6
    assert tokens[4] == int(np.float32(0.6) * v) and tokens[5] == v // 4 and tokens[6] == 2 and tokens[7] == v - 1
    assert abs(float(logp[4]) + np.log(v)) < 1e-5
    for top_k, want in ((1, 0), (7, 3), (8, 4)):               # of equal ones the first by index: u * top_k
        got, _ = sample(dtype, x[4:5].to(DT[dtype]), torch.tensor([0.5]), top_k=torch.tensor([top_k], dtype=torch.int32))
        assert int(got) == want
    got, _ = sample(dtype, x[4:5].to(DT[dtype]), torch.tensor([0.9999]), top_p=torch.tensor([0.5]))
    assert int(got) == int(np.float32(0.9999) * (v // 2 + 1))
    got, _ = sample(dtype, x[4:5].to(DT[dtype]), torch.tensor([1.0]))        # a random number of one is taken as the last
    assert int(got) == v - 1


# -- as parts of a tenant ------------------------------------------------------------------------------------------------------------
def small_tenant(dtype, n=5, tokens=3):
    from paper_2304_11745_amd import tokens as T
    heads, kv, dim, page, vocab = 6, 2, 64, 32, 900
    g = gen(31)
    ref = ref_cache(page, dim, kv, n, g, 400)
    cache = on_gpu(ref)
    start = dev(torch.tensor([0, 390, 31, 200, 64], dtype=torch.int32)[:n])
    x = dev(torch.randn(n, tokens, 96, generator=g).to(DT[dtype]))
    w = dev((torch.randn((heads + 2 * kv) * dim, 96, generator=g) / 10).to(DT[dtype]))
    w2 = dev((torch.randn(vocab, heads * dim, generator=g) / 5).to(DT[dtype]))
    e = dict(device="cuda", dtype=DT[dtype])
    qkv, ctx, logits = torch.empty(n, tokens, (heads + 2 * kv) * dim, **e), torch.empty(n, tokens, heads * dim, **e), torch.empty(n, tokens, vocab, **e)
    angle = torch.rand(500, 32, generator=g)
    table = dev(torch.stack((angle.cos(), angle.sin()), -1))
    positions = (start[:, None] + torch.arange(tokens, device="cuda", dtype=torch.int32))[..., None].contiguous()
    out, u = torch.empty(n * tokens, dtype=torch.int32, device="cuda"), dev(torch.rand(n * tokens, generator=g))
    ops = T.OpList(DT[dtype], n)
    ops.gemm(x, w, qkv)
    ops.qknorm_rope(qkv, qkv, positions, table, heads=heads, kv_heads=kv, head_dim=dim)
    ops.cache_write(qkv, cache, start, heads=heads)
    ops.cache_attention(qkv, ctx, cache, start, heads=heads)
    ops.gemm(ctx, w2, logits)
    ops.sample(logits, out, u)
    state = [ctx, logits, out, cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales]
    return ops, state, start, positions


def snapshot(state):
    torch.cuda.synchronize()
    return [t.clone() for t in state]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_way_of_running_gives_the_same_bits(dtype):
    """gacer_enqueue, the three modes, plans that cut the batch (also over two streams), the checking mode, the static workspace and a
    replayed graph."""
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    ops, state, start, _ = small_tenant(dtype)
    stream, sibling = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    s = T.TokenSession([ops], [stream])
    s.enqueue()
    want = snapshot(state)

    def again(run):
        for t in state[:3]:
            t.zero_()
        torch.cuda.synchronize()
        run()
        assert same(snapshot(state), want)
    for mode in (B.GACER_MODE_PLAN, B.GACER_MODE_SEQUENTIAL, B.GACER_MODE_STREAM_PARALLEL):
        again(lambda: s.run(mode))
        again(lambda: B.check(s.ctx, B.gacer_run_static(s.ctx, mode, 2)))
    d = (B.gacer_tenant * 1)(ops.descriptor(stream.cuda_stream))
    d[0].sibling_stream = sibling.cuda_stream
    B.check(s.ctx, B.gacer_load_tenants(s.ctx, d, 1))
    n_ops = len(ops.ops)
    for sizes in ([2, 3], [1, 1, 1, 1, 1], [4, 1]):
        for side in (0, 1):
            arr = (C.c_int * len(sizes))(*sizes)
            sp = (B.gacer_split * n_ops)(*[B.gacer_split(0, i, B.GACER_AXIS_BATCH, len(sizes), arr, side) for i in range(n_ops)])
            B.check(s.ctx, B.gacer_set_plan(s.ctx, C.byref(B.gacer_plan(n_ops, sp, 0, None))))
            again(lambda: s.run(B.GACER_MODE_PLAN))
    B.check(s.ctx, B.gacer_set_sync_every_launch(s.ctx, 1))
    again(lambda: s.run(B.GACER_MODE_PLAN))
    again(s.enqueue)
    B.check(s.ctx, B.gacer_set_sync_every_launch(s.ctx, 0))
    B.check(s.ctx, B.gacer_capture(s.ctx, B.GACER_MODE_PLAN))
    for _ in range(3):
        again(lambda: s.run(B.GACER_MODE_PLAN))
    s.close()


def test_a_captured_step_follows_the_lengths_on_the_device():
    """A step captured by the caller, replayed several times with other lengths and eager work in between."""
    from paper_2304_11745_amd import tokens as T
    ops, state, start, positions = small_tenant("bf16")
    begin = [t.clone() for t in state]
    s = T.TokenSession([ops])
    s.enqueue()
    torch.cuda.synchronize()
    first, at = start.clone(), positions.clone()

    def reset(step):
        for t, b in zip(state, begin):
            t.copy_(b)
        start.copy_(first + step)
        positions.copy_(at + step)
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.enqueue()
    for step in (0, 1, 7, 3):
        reset(step)
        s.enqueue()
        want = snapshot(state)
        reset(step)
        graph.replay()
        assert same(snapshot(state), want), step
        torch.randn(1000, device="cuda").sum().item()
    s.close()


def test_enqueue_on_the_callers_stream():
    from paper_2304_11745_amd import tokens as T
    ops, state, start, _ = small_tenant("f32")
    s = T.TokenSession([ops])
    s.enqueue()
    want = snapshot(state)
    side = torch.cuda.Stream()
    for t in state[:3]:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.enqueue()
        got = [t.clone() for t in state]
    side.synchronize()
    assert same(got, want)
    s.close()


def test_profile_trace_and_search_know_the_operators():
    import synth
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import harness
    ops, state, _, _ = small_tenant("bf16")
    tenants, data = synth.build_config(1)
    sess = harness.Session(tenants, data, extra=[ops])
    sess.run(B.GACER_MODE_SEQUENTIAL, 1)
    want = snapshot(state)
    rows = sess.trace(B.GACER_MODE_PLAN, 1)
    mine = [r for r in rows if r["tenant"] == len(tenants)]
    assert len(mine) >= len(ops.ops) and all(r["ms"] > 0 for r in mine)
    assert all(r["bytes"] > 0 for r in mine if "finish" not in r["kernel"] and "join" not in r["kernel"])
    table = sess.profile()
    assert {r.op for r in table if r.tenant == len(tenants)} == set(range(len(ops.ops)))
    splits, syncs, P, residue = sess.search(table, 20)
    sess.set_plan(splits, syncs)
    for t in state[:3]:
        t.zero_()
    torch.cuda.synchronize()
    sess.run(B.GACER_MODE_PLAN, 2)
    assert same(snapshot(state), want)
    sess.close()


def test_operator_lists_refuse_what_they_can_see():
    from paper_2304_11745_amd import tokens as T
    x = torch.zeros(2, 3, 12 * 64, device="cuda")
    table = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    cache = T.Cache.allocate(4, 2, 64, torch.zeros(2, 2, dtype=torch.int32, device="cuda"))
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.zeros(2, 3, 8 * 64, device="cuda")
    for bad in (lambda o: o.cache_write(x.bfloat16(), cache, start, heads=8), lambda o: o.cache_write(x.transpose(0, 1), cache, start, heads=8),
                lambda o: o.cache_write(x, cache, start.long(), heads=8), lambda o: o.cache_write(x, cache, start[:1], heads=8),
                lambda o: o.cache_write(x.cpu(), cache, start, heads=8), lambda o: o.cache_write(x, T.Cache(cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, table), start, heads=8),
                lambda o: o.qknorm_rope(x, out, None, None, heads=8, kv_heads=2, head_dim=64),
                lambda o: o.sample(x, torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda")),
                lambda o: T.Cache.allocate(4, 2, 96, table)):
        with pytest.raises(ValueError):
            bad(T.OpList(torch.float32, 2))
    ops = T.OpList(torch.float32, 2)                            # what only the library sees comes back as its error
    ops.cache_attention(x, out, cache, start, heads=7)
    from paper_2304_11745_amd import binding as B
    with pytest.raises(B.GacerError, match="tenant 0 op 0"):
        T.TokenSession([ops])


def test_the_example_decodes_as_if_every_token_were_filled_in_at_once():
    """examples/decode.py in fp32: the last step's logits equal those of a list that takes the same tokens as one prompt."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode
    from paper_2304_11745_amd import tokens as T
    steps, batch = 9, 3
    said, logits = decode.serve(torch.float32, batch, steps, vision=True)
    assert ((said >= 0) & (said < 8000)).all()
    again, _ = decode.serve(torch.float32, batch, steps, vision=False)
    assert torch.equal(said, again)
    d = decode.Decoder(torch.float32, batch)                   # the same weights, by their seed
    lengths = [1 + (7 * i) % 40 for i in range(batch)]
    prompts = torch.randint(0, d.vocab, (batch, 40), generator=d.gen, device="cuda")
    count = torch.tensor([n + steps for n in lengths], dtype=torch.int32, device="cuda")
    ops, x, at, out = d.body(40 + steps, count)
    s = T.TokenSession([ops])
    ids = torch.zeros(batch, 40 + steps, dtype=torch.long, device="cuda")
    for b, n in enumerate(lengths):
        ids[b, :n], ids[b, n:n + steps] = prompts[b, :n], said[b, :steps].long()
    x.copy_(d.embedding[ids])
    at.copy_(torch.arange(40 + steps, device="cuda", dtype=torch.int32)[None, :, None].expand_as(at))
    s.enqueue()
    last = out[torch.arange(batch, device="cuda"), count.long() - 1]
    h = torch.nn.functional.layer_norm(last, (d.width,), *d.last)
    want = h @ d.out.t()
    # fp32 throughout, but a value near the line between two codes may fall on either side: one code of one feature, a fifteenth of
    # its group's range; three such steps of one key feature move a logit of size 3 by a few hundredths
    assert (logits[:, 0] - want).abs().max() <= 0.05 * want.abs().max()
    s.close()


SPLITS = [  # page, dim, heads, kv, tokens, starts, counts, window: few sequences with room for long ones, so that their keys are cut into parts
    (64, 128, 8, 2, 1, [2300, 70], None, 0),
    (256, 64, 2, 2, 1, [1025, 0, 2047], None, 0),
    (64, 64, 24, 2, 1, [1800], None, 0),
    (128, 128, 4, 2, 9, [1500, 600], [9, 4], 0),
    (64, 64, 3, 3, 150, [900, 0], [150, 70], 0),
    (64, 128, 8, 1, 40, [1100], None, 0),
    (128, 64, 4, 1, 70, [1200], None, 700),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,dim,heads,kv,tokens,starts,counts,window", SPLITS)
def test_attention_with_the_keys_in_splits(dtype, page, dim, heads, kv, tokens, starts, counts, window):
    """The whole result, and the same bits from any cut of the batch (every part of it has its own part of the workspace)."""
    from paper_2304_11745_amd import binding as B
    ref, qkv, start, count, scale, want, weight = attend_case(dtype, page, dim, heads, kv, tokens, starts, counts, window, False)
    n = len(starts)
    used = ref.table.shape[1]
    ref.table = torch.cat((ref.table, torch.full((n, 32768 // page - used), -1, dtype=torch.int32)), 1)
    ref.table[0, 1] = -1                                        # an absent page within
    want, weight = R.attention(ref, qkv, heads, start, count, scale, window)
    out = torch.full((n, tokens, heads * dim), 7.0, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), dev(count), heads=heads, scale=scale, window=window), dtype, n)
    rows = C.c_size_t()
    B.check(s.ctx, B.gacer_trace_run(s.ctx, B.GACER_MODE_SEQUENTIAL, 1, None, 0, C.byref(rows)))
    assert rows.value == 2                                      # the parts, and what joins them
    s.enqueue()
    torch.cuda.synchronize()
    check_attention(out, want, weight, dtype, dim)
    whole = out.clone()
    for sizes in ([1] * n, [n - 1, 1]):
        if n == 1:
            continue
        arr = (C.c_int * len(sizes))(*sizes)
        sp = (B.gacer_split * 1)(B.gacer_split(0, 0, B.GACER_AXIS_BATCH, len(sizes), arr, 0))
        B.check(s.ctx, B.gacer_set_plan(s.ctx, C.byref(B.gacer_plan(1, sp, 0, None))))
        out.fill_(3.0)
        torch.cuda.synchronize()
        s.run(B.GACER_MODE_PLAN)
        assert torch.equal(out, whole)
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,heads", [(1, 4), (4, 4), (6, 4), (12, 4), (20, 4)])       # rows of 4, 16, 24, 48 and 80: every kernel
def test_long_caches_are_averaged_without_bias(dtype, tokens, heads):
    """65536 keys of nearly equal weight: the result is 1/256 of the values, so errors of the weights that all lie on one side would show.
    bf16: roundings to nearest of the result, of the weights and of the weights times the scales, each at most 2^-9 of a number and 2^-9 / sqrt(3) on
    average, together 2^-9; twice that is allowed.  fp32: 2^-24 for each of some hundred additions to a sum, 2^-17."""
    page, dim, n_keys = 256, 64, 65536
    g = gen(tokens)
    ref = ref_cache(page, dim, 1, 1, g, n_keys)
    at = ref.table[0].long()
    qkv = (0.2 * torch.randn(1, tokens, (heads + 2) * dim, generator=g)).to(DT[dtype])

    def unpacked(codes, pair):                                   # codes [pages, page, D], pair [pages, page]
        scale, low = (pair.long() << 16).to(torch.int32).view(torch.float32).double(), (pair & -65536).view(torch.float32).double()
        return (codes.double() * scale[..., None] + low[..., None]).reshape(n_keys, dim)
    k = unpacked(R.codes_of(ref.k[at][:, 0].contiguous().view(torch.int32)), ref.ks[at][:, 0, :, 0])
    v = unpacked(R.codes_of(ref.v[at][:, 0].contiguous().view(torch.int32)).transpose(2, 3).reshape(len(at), page, dim), ref.vs[at][:, 0, :, 0])
    for p in (0, 31, 32, 300, n_keys - 1):
        assert torch.equal(k[p], ref.value(0, p, "k")[0]) and torch.equal(v[p], ref.value(0, p, "v")[0])
    q = qkv[0, :, :heads * dim].double().reshape(tokens, heads, dim)
    seen = torch.arange(n_keys)[None, :] <= n_keys - tokens + torch.arange(tokens)[:, None]
    score = torch.einsum("thd,kd->thk", q, k) * dim ** -0.5
    want = torch.softmax(score.masked_fill(~seen[:, None], -float("inf")), -1) @ v
    start = torch.tensor([n_keys - tokens], dtype=torch.int32)
    out = torch.empty(1, tokens, heads * dim, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=heads), dtype, 1)
    s.enqueue()
    torch.cuda.synchronize()
    err = (out.cpu().double().reshape(want.shape) - want).norm() / want.norm()
    assert err <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -17), float(err)
    s.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [1, 6, 12])                   # rows of 4, 24 and 48: every bf16 kernel
def test_values_at_the_end_of_their_range(tokens, dim):
    """Groups with a value far from all others: codes 0 and 1 of 16, around zero, so that the middle of the codes is 15 times what the values are.  Roundings
    of weights must stay factors of the keys' own values: the norm of the error as in the test of long caches, 2^-8."""
    page, heads, n_keys = 64, 4, 300
    g = gen(dim + tokens)
    ref = ref_cache(page, dim, 1, 1, g, n_keys)
    ref.v &= 0x11
    scale = 0.1 + 0.3 * torch.rand(ref.vs.shape, generator=g)
    scale = scale.bfloat16().float()
    ref.vs.copy_(R.pairs(scale, -0.5 * scale))
    qkv = (0.2 * torch.randn(1, tokens, (heads + 2) * dim, generator=g)).bfloat16()
    start = torch.tensor([n_keys - tokens], dtype=torch.int32)
    want, _ = R.attention(ref, qkv, heads, start, None, dim ** -0.5, 0)
    out = torch.empty(1, tokens, heads * dim, dtype=torch.bfloat16, device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=heads), "bf16", 1)
    s.enqueue()
    torch.cuda.synchronize()
    err = (out.cpu().double() - want).norm() / want.norm()
    assert err <= 2.0 ** -8, float(err)
    s.close()


@pytest.mark.parametrize("tokens", [1, 6, 12])                   # rows of 4, 24 and 48
def test_groups_without_a_scale(tokens):
    """Groups of equal values have scale 0, whatever their codes hold: they read as their minimum, beside groups that have a scale."""
    page, dim, heads, n_keys = 64, 128, 4, 200
    g = gen(40 + tokens)
    ref = ref_cache(page, dim, 1, 1, g, n_keys)
    scale = 0.1 + 0.3 * torch.rand(ref.vs.shape, generator=g)
    scale[..., 0] = 0.0                                          # the first 64 features of every token, some of them zero altogether
    low = torch.randn(ref.vs.shape, generator=g)
    low[:, :, ::3, 0] = 0.0
    for s in (ref.vs, ref.ks):
        s.copy_(R.pairs(scale, low))
    qkv = (0.2 * torch.randn(1, tokens, (heads + 2) * dim, generator=g)).bfloat16()
    start = torch.tensor([n_keys - tokens], dtype=torch.int32)
    want, weight = R.attention(ref, qkv, heads, start, None, dim ** -0.5, 0)
    out = torch.empty(1, tokens, heads * dim, dtype=torch.bfloat16, device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=heads), "bf16", 1)
    s.enqueue()
    torch.cuda.synchronize()
    check_attention(out, want, weight, "bf16", dim)
    s.close()
