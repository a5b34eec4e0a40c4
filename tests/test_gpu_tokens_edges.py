"""Operators of a decoding tenant on the GPU where a mistake is easily overlooked: values that are not finite, single keys at the edges of what a
query sees, the sampler's ways for rows that do not fit its short ones, and what a profile leaves behind.  References in 64 bits on the CPU.

Tolerance of attention, row by row (a token's head), in the norm over its features.  With w_j the weights and |v_j| the norms of the
values: scores are off by 64 roundings of 2^-24 of sums of size 16 |q| (queries here have elements below 1/4, alpha sqrt(D) = 1), and the weights relatively
by twice that, which is at most S = 2 * 64 * 2^-24 * 16 / 4 of sum_j w_j |v_j|; fp32 sums add 2^-20 of it.  bf16 tenants round the result (2^-8 of it)
and, with many rows, each weight: errors of at most 2^-8, independent of each other, three deviations of whose sum are
3 / sqrt(3) 2^-8 sqrt(sum_j w_j^2 |v_j|^2)."""
import ctypes as C

import numpy as np
import pytest
import torch

import tokens_ref as R
from test_gpu_tokens import DT, dev, gen, on_gpu, ref_cache, sample, same, session, small_tenant, snapshot

pytestmark = pytest.mark.gpu


def unpacked(ref, b, n_keys):
    """Keys and values [n_keys, kv heads, D] of a sequence in float64, and which of its positions have a page."""
    per = min(ref.table.shape[1], -(-n_keys // ref.page))
    at = ref.table[b, :per].long()
    there = (at >= 0) & (at < ref.pages)
    at = torch.where(there, at, torch.zeros_like(at))

    def values(codes, pair):                                     # codes [pages, kv, page, D]
        scale, low = (pair.long() << 16).to(torch.int32).view(torch.float32).double(), (pair & -65536).view(torch.float32).double()
        v = codes.double().unflatten(-1, (-1, R.GROUP)) * scale[..., None] + low[..., None]
        return v.flatten(-2).transpose(1, 2).reshape(-1, ref.kv_heads, ref.dim)[:n_keys]
    k = values(R.codes_of(ref.k[at].contiguous().view(torch.int32)), ref.ks[at])
    v = R.codes_of(ref.v[at].contiguous().view(torch.int32)).transpose(3, 4).reshape(per, ref.kv_heads, ref.page, ref.dim)
    present = there.repeat_interleave(ref.page)[:n_keys]
    return k, values(v, ref.vs[at]), torch.cat((present, torch.zeros(n_keys - present.shape[0], dtype=torch.bool)))


def padded(t, n):
    return torch.cat((t, t.new_zeros(n - t.shape[0], *t.shape[1:])))


def dense_attention(ref, qkv, heads, start, count, scale, window):
    """For each sequence with tokens: (b, weights [tokens, heads, keys], values [keys, heads, D], which keys a token sees [tokens, keys])."""
    t, d, g = qkv.shape[1], ref.dim, ref.kv_heads
    for b in range(qkv.shape[0]):
        s, c = ref.span(b, start, count, t)
        if not c:
            continue
        n_keys = s + c
        k, v, present = unpacked(ref, b, n_keys)
        k, v = (padded(x, n_keys).repeat_interleave(heads // g, 1) for x in (k, v))
        at, key = torch.arange(s, s + c)[:, None], torch.arange(n_keys)[None]
        seen = (key <= at) & present[None]
        if window:
            seen &= key > at - window
        q = qkv[b, :c, :heads * d].double().reshape(c, heads, d)
        score = torch.stack([q[:, h] @ k[:, h].T for h in range(heads)], 1) * scale
        w = torch.softmax(score.masked_fill(~seen[:, None], -float("inf")), -1)
        yield b, torch.where(seen.any(-1)[:, None, None], w, torch.zeros_like(w)), v, seen


# -- norms without a rotation --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [8, 64, 128, 512])
def test_norms_alone_look_at_no_positions(dtype, dim):
    """rotary_dims = 0 through the library's own descriptor: no table, no positions, no axes."""
    from paper_2304_11745_amd import tokens as T
    heads, kv, g = 3, 1, gen(dim)
    qkv, gamma = torch.randn(2, 5, 5 * dim, generator=g).to(DT[dtype]), 1 + 0.1 * torch.randn(dim, generator=g)
    x, out = dev(qkv), torch.zeros(2, 5, 5 * dim, dtype=DT[dtype], device="cuda")
    ops = T.OpList(DT[dtype], 2)
    ops.qknorm_rope(x, out, None, None, heads=heads, kv_heads=kv, head_dim=dim, gamma_q=dev(gamma), gamma_k=dev(gamma), eps=1e-5, rotary_dims=0)
    ops._descs[0].n_axes, ops._descs[0].sections = 0, (C.c_int * 3)(-1, 2 ** 30, 7)
    s = T.TokenSession([ops])
    s.enqueue()
    torch.cuda.synchronize()
    want = R.qknorm_rope(qkv, heads, kv, dim, None, None, gamma, gamma, 1e-5, 0, [0], False)
    err = (out.cpu().double() - want).abs()
    assert (err <= (2.0 ** -8 if dtype == "bf16" else 0) * want.abs() + 2.0 ** -19 * want.abs().amax()).all()
    s.close()


# -- values that are not finite ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,page,room", [(1, 64, 0), (3, 32, 0), (6, 64, 0), (12, 64, 0), (40, 32, 0), (12, 64, 16384), (40, 64, 16384)])      # rows of 4 to 160, keys in splits
def test_a_value_group_that_is_not_finite_stays_in_its_features(dtype, tokens, page, room):
    """A group of 64 features with an infinity or a NaN reads as NaN; a query that sees it has NaN in these features and its usual result in the others, one that does
    not see it is untouched.  A key group that is not finite makes the key's score NaN, and with it the row."""
    dim, heads, kv, starts = 128, 8, 2, [150, 0, 70]
    g = gen(tokens + room)
    ref = ref_cache(page, dim, kv, 3, g, 192)
    if room:
        ref.table = torch.cat((ref.table, torch.full((3, (room - 192) // page), -1, dtype=torch.int32)), 1)
    qkv = (0.3 * torch.randn(3, tokens, (heads + 2 * kv) * dim, generator=g)).to(DT[dtype])
    start = torch.tensor(starts, dtype=torch.int32)

    def poison(scales, b, p, head, group):
        at, o = ref.where(b, p)
        scales[at, head, o, group] = 0x7FC0
    poison(ref.vs, 0, 33, 0, 0)                                 # every token sees it
    poison(ref.vs, 0, 149, 1, 1)
    poison(ref.vs, 1, tokens // 2, 0, 1)                        # tokens before it do not
    poison(ref.vs, 1, tokens - 1, 1, 0)
    poison(ref.ks, 2, 70 + tokens // 2, 1, 0)
    out = torch.full((3, tokens, heads * dim), 7.0, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=heads), dtype, 3)
    s.enqueue()
    torch.cuda.synchronize()
    got = out.cpu().double().reshape(3, tokens, heads, 2, 64)
    want, weight = R.attention(ref, qkv, heads, start, None, dim ** -0.5, 0)
    want, weight = (x.reshape(got.shape) for x in (want, weight))
    assert torch.isnan(want).any() and not torch.isnan(want).all(-1).all()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    score = 2 * 64 * 2.0 ** -24 * 16
    relative = score + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    err = (got - want).nan_to_num().abs()
    assert (err <= (relative * (weight + 6.5) + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)).nan_to_num()).all()
    s.close()


# -- single keys ---------------------------------------------------------------------------------------------------------------------
EDGES = [  # page, dim, heads, kv, tokens, starts, counts, window, room of the page table beyond the tokens (keys in splits where there is much)
    (64, 128, 8, 2, 1, [1300, 70], None, 0, 0),
    (64, 128, 8, 2, 1, [1300, 70], None, 0, 65536),
    (32, 64, 12, 12, 1, [500, 129, 64], None, 100, 0),
    (64, 128, 16, 2, 2, [1200, 63], [2, 1], 700, 0),
    (64, 128, 4, 2, 9, [900, 600], [9, 4], 0, 32768),
    (64, 128, 4, 1, 12, [1200, 64], None, 333, 0),
    (32, 128, 4, 2, 20, [700, 1, 95], None, 64, 0),
    (128, 128, 8, 2, 40, [1100], None, 0, 32768),
    (64, 64, 4, 1, 70, [1200], None, 700, 4096),
    (64, 128, 8, 1, 130, [700, 3], [130, 77], 100, 0),
    (256, 64, 3, 3, 257, [900, 300], None, 1000, 0),
]


@pytest.mark.parametrize("absent", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,dim,heads,kv,tokens,starts,counts,window,room", EDGES)
def test_no_key_is_lost_or_added(dtype, page, dim, heads, kv, tokens, starts, counts, window, room, absent):
    """Weights of nearly equal size, so that each key counts: the tolerance is less than what the result would move by without the row's own key or without the first
    key that it sees, and with the one before that or behind its own (checked on the reference)."""
    n, g = len(starts), gen(dim + tokens + window)
    ref = ref_cache(page, dim, kv, n, g, max(starts) + tokens + 1)
    if absent:
        ref.table[0, 1] = -1
    if room:
        ref.table = torch.cat((ref.table, torch.full((n, room // page), -1, dtype=torch.int32)), 1)
    scale = 0.2 + 0.05 * torch.rand(ref.vs.shape, generator=g)  # no key's values are much smaller than another's
    ref.vs.copy_(R.pairs(scale, -7.5 * scale))
    qkv = (0.05 * torch.randn(n, tokens, (heads + 2 * kv) * dim, generator=g)).to(DT[dtype])
    start = torch.tensor(starts, dtype=torch.int32)
    count = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    out = torch.full((n, tokens, heads * dim), 7.0, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), dev(count), heads=heads, window=window), dtype, n)
    s.enqueue()
    torch.cuda.synchronize()
    got = out.cpu().double().reshape(n, tokens, heads, dim)
    rows = 0
    for b, w, v, seen in dense_attention(ref, qkv, heads, start, count, dim ** -0.5, window):
        c, n_keys = seen.shape
        want = torch.stack([w[:, h] @ v[:, h] for h in range(heads)], 1)                     # [tokens, heads, D]
        size = v.norm(dim=-1).T                                                              # [heads, keys]
        all_of = (w * size[None]).sum(-1)
        bound = (2 * 64 * 2.0 ** -24 * 4 + 2.0 ** -20) * all_of
        if dtype == "bf16":
            bound = bound + 2.0 ** -8 * want.norm(dim=-1) + 3 ** 0.5 * 2.0 ** -8 * ((w * size[None]) ** 2).sum(-1).sqrt()
        err = (got[b, :c] - want).norm(dim=-1)
        assert (err <= bound).all(), float((err / bound).max())
        assert (got[b, c:] == 0).all()
        # what a key less would do: w / (1 - w) (result - value); a key more, with a weight some way below the others' mean
        less = 0.8 / (1 + seen.sum(-1)).double()
        for t in range(c):
            keys = seen[t].nonzero()[:, 0]
            if len(keys) < 2:
                continue
            for j in (int(keys[0]), int(keys[-1])):
                part = w[t, :, j]
                assert ((part / (1 - part))[:, None] * (want[t] - v[j])).norm(dim=-1).gt(bound[t]).all()
            before = int(keys[0]) - 1
            if window and before >= 0:
                assert (less[t] * (want[t] - v[before])).norm(dim=-1).gt(bound[t]).all()
            rows += heads
    assert rows
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [1, 6, 12, 40])               # rows of 4, 24, 48 and 160: every kernel
def test_large_scores_of_many_rows(tokens, dim, dtype):
    """Scores that grow to more than a thousand along the sequence and fall again, other ones for every row: the reference of each row has to follow.  A score is off by
    64 roundings of 2^-24 of three times the largest one (codes of 16 + c, minima), a weight relatively by twice that."""
    page, heads, n_keys = 32, 4, 600
    g = gen(tokens + dim)
    ref = ref_cache(page, dim, 1, 1, g, n_keys)
    base = torch.randn(dim, generator=g)
    base /= base.norm()
    q = base[None] * (4 + 4 * torch.rand(tokens * heads, 1, generator=g)) + 0.1 * torch.randn(tokens * heads, dim, generator=g)
    qkv = torch.cat((q.reshape(1, tokens, heads * dim), torch.zeros(1, tokens, 2 * dim)), -1).to(DT[dtype])
    for p in range(n_keys):
        ref.write(0, p, (base * (p if p < 400 else 800 - p) * 0.5)[None], torch.randn(1, dim, generator=g))
    start = torch.tensor([n_keys - tokens], dtype=torch.int32)
    out = torch.empty(1, tokens, heads * dim, dtype=DT[dtype], device="cuda")
    s = session(lambda o: o.cache_attention(dev(qkv), out, on_gpu(ref), dev(start), None, heads=heads, scale=1.0), dtype, 1)
    s.enqueue()
    torch.cuda.synchronize()
    (_, w, v, _), = dense_attention(ref, qkv, heads, start, None, 1.0, 0)
    k = unpacked(ref, 0, n_keys)[0][:, 0]
    largest = float((qkv[0, :, :heads * dim].double().reshape(-1, dim) @ k.T).abs().max())
    assert largest > 1000
    want = torch.stack([w[:, h] @ v[:, h] for h in range(heads)], 1)
    weight = torch.stack([w[:, h] @ v[:, h].abs() for h in range(heads)], 1)
    relative = 2 * 64 * 2.0 ** -24 * 3 * largest + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    err = (out.cpu().double().reshape(want.shape) - want).abs()
    assert (err <= relative * (weight + 1) + 2.0 ** -8 * want.abs()).all(), float(err.max())
    s.close()


# -- sampling ------------------------------------------------------------------------------------------------------------------------
def test_sampling_of_more_rows_than_a_grid_holds():
    """4194304 workgroups of 1024 threads are 2^32; the rows beyond are sampled too."""
    n, v, g = 2 ** 22 + 5, 7, gen(17)
    x, u = torch.randn(n, v, generator=g).bfloat16(), torch.rand(n, generator=g)
    tokens, logp = sample("bf16", x, u)
    w = torch.exp(x.double() - x.double().amax(-1, keepdim=True))
    cum = w.cumsum(-1)
    goal = u.double()[:, None] * cum[:, -1:]
    far = (cum - goal).abs().amin(-1) > 1e-6 * cum[:, -1]
    want = (cum <= goal).sum(-1)
    assert far[-5:].any() and far.double().mean() > 0.99
    assert torch.equal(tokens[far].long(), want[far])
    assert (logp[far].double() - (w.gather(1, want[:, None])[:, 0] / cum[:, -1]).log()[far]).abs().max() < 1e-5


def decided(x, g, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """A random number (and a top_p near the given one) at which 32 bits decide, and what it draws: (u, top_p, token, logp)."""
    for _ in range(400):
        u = float(torch.rand(1, generator=g))
        p = float(np.float32(top_p if top_p >= 1 else top_p + 0.01 * float(torch.rand(1, generator=g))))
        token, logp, margin = R.sample_row(x.float().numpy(), u, temperature, top_k, p, float(np.float32(min_p)))
        if margin > 1e-6:
            return u, p, token, logp
    raise AssertionError("no random number that decides")


def check_rows(dtype, x, cases, seed):
    """Every row of x with every one of the cases, all of which are decided."""
    g, rows, picked = gen(seed), [], []
    for row in x.to(DT[dtype]):
        for case in cases:
            case = dict(dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **case)
            case["temperature"] = float(np.float32(case["temperature"]))
            picked.append((case,) + decided(row, g, **case))
            rows.append(row)
    f = torch.tensor([[c["temperature"], p, c["min_p"], u] for c, u, p, _, _ in picked])
    k = torch.tensor([c["top_k"] for c, *_ in picked], dtype=torch.int32)
    tokens, logp = sample(dtype, torch.stack(rows), f[:, 3].contiguous(), temperature=f[:, 0].contiguous(), top_p=f[:, 1].contiguous(), min_p=f[:, 2].contiguous(), top_k=k)
    for i, (case, u, p, token, lp) in enumerate(picked):
        assert int(tokens[i]) == token, (i, case, u, p, int(tokens[i]), token)
        assert abs(float(logp[i]) - lp) <= 2e-5 * (1 + abs(lp)), (i, case)


BOTH = [dict(top_k=500), dict(top_p=0.7), dict(top_k=60000, top_p=0.6), dict(top_k=80000), dict(top_k=90000, top_p=0.9, min_p=0.01), dict(top_p=0.95, temperature=0.6)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [1.5, -1.5, 0.0])
def test_sampling_of_more_equal_logits_than_a_counter_holds(dtype, value):
    """70000 and 140000 equal logits among others: counters of 16 bits overflow, those of negative values into those of positive ones."""
    g = gen(11)
    x = value - 1 + torch.randn(2, 150001, generator=g)
    for row, n in ((0, 70000), (1, 140000)):
        x[row, torch.randperm(150001, generator=g)[:n]] = value
    check_rows(dtype, x, BOTH, 12)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [5000, 32000])
def test_sampling_with_a_large_top_k(dtype, v):
    """Beyond what the threads' largest entries can tell, with and without other filters; rows of ordinary logits, of many equal ones, and flat ones."""
    g = gen(v)
    x = 2.5 * torch.randn(3, v, generator=g)
    x[1] = torch.round(x[1])
    x[2] = 0.25
    cases = [dict(top_k=k, **more) for k in (256, 257, 900, 3000, v - 1) for more in (dict(), dict(top_p=0.8), dict(top_p=0.5, min_p=0.02, temperature=1.7))]
    check_rows(dtype, x, cases, 13)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [196608, 196617, 200001])
def test_sampling_of_rows_longer_than_the_peaks(dtype, v):
    g = gen(v)
    x = 2.5 * torch.randn(2, v, generator=g)
    x[1, 5] = 15.0
    cases = [dict(top_p=0.8), dict(top_k=50), dict(top_k=5000, top_p=0.7), dict(top_p=0.85, min_p=0.001), dict()]
    check_rows(dtype, x, [dict(c, temperature=0.5) for c in cases], 14)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [3001, 70001])
def test_sampling_where_only_divisions_are_safe(dtype, v):
    """Temperatures from 1e-38 to 1e30, and infinite logits, under every filter."""
    g = gen(v + 1)
    x = torch.round(2 * torch.randn(3, v, generator=g))
    x[1, ::50] = float("inf")
    x[2, ::7] = float("-inf")
    filters = [dict(), dict(top_k=20), dict(top_k=2500), dict(top_p=0.6), dict(top_k=700, top_p=0.7), dict(top_p=0.9, min_p=0.5)]
    check_rows(dtype, x, [dict(f, temperature=t) for f in filters for t in (1e-38, 1e-20, 1.0, 1e20, 1e30)], 15)


# -- profiles ------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lists", [1, 2])
def test_a_profile_leaves_what_a_round_leaves(dtype, lists):
    """Rotation in place, timed many times over, must not reach the cache or the tokens: after a profile everything is as after the round before it."""
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    made = [small_tenant(dtype) for _ in range(lists)]
    s = T.TokenSession([m[0] for m in made], [torch.cuda.Stream() for _ in made])
    s.run()
    everything = [t for m in made for t in m[1]] + [t for m in made for t, _ in m[0]._tensors]
    want = snapshot(everything)
    n = C.c_size_t()
    B.check(s.ctx, B.gacer_profile(s.ctx, None, 0, C.byref(n)))
    rows = (B.gacer_prof * n.value)()
    B.check(s.ctx, B.gacer_profile(s.ctx, rows, n.value, C.byref(n)))
    left = same(snapshot(everything), want)
    assert left
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_profile_turns_the_tenants_input_no_further_than_a_round(dtype):
    """A list that begins with a rotation in place of its own input (no earlier operator writes it anew): a profile turns it once, as the round that it runs first does."""
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    n, t, heads, kv, dim = 4, 3, 4, 2, 64
    g = gen(8)
    x0 = torch.randn(n, t, (heads + 2 * kv) * dim, generator=g).to(DT[dtype])
    angle = torch.rand(10, dim // 2, generator=g)
    table, pos = dev(torch.stack((angle.cos(), angle.sin()), -1)), torch.full((n, t, 1), 7, dtype=torch.int32, device="cuda")

    def make():
        x, ops = dev(x0), T.OpList(DT[dtype], n)
        ops.qknorm_rope(x, x, pos, table, heads=heads, kv_heads=kv, head_dim=dim)
        return x, ops
    (x, ops), (y, other) = make(), make()
    once = T.TokenSession([other])
    once.run()
    want = y.clone()
    s = T.TokenSession([ops])
    size = C.c_size_t()
    B.check(s.ctx, B.gacer_profile(s.ctx, None, 0, C.byref(size)))
    rows = (B.gacer_prof * size.value)()
    B.check(s.ctx, B.gacer_profile(s.ctx, rows, size.value, C.byref(size)))
    turned_once = same(snapshot([x]), [want])
    assert turned_once
    s.close()
    once.close()
