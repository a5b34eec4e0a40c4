"""Operators of a decoding tenant on the GPU where a mistake is easily overlooked.  References in 64 bits on the CPU."""
import ctypes as C

import pytest
import torch

import tokens_ref as R
from test_gpu_tokens import DT, dev, gen, on_gpu, ref_cache, sample, same, session, small_tenant, snapshot

pytestmark = pytest.mark.gpu


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
