"""Operators of a decoding tenant through the C ABI without a GPU: what gacer_load_tenants refuses, and what it accepts."""
import ctypes as C

import pytest

from paper_2304_11745_amd import binding as B

FAKE = 0x10000                                  # aligned, never dereferenced


@pytest.fixture()
def ctx():
    c = C.c_void_p()
    assert B.gacer_create(C.byref(c)) == B.GACER_OK
    yield c
    B.gacer_destroy(c)


def rope(**kw):
    d = dict(heads=8, kv_heads=2, head_dim=64, rotary_dims=64, interleaved=0, n_axes=1, sections=(32, 0, 0), n_positions=100, table=FAKE, positions=FAKE)
    d.update(kw)
    d["sections"] = (C.c_int * 3)(*d["sections"])
    return B.gacer_rope(*[d[f] for f, _ in B.gacer_rope._fields_])


def cache(**kw):
    d = dict(heads=8, kv_heads=2, head_dim=64, page_tokens=64, n_pages=10, max_pages=5, window=0, k_codes=FAKE, v_codes=FAKE, k_scales=FAKE,
             v_scales=FAKE, page_table=FAKE, start=FAKE, count=FAKE)
    d.update(kw)
    return B.gacer_cache(*[d[f] for f, _ in B.gacer_cache._fields_])


def sampling(**kw):
    d = dict(u=FAKE, temperature=None, top_k=None, top_p=None, min_p=None, tokens=FAKE, logp=None)
    d.update(kw)
    return B.gacer_sampling(*[d[f] for f, _ in B.gacer_sampling._fields_])


BATCH, TOKENS = 3, 5
QKV, OUT, KV = (BATCH, 12 * 64, TOKENS, 1), (BATCH, 8 * 64, TOKENS, 1), (BATCH, 2 * 2 * 64, TOKENS, 1)
KINDS = {"rope": (B.GACER_QKNORM_ROPE, rope, QKV, QKV), "write": (B.GACER_CACHE_WRITE, cache, QKV, None), "read": (B.GACER_CACHE_READ, cache, None, KV),
         "attend": (B.GACER_CACHE_ATTENTION, cache, QKV, OUT), "sample": (B.GACER_SAMPLE, sampling, (BATCH, 1000, 1, 1), None)}


def load(ctx, name, desc=None, op=None, x=None, y=None, dtype=B.GACER_BF16, share=False, **kw):
    """Loads a tenant of one operator; keywords change its descriptor, `op` the operator's own fields, x and y its shapes."""
    kind, make, xs, ys = KINDS[name]
    xs, ys = x or xs, y or ys
    d = make(**kw) if desc is None else desc
    tensors = (B.gacer_tensor * 2)()
    tensors[0] = B.gacer_tensor(*(xs or (BATCH, 1, 1, 1)), FAKE, 0, 0, 0)
    tensors[1] = B.gacer_tensor(*(ys or (BATCH, 1, 1, 1)), FAKE if share else FAKE + (1 << 24), 0, 0, 0)
    ops = (B.gacer_op * 1)()
    ops[0] = B.gacer_op(kind, 0 if xs else -1, -1, -1, 1 if ys else -1, C.addressof(d) if d else None, None, None, None, 0, 0, 1, 1, 1, 0, 1, 0, 1e-6)
    for k, v in (op or {}).items():
        setattr(ops[0], k, v)
    desc = (B.gacer_tenant * 1)(B.gacer_tenant(1, ops, 2, tensors, 0, 1 if ys else 0, dtype, BATCH, None, None))
    return B.gacer_load_tenants(ctx, desc, 1)


@pytest.mark.parametrize("dtype", [B.GACER_F32, B.GACER_BF16])
@pytest.mark.parametrize("name", KINDS)
def test_good_operators_load(ctx, name, dtype):
    assert load(ctx, name, dtype=dtype) == B.GACER_OK, B.gacer_last_error(ctx)
    n = C.c_int()
    assert B.gacer_launch_count(ctx, B.GACER_MODE_PLAN, C.byref(n)) == B.GACER_OK and n.value == 1


@pytest.mark.parametrize("name", ["rope"])
def test_norm_and_rotation_may_run_in_place(ctx, name):
    assert load(ctx, name, share=True) == B.GACER_OK
    assert load(ctx, "attend", share=True) == B.GACER_ESHAPE


@pytest.mark.parametrize("status,kw", [
    (B.GACER_ESHAPE, dict(heads=7)), (B.GACER_ESHAPE, dict(heads=0)), (B.GACER_ESHAPE, dict(kv_heads=0)), (B.GACER_ESHAPE, dict(head_dim=60)),
    (B.GACER_ESHAPE, dict(head_dim=1024)), (B.GACER_ESHAPE, dict(head_dim=0)), (B.GACER_ESHAPE, dict(rotary_dims=72, sections=(36, 0, 0))), (B.GACER_ESHAPE, dict(rotary_dims=24, sections=(12, 0, 0))),
    (B.GACER_ESHAPE, dict(rotary_dims=-16)), (B.GACER_ESHAPE, dict(n_axes=0)), (B.GACER_ESHAPE, dict(n_axes=4)), (B.GACER_ESHAPE, dict(sections=(31, 0, 0))),
    (B.GACER_ESHAPE, dict(n_axes=2, sections=(40, -8, 0))), (B.GACER_EINVAL, dict(table=None)), (B.GACER_EINVAL, dict(positions=None)),
    (B.GACER_EINVAL, dict(n_positions=0)), (B.GACER_EINVAL, dict(table=FAKE + 8)), (B.GACER_EINVAL, dict(positions=FAKE + 2)),
    (B.GACER_ESHAPE, dict(x=(BATCH, 11 * 64, TOKENS, 1))), (B.GACER_ESHAPE, dict(y=(BATCH, 12 * 64, TOKENS + 1, 1))), (B.GACER_ESHAPE, dict(x=(BATCH, 12 * 64, TOKENS, 2), y=(BATCH, 12 * 64, TOKENS, 2))),
    (B.GACER_ESHAPE, dict(op=dict(alpha=-1.0))), (B.GACER_ESHAPE, dict(op=dict(alpha=float("nan")))), (B.GACER_EINVAL, dict(op=dict(scale=FAKE + 4))),
    (B.GACER_EINVAL, dict(op=dict(w=None))), (B.GACER_ESHAPE, dict(op=dict(out=-1))), (B.GACER_ESHAPE, dict(op=dict(in0=1))), (B.GACER_ESHAPE, dict(op=dict(in0=7))),
    (B.GACER_ESHAPE, dict(op=dict(out=0))), (B.GACER_ESHAPE, dict(op=dict(res=0))), (B.GACER_ESHAPE, dict(op=dict(act=1)))])
def test_norm_and_rotation_refuses(ctx, status, kw):
    assert load(ctx, "rope", **kw) == status, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx)


def test_rotation_of_no_feature_needs_no_table(ctx):
    assert load(ctx, "rope", rotary_dims=0, table=None, positions=None, n_axes=0, sections=(0, 0, 0), n_positions=0) == B.GACER_OK


@pytest.mark.parametrize("name", ["write", "read", "attend"])
@pytest.mark.parametrize("status,kw", [
    (B.GACER_ESHAPE, dict(kv_heads=0)), (B.GACER_ESHAPE, dict(head_dim=96)), (B.GACER_ESHAPE, dict(head_dim=256)), (B.GACER_ESHAPE, dict(page_tokens=16)),
    (B.GACER_ESHAPE, dict(page_tokens=48)), (B.GACER_ESHAPE, dict(page_tokens=8192)), (B.GACER_ESHAPE, dict(n_pages=0)), (B.GACER_ESHAPE, dict(max_pages=0)),
    (B.GACER_ESHAPE, dict(max_pages=1 << 30)), (B.GACER_EINVAL, dict(k_codes=None)), (B.GACER_EINVAL, dict(v_codes=None)), (B.GACER_EINVAL, dict(k_scales=None)),
    (B.GACER_EINVAL, dict(v_scales=None)), (B.GACER_EINVAL, dict(page_table=None)), (B.GACER_EINVAL, dict(start=None)), (B.GACER_EINVAL, dict(k_codes=FAKE + 8)),
    (B.GACER_EINVAL, dict(v_codes=FAKE + 4)), (B.GACER_EINVAL, dict(v_scales=FAKE + 8)), (B.GACER_EINVAL, dict(start=FAKE + 1)), (B.GACER_EINVAL, dict(count=FAKE + 2)), (B.GACER_EINVAL, dict(op=dict(w=None)))])
def test_cache_operators_refuse(ctx, name, status, kw):
    assert load(ctx, name, **kw) == status, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx)


def test_cache_operators_refuse_what_does_not_fit_them(ctx):
    assert load(ctx, "write", heads=9) == B.GACER_ESHAPE
    assert load(ctx, "attend", heads=0) == B.GACER_ESHAPE
    assert load(ctx, "attend", heads=130, x=(BATCH, 134 * 64, TOKENS, 1), y=(BATCH, 130 * 64, TOKENS, 1)) == B.GACER_ESHAPE       # 65 heads per kv head
    assert load(ctx, "write", op=dict(out=1), y=KV) == B.GACER_ESHAPE
    assert load(ctx, "read", op=dict(in0=0)) == B.GACER_ESHAPE
    assert load(ctx, "read", y=(BATCH, 3 * 64, TOKENS, 1)) == B.GACER_ESHAPE
    assert load(ctx, "attend", y=(BATCH, 8 * 64, TOKENS + 1, 1)) == B.GACER_ESHAPE
    assert load(ctx, "attend", x=(2 * BATCH, 12 * 64, TOKENS, 1)) == B.GACER_ESHAPE
    assert load(ctx, "attend", window=-1) == B.GACER_ESHAPE
    assert load(ctx, "attend", op=dict(alpha=float("inf"))) == B.GACER_ESHAPE
    assert load(ctx, "read", heads=0) == B.GACER_OK
    assert load(ctx, "attend", count=None, window=7) == B.GACER_OK


@pytest.mark.parametrize("status,kw", [
    (B.GACER_EINVAL, dict(u=None)), (B.GACER_EINVAL, dict(tokens=None)), (B.GACER_EINVAL, dict(u=FAKE + 2)), (B.GACER_EINVAL, dict(tokens=FAKE + 1)),
    (B.GACER_EINVAL, dict(logp=FAKE + 1)), (B.GACER_ESHAPE, dict(x=(BATCH, (1 << 24) + 1, 1, 1))), (B.GACER_ESHAPE, dict(x=(BATCH + 1, 100, 1, 1))), (B.GACER_EINVAL, dict(op=dict(w=None)))])
def test_sampling_refuses(ctx, status, kw):
    assert load(ctx, "sample", **kw) == status, B.gacer_last_error(ctx)


@pytest.mark.parametrize("name", KINDS)
def test_they_split_along_the_batch_only(ctx, name):
    assert load(ctx, name) == B.GACER_OK
    for axis, factor, status in ((B.GACER_AXIS_BATCH, 2, B.GACER_OK), (B.GACER_AXIS_BATCH, 4, B.GACER_EPLAN), (B.GACER_AXIS_COUT, 2, B.GACER_EPLAN)):
        sp = (B.gacer_split * 1)(B.gacer_split(0, 0, axis, factor, None, 0))
        assert B.gacer_set_plan(ctx, C.byref(B.gacer_plan(1, sp, 0, None))) == status


def test_the_descriptor_is_copied_when_the_tenant_loads(ctx):
    d = cache()
    assert load(ctx, "attend", desc=d) == B.GACER_OK
    d.page_tokens = 0                            # no longer of interest
    sp = (B.gacer_split * 1)(B.gacer_split(0, 0, B.GACER_AXIS_BATCH, 2, None, 0))
    assert B.gacer_set_plan(ctx, C.byref(B.gacer_plan(1, sp, 0, None))) == B.GACER_OK


def test_enqueue_checks_its_arguments(ctx):
    assert B.gacer_enqueue(None, 0, None) == B.GACER_EINVAL
    assert B.gacer_enqueue(ctx, 0, None) == B.GACER_ESTATE
    assert load(ctx, "sample") == B.GACER_OK
    assert B.gacer_enqueue(ctx, 1, None) == B.GACER_EINVAL and B.gacer_enqueue(ctx, -1, None) == B.GACER_EINVAL
