"""Operators on 8-bit rows through the C ABI without a GPU: what gacer_load_tenants refuses, and what it accepts; and the oracle of their GPU tests."""
import ctypes as C

import numpy as np
import pytest
import torch

import fp8_ref as R
from paper_2304_11745_amd import binding as B

FAKE = 0x10000                                  # aligned, never dereferenced
AT = [FAKE + (i << 24) for i in range(16)]      # places of their own


@pytest.fixture()
def ctx():
    c = C.c_void_p()
    assert B.gacer_create(C.byref(c)) == B.GACER_OK
    yield c
    B.gacer_destroy(c)


BATCH, TOKENS, IN, OUT = 3, 5, 144, 80


def rows(at, width, **kw):
    d = dict(codes=AT[at], scales=AT[at + 1], rows=BATCH * TOKENS, features=width)
    d.update(kw)
    return B.gacer_fp8_rows(*[d[f] for f, _ in B.gacer_fp8_rows._fields_])


def weight(at, **kw):
    d = dict(codes=AT[at], scales=AT[at + 1])
    d.update(kw)
    return B.gacer_fp8_weight(d["codes"], d["scales"])


def load(ctx, kind, x=None, y=None, w=None, norm=1, codes=True, shapes=None, op=None, dtype=B.GACER_BF16, odd=False, second=None, **fields):
    """A tenant of one operator: tensors 0 (in0 of a norm), 1 (res) and 2 (out); keywords change its 8-bit operands and its fields."""
    inner, outer = (BATCH, IN, TOKENS, 1), (BATCH, IN if kind == B.GACER_RMSNORM_FP8 else OUT, TOKENS, 1)
    shapes = {0: inner, 1: outer, 2: outer, **(shapes or {})}
    tensors = (B.gacer_tensor * 3)(*[B.gacer_tensor(*shapes[i], AT[i], 0, 0, 0) for i in range(3)])
    if kind == B.GACER_RMSNORM_FP8:
        d = B.gacer_fp8_norm(norm, rows(4, IN, **(y or {})) if codes else B.gacer_fp8_rows())
        f = dict(in0=0, res=1, out=2, act=0, scale=AT[12])
    elif kind == B.GACER_GEMM_FP8:
        d = B.gacer_fp8_gemm(rows(4, IN, **(x or {})), weight(6, **(w or {})))
        f = dict(in0=-1, res=1, out=2, act=1, bias=AT[12])
    else:
        d = B.gacer_fp8_gated(rows(4, IN, **(x or {})), weight(6, **(w or {})), weight(8, **(second or {})), rows(10, OUT, **(y or {})) if codes else B.gacer_fp8_rows())
        f = dict(in0=-1, res=-1, out=-1 if codes else 2, act=6)
    f.update(op or {})
    f.update(fields)
    raw = C.create_string_buffer(C.sizeof(d) + 8)
    at = C.addressof(raw) + (1 if odd else 0)
    C.memmove(at, C.addressof(d), C.sizeof(d))
    ops = (B.gacer_op * 1)(B.gacer_op(kind, -1, -1, -1, -1, at, None, None, None, 0, 0, 1, 1, 1, 0, 1, 0, 1e-6))
    for k, v in f.items():
        setattr(ops[0], k, v)
    desc = (B.gacer_tenant * 1)(B.gacer_tenant(1, ops, 3, tensors, 0, 2 if f["out"] == 2 else 0, dtype, BATCH, None, None))
    return B.gacer_load_tenants(ctx, desc, 1)


N, G, A = B.GACER_RMSNORM_FP8, B.GACER_GEMM_FP8, B.GACER_GATED_FP8


@pytest.mark.parametrize("dtype", [B.GACER_F32, B.GACER_BF16])
@pytest.mark.parametrize("kind", [N, G, A])
@pytest.mark.parametrize("kw", [{}, dict(odd=True), dict(codes=False)])
def test_good_operators_load(ctx, kind, dtype, kw):
    assert load(ctx, kind, dtype=dtype, **kw) == B.GACER_OK, B.gacer_last_error(ctx)
    n = C.c_int()
    assert B.gacer_launch_count(ctx, B.GACER_MODE_PLAN, C.byref(n)) == B.GACER_OK and n.value == 1
    for axis, factor, status in ((B.GACER_AXIS_BATCH, 2, B.GACER_OK), (B.GACER_AXIS_BATCH, 4, B.GACER_EPLAN), (B.GACER_AXIS_COUT, 2, B.GACER_EPLAN)):
        sp = (B.gacer_split * 1)(B.gacer_split(0, 0, axis, factor, None, 0))
        assert B.gacer_set_plan(ctx, C.byref(B.gacer_plan(1, sp, 0, None))) == status


def test_what_may_be_left_out(ctx):
    assert load(ctx, N, res=-1, out=-1, scale=None) == B.GACER_OK
    assert load(ctx, N, norm=0, out=-1) == B.GACER_OK
    assert load(ctx, G, res=-1, bias=None) == B.GACER_OK
    for act in range(8):
        assert load(ctx, G, act=act) == B.GACER_OK and load(ctx, A, act=act) == B.GACER_OK
    wide = (BATCH, 81, TOKENS, 1)
    assert load(ctx, G, shapes={1: wide, 2: wide}) == B.GACER_OK                       # odd output features
    assert load(ctx, N, codes=False, shapes={0: wide, 1: wide, 2: wide}) == B.GACER_OK
    assert load(ctx, G, shapes={1: (BATCH, OUT, 1, TOKENS), 2: (BATCH, OUT, 1, TOKENS)}) == B.GACER_OK


S, E = B.GACER_ESHAPE, B.GACER_EINVAL


@pytest.mark.parametrize("status,kw", [
    (E, dict(op=dict(w=None))), (S, dict(in0=-1)), (S, dict(in0=7)), (S, dict(in0=2)), (S, dict(in1=1)), (S, dict(res=2)), (S, dict(res=9)), (S, dict(act=1)), (S, dict(out=9)),
    (S, dict(alpha=-1.0)), (S, dict(alpha=float("nan"))), (S, dict(alpha=float("inf"))), (E, dict(scale=AT[12] + 2)), (S, dict(codes=False, out=-1)),
    (S, dict(shapes={2: (BATCH, IN, TOKENS + 1, 1)})), (S, dict(shapes={1: (BATCH, IN + 16, TOKENS, 1)})), (S, dict(y=dict(features=IN + 16))), (S, dict(y=dict(rows=BATCH))),
    (E, dict(y=dict(scales=None))), (E, dict(y=dict(codes=AT[4] + 8))), (E, dict(y=dict(scales=AT[5] + 2))), (S, dict(y=dict(codes=AT[0]))), (S, dict(y=dict(codes=AT[2]))),
    (S, dict(y=dict(scales=AT[1]))), (S, dict(y=dict(scales=AT[12]))), (S, dict(y=dict(scales=AT[4]))), (S, dict(out=0)), (S, dict(out=1)),
    (S, dict(shapes={i: (BATCH, 136, TOKENS, 1) for i in range(3)}, y=dict(features=136))), (S, dict(shapes={i: (4, IN, TOKENS, 1) for i in range(3)}))])
def test_a_norm_refuses(ctx, status, kw):
    assert load(ctx, N, **kw) == status, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx)


COMMON = [(S, dict(in0=0)), (S, dict(in1=0)), (E, dict(x=dict(codes=None))), (E, dict(x=dict(scales=None))), (E, dict(x=dict(codes=AT[4] + 4))), (E, dict(x=dict(scales=AT[5] + 1))),
          (S, dict(x=dict(features=152))), (S, dict(x=dict(features=0))), (S, dict(x=dict(features=65552))), (S, dict(x=dict(features=-16))), (S, dict(x=dict(rows=0))), (S, dict(x=dict(rows=BATCH * TOKENS + 1))),
          (S, dict(x=dict(rows=-BATCH))), (S, dict(x=dict(rows=1 << 24, features=256))), (E, dict(w=dict(codes=None))), (E, dict(w=dict(scales=None))), (E, dict(w=dict(codes=AT[6] + 8))),
          (E, dict(w=dict(scales=AT[7] + 2))), (E, dict(act=8)), (E, dict(act=-1)), (E, dict(op=dict(w=None)))]


@pytest.mark.parametrize("status,kw", COMMON + [
    (S, dict(out=-1)), (S, dict(out=5)), (S, dict(res=2)), (S, dict(x=dict(rows=BATCH))), (E, dict(bias=AT[12] + 1)), (S, dict(shapes={1: (BATCH, OUT, TOKENS + 1, 1)})), (S, dict(x=dict(codes=AT[2]))), (S, dict(w=dict(scales=AT[2]))),
    (S, dict(bias=AT[2])), (S, dict(res=2)), (S, dict(shapes={1: (BATCH, 70000, TOKENS, 1), 2: (BATCH, 70000, TOKENS, 1)}, x=dict(features=32768)))])
def test_a_product_refuses(ctx, status, kw):
    assert load(ctx, G, **kw) == status, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx)


@pytest.mark.parametrize("status,kw", COMMON + [
    (E, dict(second=dict(codes=None))), (E, dict(second=dict(scales=AT[9] + 2))), (S, dict(res=1)), (S, dict(out=2)), (S, dict(codes=False, out=-1)), (S, dict(y=dict(rows=BATCH))),
    (S, dict(y=dict(features=72))), (E, dict(y=dict(scales=None))), (S, dict(y=dict(codes=AT[4]))), (S, dict(y=dict(codes=AT[8]))), (S, dict(y=dict(scales=AT[10] + 16))), (S, dict(y=dict(scales=AT[7]))),
    (S, dict(codes=False, x=dict(rows=BATCH)))])
def test_a_gated_block_refuses(ctx, status, kw):
    assert load(ctx, A, **kw) == status, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx)


@pytest.mark.parametrize("kind", [N, A])
def test_norms_and_gated_blocks_refuse_a_bias(ctx, kind):
    assert load(ctx, kind, bias=AT[13]) == S, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx) and b"bias" in B.gacer_last_error(ctx)


def test_other_operators_take_no_new_activation(ctx):
    t = (B.gacer_tensor * 2)(*[B.gacer_tensor(BATCH, 16, 1, 1, AT[i], 0, 0, 0) for i in range(2)])
    for act, status in ((5, B.GACER_OK), (6, B.GACER_EINVAL), (7, B.GACER_EINVAL)):
        ops = (B.gacer_op * 1)(B.gacer_op(B.GACER_ACT, 0, -1, -1, 1, None, None, None, None, 0, 0, 1, 1, 1, 0, 1, act, 1.0))
        d = (B.gacer_tenant * 1)(B.gacer_tenant(1, ops, 2, t, 0, 1, B.GACER_F32, BATCH, None, None))
        assert B.gacer_load_tenants(ctx, d, 1) == status


def test_a_residual_that_is_written_later_is_no_input(ctx):
    """Tensor 1 is the residual of the first operator and what the second writes."""
    t = (B.gacer_tensor * 3)(*[B.gacer_tensor(BATCH, IN, TOKENS, 1, AT[i], 0, 0, 0) for i in range(3)])
    d = B.gacer_fp8_norm(1, rows(4, IN))
    for second, status in ((1, B.GACER_ESHAPE), (2, B.GACER_OK)):
        ops = (B.gacer_op * 2)(B.gacer_op(N, 0, -1, 1, -1, C.addressof(d), None, None, None, 0, 0, 1, 1, 1, 0, 1, 0, 1e-6),
                               B.gacer_op(B.GACER_ACT, 0, -1, -1, second, None, None, None, None, 0, 0, 1, 1, 1, 0, 1, 1, 1.0))
        desc = (B.gacer_tenant * 1)(B.gacer_tenant(2, ops, 3, t, 0, second, B.GACER_F32, BATCH, None, None))
        assert B.gacer_load_tenants(ctx, desc, 1) == status, B.gacer_last_error(ctx)


# -- the oracle ------------------------------------------------------------------------------------------------------------------------
def test_the_oracles_codes_are_those_of_the_format():
    x = np.concatenate((R.GRID, -R.GRID, (R.GRID[:-1] + R.GRID[1:]) / 2, np.random.default_rng(0).normal(0, 60, 5000), 10.0 ** np.random.default_rng(1).uniform(-4, 2.6, 5000)))
    want = torch.from_numpy(x).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.nearest(x.astype(np.float32).astype(np.float64)), want)


def test_the_oracle_sees_a_wrong_code_and_a_wrong_scale():
    g = torch.Generator().manual_seed(1)
    codes, scales, y = R.rows(g, 4, 144)
    m = torch.stack([y[:, :128].abs().amax(1), y[:, 128:].abs().amax(1)])
    scales = (m / 448).float()
    of = scales.double().t().repeat_interleave(128, 1)[:, :144]
    codes = torch.from_numpy(R.nearest((y / of).numpy()))
    err = 1e-7 * y.abs()
    R.check_rows(codes, scales, y, err)
    for spoil in (lambda c, s: c.__setitem__((1, 3), c[1, 3] * 1.125 + 2.0 ** -9), lambda c, s: s.__setitem__((1, 2), s[1, 2] * 1.00001), lambda c, s: s.__setitem__((0, 0), float("nan"))):
        c, s = codes.clone(), scales.clone()
        spoil(c, s)
        with pytest.raises(AssertionError):
            R.check_rows(c, s, y, err)
