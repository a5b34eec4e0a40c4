"""Operators on 8-bit rows on the GPU against plain implementations in 64 bits (tests/fp8_ref.py).

Tolerances.  A sum of C squares is added lane by lane (at most 64 terms), then over at most 10 + 16 halves: 2^-24 each, and half of it after the root; with
the division, the root and three products y is off by at most 64 units of 2^-24 = 2^-18.  Products: fp8_ref.product.  An activation's slope is at most 1.5, its own
arithmetic within 2^-18 of its value (the exponential of up to 88 takes its argument's rounding, 88 units of 2^-24, where the value is not yet below 2^-126).
A bf16 result is one rounding, 2^-8 of it; of fp32, 2^-24 and no more than the terms before it."""
import ctypes as C

import pytest
import torch

import fp8_ref as R

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def dev(t):
    return None if t is None else t.cuda().contiguous()


def run(build, dtype, batch):
    from paper_2304_11745_amd import tokens as T
    ops = T.OpList(DT[dtype], batch)
    build(ops)
    s = T.TokenSession([ops])
    s.enqueue()
    torch.cuda.synchronize()
    s.close()


def empty_rows(batch, tokens, features, fill=0x55):
    """8-bit rows that hold something else before."""
    from paper_2304_11745_amd import tokens as T
    return T.Fp8Rows(torch.full((batch, tokens, features), fill, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                     torch.full((R.blocks(features), batch * tokens), 7.0, device="cuda"))


# -- norm and codes --------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,tokens,width,norm,gamma,res,total", [
    (1, 1, 16, True, True, True, True),
    (1, 1, 128, True, False, False, False),
    (2, 3, 144, True, True, True, False),          # a last block of 16
    (1, 5, 1008, False, False, True, True),
    (3, 1, 1040, True, True, False, True),         # more than two runs a lane of a wave
    (2, 2, 2048, True, True, True, True),
    (1, 7, 4096, True, True, True, True),
    (3, 3, 5008, True, True, True, True),
    (1, 2, 12288, False, False, False, False),
    (1, 2, 16400, True, True, True, True),         # the large workgroup
    (1, 1, 65536, True, True, True, True),
    (3, 2, 40976, True, True, True, False),        # in pieces, the last one short
    (1, 3, 32784, False, False, True, True),
])
def test_norm_and_codes(dtype, batch, tokens, width, norm, gamma, res, total):
    g = gen(width + tokens)
    n = batch * tokens
    x = (3 * torch.randn(batch, tokens, width, generator=g) * (1 + 9 * (torch.rand(width, generator=g) < 0.01))).to(DT[dtype])
    x.view(n, width)[0, :min(128, width)] = 0                                   # a block of zeros
    r = torch.randn(batch, tokens, width, generator=g).to(DT[dtype]) if res else None
    if res:
        r.view(n, width)[0, :min(128, width)] = 0
    gm = 1 + 0.3 * torch.randn(width, generator=g) if gamma else None
    rows, out = empty_rows(batch, tokens, width), torch.full((batch, tokens, width), 7.0, dtype=DT[dtype], device="cuda") if total else None
    dx, dr, dg = dev(x), dev(r), dev(gm)
    if norm:
        run(lambda o: o.rmsnorm_fp8(dx, rows, dg, eps=1e-5, res=dr, sum=out), dtype, batch)
    else:
        run(lambda o: o.quantise_fp8(dx, rows, res=dr, sum=out), dtype, batch)
    h = x.double() + (r.double() if res else 0)
    if total:
        assert (((out.cpu().double() - h).abs()) <= (HALF[dtype] + 2.0 ** -24) * h.abs()).all()
    h = h.view(n, width)
    y = h * ((h * h).mean(-1, keepdim=True) + 1e-5).rsqrt() * (gm.double() if gamma else 1) if norm else h
    R.check_rows(rows.codes.cpu().view(n, width), rows.scales.cpu(), y, (2.0 ** -18 if norm else 2.0 ** -24) * y.abs())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,width", [(1, 1), (3, 7), (5, 129), (2, 1000), (3, 4097), (2, 20001), (5, 49999), (1, 32768)])
def test_norm_in_the_tenants_type(dtype, tokens, width):
    g = gen(width)
    x, r, gm = (torch.randn(2, tokens, width, generator=g) * 4).to(DT[dtype]), torch.randn(2, tokens, width, generator=g).to(DT[dtype]), 1 + 0.2 * torch.randn(width, generator=g)
    dx, dr, dg, out = dev(x), dev(r), dev(gm), torch.full((2, tokens, width), 7.0, dtype=DT[dtype], device="cuda")
    run(lambda o: o.rmsnorm(dx, dg, out, eps=1e-6, res=dr), dtype, 2)
    h = x.double() + r.double()
    y = h * ((h * h).mean(-1, keepdim=True) + 1e-6).rsqrt() * gm.double()
    assert ((out.cpu().double() - y).abs() <= (HALF[dtype] + 2.0 ** -18) * y.abs()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_codes_of_awkward_values(dtype):
    """Infinities, NaN, values at both ends of the range, and those between two codes."""
    g = gen(3)
    x = torch.randn(1, 8, 384, generator=g)
    x[0, 0, 5], x[0, 1, 130], x[0, 2, 383], x[0, 3, 0] = float("inf"), float("nan"), float("-inf"), -3e38
    x[0, 4] *= 1e-30
    x[0, 5] = 0
    x[0, 6, :128] = torch.cat((torch.tensor([448.0]), torch.from_numpy((R.GRID[:-1] + R.GRID[1:]) / 2).float(), torch.tensor([0.0])))      # ties
    x = x.to(DT[dtype])
    rows, dx = empty_rows(1, 8, 384), dev(x)
    run(lambda o: o.quantise_fp8(dx, rows), dtype, 1)
    y = x[0].double()
    R.check_rows(rows.codes.cpu()[0], rows.scales.cpu(), y, torch.zeros_like(y))
    if dtype == "f32":
        assert torch.equal(rows.codes.cpu()[0, 6, :128].double(), torch.from_numpy(R.nearest(x[0, 6, :128].double().numpy())))
    # a row with an infinity has no norm: every block of it stands for NaNs
    run(lambda o: o.rmsnorm_fp8(dx, rows), dtype, 1)
    values = rows.values().cpu()[0]
    assert torch.isnan(values[1]).all() and torch.isnan(values[0, :128]).all() and not torch.isnan(values[4:]).any()


def test_more_rows_than_a_grid_holds():
    n, width = 3 << 20, 16
    x = torch.randn(n, 1, width, device="cuda").bfloat16()
    rows = empty_rows(n, 1, width)
    run(lambda o: o.quantise_fp8(x, rows), "bf16", n)
    pick = torch.tensor([0, 1, (1 << 20) + 5, (1 << 22) // 2 - 1, n - 1])
    y = x[pick.cuda(), 0].cpu().double()
    R.check_rows(rows.codes[pick.cuda(), 0].cpu(), rows.scales[:, pick.cuda()].cpu(), y, torch.zeros_like(y))
    assert not (rows.scales == 7.0).any()


# -- products --------------------------------------------------------------------------------------------------------------------------
SHAPES = [  # batch, tokens, in, out features
    (1, 1, 16, 1), (1, 1, 128, 32), (3, 1, 144, 33), (1, 2, 4096, 64), (2, 17, 400, 100), (5, 1, 6400, 48), (1, 31, 256, 513), (4, 8, 1040, 130),
    (3, 11, 272, 257), (1, 64, 2048, 128), (2, 35, 528, 300), (1, 127, 128, 96), (3, 43, 1168, 160), (1, 200, 784, 333), (2, 128, 512, 512), (1, 500, 272, 1000),
    (7, 73, 640, 264), (1, 1030, 384, 520),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,tokens,cin,cout", SHAPES)
def test_gemm(dtype, batch, tokens, cin, cout):
    from paper_2304_11745_amd import tokens as T
    g = gen(cin + cout + tokens)
    n = batch * tokens
    xc, xs, x = R.rows(g, n, cin)
    wc, wsc, w = R.weight(g, cout, cin)
    name = ["none", "relu", "gelu", "silu", "gelu_tanh", "hard_swish", "relu6", "hard_sigmoid"][(cin // 16 + cout) % 8]
    bias = torch.randn(cout, generator=g) if cout % 2 else None
    res = torch.randn(batch, tokens, cout, generator=g).to(DT[dtype]) if tokens % 2 else None
    rows, wt = T.Fp8Rows(dev(xc.view(batch, tokens, cin)), dev(xs)), T.Fp8Weight(dev(wc), dev(wsc))
    out, db, dr = torch.full((batch, tokens, cout), 7.0, dtype=DT[dtype], device="cuda"), dev(bias), dev(res)
    run(lambda o: o.gemm_fp8(rows, wt, out, bias=db, act=name, res=dr), dtype, batch)
    y, e = R.product(x, w)
    for more in (bias, None if res is None else res.view(n, cout)):
        if more is not None:
            e = e + 2.0 ** -24 * (y.abs() + more.abs().double() + e)
            y = y + more.double()
    want = R.act(y, name)
    err = 1.5 * e + (HALF[dtype] + 2.0 ** -18) * (want.abs() + 1.5 * e)
    assert ((out.cpu().double().view(n, cout) - want).abs() <= err).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("batch,tokens,cin,cout", SHAPES)
def test_gated(dtype, codes, batch, tokens, cin, cout):
    from paper_2304_11745_amd import tokens as T
    g = gen(cin + cout + tokens + 1)
    n = batch * tokens
    if codes:
        cout = -(-cout // 16) * 16
    xc, xs, x = R.rows(g, n, cin)
    (gc, gs, gv), (uc, us, uv) = R.weight(g, cout, cin), R.weight(g, cout, cin)
    name = ["silu", "gelu_tanh", "gelu", "relu", "none"][(cin // 16 + tokens) % 5]
    rows, gate, up = T.Fp8Rows(dev(xc.view(batch, tokens, cin)), dev(xs)), T.Fp8Weight(dev(gc), dev(gs)), T.Fp8Weight(dev(uc), dev(us))
    out = empty_rows(batch, tokens, cout) if codes else torch.full((batch, tokens, cout), 7.0, dtype=DT[dtype], device="cuda")
    run(lambda o: o.gated_fp8(rows, gate, up, out, act=name), dtype, batch)
    (a, ea), (b, eb) = R.product(x, gv), R.product(x, uv)
    f = R.act(a, name)
    ea = 1.5 * ea + 2.0 ** -18 * (f.abs() + 1.5 * ea)
    want = f * b
    err = f.abs() * eb + b.abs() * ea + ea * eb
    err = err + 2.0 ** -23 * (want.abs() + err)
    if codes:
        R.check_rows(out.codes.cpu().view(n, cout), out.scales.cpu(), want, err)
    else:
        assert ((out.cpu().double().view(n, cout) - want).abs() <= err + HALF[dtype] * (want.abs() + err)).all()


# sizes that take the other tiles and the inner extent in slices (tests/test_host_fp8_dispatch.py sees that none is left out)
WIDE_GEMMS = [(1, 1, 400, 70), (1, 17, 3088, 70), (3, 11, 3088, 71), (1, 1500, 4112, 70), (2, 1025, 144, 300), (3, 1000, 144, 1001), (4, 128, 14336, 4096), (50, 41, 144, 2068), (13, 5, 9616, 5520),
              (7, 31, 6416, 2050), (8, 165, 160, 6650), (5, 264, 656, 6656)]      # the last two end in tiles of half the rows, some of them empty
WIDE_GATED = [(1, 1, 2000, 80), (2, 1500, 144, 304), (3, 1000, 144, 704), (5, 410, 4112, 80), (50, 41, 4112, 144), (3, 16, 5120, 2064), (5, 264, 656, 3328)]


def wide(g, rows, width, spread):
    """8-bit operands made on the GPU: (float8 codes, scales, float64 values); blocks of rows (spread None) or of 128 by 128."""
    codes = (torch.randn(rows, width, generator=g, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    if spread is None:
        scales = (0.2 + torch.rand(R.blocks(width), rows, generator=g, device="cuda")) / 60
        return codes, scales, codes.double() * scales.double().t().repeat_interleave(R.BLOCK, 1)[:, :width]
    scales = (0.5 + torch.rand(R.blocks(rows), R.blocks(width), generator=g, device="cuda")) * spread / 60
    return codes, scales, codes.double() * scales.double().repeat_interleave(R.BLOCK, 0)[:rows].repeat_interleave(R.BLOCK, 1)[:, :width]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,tokens,cin,cout", WIDE_GEMMS)
def test_gemm_in_every_tile(dtype, batch, tokens, cin, cout):
    from paper_2304_11745_amd import tokens as T
    g = torch.Generator(device="cuda").manual_seed(cin + cout)
    n = batch * tokens
    xc, xs, x = wide(g, n, cin, None)
    wc, wsc, w = wide(g, cout, cin, cin ** -0.5)
    bias, res = torch.randn(cout, generator=g, device="cuda"), torch.randn(batch, tokens, cout, generator=g, device="cuda").to(DT[dtype])
    out = torch.full((batch, tokens, cout), 7.0, dtype=DT[dtype], device="cuda")
    run(lambda o: o.gemm_fp8(T.Fp8Rows(xc.view(batch, tokens, cin), xs), T.Fp8Weight(wc, wsc), out, bias=bias, act="silu", res=res), dtype, batch)
    y, e = R.product(x, w)
    y, e = y + bias.double() + res.view(n, cout).double(), e + 2.0 ** -22 * (y.abs() + 8)
    want = R.act(y, "silu")
    assert ((out.double().view(n, cout) - want).abs() <= 1.5 * e + (HALF[dtype] + 2.0 ** -18) * (want.abs() + 1.5 * e)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("batch,tokens,cin,cout", WIDE_GATED)
def test_gated_in_every_tile(dtype, codes, batch, tokens, cin, cout):
    from paper_2304_11745_amd import tokens as T
    g = torch.Generator(device="cuda").manual_seed(cin + cout)
    n = batch * tokens
    xc, xs, x = wide(g, n, cin, None)
    (gc, gs, gv), (uc, us, uv) = wide(g, cout, cin, cin ** -0.5), wide(g, cout, cin, cin ** -0.5)
    out = empty_rows(batch, tokens, cout) if codes else torch.full((batch, tokens, cout), 7.0, dtype=DT[dtype], device="cuda")
    run(lambda o: o.gated_fp8(T.Fp8Rows(xc.view(batch, tokens, cin), xs), T.Fp8Weight(gc, gs), T.Fp8Weight(uc, us), out, act="gelu"), dtype, batch)
    (a, ea), (b, eb) = R.product(x, gv), R.product(x, uv)
    f = R.act(a, "gelu")
    ea = 1.5 * ea + 2.0 ** -18 * (f.abs() + 1.5 * ea)
    want = f * b
    err = f.abs() * eb + b.abs() * ea + ea * eb
    err = err + 2.0 ** -23 * (want.abs() + err)
    if codes:
        R.check_rows(out.codes.cpu().view(n, cout), out.scales.cpu(), want.cpu(), err.cpu())
    else:
        assert ((out.double().view(n, cout) - want).abs() <= err + HALF[dtype] * (want.abs() + err)).all()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("tokens,cin,cout", [(1, 3088, 144), (1, 400, 70), (13, 3088, 144), (300, 4112, 144), (200, 144, 1008), (410, 144, 2064), (264, 656, 6656)])
def test_plans_give_the_bits_of_the_whole(gated, tokens, cin, cout):
    """Every tile, whole and in slices, with the batch cut unevenly, also over two streams."""
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    g = torch.Generator(device="cuda").manual_seed(cin + tokens)
    batch = 5
    cout = -(-cout // 16) * 16 if gated else cout
    xc, xs, _ = wide(g, batch * tokens, cin, None)
    ws = [wide(g, cout, cin, cin ** -0.5)[:2] for _ in range(2)]
    rows, out = T.Fp8Rows(xc.view(batch, tokens, cin), xs), empty_rows(batch, tokens, cout) if gated else torch.empty(batch, tokens, cout, dtype=torch.bfloat16, device="cuda")
    ops = T.OpList(torch.bfloat16, batch)
    if gated:
        ops.gated_fp8(rows, T.Fp8Weight(*ws[0]), T.Fp8Weight(*ws[1]), out)
    else:
        ops.gemm_fp8(rows, T.Fp8Weight(*ws[0]), out)
    state = [out.codes, out.scales] if gated else [out]
    stream, sibling = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    s = T.TokenSession([ops], [stream])
    d = (B.gacer_tenant * 1)(ops.descriptor(stream.cuda_stream))
    d[0].sibling_stream = sibling.cuda_stream
    B.check(s.ctx, B.gacer_load_tenants(s.ctx, d, 1))
    s.run(B.GACER_MODE_SEQUENTIAL)
    want = snapshot(state)
    for sizes in ([2, 3], [1, 1, 1, 1, 1], [4, 1]):
        for side in (0, 1):
            arr = (C.c_int * len(sizes))(*sizes)
            sp = (B.gacer_split * 1)(B.gacer_split(0, 0, B.GACER_AXIS_BATCH, len(sizes), arr, side))
            B.check(s.ctx, B.gacer_set_plan(s.ctx, C.byref(B.gacer_plan(1, sp, 0, None))))
            scrub(state)
            s.run(B.GACER_MODE_PLAN)
            assert same(snapshot(state), want), (sizes, side)
    s.close()


@pytest.mark.parametrize("tokens", [1, 40, 300])
def test_a_row_or_block_that_is_no_number_stays_alone(tokens):
    """NaN scales of one row's block and of one weight block reach that row and those features, and nothing beside them."""
    from paper_2304_11745_amd import tokens as T
    g = gen(5)
    cin, cout = 400, 300
    xc, xs, _ = R.rows(g, tokens, cin)
    wc, wsc, _ = R.weight(g, cout, cin)
    xs[1, tokens // 2] = float("nan")
    wsc[1, 3] = float("nan")
    out = torch.zeros(1, tokens, cout, device="cuda")
    rows, wt = T.Fp8Rows(dev(xc.view(1, tokens, cin)), dev(xs)), T.Fp8Weight(dev(wc), dev(wsc))
    run(lambda o: o.gemm_fp8(rows, wt, out), "f32", 1)
    bad = torch.zeros(tokens, cout, dtype=torch.bool)
    bad[tokens // 2], bad[:, 128:256] = True, True
    assert torch.equal(torch.isnan(out[0]).cpu(), bad)
    y = empty_rows(1, tokens, 304)
    w304 = [torch.nn.functional.pad(t.view(torch.uint8), (0, 0, 0, 4)).view(torch.float8_e4m3fn) for t in (wc,)][0]
    good = T.Fp8Weight(dev(w304), dev(torch.nan_to_num(wsc, nan=0.01)))
    run(lambda o: o.gated_fp8(rows, good, T.Fp8Weight(dev(w304), dev(wsc)), y), "f32", 1)
    s = torch.isnan(y.scales).cpu()
    want = torch.zeros(3, tokens, dtype=torch.bool)
    want[:, tokens // 2], want[1] = True, True
    assert torch.equal(s, want)


# -- together --------------------------------------------------------------------------------------------------------------------------
def layer(dtype, batch=5, tokens=3, width=272, heads_width=160, ffn=400, seed=4):
    """The dense half of a layer around a projection: norm -> qkv product -> (its first features as context) -> product + residual -> norm -> gated -> product + residual."""
    from paper_2304_11745_amd import tokens as T
    g = gen(seed)
    t = DT[dtype]
    w = {name: R.weight(g, o, i) for name, o, i in (("qkv", heads_width, width), ("o", width, heads_width), ("gate", ffn, width), ("up", ffn, width), ("down", width, ffn))}
    W = {name: T.Fp8Weight(dev(c), dev(s)) for name, (c, s, _) in w.items()}
    e = dict(dtype=t, device="cuda")
    x = torch.randn(batch, tokens, width, generator=g).to(t)
    gammas = [1 + 0.1 * torch.randn(width, generator=g) for _ in range(3)]
    D = dict(x=dev(x), q=torch.empty(batch, tokens, heads_width, **e), a=torch.empty(batch, tokens, width, **e), h=torch.empty(batch, tokens, width, **e),
             z=torch.empty(batch, tokens, width, **e), last=torch.empty(batch, tokens, width, **e))
    n1, c1, n2, f1 = (empty_rows(batch, tokens, k) for k in (width, heads_width, width, ffn))
    ops = T.OpList(t, batch)
    ops.rmsnorm_fp8(D["x"], n1, dev(gammas[0]))
    ops.gemm_fp8(n1, W["qkv"], D["q"])
    ops.quantise_fp8(D["q"], c1)
    ops.gemm_fp8(c1, W["o"], D["a"])
    ops.rmsnorm_fp8(D["a"], n2, dev(gammas[1]), res=D["x"], sum=D["h"])
    ops.gated_fp8(n2, W["gate"], W["up"], f1)
    ops.gemm_fp8(f1, W["down"], D["z"], res=D["h"])
    ops.rmsnorm(D["z"], dev(gammas[2]), D["last"])
    state = [D[k] for k in ("q", "a", "h", "z", "last")] + [t for r in (n1, c1, n2, f1) for t in (r.codes, r.scales)]
    return ops, state, D, (n1, c1, n2, f1), w, gammas, x


def snapshot(state):
    torch.cuda.synchronize()
    return [t.clone() for t in state]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def scrub(state):
    for t in state:
        t.view(torch.uint8).fill_(0x33)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,tokens", [(5, 3), (1, 1), (3, 150)])
def test_a_layer(dtype, batch, tokens):
    """Every operator of a layer on what the one before it left."""
    from paper_2304_11745_amd import tokens as T
    ops, state, D, (n1, c1, n2, f1), w, gammas, x = layer(dtype, batch, tokens)
    s = T.TokenSession([ops])
    s.enqueue()
    torch.cuda.synchronize()
    n = batch * tokens
    flat = {k: v.cpu().double().view(n, -1) for k, v in D.items()}

    def normed(h, gm):
        return h * ((h * h).mean(-1, keepdim=True) + 1e-6).rsqrt() * gm.double()

    def rows(r):
        return r.codes.cpu().view(n, -1), r.scales.cpu()

    def value(r):
        return r.values().cpu().double().view(n, -1)

    def close(got, want, err):
        assert ((got - want).abs() <= err + HALF[dtype] * (want.abs() + err)).all()
    y = normed(flat["x"], gammas[0])
    R.check_rows(*rows(n1), y, 2.0 ** -18 * y.abs())
    close(flat["q"], *R.product(value(n1), w["qkv"][2]))
    R.check_rows(*rows(c1), flat["q"], 0 * flat["q"])
    close(flat["a"], *R.product(value(c1), w["o"][2]))
    h = flat["a"] + flat["x"]
    close(flat["h"], h, 2.0 ** -24 * h.abs())
    y = normed(h, gammas[1])
    R.check_rows(*rows(n2), y, 2.0 ** -18 * y.abs())
    (a, ea), (b, eb) = R.product(value(n2), w["gate"][2]), R.product(value(n2), w["up"][2])
    f = R.act(a, "silu")
    ea = 1.5 * ea + 2.0 ** -18 * (f.abs() + 1.5 * ea)
    err = f.abs() * eb + b.abs() * ea + ea * eb
    R.check_rows(*rows(f1), f * b, err + 2.0 ** -23 * ((f * b).abs() + err))
    z, e = R.product(value(f1), w["down"][2])
    close(flat["z"], z + flat["h"], e + 2.0 ** -23 * (z.abs() + flat["h"].abs()))
    y = normed(flat["z"], gammas[2])
    close(flat["last"], y, 2.0 ** -18 * y.abs())
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 3, 90])
def test_every_way_of_running_gives_the_same_bits(dtype, tokens):
    """gacer_enqueue, the three modes, plans that cut the batch (also over two streams), the checking mode, the static workspace and a replayed graph."""
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    ops, state = layer(dtype, 5, tokens, width=1296, ffn=2064)[:2]
    stream, sibling = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    s = T.TokenSession([ops], [stream])
    s.enqueue()
    want = snapshot(state)

    def again(go):
        scrub(state)
        go()
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
        torch.randn(1000, device="cuda").sum().item()
    s.close()


def test_a_captured_layer_on_the_callers_stream():
    from paper_2304_11745_amd import tokens as T
    ops, state, D = layer("bf16", 4, 1)[:3]
    s = T.TokenSession([ops])
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    s.enqueue()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s.enqueue()
    for k in range(4):
        D["x"].copy_(torch.randn_like(D["x"]))
        s.enqueue()
        want = snapshot(state)
        scrub(state)
        graph.replay()
        assert same(snapshot(state), want), k
        torch.randn(1000, device="cuda").sum().item()
    s.close()


def test_profile_trace_and_search_know_the_operators():
    import synth
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import harness
    ops, state = layer("bf16", 4, 3, width=1296, ffn=2064)[:2]
    tenants, data = synth.build_config(1)
    sess = harness.Session(tenants, data, extra=[ops])
    sess.run(B.GACER_MODE_SEQUENTIAL, 1)
    want = snapshot(state)
    mine = [r for r in sess.trace(B.GACER_MODE_PLAN, 1) if r["tenant"] == len(tenants)]
    assert len(mine) >= len(ops.ops) and all(r["ms"] > 0 for r in mine)
    assert all(r["bytes"] > 0 for r in mine if "join" not in r["kernel"])
    assert sum(r["flops"] for r in mine) == sum(2.0 * 12 * o * i for o, i in ((160, 1296), (1296, 160), (2 * 2064, 1296), (1296, 2064)))
    table = sess.profile()
    assert {r.op for r in table if r.tenant == len(tenants)} == set(range(len(ops.ops)))
    assert same(snapshot(state), want)                          # a profile leaves what a round leaves
    splits, syncs, P, residue = sess.search(table, 20)
    sess.set_plan(splits, syncs)
    scrub(state)
    sess.run(B.GACER_MODE_PLAN, 2)
    assert same(snapshot(state), want)
    sess.close()


def test_a_residual_from_outside():
    """A list that begins behind a caller's own step: two tensors from outside, the residual beside the tenant's input."""
    from paper_2304_11745_amd import tokens as T
    g = gen(8)
    x, r = (dev(torch.randn(2, 3, 64, generator=g)) for _ in range(2))
    rows, total, last = empty_rows(2, 3, 64), torch.empty(2, 3, 64, device="cuda"), torch.empty(2, 3, 64, device="cuda")
    W = R.weight(g, 64, 64)
    wt = T.Fp8Weight(dev(W[0]), dev(W[1]))
    r2 = dev(torch.randn(2, 3, 64, generator=g))

    def build(o):
        o.rmsnorm_fp8(x, rows, res=r, sum=total)
        o.gemm_fp8(rows, wt, last, res=r2)
    run(build, "f32", 2)
    assert torch.equal(total, x + r)
    y, e = R.product(rows.values().cpu().double().view(6, 64), W[2])
    y = y + r2.cpu().double().view(6, 64)
    assert ((last.cpu().double().view(6, 64) - y).abs() <= e + 2.0 ** -22 * (y.abs() + 8)).all()


def test_weights_are_quantised_to_the_nearest_codes():
    from paper_2304_11745_amd import tokens as T
    w = torch.randn(300, 400, generator=gen(9)).cuda()
    w[:128, 128:256] = 0
    q = T.Fp8Weight.quantise(w)
    for b in range(3):
        for c in range(4):
            part, scale = w[b * 128:(b + 1) * 128, c * 128:(c + 1) * 128].cpu().double(), q.scales[b, c].item()
            assert abs(scale - max(part.abs().max().item(), 2.0 ** -60) / 448) <= 2.0 ** -23 * scale
            got = q.codes[b * 128:(b + 1) * 128, c * 128:(c + 1) * 128].cpu().double()
            d = 2.0 ** -22 * (part / scale).abs()
            assert (got.numpy() >= R.nearest((part / scale - d).numpy())).all() and (got.numpy() <= R.nearest((part / scale + d).numpy())).all()
    assert q.values().shape == w.shape


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_example_decodes_with_8_bit_weights(dtype):
    """examples/decode.py --weights fp8: the last step's hidden states lie where a list that takes the same tokens as one prompt puts them.  A step's rows go through
    other tiles than a prompt's, so that values next to a line between two codes may fall on either side: a step of e4m3 is 2^-3 of a value, of the 4-bit cache a
    fifteenth of a group's range, and each is one of hundreds of addends of a hidden feature; a tenth of the largest is far beyond what they add up to."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import decode
    from paper_2304_11745_amd import tokens as T
    steps, batch = 5, 3
    said, logits = decode.serve(DT[dtype], batch, steps, vision=True, fp8=True)
    assert ((said >= 0) & (said < 8000)).all() and torch.isfinite(logits).all()
    again, same_logits = decode.serve(DT[dtype], batch, steps, vision=False, fp8=True)
    assert torch.equal(said, again) and torch.equal(logits, same_logits)
    d = decode.Decoder(DT[dtype], batch, fp8=True)              # the same weights, by their seed
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
    last = out[torch.arange(batch, device="cuda"), count.long() - 1].float()
    want = (last * (last * last).mean(-1, keepdim=True).add(1e-6).rsqrt()) @ d.out.float().t()
    assert (logits[:, 0].float() - want).abs().max() <= 0.1 * want.abs().max()
    s.close()


def test_operator_lists_refuse_what_they_can_see():
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    f32 = dict(device="cuda")
    x, out, rows = torch.zeros(2, 3, 64, **f32), torch.zeros(2, 3, 48, **f32), T.Fp8Rows.allocate(2, 3, 64)
    w = T.Fp8Weight.quantise(torch.ones(48, 64, **f32))
    for bad in (lambda o: o.rmsnorm_fp8(x, T.Fp8Rows.allocate(2, 3, 80)), lambda o: o.rmsnorm_fp8(x, rows, torch.ones(48, **f32)), lambda o: o.rmsnorm_fp8(x.bfloat16(), rows),
                lambda o: o.gemm_fp8(rows, w, torch.zeros(2, 3, 40, **f32)), lambda o: o.gemm_fp8(T.Fp8Rows.allocate(2, 3, 80), w, out), lambda o: o.gemm_fp8(T.Fp8Rows.allocate(3, 2, 64), w, out),
                lambda o: o.gemm_fp8(rows, w, out, bias=torch.zeros(40, **f32)), lambda o: o.gated_fp8(rows, w, T.Fp8Weight.quantise(torch.ones(32, 64, **f32)), out),
                lambda o: T.Fp8Rows(rows.codes, rows.scales[:, :5]), lambda o: T.Fp8Rows(rows.codes.view(torch.uint8), rows.scales), lambda o: T.Fp8Weight(w.codes, w.scales.double()),
                lambda o: T.Fp8Weight(w.codes.t(), w.scales), lambda o: T.Fp8Rows(rows.codes.cpu(), rows.scales.cpu())):
        with pytest.raises(ValueError):
            bad(T.OpList(torch.float32, 2))
    for build, why in ((lambda o: o.rmsnorm_fp8(x, rows, sum=x), "shares memory"), (lambda o: o.gated_fp8(rows, T.Fp8Weight.quantise(torch.ones(64, 64, **f32)), T.Fp8Weight.quantise(torch.ones(64, 64, **f32)), rows), "shares memory"),
                       (lambda o: o.gemm_fp8(rows, w, torch.zeros(2, 4, 48, **f32)), "position for every row")):
        ops = T.OpList(torch.float32, 2)                       # what only the library sees comes back as its error
        build(ops)
        with pytest.raises(B.GacerError, match=why):
            T.TokenSession([ops])
