"""Products of 8-bit rows under scales whose product is no ordinary fp32 number, against plain implementations in 64 bits (tests/fp8_ref.py), in few and many rows,
whole and in slices."""
import ctypes as C

import pytest
import torch

import fp8_ref as R
import test_gpu_fp8 as G
from test_gpu_fp8_numbers import SIZES, rows_of, weight_of

pytestmark = pytest.mark.gpu


def extremes(g, tokens, cin, cout, tiny):
    """Operands whose scales are ordinary numbers, while some products of two are not.  tiny: every third row's and the first two weight blocks' about 2^-62 of the others.
    Otherwise block 1 of every third row and of the weights has scales 2^76 times the others, and codes that leave a product of 2^-18 or nothing."""
    xc, xs, _ = R.rows(g, tokens, cin)
    wc, ws, _ = R.weight(g, cout, cin)
    some = torch.arange(tokens) % 3 == 0
    if tiny:
        xs[:, some] *= 2.0 ** -62
        ws[:2] *= 2.0 ** -62
    else:
        xs[1, some] *= 2.0 ** 76
        ws[:, 1] *= 2.0 ** 76
        block = xc[:, 128:256].float()
        block[some] = 0
        block[torch.arange(tokens) % 6 == 3, 0] = 2.0 ** -9
        xc[:, 128:256] = block.to(xc.dtype)
        column = wc[:, 128].float()
        wc[:, 128] = (2.0 ** -9 * torch.where(column < 0, -1.0, 1.0)).to(wc.dtype)
    x = xc.double() * xs.double().t().repeat_interleave(R.BLOCK, 1)[:, :cin]
    w = wc.double() * ws.double().repeat_interleave(R.BLOCK, 0)[:cout].repeat_interleave(R.BLOCK, 1)[:, :cin]
    return (xc, xs, x), (wc, ws, w)


def bound(x, w):
    """fp8_ref.product, where each of a row's blocks may also round to a step of 2^-149 once when it is scaled, once when it is added, and once in every join."""
    y, e = R.product(x, w)
    return y, e + 4 * R.blocks(x.shape[1]) * 2.0 ** -149


@pytest.mark.parametrize("tiny", [True, False])
@pytest.mark.parametrize("tokens,cin,cout", SIZES + [(7, 4112, 80)])
def test_scales_whose_product_is_no_ordinary_number(tokens, cin, cout, tiny):
    g = G.gen(tokens + cout)
    (xc, xs, x), (wc, ws, w) = extremes(g, tokens, cin, cout, tiny)
    out, kept = torch.full((1, tokens, cout), 7.0, device="cuda"), torch.full((1, tokens, cout), 7.0, device="cuda")
    uc, us, _ = R.weight(g, cout, cin)
    if tiny:
        us *= 2.0 ** 60                                     # with the tiny rows an ordinary product
    else:
        us[:, 1] *= 2.0 ** -80
    u = uc.double() * us.double().repeat_interleave(R.BLOCK, 0)[:cout].repeat_interleave(R.BLOCK, 1)[:, :cin]
    rows, gate, up = rows_of(tokens, xc, xs), weight_of(wc, ws), weight_of(uc, us)
    if not tiny:                                            # what meets the large rows and gates must stay below the largest fp32 number
        assert (R.product(x, w)[0].abs().max() < 1e38) and (R.product(x, u)[0].abs().max() < 1e30)

    def build(o):
        o.gemm_fp8(rows, gate, out)
        o.gated_fp8(rows, gate, up, kept, act="none")
    G.run(build, "f32", 1)
    y, e = bound(x, w)
    assert torch.isfinite(out).all() and ((out[0].cpu().double() - y).abs() <= e + 2.0 ** -24 * y.abs()).all()
    b, eb = bound(x, u)
    want = y * b
    err = y.abs() * eb + b.abs() * e + e * eb
    err = err + 2.0 ** -23 * (want.abs() + err) + 2.0 ** -149
    small = want.abs() < 1e38
    assert small.float().mean() > 0.5 and torch.isfinite(kept[0].cpu()[small]).all() and ((kept[0].cpu().double() - want).abs() <= err)[small].all()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("tokens,cin,cout", [(3, 4112, 80), (30, 400, 304), (300, 400, 2064)])
def test_plans_give_the_bits_of_the_whole_beside_such_scales(gated, tokens, cin, cout):
    """Rows whose scales are ordinary keep their bits, whichever rows are computed beside them."""
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    batch = 5
    g = G.gen(tokens)
    (xc, xs, _), (wc, ws, _) = extremes(g, batch * tokens, cin, cout, True)
    rows, w = T.Fp8Rows(G.dev(xc.view(batch, tokens, cin)), G.dev(xs)), weight_of(wc, ws)
    up = weight_of(*R.weight(g, cout, cin)[:2])
    out = torch.zeros(batch, tokens, cout, device="cuda")
    ops = T.OpList(torch.float32, batch)
    if gated:
        ops.gated_fp8(rows, w, up, out)
    else:
        ops.gemm_fp8(rows, w, out)
    s = T.TokenSession([ops])
    s.run(B.GACER_MODE_SEQUENTIAL)
    want = G.snapshot([out])
    for sizes in ([2, 3], [1, 1, 1, 1, 1], [4, 1]):
        arr = (C.c_int * len(sizes))(*sizes)
        sp = (B.gacer_split * 1)(B.gacer_split(0, 0, B.GACER_AXIS_BATCH, len(sizes), arr, 0))
        B.check(s.ctx, B.gacer_set_plan(s.ctx, C.byref(B.gacer_plan(1, sp, 0, None))))
        G.scrub([out])
        s.run(B.GACER_MODE_PLAN)
        assert G.same(G.snapshot([out]), want), sizes
    s.close()
