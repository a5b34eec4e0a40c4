"""Products of 8-bit rows under plans that cut the batch, in every tile, whole and in slices, and through every join (tests/test_host_fp8_plan_sizes.py sees that the
sizes leave none out): against 64 bits (tests/fp8_ref.py), and every plan's bits against the whole's."""
import ctypes as C

import pytest
import torch

import fp8_ref as R
import test_gpu_fp8 as G

pytestmark = pytest.mark.gpu
BATCH = 5
# tokens of a sequence, in, out
GEMMS = [(1, 400, 80), (4, 3088, 80), (1, 8208, 80),                                        # few rows: whole, in two and eight slices
         (1, 144, 80), (8, 3088, 80), (4, 4112, 80), (4, 8208, 80),                         # 64x32: whole, two, four, eight
         (13, 144, 6656), (260, 4112, 80), (150, 8208, 80),                                 # 64x64: whole, four, eight
         (260, 144, 2064), (13, 8208, 6656), (13, 8208, 4096),                              # 128x128: whole, four, eight
         (410, 144, 2064), (13, 14336, 6656)]                                               # 256x128: whole, eight
GATED = [(1, 144, 80), (1, 2064, 80), (1, 4112, 80), (1, 8208, 80),                         # 256x32: whole, two, four, eight
         (600, 144, 304), (820, 3088, 80), (410, 4112, 80), (260, 8208, 80),                # 256x64
         (200, 144, 2064), (820, 4112, 144), (410, 4112, 144), (410, 8208, 80)]             # 256x128


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gated,codes,tokens,cin,cout", [(False, False, *s) for s in GEMMS] + [(True, c, *s) for s in GATED for c in (True, False)])
def test_every_tile_whole_and_in_slices_under_plans(dtype, gated, codes, tokens, cin, cout):
    from paper_2304_11745_amd import binding as B
    from paper_2304_11745_amd import tokens as T
    g = torch.Generator(device="cuda").manual_seed(cin + tokens)
    n = BATCH * tokens
    xc, xs, x = G.wide(g, n, cin, None)
    (wc, ws, w), (uc, us, u) = G.wide(g, cout, cin, cin ** -0.5), G.wide(g, cout, cin, cin ** -0.5)
    rows = T.Fp8Rows(xc.view(BATCH, tokens, cin), xs)
    out = G.empty_rows(BATCH, tokens, cout) if codes else torch.full((BATCH, tokens, cout), 7.0, dtype=G.DT[dtype], device="cuda")
    ops = T.OpList(G.DT[dtype], BATCH)
    if gated:
        ops.gated_fp8(rows, T.Fp8Weight(wc, ws), T.Fp8Weight(uc, us), out, act="silu")
    else:
        ops.gemm_fp8(rows, T.Fp8Weight(wc, ws), out, act="silu")
    state = [out.codes, out.scales] if codes else [out]
    s = T.TokenSession([ops])
    s.run(B.GACER_MODE_SEQUENTIAL)
    (y, e), (b, eb) = R.product(x, w), R.product(x, u)
    f = R.act(y, "silu")
    ef = 1.5 * e + 2.0 ** -18 * (f.abs() + 1.5 * e)
    want, err = (f * b, f.abs() * eb + b.abs() * ef + ef * eb) if gated else (f, ef)
    err = err + 2.0 ** -23 * (want.abs() + err)
    if codes:
        R.check_rows(out.codes.cpu().view(n, cout), out.scales.cpu(), want.cpu(), err.cpu())
    else:
        assert ((out.double().view(n, cout) - want).abs() <= err + G.HALF[dtype] * (want.abs() + err)).all()
    bits = G.snapshot(state)
    for sizes in ([2, 3], [1, 1, 1, 1, 1], [4, 1]):
        arr = (C.c_int * len(sizes))(*sizes)
        sp = (B.gacer_split * 1)(B.gacer_split(0, 0, B.GACER_AXIS_BATCH, len(sizes), arr, 0))
        B.check(s.ctx, B.gacer_set_plan(s.ctx, C.byref(B.gacer_plan(1, sp, 0, None))))
        G.scrub(state)
        s.run(B.GACER_MODE_PLAN)
        assert G.same(G.snapshot(state), bits), sizes
    s.close()
