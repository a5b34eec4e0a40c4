"""NaN through the activations of products of 8-bit rows, in few and many rows, whole and in slices."""
import pytest
import torch

import fp8_ref as R
import test_gpu_fp8 as G

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "relu6", "gelu", "hard_swish", "hard_sigmoid", "silu", "gelu_tanh"]
# tokens, in, out: a few rows whole and in slices, small tiles whole and in slices, large tiles
SIZES = [(1, 400, 304), (1, 4112, 304), (40, 400, 304), (300, 4112, 304), (1500, 400, 2064)]


def rows_of(tokens, xc, xs):
    from paper_2304_11745_amd import tokens as T
    return T.Fp8Rows(G.dev(xc.view(1, tokens, -1)), G.dev(xs))


def weight_of(wc, ws):
    from paper_2304_11745_amd import tokens as T
    return T.Fp8Weight(G.dev(wc), G.dev(ws))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,cin,cout", SIZES)
def test_what_is_no_number_passes_every_activation(act, tokens, cin, cout):
    """A NaN scale of a row's block or of a weight block reaches that row and those features whatever the activation, and changes no bit beside them."""
    g = G.gen(tokens + cin)
    xc, xs, _ = R.rows(g, tokens, cin)
    wc, ws, _ = R.weight(g, cout, cin)
    uc, us, _ = R.weight(g, cout, cin)
    row = tokens // 2 if tokens > 1 else None
    bad = torch.zeros(tokens, cout, dtype=torch.bool)
    bad[:, 128:256] = True
    spoilt_x, spoilt_w = xs.clone(), ws.clone()
    spoilt_w[1, 3] = float("nan")
    if row is not None:
        spoilt_x[1, row], bad[row] = float("nan"), True
    outs = []
    for x, w in ((xs, ws), (spoilt_x, spoilt_w)):
        rows, gate, up = rows_of(tokens, xc, x), weight_of(wc, w), weight_of(uc, us)
        y, z, codes = torch.zeros(1, tokens, cout, device="cuda"), torch.zeros(1, tokens, cout, device="cuda"), G.empty_rows(1, tokens, cout)

        def build(o):
            o.gemm_fp8(rows, gate, y, act=act)
            o.gated_fp8(rows, gate, up, z, act=act)
            o.gated_fp8(rows, gate, up, codes, act=act)
        G.run(build, "f32", 1)
        outs.append((y[0].cpu(), z[0].cpu(), codes.codes[0].view(torch.uint8).cpu(), codes.scales.cpu()))
    for clean, spoilt in zip(outs[0][:2], outs[1][:2]):
        assert torch.equal(torch.isnan(spoilt), bad) and not torch.isnan(clean).any()
        assert torch.equal(spoilt[~bad], clean[~bad])
    blocks = torch.stack([bad[:, b * 128] for b in range(R.blocks(cout))])
    assert torch.equal(torch.isnan(outs[1][3]), blocks) and torch.equal(outs[1][3][~blocks], outs[0][3][~blocks])
    assert torch.equal(outs[1][2][~bad], outs[0][2][~bad]) and (outs[1][2][bad] == 0).all()
