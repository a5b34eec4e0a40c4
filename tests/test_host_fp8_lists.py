"""Operator lists on 8-bit rows without a GPU: tensors that only look like ones on a GPU, to see what the lists refuse and what they write down."""
import pytest
import torch

from paper_2304_11745_amd import binding as B
from paper_2304_11745_amd import tokens as T
from test_host_token_lists import Fake

F8, F32 = torch.float8_e4m3fn, torch.float32


def rows(features, batch=3, tokens=5, device="cuda:0"):
    return T.Fp8Rows(Fake(F8, batch, tokens, features, device=device), Fake(F32, -(-features // 128), batch * tokens, device=device))


def weight(out, cin, device="cuda:0"):
    return T.Fp8Weight(Fake(F8, out, cin, device=device), Fake(F32, -(-out // 128), -(-cin // 128), device=device))


class At(Fake):
    """A tensor with a place of its own."""
    count = 0

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        At.count += 1
        self.at = At.count << 24

    def data_ptr(self):
        return self.at


def tensor(features, device="cuda:0"):
    return At(F32, 3, 5, features, device=device)


def test_rows_and_weights_are_whole_and_on_one_gpu():
    assert (rows(144).rows, rows(144).features, weight(70, 144).out) == (15, 144, 70)
    for bad in (lambda: T.Fp8Rows(Fake(F8, 3, 5, 144), Fake(F32, 1, 15)), lambda: T.Fp8Rows(Fake(F8, 3, 5, 144), Fake(F32, 2, 15, device="cuda:1")), lambda: T.Fp8Rows(Fake(F32, 3, 5, 144), Fake(F32, 2, 15)),
                lambda: T.Fp8Rows(Fake(F8, 3, 5, 2, 144), Fake(F32, 2, 30)), lambda: T.Fp8Weight(Fake(F8, 70, 144), Fake(F32, 1, 1)), lambda: T.Fp8Weight(Fake(F8, 70, 144), Fake(torch.bfloat16, 1, 2)),
                lambda: T.Fp8Weight(Fake(F8, 70, 144), Fake(F32, 1, 2, device="cuda:1"))):
        with pytest.raises(ValueError):
            bad()


def test_a_list_takes_rows_and_weights_of_its_own_gpu_only():
    here, there = "cuda:0", "cuda:1"
    for build in (lambda o: o.gemm_fp8(rows(144), weight(70, 144, there), tensor(70)), lambda o: o.gemm_fp8(rows(144), weight(70, 144), tensor(70, there)),
                  lambda o: o.gated_fp8(rows(144), weight(80, 144), weight(80, 144), rows(80, device=there)), lambda o: o.rmsnorm_fp8(tensor(144), rows(144, device=there)),
                  lambda o: o.rmsnorm_fp8(tensor(144), rows(144), res=tensor(144, there)), lambda o: o.rmsnorm_fp8(tensor(144), rows(144), At(F32, 144, device=there))):
        with pytest.raises(ValueError, match="GPU"):
            build(T.OpList(F32, 3))
    T.OpList(F32, 3).gemm_fp8(rows(144, device=here), weight(70, 144), tensor(70))


def test_what_a_list_writes_down():
    x, r, h, y, z = (tensor(144) for _ in range(5))
    n, g = rows(144), rows(80)
    o = T.OpList(F32, 3)
    o.rmsnorm_fp8(x, n, res=r, sum=h)                           # a residual from outside, beside the input
    o.gated_fp8(n, weight(80, 144), weight(80, 144), g, act="gelu_tanh")
    o.gemm_fp8(g, weight(144, 80), y, res=h)
    o.rmsnorm(y, None, z)
    kinds = [(op.kind, op.in0, op.res, op.out, op.act) for op in o.ops]
    assert kinds == [(B.GACER_RMSNORM_FP8, 0, 1, 2, 0), (B.GACER_GATED_FP8, -1, -1, -1, B.GACER_ACT_GELU_TANH), (B.GACER_GEMM_FP8, -1, 2, 3, 0), (B.GACER_RMSNORM_FP8, 3, -1, 4, 0)]
    assert (o.input, o.output) == (0, 4)
    for bad in (lambda: o.rmsnorm_fp8(tensor(144), n), lambda: o.rmsnorm_fp8(y, rows(160)), lambda: o.gemm_fp8(rows(144, batch=5, tokens=3), weight(144, 144), tensor(144)),
                lambda: o.gemm_fp8(n, weight(70, 160), tensor(70)), lambda: o.gated_fp8(n, weight(80, 144), weight(70, 144), rows(80)), lambda: o.gated_fp8(n, weight(80, 144), weight(80, 144), tensor(70))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(KeyError):
        o.gemm_fp8(n, weight(70, 144), tensor(70), act="no such")
    with pytest.raises(KeyError):
        T.OpList(F32, 3)._op(B.GACER_GEMM, act="silu")          # an activation of products of 8-bit rows alone


def test_operands_of_2_gib_are_refused():
    """The library's structures hold their extents in 32 bits."""
    for make in (lambda: rows(16, batch=2 ** 20, tokens=4096 + 1), lambda: rows(16, batch=2, tokens=2 ** 26), lambda: weight(2 ** 20, 2048), lambda: weight(2 ** 32 + 128, 16)):
        with pytest.raises(ValueError, match="2 GiB"):
            make()
    assert rows(16, batch=1, tokens=2 ** 27 - 1).rows == 2 ** 27 - 1
