"""Parameters that operators on 8-bit rows have no use for are refused, not left out (through the C ABI, without a GPU)."""
import pytest

from paper_2304_11745_amd import binding as B
from test_host_fp8 import AT, A, G, N, ctx, load  # noqa: F401  (ctx is a fixture)


@pytest.mark.parametrize("at", [AT[13], AT[13] + 4], ids=["aligned", "misaligned"])
@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("kind,field", [(N, "shift"), (G, "shift"), (A, "shift"), (G, "scale"), (A, "scale"), (N, "bias"), (A, "bias")])
def test_a_parameter_without_a_use_is_refused(ctx, kind, field, codes, at):  # noqa: F811
    """A norm with gamma and beta, as LAYERNORM takes them, would otherwise run without its beta."""
    assert load(ctx, kind, codes=codes, **{field: at}) == B.GACER_ESHAPE, B.gacer_last_error(ctx)
    assert b"tenant 0 op 0" in B.gacer_last_error(ctx) and field.encode() in B.gacer_last_error(ctx)


def test_those_with_a_use_are_taken(ctx):  # noqa: F811
    assert load(ctx, N, scale=AT[13]) == B.GACER_OK and load(ctx, G, bias=AT[13]) == B.GACER_OK
    assert load(ctx, N, norm=0, scale=AT[13]) == B.GACER_OK              # y = h: the header says that it is not read
