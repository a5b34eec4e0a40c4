"""Which tiles, slices and joins the sizes of tests/test_gpu_fp8_plans.py take, asked of the launchers without a GPU: every one there is."""
import subprocess

from test_host_fp8_dispatch import TILES, driver  # noqa: F401  (driver is a fixture)


def test_the_plans_take_every_tile_whole_and_in_slices_and_every_join(driver):  # noqa: F811
    import test_gpu_fp8_plans as P
    seen, joins = set(), set()
    for gated, sizes in ((0, P.GEMMS), (1, P.GATED)):
        for tokens, cin, cout in sizes:
            said = subprocess.run([driver, str(gated), str(P.BATCH * tokens), str(cin), str(cout)] + ["codes"] * gated, check=True, capture_output=True, text=True, timeout=60).stdout.split()
            slices = int(said[1])
            seen.add((said[0].replace("_bf16", ""), slices > 1))
            joins.add((gated, slices))
    assert seen == {(tile, cut) for tile in TILES for cut in (False, True)}, sorted(seen)
    assert {(g, s) for g, s in joins if s > 1} == {(g, s) for g in (0, 1) for s in (2, 4, 8)}, sorted(joins)
