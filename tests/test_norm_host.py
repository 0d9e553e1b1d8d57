"""Which arrays of the norm may be one another, checked before a device is touched."""
import pytest

from paper_2605_05607_amd import binding as B
from paper_2605_05607_amd import layer as L
from paper_2605_05607_amd import workloads as wl

A = 1 << 20  # addresses that are never dereferenced; arrays of at most 64 KiB
INV, ROWS, COLS = B.MOE_ERR_INVALID_ARG, 16, 1024
NORM = dict(rows=ROWS, cols=COLS, dtype=B.MOE_BF16, x=A, residual=2 * A, weight=3 * A, eps=1e-6, sum=4 * A, y=5 * A, codes=6 * A,
            scales=7 * A, rstd=8 * A, stream=None)
BACK = dict(rows=ROWS, cols=COLS, dtype=B.MOE_BF16, sum=A, weight=2 * A, rstd=3 * A, dy=4 * A, dsum=5 * A, dx=6 * A, dweight=7 * A,
            workspace=8 * A, workspace_bytes=1 << 20, stream=None)
BYTES = {"x": 2 * ROWS * COLS, "residual": 2 * ROWS * COLS, "sum": 2 * ROWS * COLS, "y": 2 * ROWS * COLS, "dy": 2 * ROWS * COLS,
         "dsum": 2 * ROWS * COLS, "dx": 2 * ROWS * COLS, "weight": 2 * COLS, "codes": ROWS * COLS, "scales": 4 * ROWS,
         "rstd": 4 * ROWS, "dweight": 4 * COLS, "workspace": 4 * ROWS * COLS}


@pytest.mark.parametrize("written,others", [
    ("y", ("x", "residual", "weight", "sum", "codes", "scales", "rstd")), ("codes", ("x", "residual", "weight", "sum", "scales", "rstd")),
    ("scales", ("x", "residual", "weight", "sum", "rstd")), ("rstd", ("x", "residual", "weight", "sum")), ("sum", ("weight",))])
def test_norm_writes_over_none_of_its_arrays(written, others):
    """A row is written while others are still to be read: codes in front of x, for one, would be read as later rows of x."""
    for other in others:
        for at in (NORM[other], NORM[other] + BYTES[other] - 16, NORM[other] - BYTES[written] + 16):
            if at % 16 == 0:
                assert B.lib().moe_rmsnorm(*{**NORM, written: at}.values()) == INV, (written, other, at - NORM[other])
    for other in ("x", "residual"):  # the sum may be either, and no part of it
        for by in (16, -16, 2 * COLS):
            assert B.lib().moe_rmsnorm(*{**NORM, "sum": NORM[other] + by}.values()) == INV


@pytest.mark.parametrize("written,others", [
    ("dx", ("sum", "weight", "rstd", "dweight", "workspace")), ("dweight", ("sum", "weight", "rstd", "dy", "dsum", "workspace")),
    ("workspace", ("sum", "weight", "rstd", "dy", "dsum"))])
def test_norm_gradients_write_over_none_of_their_arrays(written, others):
    for other in others:
        for at in (BACK[other], BACK[other] + BYTES[other] - 16, BACK[other] - BYTES[written] + 16):
            assert B.lib().moe_rmsnorm_backward(*{**BACK, written: at}.values()) == INV, (written, other, at - BACK[other])
    for other in ("dy", "dsum"):  # dx may be either
        for by in (16, -16, 2 * COLS):
            assert B.lib().moe_rmsnorm_backward(*{**BACK, "dx": BACK[other] + by}.values()) == INV
