"""The operators of ``ends.py`` where a quantity of theirs reaches a limit."""
import pytest

torch = pytest.importorskip("torch")

import ends_reference as ref  # noqa: E402
from test_gpu_ends import F32, TYPES, aq, rand, uniform  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 64, 250, 500, 512, 1000, 1024, 2050])
@pytest.mark.parametrize("rms", [True, False])
def test_norm_without_epsilon(aq, dtype, dim, rms):
    """eps = 0, which rows that are not constant allow, for every count of rows in a workgroup."""
    for rows in (1, 2, 3, 4, 5, 6, 7, 8, 9, 1101):
        x = (rand(1, rows, dim) * (0.5 + uniform(2, rows, 1)) + 0.5).to(dtype)
        dy, w, b = rand(3, rows, dim, dtype=dtype), rand(4, dim, dtype=dtype), rand(5, dim, dtype=dtype)
        y, off, *_ = ref.norm(x, w, b, 0.0, rms)
        ref.check(aq.layer_norm(x, w, b, eps=0.0, rms=rms), y, off + ref.rounded(y.abs() + off, dtype), f"y, {rows} rows")
        (dx, dx_off), (dw, dw_off), (db, db_off) = ref.norm_grad(dy, x, w, None, 0.0, rms)
        got = aq.layer_norm_backward(dy, x, w, eps=0.0, rms=rms, bias=True)
        ref.check(got[0], dx, dx_off + ref.rounded(dx.abs() + dx_off, dtype), f"dx, {rows} rows")
        ref.check(got[1], dw, dw_off + ref.rounded(dw, F32), f"dweight, {rows} rows")
        ref.check(got[2], db, db_off + ref.rounded(db, F32), f"dbias, {rows} rows")
