"""Wide rows of the layer norm: the kernels that only such sizes reach."""
import pytest

import test_gpu_norm_linear as base

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ layer norm
# Eight wavefronts a row (4097 to 8192 columns) and sixteen (beyond), more rows than one launch takes in the backward (512).  1300 rows: a workgroup walks a second row in the
# forward (1280 workgroups), 600 and 1300 of more than 8192 columns also in the backward (10 sqrt(rows), at most 256).
@pytest.mark.parametrize("R, H", [(520, 5120), (515, 8200), (600, 12000), (1300, 8200)])
@pytest.mark.parametrize("dtype, params, kept, pad", [("bf16", "f32", None, 0), ("bf16", "bf16", "e4m3", 5), ("f32", "f32", "e5m2", 0), ("f32", "bf16", None, 3)])
def test_layer_norm_of_wide_rows(R, H, dtype, params, kept, pad):
    base.test_layer_norm(R, H, dtype, params, kept, pad)
