"""The calls between two attention calls on the GPU: sizes and values that take other ways through their kernels."""
import numpy as np
import pytest

import step_util as U
from gpu_util import require_gpu
from test_gpu_step import Qkv, host
from test_step_model_paths import norm_cases

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_values_whose_squares_leave_float32(dtype, D):
    require_gpu()
    for c in norm_cases(np.random.default_rng(D), D, dtype):
        s = Qkv(c)
        U.check_qkv(c, host(s.call()), host(s.pool), 9)
