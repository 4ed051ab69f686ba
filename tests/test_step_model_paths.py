"""The kernels between two attention calls on the CPU model of the device, as in test_step_model.py: calls of sizes and
values that take other ways through them."""
import numpy as np
import pytest

import step_util as U
from test_step_model import _run, driver, pytestmark  # noqa: F401 (the fixture and the mark)


def norm_cases(rng, D, dtype):
    """Heads whose squares leave float32's range: every size of value that the type has, one a head, with an eps of 0 and
    one below the smallest normal number, and with one that is far larger than the squares."""
    sizes = [1e-20, 1e-22, 3e-30, 1e-37, 1e18, 1e20, 3e37, 1.0] + ([3e-42] if dtype == "f32" else [])
    for eps in (0.0, 1e-40, 1e-6):
        for inter in (False, True):
            c = U.qkv_case(rng, 5, 9, 3, D, dtype, D // 2, inter, eps=eps, far=1000)
            c["positions"][:], c["words"][:] = rng.integers(0, 1000, 5), rng.permutation(16)[:5]
            if eps == 1e-6:
                sizes = [s for s in sizes if s >= 1e-30]      # (below, a result is no normal number)
            heads = rng.choice(sizes, (5, 15, 1))
            heads[0, :9, 0] = np.resize(sizes, 9)
            c["rows"] = U.stored((rng.standard_normal((5, 15, D)) * heads).reshape(5, -1), c["row"])
            yield c


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_values_whose_squares_leave_float32(driver, tmp_path, dtype, D):  # noqa: F811
    cases = list(norm_cases(np.random.default_rng(D), D, dtype))
    for c, (pool, q_out) in zip(cases, _run(driver, cases, str(tmp_path / "x"))):
        U.check_qkv(c, q_out.reshape(c["n"], 9, D), pool, 9)
