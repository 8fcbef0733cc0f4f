"""The temperatures that scoring with alternatives and distillation take, on the CPU: what log2(e) / temperature is no f32 number for is refused before anything is launched."""
import numpy as np
import pytest

from paper_2603_16435_amd import binding
from test_distill_abi import OK, PRM, RANGE, TOP, at, batch, lib, query, top_call  # noqa: F401  (lib: a fixture)

GOOD = [0.0, 4.3e-39, 1e-38, 1e-30, 1.0, 3e38]
BAD = [1e-45, 1e-40, 2.9e-39, 4.2e-39, 3.1e38, float("inf"), float("nan"), -1e-30]


@pytest.mark.parametrize("t", GOOD + BAD)
def test_temperatures(lib, t):  # noqa: F811
    want = OK if t in GOOD else RANGE
    top, prm = binding.rl_top_params(**dict(TOP, temperature=t)), binding.rl_distill_params(**dict(PRM, temperature=t))
    assert query(lib.rl_token_top_logprobs_workspace_bytes, batch(), top)[0] == want
    for bwd in (0, 1):
        assert query(lib.rl_distill_workspace_bytes, batch(), prm, bwd)[0] == want
    with np.errstate(over="ignore", divide="ignore"):
        assert t == 0.0 or (want == OK) == (0 < t <= 3e38 and bool(np.isfinite(np.float32(1) / np.float32(t) * np.float32(np.log2(np.e)))))


@pytest.mark.parametrize("t", BAD)
def test_calls(lib, t):  # noqa: F811
    import ctypes as C
    out = binding.rl_top_outputs(lse=at(6))
    assert top_call(lib, batch(), out, at(20), 1 << 39, temperature=t) == RANGE
    d = binding.rl_distill_outputs(loss=at(7))
    assert lib.rl_distill_loss_fwd_bwd(C.byref(batch()), at(5), at(6), C.byref(binding.rl_distill_params(**dict(PRM, temperature=t))), C.byref(d), at(20), 1 << 39, None) == RANGE
