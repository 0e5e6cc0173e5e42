"""More refusals of the learner's operators before anything is launched: through the C ABI with addresses that are never
read, and through the binding with host tensors."""

import pytest
import torch

from paper_2609_13716_amd import rollout as R
from test_learner_abi import _at, _backward, _scan, _scan_cfg

KINDS = pytest.mark.parametrize("kind", [R.RL_SCAN_GATED, R.RL_SCAN_DIAGONAL])
DTYPES = pytest.mark.parametrize("dtype", [R.RL_F32, R.RL_BF16])


def _refused(status):
    assert status == R.RL_EINVAL and "overlaps" in R.lib.rollout_last_error().decode()


@KINDS
@DTYPES
@pytest.mark.parametrize("steps", [1, 8, 6000])
def test_a_state_in_place_may_share_with_nothing_else(kind, dtype, steps):
    """h_last may be h0 and dh0 may be dh_last; where another input lies there, too, the call is refused."""
    cfg = _scan_cfg(kind=kind, dtype=dtype, n_steps=steps, n_envs=1, n_agents=1, width=4)
    for other in ("u", "gate", "done"):
        _refused(_scan(cfg, h0=_at(3), h_last=_at(3), **{other: _at(3)}))
    for other in ("gate", "done", "h0", "h", "dh"):
        _refused(_backward(cfg, dh_last=_at(5), dh0=_at(5), **{other: _at(5)}))
    _refused(_scan(cfg, h0=_at(3), h_last=_at(3), h=_at(3)))
    _refused(_backward(cfg, dh_last=_at(5), dh0=_at(5), du=_at(5)))


@pytest.mark.parametrize("steps", [2 ** 32 + 5, 2 ** 31, -2 ** 32 + 5])
def test_steps_that_would_wrap(steps):
    with pytest.raises(ValueError, match="beyond 32 bits"):
        R.orthogonalize(torch.zeros(4, 8), steps=steps)
