"""The learner's operators at the ends of their inputs' ranges, against the float64 oracle: the lowest logits, ratios and
gates beyond float32, advantages under any mask, rows at any alignment.  Tolerances as in test_gpu_learner.py unless a
test says otherwise."""

import numpy as np
import pytest
import torch

from oracle import learner as L
from paper_2609_13716_amd import rollout as R

from parity import require_gpu
from test_gpu_learner import HYPER, U32, Scan, _check_ppo, _close, _gpu_args, _np, _ppo

pytestmark = pytest.mark.gpu

LOWEST = np.finfo(np.float32).min
FLT_MAX = float(np.finfo(np.float32).max)
ROUTES = pytest.mark.parametrize("rows", [300, 30000])  # one launch, three


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _hyper64(hyper=HYPER):
    return {k: float(np.float32(v)) for k, v in hyper.items()}


def _f64(kw):
    return {k: (v.astype(np.float64) if v is not None and v.dtype == np.float32 else v) for k, v in kw.items()}


# ---- PPO: the lowest logits ----


def _with_low(rows, seed, taken):
    """Inputs of which a third of the logits are to be lowest (never a whole row); whether taken actions may be."""
    kw = _ppo(rows, 6, seed=seed)
    rng = np.random.default_rng(seed + 1)
    low = rng.random((rows, 6)) < 0.33
    low[np.arange(rows), rng.integers(0, 6, rows)] = False
    if not taken:
        a = np.clip(kw["actions"], 0, 5)
        low[np.arange(rows), a] = False
    return kw, low


@ROUTES
def test_ppo_lowest_logits_are_never_taken(rows):
    """Logits at float32's lowest value, all of them legal: probability 0, so bit for bit what illegal ones give."""
    kw, low = _with_low(rows, rows, taken=False)
    kw["logits"][low] = LOWEST
    got = R.ppo_loss(**_gpu_args(kw), **HYPER, normalize=True)
    kw["legal"] = (~low).astype(np.uint8)
    want = R.ppo_loss(**_gpu_args(kw), **HYPER, normalize=True)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    _check_ppo(kw, got, True)


def _check_far(kw, near, rows):
    """kw's outputs against the oracle's for `near`, the same inputs with far logits so near that float64 and float32
    still give them probability 0 (exp(-150) = 7e-66).  The KL estimate, which alone holds the distance itself, is
    compared with kw's own: each row's term is rounded to float32 at most four times."""
    dx, dv, st = R.ppo_loss(**_gpu_args(kw), **HYPER)
    want = L.ppo_loss(**_f64(kw), **_hyper64())[2][4]
    assert abs(float(st[4]) - want) <= 4 * U32 * abs(want), (float(st[4]), want)
    st = st.clone()
    st[4] = L.ppo_loss(**_f64(near), **_hyper64())[2][4]
    _check_ppo(near, (dx, dv, st), False)


@ROUTES
def test_ppo_lowest_logits_may_be_taken(rows):
    """The taken action among them: its ratio is 0."""
    kw, low = _with_low(rows, rows + 2, taken=True)
    near = {k: v.copy() if v is not None else None for k, v in kw.items()}
    kw["logits"][low] = LOWEST
    near["logits"][low] = -150
    _check_far(kw, near, rows)


@ROUTES
def test_ppo_logits_further_apart_than_float32(rows):
    """One logit at 2e38, others at 0 or -2e38: their differences overflow float32."""
    kw, low = _with_low(rows, rows + 4, taken=True)
    low[:, 0] = False
    kw["logits"][:] = np.where(low, np.float32(-2e38), np.float32(0))
    kw["logits"][:, 0] = 2e38
    near = dict(kw, logits=np.where(np.arange(6) == 0, np.float32(0), np.float32(-150)).repeat(rows).reshape(6, rows).T.copy())
    _check_far(kw, near, rows)


@ROUTES
def test_ppo_rows_of_lowest_logits_only(rows):
    """Every action of a row equally lowest: a uniform policy."""
    kw = _ppo(rows, 6, seed=rows + 6)
    kw["logits"][::3] = LOWEST
    got = R.ppo_loss(**_gpu_args(kw), **HYPER)
    kw["logits"][::3] = 0
    _check_ppo(kw, got, False)
