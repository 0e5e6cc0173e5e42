"""The learner's operators at the ends of their inputs' ranges, against the float64 oracle: the lowest logits, ratios
and gates beyond float32, advantages under any mask, rows at any alignment.  Tolerances as in test_gpu_learner.py unless a
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
    near = dict(kw, logits=np.tile(np.where(np.arange(6) == 0, np.float32(0), np.float32(-150)), (rows, 1)))
    _check_far(kw, near, rows)


@ROUTES
def test_ppo_rows_of_lowest_logits_only(rows):
    """Every action of a row equally lowest: a uniform policy."""
    kw = _ppo(rows, 6, seed=rows + 6)
    kw["logits"][::3] = LOWEST
    got = R.ppo_loss(**_gpu_args(kw), **HYPER)
    kw["logits"][::3] = 0
    _check_ppo(kw, got, False)


# ---- recurrence: gates of any size ----

# segments; 16, 8 and 4 waves of a workgroup, pairs of bfloat16 and single channels; one wave
GATE_SIZES = [(6400, 1, 1, 16), (900, 33, 2, 210), (900, 16, 3, 211), (300, 28, 2, 512), (300, 150, 2, 256),
              (48, 500, 2, 256), (32, 3, 1, 5), (16, 3, 1, 5)]


def _forward_and_back(s):
    h, last = R.scan(s.u, s.gate, s.done, s.h0)
    s.check_forward(h, last)
    s.check_backward(h, *R.scan_backward(s.gate, h, s.dh, s.done, s.h0, s.dh_last))
    return h


@pytest.mark.parametrize("kind", ["gated", "diagonal"])
@pytest.mark.parametrize("size", [(32768, 1, 1, 16)] + GATE_SIZES)
def test_scan_of_nothing_is_nothing(kind, size):
    """Without inputs and state the states are 0, however large the products of the gates (here 1.03 for half of the
    run, then 0.97, or 1e20 all along)."""
    T = size[0]
    for up, down in ((1.03, 0.97), (1e20, 1e20)):
        s = Scan(kind, "f32", *size, done=None, h0=False, seed=1, radius=up)
        if kind == "gated":
            s.gate[:] = up
            s.gate[T // 2:] = down
        s.u.zero_()
        s.dh.zero_()
        h, last = R.scan(s.u, s.gate)
        assert (h == 0).all() and (last == 0).all()
        assert all((g == 0).all() for g in R.scan_backward(s.gate, h, s.dh))


@pytest.mark.parametrize("kind", ["gated", "diagonal"])
def test_scan_inputs_behind_growing_gates(kind):
    """Inputs in the last 400 steps alone, behind 6000 steps whose gates' product is 1e364 (the gradient: in the
    first)."""
    s = Scan(kind, "f32", 6400, 1, 2, 16, done=None, h0=False, seed=2, radius=1.15)
    s.u[:6000] = 0
    s.dh[400:] = 0
    _forward_and_back(s)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", GATE_SIZES)
def test_scan_gates_up_and_down(dt, size):
    """Gates whose product rises to 1e40 within 8 steps and falls back within the next 8 (values of 1e-30 to 1e10): every
    state fits float32, the products of the gates do not."""
    s = Scan("gated", dt, *size, done=0.01, seed=3)
    t = torch.arange(size[0], device="cuda")
    # half a period ahead in every second channel
    phase = (t[:, None, None, None] + 8 * (torch.arange(size[3], device="cuda") % 2)) % 16 < 8
    s.gate[:] = torch.where(phase, 2.0 ** 17, 2.0 ** -17) * torch.sign(s.gate.float())
    s.u *= 2.0 ** -100
    s.h0 *= 2.0 ** -100
    s.dh *= 2.0 ** -100
    s.dh_last *= 2.0 ** -100
    h, last = R.scan(s.u, s.gate, s.done, s.h0)
    s.check_forward(h, last)
    h = torch.randn(h.shape, generator=torch.Generator("cuda").manual_seed(5), device="cuda").to(h.dtype)
    s.h0 = torch.randn_like(s.h0)  # (states of 1: products with the smallest gradients fit float32, too)
    s.check_backward(h, *R.scan_backward(s.gate, h, s.dh, s.done, s.h0, s.dh_last))


@pytest.mark.parametrize("size", [(6400, 1, 1, 16), (6400, 3, 1, 33), (2000, 60, 1, 128)])
def test_scan_long_rise_and_fall(size):
    """A product of 1e-60 over 200 steps and back over the next 200: powers of two, so that every state is exact."""
    T = size[0]
    s = Scan("gated", "f32", *size, done=None, seed=4)
    fall = torch.arange(T, device="cuda")[:, None, None, None] % 400 < 200
    s.gate[:] = torch.where(fall, 0.5, 2.0)
    s.u.zero_()
    s.h0[:] = 2.0 ** 100
    h, last = R.scan(s.u, s.gate, None, s.h0)
    want, wlast = L.scan(_np(s.u), _np(s.gate), None, _np(s.h0))
    assert np.array_equal(_np(h), want) and np.array_equal(_np(last), wlast)
    s.dh.zero_()
    s.dh_last[:] = 2.0 ** -100
    du, dgate, dh0 = R.scan_backward(s.gate, torch.zeros_like(h), s.dh, None, torch.zeros_like(s.h0), s.dh_last)
    wdu, _, wdh0 = L.scan_backward(_np(s.gate), np.zeros(h.shape), _np(s.dh), None, None, _np(s.dh_last))
    assert np.abs(wdu).max() < FLT_MAX
    assert np.array_equal(_np(du), wdu) and np.array_equal(_np(dh0), wdh0) and (dgate == 0).all()


# ---- PPO: ratios and advantages beyond float32 ----


def _check_wide(kw, got, hyper=HYPER):
    """Against the oracle where outputs may pass float32's range (then: infinite, of that sign).  A gradient's policy part
    is slope (onehot - p): the slope is off by t + 4 u of itself, p by t (t of test_gpu_learner.py), so together at most
    (2 t + 16 u) |slope| (onehot + p), and what float32 cannot hold (below 2^-126) is lost."""
    h, f = _hyper64(hyper), _f64(kw)
    wdx, wdv, wst = L.ppo_loss(**f, **h)
    rows, na = kw["logits"].shape
    x = np.maximum(f["logits"], -150.0)
    p = np.exp(x - x.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    a = np.clip(kw["actions"], 0, na - 1)
    acts = (kw["actions"] == a).astype(float)
    t = U32 * (16 + 4 * np.abs(x).max(1) + 2 * np.abs(f["logp_old"]))
    slope = np.abs(f["adv"]) * np.exp(np.log(p[np.arange(rows), a]) - f["logp_old"]) * acts
    tol = ((2 * t + 16 * U32) * slope)[:, None] * (p + (np.arange(na) == a[:, None]))
    tol += ((t + 16 * U32) * h["entropy_coef"])[:, None] * (np.abs(np.log(p)) * p + 4)
    for name, g, want, tol in (("dlogits", _np(got[0]), wdx, tol / rows + 2.0 ** -126),
                               ("dvalue", _np(got[1]), wdv, 4 * U32 * np.abs(wdv)),
                               ("stats", _np(got[2]), wst, (2 * t.max() + 16 * U32) * (np.abs(wst) + np.abs(wst[1:4]).sum()) +
                                t.max() * (np.arange(6) != 5))):
        assert not np.isnan(g).any(), (name, np.argwhere(np.isnan(g))[:4].tolist())
        over = np.abs(want) - tol > FLT_MAX
        assert (g[over] == np.sign(want[over]) * np.inf).all(), name
        fine = np.abs(want) + tol < FLT_MAX
        _close(g[fine], want[fine], tol[fine], name)


@ROUTES
@pytest.mark.parametrize("lo,hi,scale", [(60, 85, 1e-6), (85, 95, 1e-12), (89, 200, 1e-3), (1, 3, 3e38)])
def test_ppo_ratios_beyond_float32(rows, lo, hi, scale):
    """Log ratios of lo to hi (float32's exp ends at 88.7), advantages of both signs and 0; some probabilities are tiny,
    some 0.  Gradients that fit float32 are right, also where the ratio or the slope does not fit."""
    rng = np.random.default_rng(rows + hi)
    kw = _ppo(rows, 6, seed=rows + 8, spread=3.0)
    x = kw["logits"]
    x[rng.random((rows, 6)) < 0.2] = -60
    x[rng.random((rows, 6)) < 0.2] = LOWEST
    x[:, 2] = rng.standard_normal(rows)
    kw["actions"] = np.where(rng.random(rows) < 0.7, 2, 3).astype(np.int32)
    kw["actions"][x[np.arange(rows), kw["actions"]] < -50] = 2
    x64 = np.maximum(x.astype(np.float64), -150)
    lp = x64 - np.log(np.exp(x64).sum(1, keepdims=True))
    kw["logp_old"] = (lp[np.arange(rows), kw["actions"]] - rng.uniform(lo, hi, rows)).astype(np.float32)
    kw["adv"] = (scale * rng.uniform(-1, 1, rows) * (rng.random(rows) < 0.8)).astype(np.float32)
    _check_wide(kw, R.ppo_loss(**_gpu_args(kw), **HYPER))


@ROUTES
def test_ppo_ratios_beyond_float64(rows):
    """Log ratios of 1000: an action of probability 0 has gradient 0, the taken one's is infinite, nothing is NaN."""
    kw = _ppo(rows, 6, seed=rows + 10)
    kw["actions"][:] = 1
    kw["logits"][:, 4] = LOWEST
    kw["logp_old"][:] = -1000
    kw["adv"] = (np.arange(rows) % 3 - 1).astype(np.float32)
    dx, dv, st = (_np(t) for t in R.ppo_loss(**_gpu_args(kw), **HYPER))
    assert not np.isnan(dx).any() and (dx[:, 4] == 0).all()
    assert np.isposinf(dx[::3, 1]).all() and np.isfinite(dx[1::3]).all() and np.isfinite(dx[2::3]).all()
    assert np.isposinf(st[[0, 1, 4]]).all() and np.isfinite(st[[2, 3, 5]]).all() and np.isfinite(dv).all()


@ROUTES
def test_ppo_entropy_coefficient_of_any_size(rows):
    """Probabilities of 0 add no gradient, however large the coefficient is."""
    kw, low = _with_low(rows, rows + 12, taken=False)
    kw["logits"][low] = LOWEST
    dx, _, _ = R.ppo_loss(**_gpu_args(kw), **dict(HYPER, entropy_coef=1e37))
    assert (dx[torch.from_numpy(low).cuda()] == 0).all() and not bool(torch.isnan(dx).any())


@pytest.mark.parametrize("rows,na", [(300, 6), (6000, 6), (6000, 32), (6000, 20)])
@pytest.mark.parametrize("spread,shift", [(0.01, 0.0), (2.0, 300.0), (1.0, -1e4), (30.0, 1e6)])
def test_ppo_borders_of_shifted_logits(rows, na, spread, shift):
    """Ratios within a few float32 steps of a border, logits about any value and nearly equal or far apart: the side
    (the clip fraction is exact) is float64's.  The oracle gets the logits less their row's largest, which float64 holds
    exactly: of logits about 1e6 its log of the sum would be off by up to 2^-34 = 6e-11, and one of these ratios lies
    1.6e-11 from its border (log r = 0.18232155926398; with the larger logits the oracle's is 0.18232155928854)."""
    kw = _ppo(rows, na, seed=23, spread=spread)
    kw["logits"] = (kw["logits"] + np.float32(shift)).astype(np.float32)
    x = kw["logits"].astype(np.float64)
    kw["actions"] = np.where(np.arange(rows) % 3 == 0, np.clip(kw["actions"], 0, na - 1), x.argmax(1)).astype(np.int32)
    top = x.max(1, keepdims=True)
    lp = x - top - np.log(np.exp(x - top).sum(1, keepdims=True))
    border = np.where(np.arange(rows) % 2 == 0, 0.8, 1.2)
    old = (lp[np.arange(rows), kw["actions"]] - np.log(border)).astype(np.float32)
    for k in (-2, -1, 0, 1, 2):
        kw["logp_old"] = (old + k * np.spacing(old)).astype(np.float32)
        _check_ppo(dict(kw, logits=x - top), R.ppo_loss(**_gpu_args(kw), **HYPER), False)


# ---- PPO: advantages ----


@pytest.mark.parametrize("rows", [2048, 2900, 32768, 65536])
@pytest.mark.parametrize("mean,scale", [(3000.0, 0.01), (-2e6, 1.0), (7.0, 0.0)])
def test_ppo_advantages_under_any_mask(rows, mean, scale):
    """Masks with the period of agents, and ones that leave a few rows anywhere: the mean may lie far from 0."""
    for pick in (lambda r: r % 2 == 1, lambda r: r % 4 == 2, lambda r: r >= rows - 7, lambda r: r == rows // 2 + 3,
                 lambda r: (r > 700) & (r < 760)):
        kw = _ppo(rows, 6, seed=14)
        kw["adv"] = (mean + scale * np.random.default_rng(15).standard_normal(rows)).astype(np.float32)
        kw["mask"] = pick(np.arange(rows)).astype(np.uint8)
        kw["adv"][kw["mask"] == 0] = np.nan
        _check_ppo(kw, R.ppo_loss(**_gpu_args(kw), **HYPER, normalize=True), True)


@pytest.mark.parametrize("rows", [300, 30000, 30001])
def test_ppo_rows_at_any_alignment(rows):
    """Equal values give equal bits wherever they lie: sums are taken in an order that depends on the sizes only."""
    kw = _ppo(rows, 6, seed=16, masked=True, padded=True)
    want = R.ppo_loss(**_gpu_args(kw), **HYPER, normalize=True)
    for off in (1, 2, 3, 4):
        got = R.ppo_loss(**_gpu_args(kw, off=off), **HYPER, normalize=True)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), off


@pytest.mark.parametrize("rows", [3000, 30001])
def test_ppo_sums_in_one_order(rows):
    """Advantages that cancel but for what their sum rounds off, so that any other order of it shows: the same bits
    wherever they lie."""
    rng = np.random.default_rng(21)
    kw = _ppo(rows, 6, seed=22)
    half = (rng.standard_normal(rows // 2) * 10.0 ** rng.uniform(-10, 10, rows // 2)).astype(np.float32)
    kw["adv"] = np.concatenate([half, -half, np.zeros(rows % 2, np.float32)])[rng.permutation(rows)]
    for mask in (None, np.ones(rows, np.uint8)):
        kw["mask"] = mask
        hyper = dict(HYPER, entropy_coef=0.0)
        want = R.ppo_loss(**_gpu_args(kw), **hyper, normalize=True)
        for off in (1, 2, 3, 4):
            got = R.ppo_loss(**_gpu_args(kw, off=off), **hyper, normalize=True)
            assert all(torch.equal(x, y) for x, y in zip(got, want)), off


# ---- PPO: small KL estimates, NaN ----


@pytest.mark.parametrize("rows", [500, 30000])
@pytest.mark.parametrize("delta", [0.0, 1e-4, 1e-3, 0.1, 0.3])
def test_ppo_kl_of_a_close_policy(rows, delta):
    """r - 1 - log r near r = 1 is about (log r)^2 / 2 and never negative.  log r is off by t (test_gpu_learner.py), so a
    row's term by |r - 1| t + r t^2, and by 8 u of itself."""
    rng = np.random.default_rng(rows)
    kw = _ppo(rows, 6, seed=17)
    kw["actions"] = np.clip(kw["actions"], 0, 5).astype(np.int32)
    x = kw["logits"].astype(np.float64)
    lp = (x - np.log(np.exp(x).sum(1, keepdims=True)))[np.arange(rows), kw["actions"]]
    kw["logp_old"] = (lp + delta * rng.uniform(-1, 1, rows)).astype(np.float32)
    got = R.ppo_loss(**_gpu_args(kw), **HYPER)
    old = kw["logp_old"].astype(np.float64)
    r = np.exp(lp - old)
    t = U32 * (16 + 4 * np.abs(x).max(1) + 2 * np.abs(old))
    want = L.ppo_loss(**_f64(kw), **_hyper64())[2][4]
    tol = (np.abs(r - 1) * t + r * t * t).mean() + 8 * U32 * want
    kl = float(got[2][4])
    assert kl >= 0 and abs(kl - want) <= tol, (kl, want, tol)
    _check_ppo(kw, got, False)


@ROUTES
def test_ppo_nan_in_old_values_is_not_hidden(rows):
    """A NaN among the old values makes its row's value loss and gradient NaN, and no other row's."""
    kw = _ppo(rows, 6, seed=18)
    clean = R.ppo_loss(**_gpu_args(kw), **HYPER)
    kw["value_old"][17] = np.nan
    dx, dv, st = R.ppo_loss(**_gpu_args(kw), **HYPER)
    rest = torch.arange(rows, device="cuda") != 17
    assert torch.isnan(dv[17]) and torch.equal(dv[rest], clean[1][rest]) and torch.equal(dx, clean[0])
    assert torch.isnan(st[0]) and torch.isnan(st[2])
    assert torch.equal(st[[1, 3, 4, 5]], clean[2][[1, 3, 4, 5]])


# ---- orthogonalisation ----


@pytest.mark.parametrize("size", [(3, 128, 192), (2, 32, 1024), (2, 512, 64)])
def test_orthogonalize_in_one_launch_captured(size):
    """Matrices whose one workgroup takes more than 64 KB of LDS, in a graph that is replayed with eager calls in
    between."""
    g, out = torch.empty(size, device="cuda"), torch.empty(size, device="cuda")
    rng = np.random.default_rng(19)
    fill = lambda: g.copy_(torch.from_numpy(rng.standard_normal(size).astype(np.float32)))  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    assert R.orthogonalize_workspace_bytes(g) == 0
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        R.orthogonalize(g, out=out)
    for k in range(4):
        fill()
        out.fill_(float(k))
        graph.replay()
        got = out.clone()
        assert torch.equal(got, R.orthogonalize(g)), k
        err = np.linalg.norm(_np(got) - L.orthogonalize(_np(g)), axis=(1, 2))
        m = min(size[1:])
        assert (err <= 6 * 3.4445 ** 5 * U32 + 16 * np.sqrt(max(size[1:])) * U32 * 1.21 * np.sqrt(m)).all(), err


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_orthogonalize_large_stack_repeats_itself(dt):
    """The largest tiles (128 x 128): every call, and every copy of a matrix in a stack, gives the same bits."""
    g = torch.randn(1, 1024, 1024, generator=torch.Generator("cuda").manual_seed(20), device="cuda").to(dt)
    g = g.repeat(4, 1, 1)
    first = R.orthogonalize(g)
    for i in range(1, 4):
        assert torch.equal(first[i], first[0])
    for _ in range(3):
        assert torch.equal(R.orthogonalize(g), first)
    want = torch.from_numpy(L.orthogonalize(_np(g[0]))).cuda()
    size = float(want.norm())
    tol = 6 * 3.4445 ** 5 * U32 + 16 * 32 * U32 * size + (2.0 ** -8 * size if dt == torch.bfloat16 else 0)
    assert float((first[0].double() - want).norm()) <= tol
