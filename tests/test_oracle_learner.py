"""Pins of the oracle's learner operators: every gradient against central differences of the value it belongs to, the
recurrence against its explicit sum, the orthogonalisation against the matrix iteration."""

import numpy as np
import pytest

from oracle import learner as L


def _scan_inputs(kind, seed, T=6, E=3, A=2, W=4):
    rng = np.random.default_rng(seed)
    n = lambda *s: rng.standard_normal(s) + (1j * rng.standard_normal(s) if kind == "diagonal" else 0)  # noqa: E731
    gate = 0.9 * np.exp(1j * rng.uniform(-3, 3, W)) if kind == "diagonal" else rng.uniform(-1, 1, (T, E, A, W))
    return n(T, E, A, W), gate, (rng.random((T, E)) < 0.3).astype(np.uint8), n(E, A, W), n(T, E, A, W), n(E, A, W)


@pytest.mark.parametrize("kind", ["gated", "diagonal"])
def test_scan_is_the_explicit_sum(kind):
    u, gate, done, h0, _, _ = _scan_inputs(kind, 0)
    h, last = L.scan(u, gate, done, h0)
    for t in range(6):
        for e in range(3):
            start = max([k + 1 for k in range(t) if done[k, e]], default=0)
            want = 0
            for j in range(start, t + 1):
                a = np.prod([gate if kind == "diagonal" else gate[k, e] for k in range(j + 1, t + 1)], axis=0) \
                    if j < t else 1.0
                want = want + a * u[j, e]
            if start == 0:
                want = want + np.prod([gate if kind == "diagonal" else gate[k, e] for k in range(t + 1)], axis=0) * h0[e]
            assert np.allclose(h[t, e], want, atol=1e-12)
    assert np.allclose(last, np.where(done[-1][:, None, None] != 0, 0, h[-1]))


@pytest.mark.parametrize("kind", ["gated", "diagonal"])
def test_scan_in_two_calls(kind):
    u, gate, done, h0, _, _ = _scan_inputs(kind, 1)
    cut = lambda a, b: gate if kind == "diagonal" else gate[a:b]  # noqa: E731
    h, last = L.scan(u, gate, done, h0)
    ha, mid = L.scan(u[:2], cut(0, 2), done[:2], h0)
    hb, end = L.scan(u[2:], cut(2, 6), done[2:], mid)
    assert np.allclose(h, np.concatenate([ha, hb])) and np.allclose(last, end)


@pytest.mark.parametrize("kind", ["gated", "diagonal"])
def test_scan_gradients_are_differences(kind):
    u, gate, done, h0, wh, wl = _scan_inputs(kind, 2)
    dot = lambda x, w: float((x * np.conj(w)).real.sum())  # noqa: E731
    loss = lambda u, gate, h0: sum(dot(x, w) for x, w in zip(L.scan(u, gate, done, h0), (wh, wl)))  # noqa: E731
    h, _ = L.scan(u, gate, done, h0)
    grads = L.scan_backward(gate, h, wh, done, h0, wl)
    args = [u, gate, h0]
    rng = np.random.default_rng(3)
    for i, g in enumerate(grads):
        for _ in range(25):
            at = tuple(rng.integers(0, n) for n in args[i].shape)
            for unit in (1.0, 1j) if kind == "diagonal" else (1.0,):
                up, dn = [x.copy() for x in args], [x.copy() for x in args]
                up[i][at] += 1e-6 * unit
                dn[i][at] -= 1e-6 * unit
                got = g[at].real if unit == 1.0 else g[at].imag
                assert abs((loss(*up) - loss(*dn)) / 2e-6 - got) < 1e-6


def _ppo_inputs(seed, R=40, nA=5, masked=True):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, nA))
    legal = (rng.random((R, nA)) < 0.7).astype(np.uint8)
    legal[3] = 0
    act = rng.integers(0, nA, R)
    act[5], act[6] = -1, nA
    return dict(logits=x, actions=act, logp_old=-1.6 + 0.3 * rng.standard_normal(R), adv=rng.standard_normal(R),
                value=rng.standard_normal(R), ret=rng.standard_normal(R), clip=0.2, value_coef=0.5, entropy_coef=0.02,
                value_clip=0.3, value_old=rng.standard_normal(R) * 0.2, legal=legal if masked else None,
                mask=(rng.random(R) < 0.8).astype(np.uint8) if masked else None)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("normalize", [False, True])
def test_ppo_gradients_are_differences(masked, normalize):
    k = _ppo_inputs(4, masked=masked)
    loss = lambda **kw: L.ppo_loss(**{**k, **kw}, normalize=normalize)[2][0]  # noqa: E731
    dx, dv, _ = L.ppo_loss(**k, normalize=normalize)
    eps = 1e-6
    for r in range(40):
        for a in range(5):
            up, dn = k["logits"].copy(), k["logits"].copy()
            up[r, a] += eps
            dn[r, a] -= eps
            assert abs((loss(logits=up) - loss(logits=dn)) / (2 * eps) - dx[r, a]) < 1e-7
        up, dn = k["value"].copy(), k["value"].copy()
        up[r] += eps
        dn[r] -= eps
        assert abs((loss(value=up) - loss(value=dn)) / (2 * eps) - dv[r]) < 1e-7


def test_ppo_rows_that_count_for_nothing():
    k = _ppo_inputs(5)
    k["legal"][:] = 0
    dx, _, st = L.ppo_loss(**k)
    assert (dx == 0).all() and st[1] == st[3] == st[4] == st[5] == 0 and st[2] > 0
    k = _ppo_inputs(5)
    k["mask"][:] = 0
    dx, dv, st = L.ppo_loss(**k, normalize=True)
    assert (dx == 0).all() and (dv == 0).all() and (st == 0).all()


@pytest.mark.parametrize("shape", [(4, 7), (7, 4), (1, 5), (6, 6), (3, 5, 8)])
def test_orthogonalize_is_the_matrix_iteration(shape):
    g = np.random.default_rng(6).standard_normal(shape)
    a, b, c = L.NS_COEFFICIENTS
    x = g / np.sqrt((g * g).sum((-2, -1), keepdims=True))
    if shape[-2] > shape[-1]:
        x = np.swapaxes(x, -1, -2)
    for _ in range(5):
        m = x @ np.swapaxes(x, -1, -2)
        x = a * x + (b * m + c * m @ m) @ x
    if shape[-2] > shape[-1]:
        x = np.swapaxes(x, -1, -2)
    assert np.allclose(L.orthogonalize(g), x, atol=1e-10)
    assert (L.orthogonalize(np.zeros(shape)) == 0).all()
