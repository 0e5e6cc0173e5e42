"""A learner's operators after a rollout: the recurrence over a stored trajectory with its gradient, the PPO loss with
its gradient, and the orthogonalised update (test infrastructure).

Only ``tests/`` uses this module; the device path shares no code with it.  Everything is float64 and written from the
definitions: the recurrence and its gradient step by step, the loss row by row in closed form, the Newton-Schulz
iteration on the singular values (Jordan et al., "Muon", 2024: X <- a X + (b X X^T + c (X X^T)^2) X acts on the
singular values s of X as s <- a s + b s^3 + c s^5 and leaves the singular vectors alone).

Values of the recurrence are real arrays [T, E, A, D] with gates of that shape, or complex arrays [T, E, A, P] with one
factor per channel [P].
"""

import numpy as np

NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _cut(done, t, x):
    """x where the envs go on after step t, 0 where an episode ended (done [T, E] or None)."""
    if done is None:
        return x
    return np.where((done[t] != 0)[:, None, None], 0.0, x)


def _factor(gate, t):
    return gate[None, None, :] if gate.ndim == 1 else gate[t]


def scan(u, gate, done=None, h0=None):
    """(h [T, ..], h_last): h_t = a_t k_t h_{t-1} + u_t; h_last is what the step after the last one starts from.

    Where a state is cut off the gate is not looked at (it may be NaN)."""
    T = u.shape[0]
    h = np.empty_like(u)
    prev = np.zeros_like(u[0]) if h0 is None else h0
    for t in range(T):
        a = _factor(gate, t)
        if t > 0 and done is not None:
            a = np.where((done[t - 1] != 0)[:, None, None], 0.0, a)
        h[t] = a * prev + u[t]
        prev = _cut(done, t, h[t])
    return h, prev


def scan_backward(gate, h, dh, done=None, h0=None, dh_last=None):
    """(du, dgate, dh0) of a real loss; gradients by complex values are d/d(real) + i d/d(imaginary)."""
    T = dh.shape[0]
    du = np.empty_like(dh)
    dgate = np.zeros(gate.shape, dh.dtype)
    flow = np.zeros_like(dh[0]) if dh_last is None else _cut(done, T - 1, dh_last)
    for t in range(T - 1, -1, -1):
        g = du[t] = dh[t] + flow
        if t == 0:
            prev = np.zeros_like(g) if h0 is None else h0
        else:
            prev = _cut(done, t - 1, h[t - 1])
        if gate.ndim == 1:
            dgate += (g * np.conj(prev)).sum((0, 1))
        else:
            dgate[t] = g * prev
        a = _factor(gate, t)
        if t > 0 and done is not None:
            a = np.where((done[t - 1] != 0)[:, None, None], 0.0, a)
        flow = np.conj(a) * g
    return du, dgate, flow


def path_lengths(u, gate, done=None, h0=None):
    """(S, D): S_t = sum_j |a_t .. a_{j+1}| |u_j|, the magnitude that h_t is summed from, and D_t, the same sum with
    each term weighted by the number of steps it went through (for error bounds of a rounded recurrence)."""
    S, D = np.empty(u.shape), np.empty(u.shape)
    s = np.zeros(u.shape[1:]) if h0 is None else np.abs(h0)
    d = s.copy()
    for t in range(u.shape[0]):
        a = np.abs(_factor(gate, t))
        if t > 0 and done is not None:
            a = np.where((done[t - 1] != 0)[:, None, None], 0.0, a)
        d = a * (d + s) + np.abs(u[t])
        s = a * s + np.abs(u[t])
        S[t], D[t] = s, d
    return S, D


def ppo_loss(logits, actions, logp_old, adv, value, ret, clip, value_coef, entropy_coef, value_clip=0.0,
             value_old=None, legal=None, mask=None, normalize=False):
    """(dlogits [R, nA], dvalue [R], stats [6]) for rows [R, nA] / [R], written row by row."""
    R, nA = logits.shape
    counted = np.ones(R, bool) if mask is None else mask != 0
    n = max(1, int(counted.sum()))
    adv = np.asarray(adv, np.float64)
    if normalize and counted.any():
        mean = adv[counted].mean()
        std = np.sqrt(((adv[counted] - mean) ** 2).mean())
        adv = np.where(counted, (np.where(counted, adv, 0.0) - mean) / (std + 1e-8), 0.0)
    dx, dv = np.zeros((R, nA)), np.zeros(R)
    pol = val = ent = kl = frac = 0.0
    for r in np.nonzero(counted)[0]:
        x = logits[r]
        ok = ~np.isneginf(x)
        if legal is not None:
            ok &= legal[r] != 0
        if ok.any():
            l = x[ok]
            top = l.max()
            logz = top + np.log(np.exp(l - top).sum())
            lp = np.full(nA, -np.inf)
            lp[ok] = l - logz
            p = np.where(ok, np.exp(lp), 0.0)
            h = -np.sum(p[ok] * lp[ok])
            ent += h
            dx[r, ok] += entropy_coef * p[ok] * (lp[ok] + h)
            a = int(actions[r])
            if 0 <= a < nA and ok[a]:
                diff = lp[a] - logp_old[r]
                ratio = np.exp(diff)
                surr, surr_c = ratio * adv[r], np.clip(ratio, 1 - clip, 1 + clip) * adv[r]
                pol -= min(surr, surr_c)
                kl += ratio - 1 - diff
                frac += float(ratio < 1 - clip or ratio > 1 + clip)
                if surr <= surr_c:
                    d = -p * ok
                    d[a] += 1.0
                    dx[r] -= adv[r] * ratio * d
        e = value[r] - ret[r]
        loss, grad = 0.5 * e * e, e
        if value_clip > 0 and abs(value[r] - value_old[r]) > value_clip:
            ec = value_old[r] + np.sign(value[r] - value_old[r]) * value_clip - ret[r]
            if 0.5 * ec * ec > loss:
                loss, grad = 0.5 * ec * ec, 0.0
        val += loss
        dv[r] = value_coef * grad
    stats = np.array([pol + value_coef * val - entropy_coef * ent, pol, val, ent, kl, frac]) / n
    return dx / n, dv / n, stats


def orthogonalize(g, steps=5):
    """The Newton-Schulz iteration of g [.., rows, cols] on its singular values."""
    a, b, c = NS_COEFFICIENTS
    u, s, v = np.linalg.svd(g, full_matrices=False)
    norm = np.sqrt((g * g).sum((-2, -1)))[..., None]
    s = np.where(norm > 0, s / np.where(norm > 0, norm, 1.0), 0.0)
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (u * s[..., None, :]) @ v
