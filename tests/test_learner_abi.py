"""Refusals of the learner's operators, before anything is launched: through the C ABI with addresses that are never
read, and through the binding with host tensors."""

import ctypes

import pytest
import torch

from paper_2609_13716_amd import rollout as R

L = R.lib
P = 0x10000000  # arrays of the calls below start here, far apart
GAP = 0x1000000


def _at(i):
    return P + i * GAP


def _scan_cfg(**kw):
    v = dict(kind=R.RL_SCAN_GATED, dtype=R.RL_F32, n_steps=8, n_envs=4, n_agents=2, width=16, **{})
    v.update(kw)
    return R._ScanConfig(**v)


def _scan(cfg=None, u=_at(0), gate=_at(1), done=_at(2), h0=_at(3), h=_at(4), h_last=_at(5), ws=_at(6), n=1 << 20):
    return L.rl_scan(None if cfg is None else ctypes.byref(cfg), u, gate, done, h0, h, h_last, ws, n, None)


def _backward(cfg, gate=_at(0), done=_at(1), h0=_at(2), h=_at(3), dh=_at(4), dh_last=_at(5), du=_at(6), dgate=_at(7),
              dh0=_at(8), ws=_at(9), n=1 << 20):
    return L.rl_scan_backward(ctypes.byref(cfg), gate, done, h0, h, dh, dh_last, du, dgate, dh0, ws, n, None)


BAD_SCAN = [(dict(kind=2), R.RL_EUNSUPPORTED), (dict(kind=-1), R.RL_EUNSUPPORTED), (dict(dtype=2), R.RL_EUNSUPPORTED),
            (dict(n_steps=0), R.RL_EINVAL), (dict(n_steps=(1 << 30) + 1), R.RL_EINVAL),
             (dict(n_envs=0), R.RL_EINVAL), (dict(n_agents=-1), R.RL_EINVAL),
            (dict(width=0), R.RL_EINVAL), (dict(n_envs=1 << 20, width=1 << 10), R.RL_EINVAL),
            (dict(n_envs=1 << 30, n_agents=1 << 30, width=1 << 30), R.RL_EINVAL),
            (dict(kind=R.RL_SCAN_DIAGONAL, n_envs=1 << 20, width=1 << 9), R.RL_EINVAL)]


@pytest.mark.parametrize("kw,code", BAD_SCAN)
def test_scan_config(kw, code):
    cfg = _scan_cfg(**kw)
    assert _scan(cfg) == code and _backward(cfg) == code
    assert L.rl_scan_workspace_bytes(ctypes.byref(cfg), 0) == 0 and L.rollout_last_error()


def test_scan_arguments():
    cfg = _scan_cfg()
    assert _scan(None) == R.RL_EINVAL
    for kw in (dict(u=None), dict(gate=None), dict(h=None, h_last=None), dict(h=_at(0)), dict(h=_at(1) + 64),
               dict(h_last=_at(3) + 4), dict(h_last=_at(4)), dict(h_last=_at(2)), dict(u=_at(0) + 2),
               dict(h0=_at(3) + 2), dict(ws=_at(0))):
        assert _scan(cfg, **kw) == R.RL_EINVAL, kw
    for kw in (dict(gate=None), dict(dh=None), dict(du=None), dict(h=None), dict(du=_at(4)), dict(dgate=_at(3)),
               dict(dh0=_at(2)), dict(dh0=_at(6)), dict(du=_at(6) + 1), dict(dgate=_at(7) + 2), dict(ws=_at(7))):
        assert _backward(cfg, **kw) == R.RL_EINVAL, kw


def test_scan_workspace():
    """A call that needs a workspace refuses one that is missing, too small or not 16-byte aligned."""
    for backward in (0, 1):
        call = _backward if backward else _scan
        for cfg in (_scan_cfg(n_steps=100000, n_envs=1, n_agents=1, width=4),
                    _scan_cfg(kind=R.RL_SCAN_DIAGONAL, width=4)):
            need = L.rl_scan_workspace_bytes(ctypes.byref(cfg), backward)
            if need:
                assert call(cfg, ws=None) == R.RL_EINVAL
                assert call(cfg, n=need - 1) == R.RL_EINVAL
                assert call(cfg, ws=_at(9) + 8) == R.RL_EINVAL
                assert "workspace" in L.rollout_last_error().decode()
    assert L.rl_scan_workspace_bytes(ctypes.byref(_scan_cfg(kind=R.RL_SCAN_DIAGONAL)), 1) > 0


def _ppo_cfg(**kw):
    v = dict(n_rows=20000, n_actions=6, normalize_adv=1, clip=0.2, value_clip=0.2, value_coef=0.5, entropy_coef=0.01)
    v.update(kw)
    return R._PpoConfig(**v)


PPO = ("logits", "legal", "mask", "actions", "logp_old", "adv", "value", "value_old", "ret", "dlogits", "dvalue",
       "stats", "workspace")


def _ppo(cfg, n=1 << 20, **kw):
    p = [kw.get(name, _at(i)) for i, name in enumerate(PPO)]
    return L.rl_ppo_loss(ctypes.byref(cfg) if cfg else None, *p, n, None)


def test_ppo_refusals():
    inf, nan = float("inf"), float("nan")
    assert _ppo(None) == R.RL_EINVAL
    for kw, code in ((dict(n_rows=0), R.RL_EINVAL), (dict(n_rows=(1 << 40) + 1), R.RL_EINVAL),
                     (dict(n_actions=0), R.RL_EUNSUPPORTED), (dict(n_actions=33), R.RL_EUNSUPPORTED),
                     (dict(normalize_adv=2), R.RL_EINVAL), (dict(clip=0.0), R.RL_EINVAL), (dict(clip=nan), R.RL_EINVAL),
                     (dict(clip=inf), R.RL_EINVAL), (dict(value_clip=-0.1), R.RL_EINVAL),
                     (dict(value_clip=inf), R.RL_EINVAL), (dict(value_coef=nan), R.RL_EINVAL),
                     (dict(entropy_coef=inf), R.RL_EINVAL)):
        cfg = _ppo_cfg(**kw)
        assert _ppo(cfg) == code, kw
        assert L.rl_ppo_workspace_bytes(ctypes.byref(cfg)) == 0, kw
    cfg = _ppo_cfg()
    for name in PPO:
        if name not in ("legal", "mask"):
            assert _ppo(cfg, **{name: None}) == R.RL_EINVAL, name
        if name not in ("legal", "mask", "workspace"):
            assert _ppo(cfg, **{name: _at(PPO.index(name)) + 2}) == R.RL_EINVAL, name
    need = L.rl_ppo_workspace_bytes(ctypes.byref(cfg))
    assert need > 0
    assert _ppo(cfg, n=need - 1) == R.RL_EINVAL and _ppo(cfg, workspace=_at(12) + 4) == R.RL_EINVAL
    for name, other in (("dlogits", "logits"), ("dvalue", "value"), ("stats", "adv"), ("dvalue", "dlogits"),
                        ("workspace", "ret"), ("dlogits", "legal")):
        assert _ppo(cfg, **{name: _at(PPO.index(other))}) == R.RL_EINVAL, (name, other)


def _ortho(n=2, rows=16, cols=32, dtype=R.RL_F32, steps=5, g=_at(0), out=_at(1), ws=_at(2), size=1 << 23):
    return L.rl_orthogonalize(n, rows, cols, dtype, steps, g, out, ws, size, None)


def test_orthogonalize_refusals():
    for kw, code in ((dict(n=0), R.RL_EINVAL), (dict(n=65536), R.RL_EINVAL), (dict(rows=0), R.RL_EINVAL),
                     (dict(cols=16385), R.RL_EINVAL), (dict(dtype=2), R.RL_EUNSUPPORTED), (dict(steps=0), R.RL_EINVAL),
                     (dict(steps=33), R.RL_EINVAL), (dict(g=None), R.RL_EINVAL), (dict(out=None), R.RL_EINVAL),
                     (dict(out=_at(0) + 4), R.RL_EINVAL), (dict(g=_at(0) + 2), R.RL_EINVAL),
                     (dict(ws=_at(1)), R.RL_EINVAL)):
        assert _ortho(**kw) == code, kw
    need = L.rl_orthogonalize_workspace_bytes(2, 512, 640, R.RL_F32)
    assert need > 0
    big = dict(rows=512, cols=640)
    assert _ortho(**big, size=need - 1) == R.RL_EINVAL
    assert _ortho(**big, ws=None) == R.RL_EINVAL and _ortho(**big, ws=_at(2) + 8) == R.RL_EINVAL
    for bad in ((0, 4, 4, R.RL_F32), (1, 0, 4, R.RL_F32), (1, 4, 20000, R.RL_F32), (1, 4, 4, 9)):
        assert L.rl_orthogonalize_workspace_bytes(*bad) == 0


def test_binding_refusals():
    z = torch.zeros
    with pytest.raises(ValueError, match="device tensor"):
        R.scan(z(4, 2, 2, 8), z(4, 2, 2, 8))
    with pytest.raises(ValueError, match="device tensor"):
        R.scan_backward(z(4, 2, 2, 8), z(4, 2, 2, 8), z(4, 2, 2, 8))
    with pytest.raises(ValueError, match="device tensor"):
        R.orthogonalize(z(4, 8))
    with pytest.raises(ValueError, match="device tensor"):
        R.ppo_loss(z(4, 6), z(4, dtype=torch.int32), z(4), z(4), z(4), z(4))
    for u, gate, what in ((z(4, 2, 8), z(4, 2, 8), "T, E, A, D"), (z(4, 2, 2, 3, 8), z(2, 8), "2, P"),
                          (z(4, 2, 2, 8), z(2, 8), "2, P"),
                          (z(4, 2, 2, 8, dtype=torch.float16), z(4, 2, 2, 8), "bfloat16")):
        with pytest.raises(ValueError, match=what):
            R.scan(u, gate)
    for g, what in ((z(4), "rows, cols"), (z(2, 2, 2, 2), "rows, cols"), (z(4, 4, dtype=torch.float64), "bfloat16")):
        with pytest.raises(ValueError, match=what):
            R.orthogonalize(g)
