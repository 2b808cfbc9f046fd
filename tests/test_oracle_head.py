"""Pins of the float64 definitions in oracle/head_oracle.py: closed forms, library routines, finite
differences, invariants.  And the host-side argument checks of the operators' entry points (no GPU:
they are found before any launch)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from oracle import sapo_oracle as orc
from paper_2509_08721_b200 import binding as B


# ------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_matches_the_library_and_its_gradient_matches_differences(kind):
    rng = np.random.default_rng(0)
    T, H, eps = 5, 12, 1e-5
    x, gamma, beta, dy = rng.normal(size=(T, H)) * 3 + 1, rng.normal(size=H), rng.normal(size=H), rng.normal(size=(T, H))
    f = ho.norm_fwd(x, gamma, beta, eps, kind)
    t = lambda a: torch.from_numpy(a)
    lib = (torch.nn.functional.layer_norm(t(x), (H,), t(gamma), t(beta), eps) if kind == "layer"
           else torch.nn.functional.rms_norm(t(x), (H,), t(gamma), eps) + t(beta))
    assert np.allclose(f["y"], lib.numpy(), rtol=1e-12, atol=1e-12)
    b = ho.norm_bwd(dy, x, gamma, f["mean"], f["rstd"], kind)
    obj = lambda x, g, be: float((ho.norm_fwd(x, g, be, eps, kind)["y"] * dy).sum())
    def numeric(a, call, h=1e-6):
        out = np.zeros_like(a)
        for i in np.ndindex(a.shape):
            up, dn = a.copy(), a.copy()
            up[i] += h
            dn[i] -= h
            out[i] = (call(up) - call(dn)) / (2 * h)
        return out
    assert np.allclose(b["dx"], numeric(x, lambda a: obj(a, gamma, beta)), atol=1e-7)
    assert np.allclose(b["dgamma"], numeric(gamma, lambda a: obj(x, a, beta)), atol=1e-7)
    assert np.allclose(b["dbeta"], numeric(beta, lambda a: obj(x, gamma, a)), atol=1e-7)
    # a layer norm does not see an offset of the row, and neither does any norm (eps 0) its scale
    if kind == "layer":
        assert np.abs(b["dx"].sum(axis=1)).max() < 1e-12
    assert np.abs((ho.norm_bwd(dy, x, gamma, f["mean"], ho.norm_fwd(x, gamma, beta, 0.0, kind)["rstd"], kind)["dx"]
                   * x).sum(axis=1)).max() < 1e-10


# ------------------------------------------------------------------------------------------ 8 bits
def test_ckpt8_error_is_within_half_a_step_and_special_groups_are_kept():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(7, 300)) * 10.0 ** rng.integers(-6, 6, size=(7, 1))).astype(np.float32)
    x[2, 128:256] = 0
    x[3, :128] = 1e-37
    x[4, 5] = np.inf
    x[5, 290] = np.nan
    data, scale = ho.ckpt8_store(x)
    v = ho.ckpt8_values(data, scale)
    assert np.all(v[2, 128:256] == 0) and np.all(v[3, :128] == 0)
    assert np.all(np.isnan(v[4, :128])) and np.all(np.isnan(v[5, 256:])) and np.isfinite(v[4, 128:]).all()
    for t in (0, 1, 6):
        for k in range(3):
            p = slice(128 * k, 128 * (k + 1))
            top = np.abs(x[t, p]).max()
            assert np.abs(v[t, p] - x[t, p]).max() <= top * (1 / 254 + 1e-6)
            assert np.abs(data[t, p].astype(int)).max() == 127      # the largest magnitude uses the whole range


# ------------------------------------------------------------------------------------------ preference
CASES = [("sigmoid", "all", 0.0, False), ("sigmoid", "best_worst", 0.1, False), ("squared", "all", 0.0, True),
         ("hinge", "all", 0.0, False), ("sigmoid", "all", 0.2, True)]


@pytest.mark.parametrize("kind,pairs,smoothing,length_norm", CASES)
def test_preference_gradient_matches_differences(kind, pairs, smoothing, length_norm):
    rng = np.random.default_rng(2)
    L = rng.integers(1, 6, size=9)
    cu, go = np.concatenate([[0], np.cumsum(L)]), np.array([0, 3, 4, 9])
    ref = -rng.random(cu[-1]) * 3
    logp = ref + rng.normal(size=cu[-1])
    rewards = rng.integers(0, 3, size=9) / 2.0
    call = lambda lp: ho.preference_loss(lp, ref, cu, rewards, go, 0.3, kind, pairs, smoothing, length_norm, 1.0)
    r = call(logp)
    num = np.zeros_like(logp)
    for t in range(len(logp)):
        up, dn = logp.copy(), logp.copy()
        up[t] += 1e-6
        dn[t] -= 1e-6
        num[t] = (call(up)["loss"] - call(dn)["loss"]) / 2e-6
    assert np.allclose(r["gscale"], num, atol=1e-8)
    assert r["q_pairs"][1] == 0 and r["q_loss"][1] == 0                  # one completion: no pair
    # every pair moves its two sequences against each other
    for q in range(3):
        assert abs(r["seq_grad"][go[q]:go[q + 1]].sum()) < 1e-12
    # through a head: the chain rule equals the policy-gradient backward on gscale
    h, W = rng.normal(size=(len(logp), 4)), rng.normal(size=(7, 4))
    ids = rng.integers(0, 7, size=len(logp))
    s = orc.token_logprobs(h, W, ids)
    g = ho.preference_loss(s["logp"], ref, cu, rewards, go, 0.3, kind, pairs, smoothing, length_norm, 1.0)
    grads = orc.policy_loss_bwd(h, W, ids, s["lse"], g["gscale"])
    loss = lambda W: ho.preference_loss(orc.token_logprobs(h, W, ids)["logp"], ref, cu, rewards, go, 0.3, kind, pairs,
                                        smoothing, length_norm, 1.0)["loss"]
    for i in [(0, 0), (3, 2), (6, 3)]:
        up, dn = W.copy(), W.copy()
        up[i] += 1e-6
        dn[i] -= 1e-6
        assert abs(grads["dW"][i] - (loss(up) - loss(dn)) / 2e-6) < 1e-7


def test_preference_closed_forms():
    # policy equal to the reference: every pair costs ln 2 and pulls with beta / 2
    cu, go = np.array([0, 2, 5, 6]), np.array([0, 3])
    z = np.zeros(6)
    r = ho.preference_loss(z, z, cu, np.array([1.0, 0.0, 0.0]), go, 0.5)
    assert abs(r["loss"] - math.log(2)) < 1e-15 and r["q_pairs"][0] == 2
    assert np.allclose(r["seq_grad"], [-0.25, 0.125, 0.125])
    # equal rewards: no pair, no gradient
    r = ho.preference_loss(z, z, cu, np.ones(3), go, 0.5)
    assert r["loss"] == 0 and not r["gscale"].any()
    # ties of the best reward: the first completion stands for it
    assert ho.preference_pairs([0.5, 1.0, 1.0, 0.0, 0.0], [0, 1, 2, 3, 4], "best_worst") == [(1, 3)]


# ------------------------------------------------------------------------------------------ refusals
INVALID, SHAPE, SMALL = -1, -2, -3
P = 0x10000                                 # a non-NULL, aligned value: nothing dereferences it on the host


def _fwd(**kw):
    a = dict(x=P, x_dtype=0, T=4, H=64, ld_x=64, gamma=P, beta=P, kind=0, eps=1e-6, w_dtype=1, y=P, y_dtype=0, ld_y=64,
             mean=P, rstd=P, ckpt=None, status=None)
    a.update(kw)
    cfg = B.NormCfgC(a["kind"], a["eps"], a["w_dtype"])
    return B.load().sapo_norm_fwd(a["x"], a["x_dtype"], a["T"], a["H"], a["ld_x"], a["gamma"], a["beta"], C.byref(cfg), a["y"],
                                  a["y_dtype"], a["ld_y"], a["mean"], a["rstd"],
                                  C.byref(a["ckpt"]) if a["ckpt"] else None, a["status"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(x_dtype=2), INVALID), (dict(y_dtype=-1), INVALID),
    (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(H=16385, ld_x=16385, ld_y=16385), SHAPE), (dict(ld_x=63), INVALID),
    (dict(ld_y=63), INVALID), (dict(kind=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(w_dtype=5), INVALID), (dict(x=P + 1), INVALID), (dict(gamma=P + 2), INVALID),
    (dict(ckpt=B.Ckpt8C(P, P, 64, 1)), INVALID),                                # a checkpoint needs a status word
    (dict(ckpt=B.Ckpt8C(None, P, 64, 1), status=P), INVALID), (dict(ckpt=B.Ckpt8C(P, P, 63, 1), status=P), INVALID),
    (dict(ckpt=B.Ckpt8C(P, P, 64, 0), status=P), INVALID), (dict(ckpt=B.Ckpt8C(P, P + 2, 64, 1), status=P), INVALID)])
def test_norm_fwd_refuses(bad, code):
    assert _fwd(**bad) == code


def _bwd(**kw):
    a = dict(dy=P, dy_dtype=0, ld_dy=64, x=P, x_dtype=0, ld_x=64, ckpt=None, T=4000, H=64, gamma=P, kind=0, w_dtype=1,
             mean=P, rstd=P, dx=P, dx_dtype=0, ld_dx=64, dgamma=P, dbeta=P, acc=0, ws=P, bytes=1 << 30)
    a.update(kw)
    cfg = B.NormCfgC(a["kind"], 0.0, a["w_dtype"])
    return B.load().sapo_norm_bwd(a["dy"], a["dy_dtype"], a["ld_dy"], a["x"], a["x_dtype"], a["ld_x"],
                                  C.byref(a["ckpt"]) if a["ckpt"] else None, a["T"], a["H"], a["gamma"], C.byref(cfg),
                                  a["mean"], a["rstd"], a["dx"], a["dx_dtype"], a["ld_dx"], a["dgamma"], a["dbeta"],
                                  a["acc"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(dy=None), INVALID), (dict(dx=None), INVALID), (dict(x=None), INVALID),
    (dict(ckpt=B.Ckpt8C(P, P, 64, 1)), INVALID),                                # both x and its checkpoint
    (dict(x=None, ckpt=B.Ckpt8C(P, P, 32, 1)), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID),
    (dict(ld_dy=10), INVALID), (dict(ld_dx=10), INVALID), (dict(ld_x=10), INVALID), (dict(H=1 << 20, ld_x=1 << 20), SHAPE),
    (dict(dx_dtype=3), INVALID), (dict(kind=-1), INVALID)])
def test_norm_bwd_refuses(bad, code):
    assert _bwd(**bad) == code


def test_norm_workspace_query():
    assert B.sapo_norm_workspace_bytes(-1, 64) == 0 and B.sapo_norm_workspace_bytes(4, 16385) == 0
    assert B.sapo_norm_workspace_bytes(4, 64) >= 2 * 64 * 4
    assert B.sapo_norm_workspace_bytes(1 << 20, 896) >= 2 * 896 * 4 * 148


@pytest.mark.parametrize("bad", [dict(data=None), dict(scale=None), dict(ld=99), dict(ld_scale=0), dict(x=None),
                                 dict(x_dtype=7), dict(ld_x=99), dict(T=-1), dict(H=0)])
def test_ckpt8_refuses(bad):
    a = dict(x=P, x_dtype=0, T=3, H=100, ld_x=100, data=P, scale=P, ld=104, ld_scale=1)
    a.update(bad)
    c = B.Ckpt8C(a["data"], a["scale"], a["ld"], a["ld_scale"])
    assert B.load().sapo_ckpt8_store(a["x"], a["x_dtype"], a["T"], a["H"], a["ld_x"], C.byref(c), P, None) == INVALID
    assert B.load().sapo_ckpt8_restore(C.byref(c), a["T"], a["H"], a["x"], a["x_dtype"], a["ld_x"], None) == INVALID


def _pref(**kw):
    a = dict(logp=P, ref=P, T=8, cu=P, S=2, rewards=P, go=P, Q=1, beta=0.1, e=0.0, scale=1.0, kind=0, pairs=0, norm=0,
             gscale=P, ratio=P, grad=P, q_loss=P, loss=P, status=P)
    a.update(kw)
    cfg = B.PrefCfgC(a["beta"], a["e"], a["scale"], a["kind"], a["pairs"], a["norm"])
    return B.load().sapo_preference_loss(a["logp"], a["ref"], a["T"], a["cu"], a["S"], a["rewards"], a["go"], a["Q"],
                                         C.byref(cfg), a["gscale"], a["ratio"], a["grad"], a["q_loss"], None, None,
                                         a["loss"], a["status"], None)


@pytest.mark.parametrize("bad", [dict(logp=None), dict(ref=None), dict(T=-1), dict(cu=None), dict(S=0), dict(Q=0),
                                 dict(rewards=None), dict(go=None), dict(beta=0.0), dict(beta=-1.0), dict(beta=float("nan")),
                                 dict(beta=float("inf")), dict(e=0.5), dict(e=-0.1), dict(e=0.1, kind=1), dict(kind=3),
                                 dict(pairs=2), dict(norm=2), dict(scale=float("inf")), dict(gscale=None), dict(ratio=None),
                                 dict(grad=None), dict(q_loss=None), dict(loss=None), dict(status=None)])
def test_preference_loss_refuses(bad):
    assert _pref(**bad) == INVALID


def test_preference_head_refuses_and_its_workspace_query():
    def call(**kw):
        a = dict(hidden=P, W=P, dtype=0, T=256, H=64, V=1000, ldh=64, ldw=64, ids=P, ref=P, cu=P, S=2, rewards=P, go=P, Q=1,
                 beta=0.1, out=P, dh=P, dW=P, od=1, ws=P, bytes=1 << 40)
        a.update(kw)
        cfg = B.PrefCfgC(a["beta"], 0.0, 1.0, 0, 0, 0)
        o = a["out"]
        return B.load().sapo_preference_loss_fwd_bwd(
            a["hidden"], a["W"], a["dtype"], a["T"], a["H"], a["V"], a["ldh"], a["ldw"], a["ids"], a["ref"], a["cu"], a["S"],
            a["rewards"], a["go"], a["Q"], C.byref(cfg), o, o, o, o, o, o, o, o, o, a["dh"], a["dW"], a["od"], 0, a["ws"],
            a["bytes"], P, None)
    for bad in (dict(hidden=None), dict(W=None), dict(dtype=2), dict(T=0), dict(ldh=32), dict(ldw=65), dict(ids=None),
                dict(ref=None), dict(cu=None), dict(S=0), dict(rewards=None), dict(go=None), dict(Q=0), dict(beta=0.0),
                dict(out=None), dict(dh=None), dict(dW=P + 8), dict(od=5), dict(ws=None), dict(hidden=P + 4)):
        assert call(**bad) == INVALID, bad
    assert call(H=60, ldh=64, ldw=64) == SHAPE
    assert call(dtype=1, ldh=64, ldw=64) == SHAPE                        # bf16 operands only
    assert B.sapo_workspace_bytes(B.WS_PREFERENCE, 9216, 896, 151936, B.DTYPE_F32) == 0
    for out in (0, B.WS_OUT_BF16):
        full = B.sapo_workspace_bytes(B.WS_PREFERENCE | out, 9216, 896, 151936, B.DTYPE_BF16)
        least = B.sapo_workspace_bytes_min(B.WS_PREFERENCE | out, 9216, 896, 151936, B.DTYPE_BF16)
        assert 0 < least <= full
    assert B.sapo_workspace_bytes(B.WS_PREFERENCE, 9216, 12, 1000, B.DTYPE_BF16) == 0
