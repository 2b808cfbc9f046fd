"""The preference loss on the device against the float64 oracle: on per-token log-probs, and through the
LM head with both gradients.

Bounds on the call that takes log-probs.  u = 2^-24.  A sequence's sum adds at most ceil(T_s / 32) terms
in a thread and joins 64 such sums in trees or chains, of differences that are off by u |d| themselves:
  tR_s = (T_s / 32 + 70) u sum |d|      (divided by T_s with length_norm, one more rounding)
  th   = beta (tR_i + tR_j) + 4 u |h|
l changes by at most |l'| th, l' by at most |l''| th, plus 8 roundings of values of their size (a pair's own and
those of joining the pairs' sums, which a lane keeps in 64 bits)."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from oracle import sapo_oracle as orc
from paper_2509_08721_b200 import binding as B
from paper_2509_08721_b200 import inputs as gen
from tests import util as TU

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def case(lengths, groups, seed, levels=4, noise=0.3):
    """lengths: tokens of each sequence; groups: sequences of each question."""
    rng = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    go = np.concatenate([[0], np.cumsum(groups)]).astype(np.int32)
    T, S = int(cu[-1]), len(lengths)
    ref = (-rng.exponential(1.5, size=T)).astype(np.float32)
    logp = (ref + rng.normal(size=T) * noise).astype(np.float32)
    rewards = (rng.integers(0, levels + 1, size=S) / levels).astype(np.float32)
    return dict(logp=logp, ref=ref, cu=cu, go=go, rewards=rewards, T=T, S=S, Q=len(groups))


def run(c, beta, **kw):
    d = {k: torch.from_numpy(c[k]).cuda() for k in ("logp", "ref", "cu", "go", "rewards")}
    out, status = B.alloc_preference_outputs(c["T"], c["S"], c["Q"]), B.new_status()
    for k, v in out.items():
        v.fill_(-7) if v.dtype == torch.int32 else v.fill_(float("nan"))
    B.sapo_preference_loss(d["logp"], d["ref"], d["cu"], d["rewards"], d["go"], beta, out, status, **kw)
    got = {k: v.cpu().numpy() for k, v in out.items()}
    got["status"] = status.item()
    return got


def check(c, got, beta, kind="sigmoid", pairs="all", label_smoothing=0.0, length_norm=False, grad_scale=1.0):
    r = ho.preference_loss(c["logp"], c["ref"], c["cu"], c["rewards"], c["go"], beta, kind, pairs, label_smoothing,
                           length_norm, grad_scale)
    cu, go, S, Q = c["cu"], c["go"], c["S"], c["Q"]
    with np.errstate(invalid="ignore"):
        d = np.abs(c["logp"].astype(np.float64) - c["ref"])
    d[~np.isfinite(d)] = 0
    n = np.diff(cu)
    tR = np.array([(n[s] / 32 + 70) * U * d[cu[s]:cu[s + 1]].sum() for s in range(S)])
    if length_norm:
        tR = tR / np.maximum(n, 1) + U * np.abs(r["seq_logratio"])
    assert np.all(np.abs(got["seq_logratio"] - r["seq_logratio"]) <= tR + 1e-37)
    assert np.array_equal(got["q_pairs"], r["q_pairs"])
    tg, tq, tm = np.zeros(S), np.zeros(Q), np.zeros(Q)
    R = r["seq_logratio"]
    for q in range(Q):
        members = [s for s in range(go[q], go[q + 1]) if n[s] > 0 and np.isfinite(c["rewards"][s])]
        P = ho.preference_pairs(c["rewards"], members, pairs)
        for i, j in P:
            D = R[i] - R[j]
            l, dl = ho.pair_loss(D, beta, kind, label_smoothing)
            tD = tR[i] + tR[j] + 4 * U * abs(D)
            curve = {"sigmoid": beta * beta / 4, "squared": 2.0, "hinge": 0.0}[kind]
            big = {"sigmoid": beta, "squared": 2 * (abs(D) + 1 / beta), "hinge": beta}[kind]
            if kind == "hinge":
                assert abs(beta * D - 1) > 1e-4                       # no pair of the test sits on the kink
            tl = big * tD + curve * tD ** 2 + 8 * U * (abs(l) + {"squared": (abs(D) + 1 / beta) ** 2}.get(kind, 1.0))
            tq[q] += tl / len(P)
            tm[q] += beta * tD / len(P)
            e = abs(grad_scale) * (curve * tD + 8 * U * big) / (Q * len(P))
            tg[i] += e
            tg[j] += e
    assert np.all(np.abs(got["q_loss"] - r["q_loss"]) <= tq + U * np.abs(r["q_loss"]) + 1e-37)
    assert np.all(np.abs(got["q_margin"] - r["q_margin"]) <= tm + U * np.abs(r["q_margin"]) + 1e-37)
    assert abs(got["loss"][0] - r["loss"]) <= tq.sum() / Q + 2 * U * abs(r["loss"]) + 1e-37
    tg = tg + 4 * U * np.abs(r["seq_grad"])
    assert np.all(np.abs(got["seq_grad"] - r["seq_grad"]) <= tg + 1e-37)
    per = tg / np.maximum(n, 1) if length_norm else tg
    tt = np.repeat(per, n) + 2 * U * np.abs(r["gscale"][cu[0]:cu[-1]])
    assert np.all(np.abs(got["gscale"][cu[0]:cu[-1]] - r["gscale"][cu[0]:cu[-1]]) <= tt + 1e-37)
    return r


VARIANTS = [dict(), dict(pairs="best_worst", label_smoothing=0.1), dict(kind="squared", length_norm=True),
            dict(kind="hinge", grad_scale=-2.5), dict(label_smoothing=0.3, length_norm=True, grad_scale=0.5),
            dict(kind="squared", pairs="best_worst")]
# tokens per sequence and sequences per question: single tokens, ragged, empty sequences, questions of one or
# no completion, more completions than threads, long rows, very long ones with few questions
RNG = np.random.default_rng(77)
BATCHES = {
    "one_token": ([1, 1], [2]),
    "ragged": (list(RNG.integers(1, 90, size=24)), [8, 8, 8]),
    "empty_and_single": ([0, 5, 0, 7, 3, 0, 9, 4, 1], [3, 0, 1, 0, 5]),
    "many_per_question": (list(RNG.integers(1, 5, size=700)), [1, 300, 399]),
    "many_questions": (list(RNG.integers(1, 40, size=3000)), [2] * 1500),
    "long_rows": (list(RNG.integers(3000, 9000, size=8)), [4, 4]),
    "one_question_very_long": ([70001, 33, 50000, 1], [4]),
    "long_next_to_short": ([100000, 3, 2, 5, 1, 8], [2, 4]),
}


@pytest.mark.parametrize("kw", VARIANTS, ids=["default", "best_smooth", "squared_norm", "hinge", "smooth_norm", "squared_best"])
@pytest.mark.parametrize("name", list(BATCHES))
def test_preference_loss(name, kw):
    c = case(*BATCHES[name], seed=5)
    got = run(c, 0.1, **kw)
    check(c, got, 0.1, **kw)
    assert got["status"] == 0
    again = run(c, 0.1, **kw)
    for k in got:
        assert np.array_equal(got[k], again[k]), k


def test_equal_rewards_give_no_pair_and_extreme_margins_stay_finite():
    c = case([40] * 8, [4, 4], seed=1)
    c["rewards"][:4] = 0.5
    c["logp"][160:200] -= 60.0                                          # |h| in the hundreds, both signs
    c["logp"][200:240] += 60.0
    got = run(c, 0.5)
    check(c, got, 0.5)
    assert got["q_pairs"][0] == 0 and got["q_loss"][0] == 0 and not got["gscale"][:160].any()
    assert np.isfinite(got["gscale"]).all() and np.isfinite(got["loss"]).all()


def test_values_that_are_not_finite():
    c = case([30, 20, 25, 15, 10, 10], [3, 3], seed=2)
    c["logp"][3], c["ref"][40], c["logp"][60] = np.nan, np.inf, -np.inf
    c["rewards"][4] = np.nan
    c["rewards"][1], c["rewards"][2] = 1.0, 0.0
    got = run(c, 0.2)
    check(c, got, 0.2)
    assert got["gscale"][3] == 0 and got["gscale"][40] == 0 and got["gscale"][60] == 0
    assert got["gscale"][2] != 0 or got["seq_grad"][0] == 0
    assert not got["gscale"][c["cu"][4]:c["cu"][5]].any() and got["seq_grad"][4] == 0
    assert set(B.decode_status(got["status"])) == {"NONFINITE_INPUT", "NONFINITE_REWARD"}


def test_tokens_and_sequences_outside_every_question():
    c = case([10, 20, 30, 40, 50], [5], seed=3)
    c["go"] = np.array([1, 4], dtype=np.int32)
    c["Q"] = 1
    extra = 9                                                           # capacity behind the last token
    c["logp"], c["ref"] = np.concatenate([c["logp"], np.full(extra, np.nan, np.float32)]), np.concatenate([c["ref"], np.zeros(extra, np.float32)])
    c["T"] += extra
    got = run(c, 0.1)
    inner = dict(c, go=np.array([0, 3], np.int32), cu=(c["cu"][1:5] - 10).astype(np.int32), logp=c["logp"][10:100], ref=c["ref"][10:100],
                 rewards=c["rewards"][1:4], S=3, T=90)
    r = ho.preference_loss(inner["logp"], inner["ref"], inner["cu"], inner["rewards"], inner["go"], 0.1)
    assert np.allclose(got["gscale"][10:100], r["gscale"], rtol=1e-4, atol=1e-9)
    assert not got["gscale"][:10].any() and not got["gscale"][100:].any()
    assert got["seq_logratio"][0] == 0 and got["seq_logratio"][4] == 0 and got["seq_grad"][0] == 0 and got["seq_grad"][4] == 0
    assert got["status"] == 0


def test_bad_offsets_are_clamped_and_reported():
    c = case([16, 16, 16, 16], [2, 2], seed=4)
    for k, i, v in (("cu", 4, 1000), ("cu", 0, -5), ("go", 2, 9), ("go", 1, 3), ("cu", 2, 3)):
        b = dict(c)
        b[k] = c[k].copy()
        b[k][i] = v
        got = run(b, 0.1)
        assert ("BAD_INDEX" in B.decode_status(got["status"])) == (k != "go" or i != 1)
        assert np.isfinite(got["loss"]).all()


def test_empty_batch_of_tokens():
    out, status = B.alloc_preference_outputs(0, 2, 1), B.new_status()
    z = torch.zeros(0, device="cuda")
    B.sapo_preference_loss(z, z, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.tensor([1.0, 0.0], device="cuda"),
                           torch.tensor([0, 2], dtype=torch.int32, device="cuda"), 0.1, out, status)
    assert out["loss"].item() == 0 and out["q_pairs"].item() == 0 and status.item() == 0


# ------------------------------------------------------------------------------------------ through the head
def head_case(H, V, lengths, groups, seed, dtype=gen.DTYPE_BF16, noise=0.3):
    rng = np.random.default_rng(seed)
    c = case(lengths, groups, seed)
    h = rng.normal(size=(c["T"], H)).astype(np.float32)
    W = (rng.normal(size=(V, H)) * 0.05).astype(np.float32)
    if dtype == gen.DTYPE_BF16:
        h, W = gen.f32_to_bf16_bits(h), gen.f32_to_bf16_bits(W)
    c.update(h=h, W=W, ids=rng.integers(0, V, size=c["T"]).astype(np.int32))
    h64, W64 = (gen.as_f32(a).astype(np.float64) for a in (h, W))
    s = orc.token_logprobs(h64, W64, c["ids"])
    c["logp"], c["lse"], c["h64"], c["W64"] = s["logp"], s["lse"], h64, W64
    c["ref"] = (s["logp"] + rng.normal(size=c["T"]) * noise).astype(np.float32)
    return c


def head_run(c, beta, out_dtype=torch.float32, workspace=None, accumulate=None, T=None, **kw):
    t = TU.to_torch
    hidden, W = t(c["h"]), t(c["W"])
    T, V, H = c["T"], W.shape[0], W.shape[1]
    dcode = B.DTYPE_F32 if hidden.dtype == torch.float32 else B.DTYPE_BF16
    kind = B.WS_PREFERENCE | (B.WS_OUT_BF16 if out_dtype == torch.bfloat16 else 0)
    ws = TU.poisoned_workspace(B.sapo_workspace_bytes(kind, T, H, V, dcode) if workspace is None else workspace)
    out, status = B.alloc_preference_outputs(T, c["S"], c["Q"], scores=True), B.new_status()
    for v in out.values():
        v.fill_(-7) if v.dtype == torch.int32 else v.fill_(float("nan"))
    dh = torch.full((T, H), float("nan"), dtype=out_dtype, device="cuda")
    dW = torch.full((V, H), float("nan"), dtype=out_dtype, device="cuda") if accumulate is None else accumulate
    B.sapo_preference_loss_fwd_bwd(hidden, W, t(c["ids"]), t(c["ref"]), t(c["cu"]), t(c["rewards"]), t(c["go"]), beta, out,
                                   dh, dW, accumulate is not None, ws, status, **kw)
    torch.cuda.synchronize()
    return dict(out, dhidden=dh, dW=dW, status=status.item())


def head_check(c, got, beta, masked=None, dW_base=0.0, **kw):
    """Log-probs, loss and gradients under the bars of the policy loss: 2e-3 absolute on log-probs (so
    2e-3 sqrt(T_s) and more on a sum is generous; 1e-5 T_s is what fp32 accumulation leaves), 2e-2
    relative Frobenius error on the gradients."""
    r = ho.preference_loss(np.where(masked, 0, c["logp"]) if masked is not None else c["logp"], c["ref"], c["cu"], c["rewards"],
                           c["go"], beta, masked=masked, **kw)
    n = lambda k: got[k].float().cpu().numpy().astype(np.float64)
    ok = np.ones(c["T"], bool) if masked is None else ~masked
    assert np.abs(n("logp") - c["logp"])[ok].max() <= 2e-3 and np.abs(n("lse") - c["lse"]).max() <= 2e-3
    L = np.diff(c["cu"])
    assert np.all(np.abs(n("seq_logratio") - r["seq_logratio"]) <= 1e-5 * np.maximum(L, 1))
    assert abs(n("loss")[0] - r["loss"]) <= 1e-3 * abs(r["loss"]) + 1e-6
    assert np.array_equal(got["q_pairs"].cpu().numpy(), r["q_pairs"])
    gs = np.abs(r["gscale"]).max()
    assert np.abs(n("gscale") - r["gscale"]).max() <= 2e-3 * gs
    grads = orc.policy_loss_bwd(c["h64"], c["W64"], c["ids"].clip(0, c["W64"].shape[0] - 1), c["lse"], r["gscale"])
    if gs > 0:
        assert TU.rel_fro(n("dhidden"), grads["dhidden"]) <= 2e-2
        assert TU.rel_fro(n("dW"), grads["dW"] + dW_base) <= 2e-2
    else:
        assert not got["dhidden"].any() and (np.ndim(dW_base) > 0 or not got["dW"].any())
    return r


HEADS = [(64, 1000, [32] * 16, [8, 8]), (128, 2500, list(RNG.integers(1, 90, size=9)), [2, 0, 3, 4]),
         (328, 2000, [1, 2, 300, 5], [2, 2]), (896, 3001, list(RNG.integers(30, 120, size=6)), [2, 2, 2])]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,V,lengths,groups", HEADS)
@pytest.mark.parametrize("kw", VARIANTS[:3], ids=["default", "best_smooth", "squared_norm"])
def test_preference_through_the_head(H, V, lengths, groups, kw, out_dtype):
    c = head_case(H, V, lengths, groups, seed=H)
    got = head_run(c, 0.1, out_dtype, **kw)
    head_check(c, got, 0.1, **kw)
    assert got["status"] == 0


def test_head_smallest_workspace_accumulation_and_refusals():
    c = head_case(256, 2100, [100, 60, 140, 90], [2, 2], seed=8)
    least = B.sapo_workspace_bytes_min(B.WS_PREFERENCE, c["T"], 256, 2100, B.DTYPE_BF16)
    got = head_run(c, 0.1, workspace=least)                             # several chunks of 128 tokens
    head_check(c, got, 0.1)
    base = torch.randn(2100, 256, device="cuda") * 1e-4
    got = head_run(c, 0.1, accumulate=base.clone())
    head_check(c, got, 0.1, dW_base=base.cpu().numpy())
    with pytest.raises(B.SapoError, match="workspace"):
        head_run(c, 0.1, workspace=1024)
    with pytest.raises(B.SapoError, match="shape"):                     # bf16 operands only
        head_run(head_case(64, 1000, [32] * 8, [4, 4], seed=9, dtype=gen.DTYPE_F32), 0.1, workspace=1 << 30)


@pytest.mark.parametrize("small", [False, True])
def test_head_masked_tokens(small):
    c = head_case(128, 1500, [40, 50, 30, 60], [2, 2], seed=10)
    c["rewards"][:] = [1, 0, 0, 1]
    masked = np.zeros(c["T"], bool)
    c["ids"][7], c["ids"][100] = -1, 1500
    c["ref"][20], c["ref"][130] = np.nan, -np.inf
    masked[[7, 20, 100, 130]] = True
    ws = B.sapo_workspace_bytes_min(B.WS_PREFERENCE, c["T"], 128, 1500, B.DTYPE_BF16) if small else None
    got = head_run(c, 0.1, workspace=ws)
    keep = {k: c[k].copy() for k in ("logp",)}
    r = head_check(c, got, 0.1, masked=masked)
    assert not got["gscale"][torch.from_numpy(masked)].any() and not got["dhidden"][torch.from_numpy(masked)].any()
    assert got["logp"][7] == 0 and got["logp"][100] == 0
    assert set(B.decode_status(got["status"])) == {"BAD_TOKEN_ID", "NONFINITE_INPUT"}
    assert np.array_equal(keep["logp"], c["logp"]) and r["q_pairs"].sum() == 2


def test_head_questions_without_pairs_get_zero_gradients():
    c = head_case(256, 2000, [130, 140, 150, 160], [2, 2], seed=12)
    c["rewards"][:] = [1, 1, 0, 1]
    got = head_run(c, 0.1)
    head_check(c, got, 0.1)
    assert not got["dhidden"][:270].any() and got["dhidden"][270:].any()
    c["rewards"][:] = 0.5
    got = head_run(c, 0.1)
    head_check(c, got, 0.1)


def test_gscale_feeds_the_policy_backward():
    """sapo_preference_loss on the forward's log-probs, then sapo_policy_loss_bwd: the same gradients."""
    c = head_case(128, 2000, [50, 70, 40, 60], [2, 2], seed=14)
    one = head_run(c, 0.1)
    t = TU.to_torch
    hidden, W, ids = t(c["h"]), t(c["W"]), t(c["ids"])
    T, S = c["T"], c["S"]
    fwd, status = B.alloc_fwd_outputs(T, S), B.new_status()
    ws = TU.poisoned_workspace(B.sapo_workspace_bytes(B.WS_BWD, T, 128, 2000, B.DTYPE_BF16) + (1 << 20))
    B.sapo_policy_loss_fwd(hidden, W, ids, t(c["ref"]), torch.zeros(S, device="cuda"), t(c["cu"]), 0.2, 0.2, 1.0, fwd, ws, status)
    out = B.alloc_preference_outputs(T, S, c["Q"])
    B.sapo_preference_loss(fwd["logp"], t(c["ref"]), t(c["cu"]), t(c["rewards"]), t(c["go"]), 0.1, out, status)
    dh, dW = torch.empty(T, 128, device="cuda"), torch.empty(2000, 128, device="cuda")
    B.sapo_policy_loss_bwd(hidden, W, ids, fwd["lse"], out["gscale"], dh, dW, False, ws, status)
    assert status.item() == 0
    assert TU.rel_fro(dh.cpu().numpy(), one["dhidden"].cpu().numpy()) <= 1e-2
    assert TU.rel_fro(dW.cpu().numpy(), one["dW"].cpu().numpy()) <= 1e-2
    assert abs(out["loss"].item() - one["loss"].item()) <= 1e-5


@pytest.mark.parametrize("pairs", ["all", "best_worst"])
def test_head_leaves_out_blocks_without_a_pair(pairs):
    """Wide tiles: runs of more than 128 tokens that enter no pair (ties, single completions, completions between the
    best and the worst) are left out of the contractions, whose panel rows for them were never written."""
    c = head_case(512, 1800, [300, 280, 150, 400, 200, 310, 260], [2, 1, 4], seed=16)
    c["rewards"][:] = [0.5, 0.5, 1.0, 0.5, 0.25, 1.0, 0.5]
    got = head_run(c, 0.1, pairs=pairs)
    r = head_check(c, got, 0.1, pairs=pairs)
    assert list(r["q_pairs"]) == [0, 0, 5 if pairs == "all" else 1]
    assert not got["dhidden"][:730].any() and torch.isfinite(got["dW"]).all() and got["status"] == 0


def test_many_calls_on_two_streams_repeat_bit_for_bit():
    """Calls on two streams at once, more of them than the library has counters: every loss is the first one's."""
    c = case(list(RNG.integers(20, 60, size=80)), [2] * 40, seed=18)
    d = {k: torch.from_numpy(c[k]).cuda() for k in ("logp", "ref", "cu", "go", "rewards")}
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    n = 9000
    losses = torch.full((2 * n,), float("nan"), device="cuda")
    status = B.new_status()
    outs = [B.alloc_preference_outputs(c["T"], c["S"], c["Q"]) for _ in streams]
    torch.cuda.synchronize()
    for i in range(n):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                out = dict(outs[k], loss=losses[2 * i + k:2 * i + k + 1])
                B.sapo_preference_loss(d["logp"], d["ref"], d["cu"], d["rewards"], d["go"], 0.1, out, status)
    torch.cuda.synchronize()
    assert torch.isfinite(losses).all() and (losses == losses[0]).all() and status.item() == 0
    check(c, dict(run(c, 0.1)), 0.1)


def test_binding_refuses_arrays_that_do_not_fit():
    c = case([3, 4, 5], [2, 1], 5)
    good = {k: torch.from_numpy(c[k]).cuda() for k in ("logp", "ref", "cu", "go", "rewards")}
    out, status = B.alloc_preference_outputs(c["T"], c["S"], c["Q"]), B.new_status()
    for key, bad in [("ref", good["ref"][:-1]), ("ref", good["ref"].double()), ("ref", good["ref"].cpu()),
                     ("logp", torch.zeros(2 * c["T"], device="cuda")[::2]), ("cu", good["cu"].long()),
                     ("go", good["go"].float()), ("rewards", good["rewards"][:2])]:
        d = dict(good, **{key: bad})
        with pytest.raises(B.SapoError):
            B.sapo_preference_loss(d["logp"], d["ref"], d["cu"], d["rewards"], d["go"], 0.1, out, status)
    for key in ("gscale", "seq_logratio", "seq_grad", "q_loss"):
        with pytest.raises(B.SapoError):
            B.sapo_preference_loss(good["logp"], good["ref"], good["cu"], good["rewards"], good["go"], 0.1,
                                   dict(out, **{key: out[key][:-1]}), status)
    hidden, W = torch.zeros(c["T"], 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(128, 64, dtype=torch.bfloat16, device="cuda")
    ids, out = torch.zeros(c["T"], dtype=torch.int32, device="cuda"), B.alloc_preference_outputs(c["T"], c["S"], c["Q"], scores=True)
    ws = torch.empty(B.sapo_workspace_bytes(B.WS_PREFERENCE | B.WS_OUT_BF16, c["T"], 64, 128, B.DTYPE_BF16), dtype=torch.uint8, device="cuda")

    def through_head(hidden=hidden, W=W, ids=ids, ref=good["ref"], dhidden=torch.empty_like(hidden), dW=torch.empty_like(W)):
        B.sapo_preference_loss_fwd_bwd(hidden, W, ids, ref, good["cu"], good["rewards"], good["go"], 0.1, out, dhidden, dW,
                                       False, ws, status)
    through_head()
    assert status.item() == 0 and torch.isfinite(out["loss"]).all()
    for bad in [dict(W=W.float()), dict(W=W[:, :32]), dict(ids=ids.long()), dict(ids=ids[:-1]), dict(ref=good["ref"].cpu()),
                dict(dhidden=torch.empty(c["T"], 32, dtype=torch.bfloat16, device="cuda")), dict(dhidden=torch.empty(c["T"] - 1, 64, dtype=torch.bfloat16, device="cuda")),
                dict(dW=torch.empty(64, 64, dtype=torch.bfloat16, device="cuda")), dict(dW=torch.empty(64, 128, dtype=torch.bfloat16, device="cuda").t())]:
        with pytest.raises(B.SapoError):
            through_head(**bad)


def test_captured_calls_replay():
    """Captured in a graph (both forms, and the call through the head), calls beside the replays, new inputs: the
    results of direct calls, bit for bit."""
    cases = [case([9, 30, 4, 17], [2, 2], 21), case(list(RNG.integers(20, 60, size=80)), [2] * 40, seed=22)]
    H, V, status = 64, 300, B.new_status()
    gen_ = torch.Generator(device="cuda").manual_seed(23)
    data = []
    for c in cases:
        d = {k: torch.from_numpy(c[k]).cuda() for k in ("logp", "ref", "cu", "go", "rewards")}
        d["out"] = B.alloc_preference_outputs(c["T"], c["S"], c["Q"])
        d["hidden"] = torch.randn(c["T"], H, generator=gen_, device="cuda").bfloat16()
        d["W"] = torch.randn(V, H, generator=gen_, device="cuda").bfloat16()
        d["ids"] = torch.randint(0, V, (c["T"],), generator=gen_, device="cuda").int()
        d["scored"] = B.alloc_preference_outputs(c["T"], c["S"], c["Q"], scores=True)
        d["dh"], d["dW"] = torch.empty_like(d["hidden"]), torch.empty_like(d["W"])
        d["ws"] = torch.empty(B.sapo_workspace_bytes(B.WS_PREFERENCE | B.WS_OUT_BF16, c["T"], H, V, B.DTYPE_BF16),
                              dtype=torch.uint8, device="cuda")
        data.append(d)

    def calls():
        for d in data:
            B.sapo_preference_loss(d["logp"], d["ref"], d["cu"], d["rewards"], d["go"], 0.1, d["out"], status)
            B.sapo_preference_loss_fwd_bwd(d["hidden"], d["W"], d["ids"], d["ref"], d["cu"], d["rewards"], d["go"], 0.1,
                                           d["scored"], d["dh"], d["dW"], False, d["ws"], status)

    def results():
        torch.cuda.synchronize()
        return [v.clone() for d in data for v in (*d["out"].values(), *d["scored"].values(), d["dh"], d["dW"])]

    calls()                                                    # first calls set up what a capture may not
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(2):
        for d in data:
            d["ref"].add_(0.25 * torch.randn(d["ref"].shape, generator=gen_, device="cuda"))
        calls()
        want = results()
        for d in data:
            for v in (*d["out"].values(), *d["scored"].values(), d["dh"], d["dW"]):
                v.zero_()
        for _ in range(3):
            graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, results())) and status.item() == 0
