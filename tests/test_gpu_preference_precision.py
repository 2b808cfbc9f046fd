"""How exact the log ratios of the preference call through the head are on average.

The tensor cores truncate when they add to a logit, always towards zero: the log-sum-exp of a token comes out short,
with one sign, and a sequence's sum collects that.  The call takes a part of it out (a factor on the logits, from the
truncation of a sum whose parts all have about the same share of the logit); the policy forward does not.  Against 64
bits, b0 is the mean error of the policy forward's lse over the tokens of a case, b1 that of this call's log ratios, which
have the other sign.  NOISE: the mean over 1024 tokens of roundings of lse to fp32 (5e-7 each, 2e-8 in the mean), of log
ratios, and the factor's own rounding to fp32 (up to 4.2e-8 of a logit, and logits are about 4 where it counts).
  logits whose running sums grow evenly:  at least 60 % of b0 is gone
  any others (sums that cancel, one logit far above all):  no worse than without it"""
import pytest
import torch

from paper_2509_08721_b200 import binding as B

pytestmark = pytest.mark.gpu
NOISE = 2e-7
T = 1024


def make(H, V, kind):
    g = torch.Generator(device="cuda").manual_seed(H + V)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    h, W = r(T, H), r(V, H) / H ** 0.5
    ids = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    if kind.startswith("std"):                                       # logits of this standard deviation
        W *= float(kind[3:])
    if kind == "offset":                                             # the hidden states and the head have a common offset
        h += 0.3
        W += 0.03 / H ** 0.5
    if kind == "channels":                                           # a few channels twenty times as large
        h *= torch.where(torch.rand(H, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    if kind == "cancel":                                             # one half of the columns adds 20 to every logit, the other takes it away
        h[:, :H // 2] += 1
        h[:, H // 2:] -= 1
        W += 40.0 / H
    if kind == "peaked":                                             # the chosen token's logit is 20
        w = W[ids.long()].bfloat16().float()
        h = 0.3 * h + 20.0 * w / w.square().sum(1, keepdim=True)
    return h.bfloat16(), W.bfloat16(), ids, r(T)


@pytest.mark.parametrize("kind", ["std0.5", "std1", "std2", "offset", "channels", "cancel", "peaked"])
@pytest.mark.parametrize("H", [64, 896, 3584, 16384])
def test_mean_error_of_the_log_ratios(H, kind):
    V = 8000 if H <= 3584 else 4000
    h, W, ids, noise = make(H, V, kind)
    z = h.double() @ W.double().T
    lse = torch.logsumexp(z, 1)
    logp = z.gather(1, ids.long()[:, None])[:, 0] - lse
    ref = logp.float() + 0.2 * noise
    one = torch.arange(T + 1, device="cuda").int()                   # a token a sequence: the log ratios come out one by one
    two = torch.arange(0, T + 1, 2, device="cuda").int()
    status = B.new_status()
    out = B.alloc_preference_outputs(T, T, T // 2, scores=True)
    ws = torch.empty(B.sapo_workspace_bytes(B.WS_PREFERENCE, T, H, V, B.DTYPE_BF16), dtype=torch.uint8, device="cuda")
    dh, dW = torch.empty(T, H, device="cuda"), torch.empty(V, H, device="cuda")
    B.sapo_preference_loss_fwd_bwd(h, W, ids, ref, one, torch.zeros(T, device="cuda"), two, 0.1, out, dh, dW, False, ws, status)
    fwd = B.alloc_fwd_outputs(T, T)
    ws = torch.empty(B.sapo_workspace_bytes(B.WS_FWD, T, H, V, B.DTYPE_BF16), dtype=torch.uint8, device="cuda")
    B.sapo_policy_loss_fwd(h, W, ids, ref, torch.zeros(T, device="cuda"), one, 0.2, 0.2, 1.0, fwd, ws, status)
    b0 = (fwd["lse"].double() - lse).mean().item()
    b1 = -(out["seq_logratio"].double() - (logp - ref.double())).mean().item()
    print(f"\n[bias] H={H} {kind}: E_p z {(torch.softmax(z, 1) * z).sum(1).mean().item():.2f}, "
          f"policy forward's lse {b0:.2e}, log ratios {b1:.2e}")
    assert status.item() == 0 and b0 < NOISE                         # truncation: never upwards
    kept = 1.0 if kind in ("cancel", "peaked") else 0.4
    assert abs(b1) <= kept * abs(b0) + NOISE, (b0, b1)
