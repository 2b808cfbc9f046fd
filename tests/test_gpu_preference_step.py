"""The operators around the head in one preference-training step (pipeline.PreferenceScorer): pack, norm with
an 8-bit checkpoint, preference loss through the head, norm backward, against the float64 oracle run on the
same packed batch, and as a descent direction."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from oracle import sapo_oracle as orc
from paper_2509_08721_b200 import binding as B
from paper_2509_08721_b200 import inputs as gen
from paper_2509_08721_b200.pipeline import PreferenceScorer
from tests import util as TU

pytestmark = pytest.mark.gpu


def make(seed, H=256, V=2000):
    recipe = gen.Recipe("pref", gen.DTYPE_BF16, H, V, 4, 2, 2, ("uniform", 5, 90), ("bernoulli", 0.5))
    batch = gen.make_batch(recipe, seed)
    rng = np.random.default_rng(seed)
    gamma = (1 + 0.2 * rng.normal(size=H)).astype(np.float32)
    nbeta = (0.1 * rng.normal(size=H)).astype(np.float32)
    return batch, gamma, nbeta


def reference(batch, gamma, nbeta, norm, eps, ref_lp, beta, x_read):
    """hidden as the device rounds it (bf16), then the loss and all gradients; x_read: what the norm's backward reads."""
    b = batch.built
    x = gen.as_f32(b.hidden).astype(np.float64)
    f = ho.norm_fwd(x, gamma, nbeta, eps, norm)
    h = gen.as_f32(gen.f32_to_bf16_bits(f["y"].astype(np.float32))).astype(np.float64)
    W = gen.as_f32(batch.W).astype(np.float64)
    s = orc.token_logprobs(h, W, b.ids)
    r = ho.preference_loss(s["logp"], ref_lp, b.cu_seqlens, b.rewards, b.group_offsets, beta)
    g = orc.policy_loss_bwd(h, W, b.ids, s["lse"], r["gscale"])
    n = ho.norm_bwd(g["dhidden"], x_read, gamma, f["mean"], f["rstd"], norm)
    return r, g, n


@pytest.mark.parametrize("norm,keep,dt", [("layer", "bits8", torch.float32), ("rms", "bits8", torch.bfloat16), ("layer", "exact", torch.bfloat16)])
def test_step_matches_the_oracle(norm, keep, dt):
    batch, gamma, nbeta = make(21)
    b = batch.built
    nbeta = nbeta if norm == "layer" else None
    x = gen.as_f32(b.hidden)
    f = ho.norm_fwd(x, gamma, nbeta, 1e-6, norm)
    cur = orc.token_logprobs(f["y"], gen.as_f32(batch.W).astype(np.float64), b.ids)["logp"].astype(np.float32)
    gen.install_old_logp(batch, cur)                       # the reference policy: the current one, with noise
    x_read = x.astype(np.float64) if keep == "exact" else ho.ckpt8_values(*ho.ckpt8_store(x))
    r, g, n = reference(batch, gamma, nbeta, norm, 1e-6, b.old_logp, 0.5, x_read)
    sc = PreferenceScorer(TU.to_torch(batch.W), torch.from_numpy(gamma).cuda(), None if nbeta is None else torch.from_numpy(nbeta).cuda(),
                          batch.T + 37, batch.S + 2, 6, beta=0.5, norm=norm, keep=keep, grad_dtype=dt)
    for _ in range(2):                                     # the second step finds the first one's buffers
        res = sc.step(TU.dev_rollouts(batch.local), TU.dev_rollouts(batch.ext), TU.dev_selection(batch.sel), batch.T, batch.S)
        torch.cuda.synchronize()
        sc.check_status()
        f64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(res.out["q_pairs"].cpu().numpy(), r["q_pairs"]) and r["q_pairs"].sum() > 0
        assert abs(res.loss.item() - r["loss"]) <= 1e-3 * abs(r["loss"]) + 1e-5
        assert TU.rel_fro(f64(res.dW), g["dW"]) <= 2e-2
        assert TU.rel_fro(f64(res.dx), n["dx"]) <= 2e-2
        assert TU.rel_fro(f64(res.dgamma), n["dgamma"]) <= 2e-2
        if nbeta is not None:
            assert TU.rel_fro(f64(res.dbeta), n["dbeta"]) <= 2e-2


def test_steps_along_the_gradient_lower_the_loss():
    """The head and the norm's weights follow their gradients (a line search's first step): the loss falls by what
    the gradient says, to first order."""
    batch, gamma, _ = make(22)
    b = batch.built
    f = ho.norm_fwd(gen.as_f32(b.hidden), gamma, None, 1e-6, "rms")
    gen.install_old_logp(batch, orc.token_logprobs(f["y"], gen.as_f32(batch.W).astype(np.float64), b.ids)["logp"].astype(np.float32))
    args = (TU.dev_rollouts(batch.local), TU.dev_rollouts(batch.ext), TU.dev_selection(batch.sel), batch.T, batch.S)
    W32 = TU.to_torch(batch.W).float()
    run = lambda W, g: PreferenceScorer(W.bfloat16(), g, None, batch.T, batch.S, 4, beta=0.5, grad_dtype=torch.float32).step(*args)
    g0 = torch.from_numpy(gamma).cuda()
    r = run(W32, g0)
    l0, dW, dg = r.loss.item(), r.dW.clone(), r.dgamma.clone()
    step = 0.05 / float((dW ** 2).sum() + (dg ** 2).sum())
    W1 = W32 - step * dW
    l1 = run(W1, g0 - step * dg).loss.item()
    # the change that the head sees is that of its bf16 weights
    says = float((dW * (W32 - W1.bfloat16().float())).sum() + step * (dg ** 2).sum())
    assert says > 0 and 0.6 * says <= l0 - l1 <= 1.4 * says, (l0, l1, says)


def test_bad_arguments():
    batch, gamma, _ = make(23)
    W, g = TU.to_torch(batch.W), torch.from_numpy(gamma).cuda()
    with pytest.raises(ValueError):
        PreferenceScorer(W, g, None, 128, 4, 2, keep="half")
    with pytest.raises(B.SapoError):
        PreferenceScorer(W.float(), g, None, 128, 4, 2)
    sc = PreferenceScorer(W, g, None, batch.T, batch.S, 4, kind="other")
    with pytest.raises(B.SapoError):
        sc.step(TU.dev_rollouts(batch.local), TU.dev_rollouts(batch.ext), TU.dev_selection(batch.sel), batch.T, batch.S)
