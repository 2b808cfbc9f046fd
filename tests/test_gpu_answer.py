"""The operators that update a policy's last layers and answer with them, run together as a node would
(pipeline.PreferenceScorer -> HeadOptimizer -> AnswerHead), against the float64 oracle at every seam.

Logits: the device's product of the device's own 8-bit operands is held to the bound of test_gpu_fp8.py; the ids and log-probs to those
of the oracle on the device's own logits, with the bound of test_gpu_sample.py."""
import numpy as np
import pytest
import torch

from oracle import answer_oracle as ao
from oracle import head_oracle as ho
from paper_2509_08721_b200 import binding as B
from paper_2509_08721_b200 import inputs as gen
from paper_2509_08721_b200.pipeline import AnswerHead, HeadOptimizer, PreferenceScorer
from tests import util as TU
from tests.test_gpu_fp8 import check_product, host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("bits,norm", [(8, "rms"), (32, "layer")])
def test_train_update_answer(bits, norm):
    H, V = 256, 2001
    recipe = gen.Recipe("answer", gen.DTYPE_BF16, H, V, 4, 2, 2, ("uniform", 5, 60), ("bernoulli", 0.5))
    batch = gen.make_batch(recipe, 3)
    rng = np.random.default_rng(4)
    gen.install_old_logp(batch, np.log(rng.uniform(1e-4, 1e-3, size=batch.T)).astype(np.float32))
    W = TU.to_torch(batch.W)
    gamma = torch.from_numpy((1 + 0.1 * rng.normal(size=H)).astype(np.float32)).cuda()
    nbeta = torch.from_numpy((0.1 * rng.normal(size=H)).astype(np.float32)).cuda() if norm == "layer" else None
    trainer = PreferenceScorer(W, gamma, nbeta, batch.T, batch.S, recipe.Q, beta=0.5, norm=norm)
    opt = HeadOptimizer(W, gamma, nbeta, lr=1e-2, weight_decay=0.1, bits=bits, seed=11)
    head = AnswerHead(W, gamma, nbeta, 50, norm=norm)
    dev = TU.dev_rollouts(batch.local), TU.dev_rollouts(batch.ext), TU.dev_selection(batch.sel)
    x = TU.to_torch(batch.built.hidden)[:40]
    for step in (1, 2):
        before = [p.cpu().numpy().astype(np.float64) for p in opt.tensors.params]
        res = trainer.step(*dev, batch.T, batch.S)
        opt.step(res.dW, res.dgamma, res.dbeta)
        head.refresh()
        seeds = torch.from_numpy(rng.integers(-2 ** 63, 2 ** 63 - 1, size=40)).cuda()
        ids, logp = head.next_tokens(x, seeds, temperature=0.9, top_k=500, top_p=0.95)
        torch.cuda.synchronize()
        for part in (trainer, opt, head):
            part.check_status()
        if step == 1:                      # the first step moves every weight with a gradient by lr, less eps
            g = res.dW.float().cpu().numpy().astype(np.float64).reshape(before[0].shape)
            want = before[0] * (1 - 1e-2 * 0.1) - 1e-2 * g / (np.abs(g) + 1e-8)
            got = opt.master.cpu().numpy()
            # 0.1 g and 0.001 g g in fp32 and back: 16 u of the update; eps weighs g where it is tiny; 3 u of the weight
            assert np.all(np.abs(got - want) <= 16 * U * 1e-2 + 3 * U * np.abs(want))
        assert torch.equal(W, opt.master.bfloat16())
        wc, ws = ao.fp8_store(W.float().cpu().numpy(), True)
        codes, scale = host(head.w8)
        assert np.array_equal(codes & 127, wc & 127) and np.array_equal(scale, ws)
        f = ho.norm_fwd(x.float().cpu().numpy(), gamma.cpu().numpy(), None if nbeta is None else nbeta.cpu().numpy(), 1e-6, norm)
        hidden = head.hidden[:40].float().cpu().numpy()
        assert np.abs(hidden - f["y"]).max() <= 2.0 ** -8 * np.abs(f["y"]).max()
        x8 = B.Fp8(head.x8.data[:40], head.x8.scale[:40], H)
        xc, xs = ao.fp8_store(hidden)
        codes, scale = host(x8)
        assert np.array_equal(codes & 127, xc & 127) and np.array_equal(scale, xs)
        z = head.logits[:40, :V]
        check_product(x8, head.w8, z)
        z, ids, logp, seeds = z.cpu().numpy(), ids.cpu().numpy(), logp.cpu().numpy(), seeds.cpu().numpy()
        for b in range(40):
            i, lp, _ = ao.sample(z[b], int(seeds[b]) % 2 ** 64, 0.9, 500, 0.95)
            assert ids[b] == i and abs(logp[b] - lp) <= 2.0 ** -22 + 477 * U + 2 * U * (abs(lp) + 30)
