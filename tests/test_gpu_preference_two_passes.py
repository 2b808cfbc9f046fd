"""The preference call through the head with a panel smaller than the batch: the forward keeps sums only and the backward
recomputes the logits, in several chunks each.  The same bars as with one pass (test_gpu_preference.py), bf16 outputs,
accumulation, tokens that are masked or too far from the reference, and replays of a graph."""
import numpy as np
import pytest
import torch

from paper_2509_08721_b200 import binding as B
from tests import util as TU
from tests.test_gpu_preference import head_case, head_check, head_run

pytestmark = pytest.mark.gpu


def small_workspace(c, H, V, out_dtype, blocks=1):
    """Bytes for a panel of `blocks` blocks of 128 tokens."""
    kind = B.WS_PREFERENCE | (B.WS_OUT_BF16 if out_dtype == torch.bfloat16 else 0)
    least = B.sapo_workspace_bytes_min(kind, c["T"], H, V, B.DTYPE_BF16)
    whole = B.sapo_workspace_bytes(kind, c["T"], H, V, B.DTYPE_BF16)
    per_block = (whole - least) // (-(-c["T"] // 128) - 1)
    n = least + (blocks - 1) * per_block
    assert n < whole
    return n


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,blocks", [(64, 1), (328, 2), (896, 3)])
@pytest.mark.parametrize("kw", [dict(), dict(kind="squared", pairs="best_worst", length_norm=True)])
def test_chunks(H, blocks, kw, out_dtype):
    V = 2500
    c = head_case(H, V, [100, 1, 60, 190, 90, 130, 64], [2, 1, 4], seed=31 + H)
    got = head_run(c, 0.1, out_dtype, workspace=small_workspace(c, H, V, out_dtype, blocks), **kw)
    head_check(c, got, 0.1, **kw)
    assert got["status"] == 0
    base = (torch.randn(V, H, device="cuda") * 1e-3).to(out_dtype)
    got = head_run(c, 0.1, out_dtype, workspace=small_workspace(c, H, V, out_dtype, blocks), accumulate=base.clone(), **kw)
    head_check(c, got, 0.1, dW_base=base.double().cpu().numpy(), **kw)


@pytest.mark.parametrize("small", [False, True])
def test_tokens_too_far_from_the_reference_are_masked(small):
    """A log ratio beyond 69 either way: reported, no gradient, out of its sequence's sum; everything else as without it."""
    H, V = 256, 1500
    c = head_case(H, V, [150, 40, 130, 60], [2, 2], seed=41)
    c["rewards"][:] = [1, 0, 0, 1]
    masked = np.zeros(c["T"], bool)
    for t, far in ((5, 200.0), (160, -200.0), (300, 90.0)):
        c["ref"][t] += far
        masked[t] = True
    got = head_run(c, 0.1, workspace=small_workspace(c, H, V, torch.float32) if small else None)
    lse = got["lse"].clone()
    assert not lse[torch.from_numpy(masked)].any() and not got["logp"][torch.from_numpy(masked)].any()
    got["lse"][torch.from_numpy(masked).cuda()] = torch.from_numpy(c["lse"][masked]).float().cuda()
    r = head_check(c, got, 0.1, masked=masked)
    assert not got["gscale"][torch.from_numpy(masked)].any() and not got["dhidden"][torch.from_numpy(masked)].any()
    assert B.decode_status(got["status"]) == ["EXP_RANGE"] and r["q_pairs"].sum() == 2


def test_captured_call_replays():
    H, V = 128, 1200
    c = head_case(H, V, [100, 60, 140, 90], [2, 2], seed=51)
    t = TU.to_torch
    d = {k: t(c[k]) for k in ("h", "W", "ids", "ref", "cu", "rewards", "go")}
    out, status = B.alloc_preference_outputs(c["T"], c["S"], c["Q"], scores=True), B.new_status()
    dh, dW = torch.empty(c["T"], H, device="cuda"), torch.empty(V, H, device="cuda")
    ws = torch.empty(small_workspace(c, H, V, torch.float32), dtype=torch.uint8, device="cuda")

    def call():
        B.sapo_preference_loss_fwd_bwd(d["h"], d["W"], d["ids"], d["ref"], d["cu"], d["rewards"], d["go"], 0.1, out, dh, dW,
                                       False, ws, status)
    results = lambda: [v.clone() for v in (*out.values(), dh, dW)]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for shift in (0.1, -0.2):
        d["ref"].add_(shift)
        call()
        torch.cuda.synchronize()
        want = results()
        for v in (*out.values(), dh, dW):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, results())) and status.item() == 0
