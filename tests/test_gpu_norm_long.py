"""The norm's kernels and the checkpoints on batches long enough for their steady state: every group of warps goes
through 16 rows and more (a ring of shared-memory stages is refilled several times, a thread adds up that many rows' weight
gradients), no row is zero, and every output is compared with 64-bit arithmetic (torch on the device, elementary operations).

Bounds as in test_gpu_norm.py, u = 2^-24, but the weight gradients': a column's sum passes through one thread's chain of
at most n rows (a row is spread over ceil(H / 512) warps at most, an SM takes 8 warps' rows at least at a time), 16 groups
of a block, then 5 parts, 3 lanes and 16 warps of the reduction, 48 roundings in all with those of a term itself:
  n = ceil(T / (148 max(1, 8 // ceil(H / 512))));  dgamma, dbeta: (n + 48) u sum_t |terms|, and what xh itself is off by.
A row that is left out or read twice changes a column by 1 of T terms; the bound is below a quarter of their mean."""
import pytest
import torch

from paper_2509_08721_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# rows and columns: one vector a thread (200 ragged, 256 whole), two with 1, 2, 3, 5, 7, 8 and 16 warps a row (512, 1536,
# 3584 and 8192 whole), four (9000, 16384), rows on no vector boundary (1001), short ones (72), widths between (264)
SHAPES = [(40000, 72), (40000, 200), (40000, 256), (40000, 264), (40000, 512), (30000, 896), (20000, 1001), (20000, 1280), (20000, 1536),
          (15000, 2304), (15000, 3584), (15000, 4096), (6000, 8192), (6000, 9000), (4000, 16384)]
TYPES = [("layer", "bf16", "bf16"), ("rms", "bf16", "f32"), ("rms", "f32", "bf16"), ("layer", "f32", "f32")]


def data(T, H, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(T, H, generator=g, device="cuda") * scale + shift).to(dtype)


def within(got, want, tol):
    """Every element of `got` is the rounding, to its own type, of a value in want +- tol."""
    lo, hi = want - tol, want + tol
    if got.dtype == torch.bfloat16:
        lo, hi = lo.bfloat16().double(), hi.bfloat16().double()
    v = got.double()
    return bool(((lo <= v) & (v <= hi)).all())


def check_fwd(x, gamma, beta, eps, layer, y, mean, rstd):
    X = x.double()
    m = X.mean(1, keepdim=True) if layer else torch.zeros(len(X), 1, dtype=torch.float64, device="cuda")
    dm = 64 * U * X.abs().mean(1, keepdim=True) if layer else torch.zeros_like(m)
    xc = X - m
    rs = (xc.square().mean(1, keepdim=True) + eps).rsqrt()
    dr = 68 * U + (rs * dm).square()
    G = gamma.double()
    want = xc * rs * G + (0.0 if beta is None else beta.double())
    assert within(y, want, G.abs() * rs * (dm + 2 * U * xc.abs()) + (xc * rs * G).abs() * dr + 2 * U * want.abs())
    assert mean is None or bool(((mean.double() - m[:, 0]).abs() <= dm[:, 0]).all())
    assert bool(((rstd.double() - rs[:, 0]).abs() <= (rs * dr)[:, 0]).all())


def check_bwd(dy, X, gamma, mean, rstd, layer, dx, dgamma, dbeta):
    """X: the values that the backward reads, in 64 bits."""
    T = len(X)
    M = mean.double()[:, None] if layer else torch.zeros(T, 1, dtype=torch.float64, device="cuda")
    rs, D = rstd.double()[:, None], dy.double()
    xh, g = (X - M) * rs, D * gamma.double()
    c1, c2 = (g.mean(1, keepdim=True) if layer else torch.zeros_like(M)), (g * xh).mean(1, keepdim=True)
    dxh = 3 * U * (X.abs() + M.abs()) * rs
    tol = rs * (8 * U * (g.abs() + c1.abs() + (xh * c2).abs()) + 72 * U * (g.abs().mean(1, keepdim=True) +
                xh.abs() * (g * xh).abs().mean(1, keepdim=True)))
    tol += rs * (dxh * c2.abs() + xh.abs() * (g.abs() * dxh).mean(1, keepdim=True))
    assert within(dx, rs * (g - c1 - xh * c2), tol)
    chain = (-(-T // (148 * max(1, 8 // -(-X.shape[1] // 512)))) + 48) * U
    assert chain * T < 0.25                                       # a row too few or too many would show
    assert bool(((dgamma.double() - (D * xh).sum(0)).abs() <= chain * (D * xh).abs().sum(0) + (D.abs() * dxh).sum(0)).all())
    assert bool(((dbeta.double() - D.sum(0)).abs() <= chain * D.abs().sum(0)).all())


def checkpoint(x):
    """(data, scale) of the format, each step rounded to fp32."""
    T, H = x.shape
    n = -(-H // B.Q8_GROUP)
    p = torch.zeros(T, n * B.Q8_GROUP, device="cuda")
    p[:, :H] = x.float()
    p = p.view(T, n, B.Q8_GROUP)
    a = p.abs().amax(2, keepdim=True)
    one = torch.ones((), device="cuda")
    return torch.round(p * (127.0 * (one / a))).view(T, -1)[:, :H].to(torch.int8), (a * (one / 127.0))[:, :, 0]


@pytest.mark.parametrize("kind,xt,dt", TYPES)
@pytest.mark.parametrize("T,H", SHAPES)
def test_long_batches(T, H, kind, xt, dt):
    layer = kind == "layer"
    x, dy = data(T, H, DT[xt], T + H, 2.0, 0.5), data(T, H, DT[dt], 3)
    gamma, beta = 1 + 0.3 * data(1, H, torch.float32, 9)[0], (0.3 * data(1, H, torch.float32, 10)[0] if layer else None)
    new = lambda *n, dtype=torch.float32: torch.full(n, float("nan"), dtype=dtype, device="cuda")
    mean, rstd = new(T) if layer else None, new(T)
    y, c, status = new(T, H, dtype=DT[xt]), B.alloc_ckpt8(T, H), B.new_status()
    B.sapo_norm_fwd(x, gamma, beta, 1e-5, kind, y, mean, rstd)
    check_fwd(x, gamma, beta, 1e-5, layer, y, mean, rstd)
    kept = new(T, H, dtype=DT[xt])
    B.sapo_norm_fwd(x, gamma, beta, 1e-5, kind, kept, mean, rstd, c, status)
    assert torch.equal(kept, y) and status.item() == 0
    q, scale = checkpoint(x)
    assert torch.equal(c.data[:, :H], q) and torch.equal(c.scale, scale)
    stored, back = B.alloc_ckpt8(T, H), new(T, H, dtype=DT[xt])
    B.sapo_ckpt8_store(x, stored, status)
    assert torch.equal(stored.data[:, :H], q) and torch.equal(stored.scale, scale)
    B.sapo_ckpt8_restore(stored, back)
    value = q.double() * scale.double().repeat_interleave(B.Q8_GROUP, 1)[:, :H]
    assert within(back, value, U * value.abs())
    again = new(T, H)
    B.sapo_norm_replay(c, gamma, beta, kind, mean, rstd, again)
    M, rs, G = (mean.double()[:, None] if layer else 0.0), rstd.double()[:, None], gamma.double()
    want = (value - M) * rs * G + (beta.double() if layer else 0.0)
    off = value.abs() + (M.abs() if layer else 0.0)
    assert within(again, want, 4 * U * (off * rs * G.abs() + want.abs()))
    ws = torch.full((B.sapo_norm_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
    for source, X in ((x, x.double()), (c, value)):
        dx, dg, db = new(T, H, dtype=DT[xt]), new(H), new(H)
        B.sapo_norm_bwd(dy, source, gamma, mean, rstd, kind, dx, dg, db, ws)
        check_bwd(dy, X, gamma, mean, rstd, layer, dx, dg, db)


@pytest.mark.parametrize("H", [64, 200, 264, 896, 4096, 9000])
def test_weights_statistics_and_checkpoints_off_sixteen_bytes(H):
    """Arrays that start 4 bytes behind a 16-byte boundary (weights, statistics, scales), 8-bit rows on odd bytes, scales
    with a pitch of their own: other kernels, or other instructions, the same bounds."""
    T = 700
    x, dy = data(T, H, torch.bfloat16, H, 2.0, 0.5), data(T, H, torch.float32, 3)
    off = lambda n: torch.full((n + 1,), float("nan"), device="cuda")[1:]
    gamma, beta, mean, rstd = off(H), off(H), off(T), off(T)
    gamma.copy_(1 + 0.3 * data(1, H, torch.float32, 9)[0])
    beta.copy_(0.3 * data(1, H, torch.float32, 10)[0])
    n, status = -(-H // B.Q8_GROUP), B.new_status()
    for first in (0, 1):                                          # 8-bit rows on 16-byte boundaries, and on odd bytes
        q = torch.full((T, -(-H // 16) * 16 + 16), -128, dtype=torch.int8, device="cuda")
        s = torch.full((T, n + 3), float("nan"), device="cuda")
        c = B.Ckpt8(q[:, first:first + H], s[:, 1:1 + n], H)
        y, dx, dg, db = torch.empty_like(x), torch.empty_like(x), off(H), off(H)
        B.sapo_norm_fwd(x, gamma, beta, 1e-5, "layer", y, mean, rstd, c, status)
        check_fwd(x, gamma, beta, 1e-5, True, y, mean, rstd)
        data_, scale = checkpoint(x)
        assert torch.equal(c.data, data_) and torch.equal(c.scale, scale) and status.item() == 0
        assert (q[:, :first] == -128).all() and (q[:, first + H:] == -128).all()
        assert torch.isnan(s[:, 0]).all() and torch.isnan(s[:, 1 + n:]).all()
        ws = torch.full((B.sapo_norm_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
        value = data_.double() * scale.double().repeat_interleave(B.Q8_GROUP, 1)[:, :H]
        for source, X in ((x, x.double()), (c, value)):
            B.sapo_norm_bwd(dy, source, gamma, mean, rstd, "layer", dx, dg, db, ws)
            check_bwd(dy, X, gamma, mean, rstd, True, dx, dg, db)
