"""The norm in front of the LM head and 8-bit activation checkpoints on the device, against the
float64 oracle.

Bounds.  u = 2^-24 is the rounding of one fp32 operation.  A row's sums add at most 32 terms in a
thread, 5 in a warp's tree and 16 warps: 53 roundings, taken as 64.
  mean:  dm = 64 u mean|x|;  rstd: relative dr = 64 u (half of it would do: a square root), plus what
  dm adds to the variance, at most rstd^2 dm^2, plus 4 roundings;
  y:     |gamma| rstd (dm + 2 u |x - m|) + |xh gamma| dr + 2 u |y|
  dx:    rstd (8 u (|g| + |c1| + |xh c2|) + 72 u (mean|g| + |xh| mean|g xh|)) with c1 = mean g, c2 = mean g xh
  dgamma, dbeta: (T + 64) u sum_t |terms| (as if one thread added all rows), 4 more for xh.
An output in bf16 lies between the bf16 roundings of both ends of that interval."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from paper_2509_08721_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(T, H, dtype, ld=None, seed=0, scale=1.0, shift=0.0):
    """[T, H] with row pitch ld, NaN in the gaps: nothing between the rows may be read into a result."""
    g = torch.Generator().manual_seed(seed)
    full = torch.full((T, ld or H), float("nan"), dtype=dtype)
    full[:, :H] = (torch.randn(T, H, generator=g) * scale + shift).to(dtype)
    return full.cuda()[:, :H]


def within(got, want, tol):
    """Every element of `got` is the rounding, to its own type, of a value in want +- tol."""
    lo, hi = want - tol, want + tol
    if got.dtype == torch.bfloat16:
        lo, hi = (f64(torch.from_numpy(v).bfloat16()) for v in (lo, hi))
    v = f64(got)
    return bool(np.all((lo <= v) & (v <= hi)))


def check_fwd(x, gamma, beta, eps, kind, y, mean, rstd):
    X = f64(x)
    r = ho.norm_fwd(X, None if gamma is None else f64(gamma), None if beta is None else f64(beta), eps, kind)
    G = 1.0 if gamma is None else np.abs(f64(gamma))
    m, rs = r["mean"][:, None], r["rstd"][:, None]
    dm = 64 * U * np.abs(X).mean(1, keepdims=True) if kind == "layer" else np.zeros((X.shape[0], 1))
    dr = 68 * U + (rs * dm) ** 2
    xh = (X - m) * rs
    tol = G * rs * (dm + 2 * U * np.abs(X - m)) + np.abs(xh) * G * dr + 2 * U * np.abs(r["y"]) + 1e-37
    assert within(y, r["y"], tol)
    if mean is not None:
        assert np.all(np.abs(f64(mean) - r["mean"]) <= dm[:, 0] + 1e-37)
    if rstd is not None:
        assert np.all(np.abs(f64(rstd) - r["rstd"]) <= (r["rstd"] * dr[:, 0]))


def check_bwd(dy, X, gamma, mean, rstd, kind, dx, dgamma, dbeta, base=(None, None)):
    """X: float64 values that the backward reads."""
    M = np.zeros(X.shape[0]) if mean is None else f64(mean)
    r = ho.norm_bwd(f64(dy), X, None if gamma is None else f64(gamma), M, f64(rstd), kind)
    g, xh, rs, T = r["g"], r["xh"], f64(rstd)[:, None], X.shape[0]
    c1 = np.abs(g.mean(1, keepdims=True)) if kind == "layer" else 0.0
    c2 = np.abs((g * xh).mean(1, keepdims=True))
    tol = rs * (8 * U * (np.abs(g) + c1 + np.abs(xh) * c2) + 72 * U * (np.abs(g).mean(1, keepdims=True) +
                np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True))) + 1e-37
    # xh itself: the difference x - mean and one product, a few roundings of values as large as x
    dxh = 3 * U * (np.abs(X) + np.abs(M[:, None])) * rs
    tol = tol + rs * (dxh * c2 + np.abs(xh) * (np.abs(g) * dxh).mean(1, keepdims=True))
    assert within(dx, r["dx"], tol)
    D = np.abs(f64(dy))
    if dgamma is not None:
        add = 0.0 if base[0] is None else f64(base[0])
        assert np.all(np.abs(f64(dgamma) - (r["dgamma"] + add)) <= (T + 68) * U * (D * np.abs(xh)).sum(0) + (D * dxh).sum(0) + 2 * U * np.abs(add) + 1e-37)
    if dbeta is not None:
        add = 0.0 if base[1] is None else f64(base[1])
        assert np.all(np.abs(f64(dbeta) - (r["dbeta"] + add)) <= (T + 68) * U * D.sum(0) + 2 * U * np.abs(add) + 1e-37)


def weights(H, kind, wt, affine=True):
    g = torch.Generator().manual_seed(9)
    if not affine:
        return None, None
    gamma = (1 + 0.3 * torch.randn(H, generator=g)).to(wt).cuda()
    return gamma, ((0.3 * torch.randn(H, generator=g)).to(wt).cuda() if kind == "layer" else None)


def stats(T, kind):
    return (torch.full((T,), float("nan"), device="cuda") if kind == "layer" else None,
            torch.full((T,), float("nan"), device="cuda"))


# (T, H, extra columns of pitch): one column to the widest row, odd widths, pitches on and off 16 bytes
SHAPES = [(1, 1, 0), (1, 896, 0), (3, 7, 0), (5, 17, 3), (29, 64, 0), (33, 128, 8), (9, 130, 0), (40, 328, 8), (4, 1000, 0),
          (700, 896, 0), (6, 1001, 0), (9, 1536, 16), (7, 3584, 0), (5, 4104, 1), (3, 8200, 0), (2, 16384, 0), (3, 16383, 5)]
TYPES = [("layer", "bf16", "bf16", "f32"), ("rms", "f32", "f32", "bf16"), ("layer", "f32", "bf16", "bf16"), ("rms", "bf16", "f32", "f32")]


@pytest.mark.parametrize("kind,xt,yt,wt", TYPES)
@pytest.mark.parametrize("T,H,pad", SHAPES)
def test_norm_forward_and_backward(T, H, pad, kind, xt, yt, wt):
    """yt is the type of y, of dy and (mixed with x's) of dx."""
    x = rows(T, H, DT[xt], H + pad, seed=T + H, scale=2.0, shift=0.5)
    gamma, beta = weights(H, kind, DT[wt])
    mean, rstd = stats(T, kind)
    y = rows(T, H, DT[yt], H + pad)
    B.sapo_norm_fwd(x, gamma, beta, 1e-5, kind, y, mean, rstd)
    check_fwd(x, gamma, beta, 1e-5, kind, y, mean, rstd)
    if pad:
        assert torch.isnan(y._base[:, H:].float()).all()              # the gap between the rows is left alone
    dy = rows(T, H, DT[yt], H + pad, seed=3)
    dx = rows(T, H, DT[xt], H + pad)
    dg, db = torch.full((H,), float("nan"), device="cuda"), torch.full((H,), float("nan"), device="cuda")
    ws = torch.full((B.sapo_norm_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
    B.sapo_norm_bwd(dy, x, gamma, mean, rstd, kind, dx, dg, db, ws)
    check_bwd(dy, f64(x), gamma, mean, rstd, kind, dx, dg, db)
    if pad:
        assert torch.isnan(dx._base[:, H:].float()).all()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("T,H", [(1, 64), (1000, 200), (2500, 896), (4097, 72)])
def test_norm_backward_accumulates_aliases_and_repeats(kind, T, H):
    x, dy = rows(T, H, torch.bfloat16, seed=1), rows(T, H, torch.float32, seed=2)
    gamma, beta = weights(H, kind, torch.float32)
    mean, rstd = stats(T, kind)
    y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    B.sapo_norm_fwd(x, gamma, beta, 1e-6, kind, y, mean, rstd)
    ws = torch.empty(B.sapo_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    base = [torch.randn(H, device="cuda") * 10, torch.randn(H, device="cuda") * 10]
    got = [b.clone() for b in base]
    inplace = dy.clone()
    B.sapo_norm_bwd(inplace, x, gamma, mean, rstd, kind, inplace, got[0], got[1], ws, accumulate=True)
    check_bwd(dy, f64(x), gamma, mean, rstd, kind, inplace, got[0], got[1], base)
    # the same inputs give the same bits, whatever else ran before; each weight gradient may be left out
    first = None
    for _ in range(3):
        ws.fill_(0xFF)
        dx, dg = torch.empty_like(dy), torch.empty(H, device="cuda")
        B.sapo_norm_bwd(dy, x, gamma, mean, rstd, kind, dx, dg, None, ws)
        first = first or (dx, dg)
        assert torch.equal(dx, first[0]) and torch.equal(dg, first[1])
    dx2 = torch.empty_like(dy)
    B.sapo_norm_bwd(dy, x, gamma, mean, rstd, kind, dx2, None, None, None)
    assert torch.equal(dx2, first[0])
    # y may be x
    B.sapo_norm_fwd(x, gamma, beta, 1e-6, kind, x, None, None)
    assert torch.equal(x, y)


def test_norm_without_weights_constant_rows_and_large_offsets():
    T, H = 6, 256
    x = rows(T, H, torch.float32, seed=4)
    x[1] = 3.25                                                       # no variance: rstd = eps^-1/2, y = 0
    x[2] += 1000.0                                                    # two passes: the offset costs dm, not the variance
    x[3] = 0.0
    x[4] *= 1e-20
    mean, rstd = stats(T, "layer")
    y = torch.empty_like(x)
    B.sapo_norm_fwd(x, None, None, 1e-5, "layer", y, mean, rstd)
    check_fwd(x, None, None, 1e-5, "layer", y, mean, rstd)
    assert (y[1] == 0).all() and (y[3] == 0).all()
    dy, dx = rows(T, H, torch.float32, seed=5), torch.empty_like(x)
    B.sapo_norm_bwd(dy, x, None, mean, rstd, "layer", dx, None, None, None)
    check_bwd(dy, f64(x), None, mean, rstd, "layer", dx, None, None)


def test_a_row_that_is_not_finite_spoils_no_other_row():
    T, H = 9, 896
    x = rows(T, H, torch.bfloat16, seed=6)
    ref, y = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = stats(T, "layer")
    B.sapo_norm_fwd(x, None, None, 1e-5, "layer", ref, mean, rstd)
    bad = x.clone()
    bad[3, 5], bad[7, 890] = float("nan"), float("inf")
    B.sapo_norm_fwd(bad, None, None, 1e-5, "layer", y, mean, rstd)
    ok = [t for t in range(T) if t not in (3, 7)]
    assert torch.equal(y[ok], ref[ok]) and torch.isnan(y[3].float()).all() and torch.isnan(y[7].float()).all()


def test_empty_batch():
    H = 64
    x = torch.empty(0, H, dtype=torch.bfloat16, device="cuda")
    e = torch.empty(0, device="cuda")
    B.sapo_norm_fwd(x, None, None, 1e-5, "layer", x.clone(), e, e)
    dg, db = torch.ones(H, device="cuda"), torch.ones(H, device="cuda")
    B.sapo_norm_bwd(x, x, None, e, e, "layer", x.clone(), dg, db, None, accumulate=True)
    assert (dg == 1).all()
    B.sapo_norm_bwd(x, x, None, e, e, "layer", x.clone(), dg, db, None)
    assert not dg.any() and not db.any()
    c = B.alloc_ckpt8(0, H)
    B.sapo_ckpt8_store(x, c, B.new_status())
    B.sapo_ckpt8_restore(c, x)


# ------------------------------------------------------------------------------------------ 8 bits
@pytest.mark.parametrize("xt", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,pad", SHAPES)
def test_ckpt8_store_is_exact_and_restores(T, H, pad, xt):
    x = rows(T, H, DT[xt], H + pad, seed=T * 7 + H, scale=3.0)
    if T > 2:
        x[1] = 0
        x[2, : max(1, H // 2)] *= 1e-37 if xt == "f32" else 0.5
    c, status = B.alloc_ckpt8(T, H), B.new_status()
    if pad:
        c = B.Ckpt8(torch.empty(T, H + pad, dtype=torch.int8, device="cuda"), c.scale, H)
    c.data.fill_(-128)
    B.sapo_ckpt8_store(x, c, status)
    data, scale = ho.ckpt8_store(f64(x).astype(np.float32))
    assert np.array_equal(c.data[:, :H].cpu().numpy(), data)
    assert np.array_equal(c.scale.cpu().numpy(), scale)
    if c.data.shape[1] > H:
        assert (c.data[:, H:] == -128).all()
    back = rows(T, H, DT[xt], H + pad)
    B.sapo_ckpt8_restore(c, back)
    v = ho.ckpt8_values(data, scale)
    assert within(back, v, U * np.abs(v) + 1e-45)
    assert status.item() == 0


def test_ckpt8_groups_that_are_not_finite():
    x = rows(4, 300, torch.float32, seed=8)
    x[1, 130], x[2, 299] = float("-inf"), float("nan")
    c, status = B.alloc_ckpt8(4, 300), B.new_status()
    B.sapo_ckpt8_store(x, c, status)
    assert B.decode_status(status.item()) == ["NONFINITE_INPUT"]
    data, scale = ho.ckpt8_store(f64(x).astype(np.float32))
    assert np.array_equal(c.data[:, :300].cpu().numpy(), data)
    assert np.array_equal(c.scale.cpu().numpy(), scale, equal_nan=True)
    back = torch.empty_like(x)
    B.sapo_ckpt8_restore(c, back)
    assert torch.isnan(back[1, 128:256]).all() and torch.isnan(back[2, 256:]).all() and torch.isfinite(back[[0, 3]]).all()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("T,H,pad", [(1, 896, 0), (37, 64, 0), (300, 1000, 0), (21, 1001, 0), (70, 1536, 8), (5, 3584, 0), (3, 9000, 0)])
def test_norm_training_pass_on_a_checkpoint(T, H, pad, kind):
    """The forward's checkpoint equals the stored one bit for bit and changes nothing else; the replay
    and the backward read exactly the values it stands for."""
    x = rows(T, H, torch.bfloat16, H + pad, seed=T + H, shift=0.3)
    gamma, beta = weights(H, kind, torch.float32)
    mean, rstd = stats(T, kind)
    y, y0 = torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    c, c2, status = B.alloc_ckpt8(T, H), B.alloc_ckpt8(T, H), B.new_status()
    B.sapo_norm_fwd(x, gamma, beta, 1e-5, kind, y, mean, rstd, c, status)
    B.sapo_norm_fwd(x, gamma, beta, 1e-5, kind, y0, None, None)
    B.sapo_ckpt8_store(x, c2, status)
    assert torch.equal(y, y0) and torch.equal(c.data[:, :H], c2.data[:, :H]) and torch.equal(c.scale, c2.scale)
    assert status.item() == 0
    X = ho.ckpt8_values(c.data[:, :H].cpu().numpy(), c.scale.cpu().numpy())
    # replay: the values, minus the stored mean, times the stored rstd
    again = torch.empty(T, H, device="cuda")
    B.sapo_norm_replay(c, gamma, beta, kind, mean, rstd, again)
    M = np.zeros(T) if mean is None else f64(mean)
    want = ho.norm_apply(X, M, f64(rstd), f64(gamma), None if beta is None else f64(beta))
    tol = 4 * U * ((np.abs(X) + np.abs(M)[:, None]) * f64(rstd)[:, None] * np.abs(f64(gamma)) + np.abs(want))
    assert np.all(np.abs(f64(again) - want) <= tol)
    dy = rows(T, H, torch.float32, H + pad, seed=11)
    dx, dg, db = torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    ws = torch.full((B.sapo_norm_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
    B.sapo_norm_bwd(dy, c, gamma, mean, rstd, kind, dx, dg, db, ws)
    check_bwd(dy, X, gamma, mean, rstd, kind, dx, dg, db)


def test_rows_beyond_two_to_the_31_elements():
    """Offsets that need 64 bits: 2.2e9 elements, only the last rows are not zero."""
    T, H = 620_000, 3584
    assert T * H > 2 ** 31
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    x[-3:] = rows(3, H, torch.bfloat16, seed=12)
    c, status = B.alloc_ckpt8(T, H), B.new_status()
    mean, rstd = stats(T, "layer")
    y = torch.empty_like(x)
    B.sapo_norm_fwd(x, None, None, 1e-5, "layer", y, mean, rstd, c, status)
    check_fwd(x[-5:], None, None, 1e-5, "layer", y[-5:], mean[-5:], rstd[-5:])
    assert not y[:-3].any()
    data, scale = ho.ckpt8_store(f64(x[-4:]).astype(np.float32))
    assert np.array_equal(c.data[-4:].cpu().numpy(), data) and np.array_equal(c.scale[-4:].cpu().numpy(), scale)
    dg, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    ws = torch.empty(B.sapo_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    B.sapo_norm_bwd(y, c, None, mean, rstd, "layer", y, dg, db, ws)          # dy = y, in place
    ref = torch.empty(5, H, dtype=torch.bfloat16, device="cuda")
    B.sapo_norm_fwd(x[-5:], None, None, 1e-5, "layer", ref, None, None)
    check_bwd(ref, ho.ckpt8_values(c.data[-5:].cpu().numpy(), c.scale[-5:].cpu().numpy()), None, mean[-5:], rstd[-5:],
              "layer", y[-5:], None, None)
    B.sapo_ckpt8_restore(c, x)
    assert not x[:-3].any() and status.item() == 0


def test_on_a_stream_of_its_own_and_small_workspace():
    T, H = 5000, 896
    x, dy = rows(T, H, torch.bfloat16, seed=1), rows(T, H, torch.bfloat16, seed=2)
    want = None
    for st in (torch.cuda.current_stream(), torch.cuda.Stream()):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            mean, rstd = stats(T, "layer")
            y, dx = torch.empty_like(x), torch.empty_like(x)
            dg, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
            ws = torch.empty(B.sapo_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
            B.sapo_norm_fwd(x, None, None, 1e-5, "layer", y, mean, rstd)
            B.sapo_norm_bwd(dy, x, None, mean, rstd, "layer", dx, dg, db, ws)
        st.synchronize()
        want = want or (y, dx, dg, db)
        for a, b in zip(want, (y, dx, dg, db)):
            assert torch.equal(a, b)
    with pytest.raises(B.SapoError, match="workspace"):
        B.sapo_norm_bwd(dy, x, None, mean, rstd, "layer", dx, dg, db, ws[:64])
    with pytest.raises(B.SapoError):
        B.sapo_norm_bwd(dy, x, None, mean, rstd, "layer", dx, dg, db, None)


def test_binding_refuses_wrong_shapes_and_types():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    m = torch.zeros(4, device="cuda")
    y = torch.empty_like(x)
    for call in (lambda: B.sapo_norm_fwd(x.half(), None, None, 1e-5, "layer", y, m, m),
                 lambda: B.sapo_norm_fwd(x, None, None, 1e-5, "batch", y, m, m),
                 lambda: B.sapo_norm_fwd(x, torch.zeros(63, device="cuda"), None, 1e-5, "layer", y, m, m),
                 lambda: B.sapo_norm_fwd(x, None, None, 1e-5, "layer", y[:3], m, m),
                 lambda: B.sapo_norm_fwd(x, None, None, 1e-5, "layer", y, m.double(), m),
                 lambda: B.sapo_norm_fwd(x.t(), None, None, 1e-5, "layer", y.t(), None, None),
                 lambda: B.sapo_norm_fwd(x, m.new_zeros(64), m.new_zeros(64).bfloat16(), 1e-5, "layer", y, m, m),
                 lambda: B.sapo_norm_fwd(x, None, None, 1e-5, "layer", y, m, m, B.alloc_ckpt8(4, 63), B.new_status()),
                 lambda: B.sapo_norm_bwd(x, B.alloc_ckpt8(3, 64), None, m, m, "layer", y, None, None, None),
                 lambda: B.sapo_norm_replay(B.alloc_ckpt8(4, 32), None, None, "rms", None, m, y)):
        with pytest.raises(B.SapoError):
            call()


def test_captured_calls_replay():
    """Norm forward with a checkpoint, replay and backward in a graph, on new inputs: the results of direct calls, bit for bit."""
    data = []
    for T, H, kind in [(1, 8, "rms"), (37, 1001, "layer"), (500, 896, "rms")]:
        x = torch.randn(T, H, device="cuda").bfloat16()
        e = lambda *s: torch.empty(*s, device="cuda")
        data.append(dict(x=x, dy=torch.randn(T, H, device="cuda"), gamma=torch.randn(H, device="cuda"), kind=kind,
                         y=torch.empty_like(x), back=torch.empty_like(x), mean=e(T) if kind == "layer" else None, rstd=e(T),
                         ckpt=B.alloc_ckpt8(T, H), dx=e(T, H), dgamma=e(H), dbeta=e(H),
                         ws=torch.empty(B.sapo_norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")))
    status = B.new_status()
    outputs = ("y", "back", "dx", "dgamma", "dbeta")

    def calls():
        for d in data:
            B.sapo_norm_fwd(d["x"], d["gamma"], None, 1e-6, d["kind"], d["y"], d["mean"], d["rstd"], d["ckpt"], status)
            B.sapo_ckpt8_restore(d["ckpt"], d["back"])
            B.sapo_norm_bwd(d["dy"], d["ckpt"], d["gamma"], d["mean"], d["rstd"], d["kind"], d["dx"], d["dgamma"],
                            d["dbeta"], d["ws"])

    def results():
        torch.cuda.synchronize()
        return [d[k].clone() for d in data for k in outputs]

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(2):
        for d in data:
            d["x"].copy_(torch.randn(d["x"].shape, device="cuda"))
        calls()
        want = results()
        for d in data:
            for k in outputs:
                d[k].zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, results())) and status.item() == 0
