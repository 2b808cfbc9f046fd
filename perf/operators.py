"""Cases of the operators around the LM head: the norm in front of it (forward, backward), 8-bit activation
checkpoints and their use in the backward pass, and the preference loss (on per-token log-probs, and
through the head).

With own = False every operator is computed in its plain form: elementary torch operations in 32 bits,
rounded once at the end.  With own = True the calls are those of the package's binding."""
import math

import torch

own = False

GROUP = 128          # columns that share one scale of an 8-bit checkpoint
TINY = 2.0 ** -119   # a group whose largest magnitude is below this is stored as zero
EPS = 1e-6


def _types(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the final norm of one decoded token: launch latency is all there is
        {"name": "norm_fwd one token", "op": "norm_fwd", "T": 1, "H": 896, "kind": "rms", "x": "bf16", "y": "bf16"},
        # the final norm of a whole packed batch of 256 completions at hidden 1536
        {"name": "norm_fwd batch", "op": "norm_fwd", "T": 146382, "H": 1536, "kind": "layer", "x": "bf16", "y": "bf16"},
        # a tiny fp32 model under test: one ragged handful of tokens
        {"name": "norm_bwd tiny f32", "op": "norm_bwd", "T": 29, "H": 64, "kind": "layer", "x": "f32", "dy": "f32"},
        # a batch of 64 completions at hidden 896, gradient in fp32 as the loss call returns it by default
        {"name": "norm_bwd batch", "op": "norm_bwd", "T": 16527, "H": 896, "kind": "rms", "x": "bf16", "dy": "f32"},
        # 256 long completions at hidden 3584, bf16 throughout
        {"name": "norm_bwd wide", "op": "norm_bwd", "T": 143347, "H": 3584, "kind": "layer", "x": "bf16", "dy": "bf16"},
        # an activation kept in 8 bits between forward and backward, and brought back
        {"name": "ckpt8 batch", "op": "ckpt8", "T": 16527, "H": 896, "x": "bf16"},
        # the norm's training pass with its input kept in 8 bits: forward stores, backward reads it in place
        {"name": "ckpt8 norm training", "op": "norm_ckpt8", "T": 65537, "H": 1536, "kind": "layer", "x": "bf16",
         "dy": "bf16"},
        # 4 questions x 8 completions of 32 tokens
        {"name": "pref tiny", "op": "pref", "Q": 4, "G": 8, "lo": 32, "hi": 32, "loss": "sigmoid", "pairs": "all"},
        # 64 questions x 8 completions of 256 to 1024 tokens, all pairs of a question
        {"name": "pref batch", "op": "pref", "Q": 64, "G": 8, "lo": 256, "hi": 1024, "loss": "sigmoid", "pairs": "all"},
        # classic pairs of very long completions: few rows, a long axis
        {"name": "pref long", "op": "pref", "Q": 2, "G": 2, "lo": 40000, "hi": 65000, "loss": "squared", "pairs": "best_worst"},
        # a small vocabulary: launches count as much as the contractions
        {"name": "pref_head small", "op": "pref_head", "Q": 4, "G": 8, "lo": 32, "hi": 32, "H": 64, "V": 1000,
         "loss": "sigmoid", "pairs": "all"},
        # chosen and rejected completions of 64 to 512 tokens at hidden 896 and the full vocabulary
        {"name": "pref_head batch", "op": "pref_head", "Q": 16, "G": 2, "lo": 64, "hi": 512, "H": 896, "V": 151936,
         "loss": "sigmoid", "pairs": "best_worst"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "ckpt8", "norm_ckpt8", "pref", "pref_head"])
    if op in ("norm_fwd", "norm_bwd", "ckpt8", "norm_ckpt8"):
        H = _log_int(rng, 33, 8192)
        if rng.random() < 0.7:                       # most models: a multiple of 8; the rest odd sizes
            H = -(-H // 8) * 8
        T = _log_int(rng, 1, max(1, min(262144, int(2.0e8 / H))))
        c = {"op": op, "T": T, "H": H, "x": rng.choice(["bf16", "bf16", "f32"])}
        if op != "ckpt8":
            c["kind"] = rng.choice(["layer", "rms"])
        if op == "norm_fwd":
            c["y"] = c["x"]
        if op in ("norm_bwd", "norm_ckpt8"):
            c["dy"] = rng.choice(["bf16", "f32"])
        return c
    loss = rng.choice(["sigmoid", "sigmoid", "squared", "hinge"])
    pairs = rng.choice(["all", "best_worst"])
    if op == "pref":
        Q = _log_int(rng, 1, 512)
        G = rng.randint(2, 16)
        hi = _log_int(rng, 8, max(8, min(65536, int(4.0e6 / (Q * G)))))
        return {"op": op, "Q": Q, "G": G, "lo": max(1, hi // rng.randint(1, 8)), "hi": hi, "loss": loss, "pairs": pairs}
    H = 8 * _log_int(rng, 8, 192)
    V = _log_int(rng, 1000, 152064)
    Q, G = _log_int(rng, 1, 16), rng.randint(2, 8)
    most = min(12000.0, 5.0e12 / (6.0 * V * H), 1.2e9 / V)
    hi = _log_int(rng, 8, max(8, min(512, int(most / (Q * G)))))
    return {"op": op, "Q": Q, "G": G, "lo": max(1, hi // rng.randint(1, 8)), "hi": hi, "H": H, "V": V, "loss": loss,
            "pairs": pairs}


# ------------------------------------------------------------------------------------------ inputs
def _lengths(case, gen):
    """Ragged lengths between lo and hi that add up to the same total for every seed: half of them are
    drawn, the other half mirrored, all in random order."""
    n, lo, hi = case["Q"] * case["G"], case["lo"], case["hi"]
    a = torch.randint(lo, hi + 1, (n // 2,), generator=gen)
    L = torch.cat([a, lo + hi - a, torch.full((n % 2,), (lo + hi) // 2)])[torch.randperm(n, generator=gen)]
    cu = torch.zeros(n + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(L, 0)
    return L, cu


def _activation(T, H, g, dtype):
    """A residual stream: unit variance, a slow offset, a few channels twenty times as large."""
    x = torch.randn(T, H, generator=g, device="cuda")
    x.mul_(torch.where(torch.rand(H, generator=g, device="cuda") < 0.01, 20.0, 1.0))
    x.add_(0.25 * torch.randn(H, generator=g, device="cuda"))
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op = case["op"]
    s = {"case": case, "op": op}
    if op in ("norm_fwd", "norm_bwd", "ckpt8", "norm_ckpt8"):
        T, H = case["T"], case["H"]
        xt = _types(case["x"])
        s["x"] = _activation(T, H, g, xt)
        if op == "ckpt8":
            s["back"] = torch.empty(T, H, dtype=xt, device="cuda")
        else:
            s["gamma"] = 1.0 + 0.1 * torch.randn(H, generator=g, device="cuda")
            s["beta"] = 0.1 * torch.randn(H, generator=g, device="cuda") if case["kind"] == "layer" else None
            s["mean"] = torch.empty(T, device="cuda") if case["kind"] == "layer" else None
            s["rstd"] = torch.empty(T, device="cuda")
        if op in ("norm_bwd", "norm_ckpt8"):
            s["dy"] = (1e-3 * torch.randn(T, H, generator=g, device="cuda")).to(_types(case["dy"]))
            s["dx"] = torch.empty(T, H, dtype=xt, device="cuda")
            s["dgamma"] = torch.empty(H, device="cuda")
            s["dbeta"] = torch.empty(H, device="cuda") if case["kind"] == "layer" else None
        if op in ("norm_fwd", "norm_ckpt8"):
            s["y"] = torch.empty(T, H, dtype=_types(case.get("y", case["x"])), device="cuda")
        if op == "norm_bwd":       # the forward has left its statistics
            step = max(1, (1 << 27) // H)
            for a in range(0, T, step):
                xs = s["x"][a:a + step].float()
                if case["kind"] == "layer":
                    s["mean"][a:a + step] = xs.mean(1)
                    xs = xs - s["mean"][a:a + step, None]
                s["rstd"][a:a + step] = torch.rsqrt(xs.square().mean(1) + EPS)
    else:
        host = torch.Generator()
        host.manual_seed(int(seed))
        L, cu = _lengths(case, host)
        T, Q, G = int(cu[-1]), case["Q"], case["G"]
        S = Q * G
        s["T"], s["S"] = T, S
        s["cu"] = cu.cuda()
        s["seq"] = torch.repeat_interleave(torch.arange(S), L).cuda()      # sequence of each token
        s["go"] = torch.arange(0, S + 1, G, dtype=torch.int32).cuda()
        # a graded reward with ties, as rule-checked answers get
        s["rewards"] = (torch.randint(0, 5, (S,), generator=host).float() / 4).cuda()
        if op == "pref":
            s["ref"] = 1.5 * torch.log(torch.rand(T, generator=g, device="cuda") + 1e-3)
            s["logp"] = s["ref"] + 0.2 * torch.randn(T, generator=g, device="cuda")
        else:
            H, V = case["H"], case["V"]
            s["hidden"] = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
            s["W"] = (0.02 * torch.randn(V, H, generator=g, device="cuda")).to(torch.bfloat16)
            s["ids"] = torch.randint(0, V, (T,), generator=g, device="cuda").to(torch.int32)
            ref = torch.empty(T, device="cuda")
            for a in range(0, T, 2048):              # a reference policy a few updates away
                z = (s["hidden"][a:a + 2048] @ s["W"].T).float()
                ref[a:a + 2048] = z.gather(1, s["ids"][a:a + 2048].long()[:, None])[:, 0] - torch.logsumexp(z, 1)
            s["ref"] = ref + 0.2 * torch.randn(T, generator=g, device="cuda")
            s["dhidden"] = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
            s["dW"] = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
    if own:
        _plan(s)
    return s


def _plan(s):
    """The buffers and the scratch that a program keeps for its calls."""
    from paper_2509_08721_b200 import binding as B
    op, case = s["op"], s["case"]
    s["status"] = B.new_status()
    if op in ("ckpt8", "norm_ckpt8"):
        s["ckpt"] = B.alloc_ckpt8(case["T"], case["H"])
    if op in ("norm_bwd", "norm_ckpt8"):
        s["ws"] = torch.empty(B.sapo_norm_workspace_bytes(case["T"], case["H"]), dtype=torch.uint8, device="cuda")
    if op in ("pref", "pref_head"):
        s["out"] = B.alloc_preference_outputs(s["T"], s["S"], case["Q"], scores=op == "pref_head")
    if op == "pref_head":
        n = B.sapo_workspace_bytes(B.WS_PREFERENCE | B.WS_OUT_BF16, s["T"], case["H"], case["V"], B.DTYPE_BF16)
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")


BETA = 0.1


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2509_08721_b200 import binding as B
    op, case = s["op"], s["case"]
    if op == "norm_fwd":
        B.sapo_norm_fwd(s["x"], s["gamma"], s["beta"], EPS, case["kind"], s["y"], s["mean"], s["rstd"])
        return _named(s, "y", "mean", "rstd")
    if op == "norm_bwd":
        B.sapo_norm_bwd(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], case["kind"], s["dx"], s["dgamma"],
                        s["dbeta"], s["ws"])
        return _named(s, "dx", "dgamma", "dbeta")
    if op == "ckpt8":
        B.sapo_ckpt8_store(s["x"], s["ckpt"], s["status"])
        B.sapo_ckpt8_restore(s["ckpt"], s["back"])
        return {"back": s["back"], "scale": s["ckpt"].scale}
    if op == "norm_ckpt8":
        B.sapo_norm_fwd(s["x"], s["gamma"], s["beta"], EPS, case["kind"], s["y"], s["mean"], s["rstd"], s["ckpt"],
                        s["status"])
        B.sapo_norm_bwd(s["dy"], s["ckpt"], s["gamma"], s["mean"], s["rstd"], case["kind"], s["dx"], s["dgamma"],
                        s["dbeta"], s["ws"])
        return _named(s, "y", "mean", "rstd", "dx", "dgamma", "dbeta")
    out = s["out"]
    if op == "pref":
        B.sapo_preference_loss(s["logp"], s["ref"], s["cu"], s["rewards"], s["go"], BETA, out, s["status"],
                               kind=case["loss"], pairs=case["pairs"])
        return {k: out[k] for k in ("loss", "gscale", "seq_logratio", "seq_grad", "q_loss", "q_margin", "q_pairs")}
    B.sapo_preference_loss_fwd_bwd(s["hidden"], s["W"], s["ids"], s["ref"], s["cu"], s["rewards"], s["go"], BETA, out,
                                   s["dhidden"], s["dW"], False, s["ws"], s["status"], kind=case["loss"],
                                   pairs=case["pairs"])
    r = {k: out[k] for k in ("loss", "logp", "lse", "gscale", "seq_logratio", "seq_grad", "q_loss", "q_margin",
                             "q_pairs")}
    r["dhidden"], r["dW"] = s["dhidden"], s["dW"]
    return r


def _named(s, *names):
    return {n: s[n] for n in names if s[n] is not None}


def _norm_plain(x, gamma, beta, layer):
    mean = x.mean(1) if layer else None
    xc = x - mean[:, None] if layer else x
    rstd = torch.rsqrt(xc.square().mean(1) + EPS)
    y = xc * rstd[:, None] * gamma
    return (y + beta if beta is not None else y), mean, rstd


def _norm_bwd_plain(dy, x, gamma, mean, rstd):
    xh = (x - mean[:, None] if mean is not None else x) * rstd[:, None]
    g = dy * gamma
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if mean is not None:
        dx = dx - g.mean(1, keepdim=True)
    return dx * rstd[:, None], (dy * xh).sum(0), dy.sum(0)


def _ckpt8_plain(x):
    """(values the 8-bit checkpoint stands for, scales)"""
    T, H = x.shape
    n = -(-H // GROUP)
    p = torch.zeros(T, n * GROUP, dtype=x.dtype, device=x.device)
    p[:, :H] = x
    p = p.view(T, n, GROUP)
    a = p.abs().amax(2, keepdim=True)
    big = a >= TINY
    inv = torch.where(big, 127.0 / a, torch.zeros_like(a))
    scale = torch.where(big, a / 127.0, torch.zeros_like(a))
    return (torch.round(p * inv) * scale).view(T, n * GROUP)[:, :H], scale[:, :, 0]


def _pairs(case, rewards):
    """[Q, G, G]: 1 where completion i of a question is preferred to its completion j"""
    r = rewards.view(case["Q"], case["G"])
    P = r[:, :, None] > r[:, None, :]
    if case["pairs"] == "best_worst":
        k = torch.arange(case["G"], device=r.device)
        best = (r == r.amax(1, keepdim=True))
        worst = (r == r.amin(1, keepdim=True))
        first = lambda m: torch.where(m, k, case["G"]).amin(1, keepdim=True) == k
        P = P & first(best)[:, :, None] & first(worst)[:, None, :]
    return P


def _pref_plain(case, d, seq, cu, T, S, rewards):
    """d: log ratio of each token; everything that follows from the log ratios"""
    Q, G = case["Q"], case["G"]
    longest = case["hi"]                             # the ragged rows side by side, zeros behind their ends
    at = seq * longest + torch.arange(T, device=d.device) - cu.long()[seq]
    R = torch.zeros(S * longest, dtype=d.dtype, device=d.device).scatter_(0, at, d).view(S, longest).sum(1)
    P = _pairs(case, rewards).to(d.dtype)
    Rq = R.view(Q, G)
    delta = Rq[:, :, None] - Rq[:, None, :]
    h = BETA * delta
    if case["loss"] == "sigmoid":
        e = torch.exp(-h.abs())
        l = torch.clamp(-h, min=0) + torch.log1p(e)
        dl = -torch.where(h > 0, e, torch.ones_like(e)) / (1 + e) * BETA
    elif case["loss"] == "squared":
        u = delta - 1 / (2 * BETA)
        l, dl = u * u, 2 * u
    else:
        l = torch.clamp(1 - h, min=0)
        dl = torch.where(h < 1, -BETA * torch.ones_like(h), torch.zeros_like(h))
    n = P.sum((1, 2))
    per = torch.clamp(n, min=1)
    q_loss = (P * l).sum((1, 2)) / per
    q_margin = (P * h).sum((1, 2)) / per
    f = P * dl
    grad = (f.sum(2) - f.sum(1)) / (Q * per[:, None])
    grad = grad.reshape(S)
    return {"loss": (q_loss.sum() / Q).view(1), "gscale": grad[seq], "seq_logratio": R, "seq_grad": grad, "q_loss": q_loss,
            "q_margin": q_margin, "q_pairs": n.to(torch.int32)}


def _head_plain(hidden, W, ids):
    z = hidden @ W.T
    m = z.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))[:, 0]
    zy = torch.gather(z, 1, ids.long()[:, None])[:, 0]
    return z, lse, zy - lse


def _head_bwd_plain(z, lse, g, ids, hidden, W):
    dz = torch.exp(z - lse[:, None]).mul_(-g[:, None])
    dz[torch.arange(len(ids), device=ids.device), ids.long()] += g
    return dz @ W, dz.T @ hidden


def _run_plain(s):
    op, case = s["op"], s["case"]
    if op == "norm_fwd":
        y, mean, rstd = _norm_plain(s["x"].float(), s["gamma"], s["beta"], case["kind"] == "layer")
        return _only({"y": y.to(s["y"].dtype), "mean": mean, "rstd": rstd})
    if op == "norm_bwd":
        dx, dgamma, dbeta = _norm_bwd_plain(s["dy"].float(), s["x"].float(), s["gamma"], s["mean"], s["rstd"])
        return _only({"dx": dx.to(s["dx"].dtype), "dgamma": dgamma, "dbeta": dbeta if case["kind"] == "layer" else None})
    if op == "ckpt8":
        v, scale = _ckpt8_plain(s["x"].float())
        return {"back": v.to(s["back"].dtype), "scale": scale}
    if op == "norm_ckpt8":
        x = s["x"].float()
        y, mean, rstd = _norm_plain(x, s["gamma"], s["beta"], case["kind"] == "layer")
        dx, dgamma, dbeta = _norm_bwd_plain(s["dy"].float(), _ckpt8_plain(x)[0], s["gamma"], mean, rstd)
        return _only({"y": y.to(s["y"].dtype), "mean": mean, "rstd": rstd, "dx": dx.to(s["dx"].dtype), "dgamma": dgamma,
                      "dbeta": dbeta if case["kind"] == "layer" else None})
    if op == "pref":
        return _pref_plain(case, s["logp"] - s["ref"], s["seq"], s["cu"], s["T"], s["S"], s["rewards"])
    hidden, W = s["hidden"].float(), s["W"].float()
    z, lse, logp = _head_plain(hidden, W, s["ids"])
    r = _pref_plain(case, logp - s["ref"], s["seq"], s["cu"], s["T"], s["S"], s["rewards"])
    dh, dW = _head_bwd_plain(z, lse, r["gscale"], s["ids"], hidden, W)
    r.update(logp=logp, lse=lse, dhidden=dh.to(torch.bfloat16), dW=dW.to(torch.bfloat16))
    return r


def _only(d):
    return {k: v for k, v in d.items() if v is not None}


# ------------------------------------------------------------------------------------------ work
def work(case):
    size = {"bf16": 2, "f32": 4}
    op = case["op"]
    if op in ("norm_fwd", "norm_bwd", "ckpt8", "norm_ckpt8"):
        T, H = case["T"], case["H"]
        n, b = T * H, size[case["x"]]
        stats = 4 * T * (2 if case.get("kind") == "layer" else 1)
        weights = 4 * H * (2 if case.get("kind") == "layer" else 1)
        scales = 4 * T * -(-H // GROUP)
        if op == "norm_fwd":
            return {"bytes": n * (b + size[case["y"]]) + stats + weights, "flops": 7 * n}
        if op == "norm_bwd":
            return {"bytes": n * (b + size[case["dy"]] + b) + stats + 4 * H + weights, "flops": 13 * n}
        if op == "ckpt8":
            return {"bytes": n * (b + 1 + 1 + b) + 2 * scales, "flops": 4 * n}
        return {"bytes": n * (b + b + 1 + 1 + size[case["dy"]] + b) + 2 * scales + 2 * stats + 2 * weights + 4 * H,
                "flops": 24 * n}
    S = case["Q"] * case["G"]
    T = S * (case["lo"] + case["hi"]) / 2
    if op == "pref":
        return {"bytes": 12 * T + 20 * S + 16 * case["Q"], "flops": 3 * T}
    H, V = case["H"], case["V"]
    return {"bytes": 2 * (2 * T * H + 2 * V * H) + 20 * T + 20 * S, "flops": 6 * T * V * H}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm_fwd", "norm_bwd", "ckpt8", "norm_ckpt8"):
        return _exact_rows(case, s)
    d = (s["logp"].double() - s["ref"].double()) if op == "pref" else None
    if op == "pref_head":
        T, V = s["T"], case["V"]
        h, W, ids = s["hidden"].double(), s["W"].double(), s["ids"].long()
        step = max(1, (1 << 29) // V)
        lse, logp = torch.empty(T, dtype=torch.float64, device="cuda"), torch.empty(T, dtype=torch.float64, device="cuda")
        for a in range(0, T, step):
            z = h[a:a + step] @ W.T
            lse[a:a + step] = torch.logsumexp(z, 1)
            logp[a:a + step] = z.gather(1, ids[a:a + step, None])[:, 0] - lse[a:a + step]
        d = logp - s["ref"].double()
    r = _exact_pref(case, s, d)
    if op == "pref_head":
        dh, dW = torch.empty_like(h), torch.zeros_like(W)
        for a in range(0, T, step):
            g = r["gscale"][a:a + step, None]
            p = torch.exp(h[a:a + step] @ W.T - lse[a:a + step, None])
            one = torch.zeros_like(p).scatter_(1, ids[a:a + step, None], 1.0)
            dz = g * (one - p)
            dh[a:a + step] = dz @ W
            dW += dz.T @ h[a:a + step]
        r.update(logp=logp, lse=lse, dhidden=dh, dW=dW)
    return r


def _exact_pref(case, s, d):
    """Question by question on the host, pair by pair."""
    Q, G = case["Q"], case["G"]
    cu, d, rew = s["cu"].tolist(), d.cpu(), s["rewards"].cpu().tolist()
    R = [float(d[cu[i]:cu[i + 1]].sum()) for i in range(Q * G)]
    grad, q_loss, q_margin, q_pairs = [0.0] * (Q * G), [], [], []
    for q in range(Q):
        members = list(range(q * G, (q + 1) * G))
        if case["pairs"] == "best_worst":
            i = max(members, key=lambda k: (rew[k], -k))
            j = min(members, key=lambda k: (rew[k], k))
            pairs = [(i, j)] if rew[i] > rew[j] else []
        else:
            pairs = [(i, j) for i in members for j in members if rew[i] > rew[j]]
        total = margin = 0.0
        for i, j in pairs:
            D = R[i] - R[j]
            h = BETA * D
            if case["loss"] == "sigmoid":
                l = max(-h, 0.0) + math.log1p(math.exp(-abs(h)))
                dD = -BETA / (1 + math.exp(h)) if h < 700 else 0.0
            elif case["loss"] == "squared":
                l, dD = (D - 0.5 / BETA) ** 2, 2 * (D - 0.5 / BETA)
            else:
                l, dD = max(0.0, 1 - h), -BETA if h < 1 else 0.0
            total, margin = total + l, margin + h
            grad[i] += dD / (Q * len(pairs))
            grad[j] -= dD / (Q * len(pairs))
        n = max(1, len(pairs))
        q_loss.append(total / n)
        q_margin.append(margin / n)
        q_pairs.append(len(pairs))
    t = lambda v: torch.tensor(v, dtype=torch.float64, device="cuda")
    return {"loss": t([sum(q_loss) / Q]), "gscale": t(grad)[s["seq"]], "seq_logratio": t(R), "seq_grad": t(grad),
            "q_loss": t(q_loss), "q_margin": t(q_margin), "q_pairs": torch.tensor(q_pairs, dtype=torch.int32)}


def _exact_rows(case, s):
    """The row operators, a block of rows at a time."""
    op, T, H = case["op"], case["T"], case["H"]
    layer = case.get("kind") == "layer"
    new = lambda *n: torch.zeros(*n, dtype=torch.float64, device="cuda")
    small = {"mean": new(T), "rstd": new(T), "dgamma": new(H), "dbeta": new(H), "scale": new(T, -(-H // GROUP))}
    big = {k: [] for k in ("y", "dx", "back")}
    step = max(1, (1 << 26) // H)
    for a in range(0, T, step):
        b = min(T, a + step)
        x = s["x"][a:b].double()
        kept = x
        if op in ("ckpt8", "norm_ckpt8"):
            kept = torch.empty_like(x)
            for k in range(-(-H // GROUP)):
                part = x[:, k * GROUP:(k + 1) * GROUP]
                top = part.abs().max(1, keepdim=True).values
                sc = torch.where(top >= TINY, top / 127, torch.zeros_like(top))
                kept[:, k * GROUP:(k + 1) * GROUP] = torch.where(sc > 0, torch.round(part / sc) * sc, torch.zeros_like(part))
                small["scale"][a:b, k] = sc[:, 0]
            if op == "ckpt8":
                big["back"].append(kept)
                continue
        if op == "norm_bwd":                       # the statistics are inputs
            mean = s["mean"][a:b].double()[:, None] if layer else 0.0
            rstd = s["rstd"][a:b].double()[:, None]
        else:
            mean = x.mean(1, keepdim=True) if layer else 0.0
            rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
            if layer:
                small["mean"][a:b] = mean[:, 0]
            small["rstd"][a:b] = rstd[:, 0]
        gamma = s["gamma"].double()
        if op != "norm_bwd":
            y = (x - mean) * rstd * gamma
            big["y"].append(y + s["beta"].double() if layer else y)
        if op != "norm_fwd":
            dy = s["dy"][a:b].double()
            xh = (kept - mean) * rstd
            u = dy * gamma
            v = u - xh * ((u * xh).sum(1, keepdim=True) / H)
            big["dx"].append(rstd * (v - u.sum(1, keepdim=True) / H if layer else v))
            small["dgamma"] += (dy * xh).sum(0)
            small["dbeta"] += dy.sum(0)
    names = {"norm_fwd": ("y", "mean", "rstd"), "norm_bwd": ("dx", "dgamma", "dbeta"), "ckpt8": ("back", "scale"),
             "norm_ckpt8": ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}[op]
    return {n: torch.cat(big[n]) if n in big else small[n] for n in names if layer or n not in ("mean", "dbeta")}
