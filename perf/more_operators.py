"""Cases of the operators that answer with a policy and update it: drawing tokens from logits (temperature, top-k,
top-p, min-p) with given random numbers, matrices in 8-bit floating point with a scale for each block of 128 and their
product, and an AdamW step over many tensors with states in 32 or 8 bits.

With own = False every operator is computed in its plain form: elementary torch operations in 32 bits (64 where a
choice between tokens hangs on them), rounded once at the end.  With own = True the calls are those of the package's
binding."""
import math

import numpy as np
import torch

own = False

GROUP = 128            # columns (elements) that share one scale
TOP = 448.0            # largest value of the 8-bit type (4 bits of exponent, 3 of fraction)
TINY = 2.0 ** -119     # a group whose largest magnitude is below this is stored as zeros
LEAST = 2.0 ** -6      # a root of v that is not zero is not stored below this part of 448
F8 = torch.float8_e4m3fn
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
ADAM_SEED = 0x5EED0123456789AB


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the next token of a single answer, with the filters that serving programs set
        {"name": "sample one token", "op": "sample", "B": 1, "V": 151936, "x": "bf16", "temperature": 0.8, "top_k": 50,
         "top_p": 0.95, "min_p": 0.0, "masked": 0.0, "mixed": False},
        # 64 questions x 8 answers, one token of each, from the policy's own distribution (what training assumes)
        {"name": "sample rollouts", "op": "sample", "B": 512, "V": 151936, "x": "bf16", "temperature": 1.0, "top_k": 0,
         "top_p": 1.0, "min_p": 0.0, "masked": 0.0, "mixed": False},
        # requests of different users in one batch: each row has its own settings, some tokens are ruled out
        {"name": "sample mixed", "op": "sample", "B": 96, "V": 152064, "x": "f32", "temperature": 0.7, "top_k": 200,
         "top_p": 0.9, "min_p": 0.02, "masked": 0.05, "mixed": True},
        # activations of 64 completions at hidden 3584, in front of a product
        {"name": "fp8_store rows", "op": "fp8_store", "R": 16527, "C": 3584, "x": "bf16", "blocks": False},
        # an LM head laid out again after its update
        {"name": "fp8_store head", "op": "fp8_store", "R": 151936, "C": 896, "x": "bf16", "blocks": True},
        # the logits of one token at hidden 896: the head is read once, latency shows
        {"name": "fp8_matmul one token", "op": "fp8_matmul", "T": 1, "N": 151936, "K": 896, "y": "f32"},
        # the logits of 64 answers at hidden 3584
        {"name": "fp8_matmul 64 tokens", "op": "fp8_matmul", "T": 64, "N": 152064, "K": 3584, "y": "f32"},
        # the logits of a batch of completions: short sums, a large result
        {"name": "fp8_matmul head", "op": "fp8_matmul", "T": 4096, "N": 151936, "K": 896, "y": "bf16"},
        # a layer of a model of hidden 3584 over a batch: long sums
        {"name": "fp8_matmul layer", "op": "fp8_matmul", "T": 8192, "N": 14336, "K": 3584, "y": "bf16"},
        # the norms of a small model: many small tensors, latency
        {"name": "adamw norms", "op": "adamw", "shapes": "896*24 64 1001", "bits": 32, "g": "f32"},
        # head and norm of a policy of hidden 896, states in 32 bits, bf16 gradients
        {"name": "adamw head", "op": "adamw", "shapes": "151936x896 896*2", "bits": 32, "g": "bf16"},
        # the same with states in 8 bits and some layers' weights, fp32 gradients
        {"name": "adamw 8-bit", "op": "adamw", "shapes": "151936x896 896x4864*6 896x896*4 896*12 1151", "bits": 8, "g": "f32"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "fp8_store", "fp8_matmul", "fp8_matmul", "adamw"])
    if op == "sample":
        V = _log_int(rng, 700, 262144)
        B = _log_int(rng, 1, max(1, min(1024, int(5.0e7 / V))))
        return {"op": op, "B": B, "V": V, "x": rng.choice(["bf16", "f32"]), "temperature": rng.choice([1.0, 1.0, 0.6, 0.3, 1.4]),
                "top_k": rng.choice([0, 0, 1, 20, 64, 1000]), "top_p": rng.choice([1.0, 0.99, 0.9, 0.5]),
                "min_p": rng.choice([0.0, 0.0, 0.05, 0.2]), "masked": rng.choice([0.0, 0.3]), "mixed": rng.random() < 0.4}
    if op == "fp8_store":
        C = _log_int(rng, 40, 16384)
        R = _log_int(rng, 1, max(1, min(160000, int(1.2e8 / C))))
        return {"op": op, "R": R, "C": C, "x": rng.choice(["bf16", "bf16", "f32"]), "blocks": rng.random() < 0.4}
    if op == "fp8_matmul":
        K, N = _log_int(rng, 100, 8192), _log_int(rng, 100, 152064)
        T = _log_int(rng, 1, max(1, min(8192, int(4.0e11 / (N * K)))))
        return {"op": op, "T": T, "N": N, "K": K, "y": rng.choice(["bf16", "f32"])}
    shapes = ["%d*%d" % (_log_int(rng, 1, 5000), rng.randint(1, 12)) for _ in range(rng.randint(1, 4))]
    if rng.random() < 0.7:
        shapes.append("%dx%d*%d" % (_log_int(rng, 64, 8192), _log_int(rng, 64, 2048), rng.randint(1, 4)))
    return {"op": op, "shapes": " ".join(shapes), "bits": rng.choice([8, 8, 32]), "g": rng.choice(["bf16", "f32"])}


def _sizes(case):
    """Elements of each tensor: "896x4864*6" are six matrices."""
    n = []
    for part in case["shapes"].split():
        shape, _, times = part.partition("*")
        n += [math.prod(int(d) for d in shape.split("x"))] * int(times or 1)
    return n


# ------------------------------------------------------------------------------------------ inputs
def _settings(case, g):
    """Each row's temperature, top_k, top_p and min_p: the case's, or a mixture around it with greedy rows."""
    B = case["B"]
    if not case["mixed"]:
        return [case["temperature"], case["top_k"], case["top_p"], case["min_p"]]
    u = torch.rand(4, B, generator=g, device="cuda")
    T = torch.where(u[0] < 0.15, 0.0, case["temperature"] * (0.5 + u[0]))
    k = torch.where(u[1] < 0.3, 0, 1 + (u[1] * max(2 * case["top_k"], 8)).to(torch.int32)).to(torch.int32)
    p = torch.where(u[2] < 0.3, 1.0, 1 - (1 - 0.9 * case["top_p"]) * u[2])
    return [T, k, p, torch.where(u[3] < 0.6, 0.0, case["min_p"] * u[3])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op = case["op"]
    s = {"case": case, "op": op, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    randn = lambda *n: torch.randn(*n, generator=g, device="cuda")
    if op == "sample":
        B, V = case["B"], case["V"]
        z = 2.5 * randn(B, V)                          # the bulk of a vocabulary, and some tokens that fit
        fit = torch.randint(0, V, (B, 24), generator=g, device="cuda")
        z.scatter_add_(1, fit, 4.0 + 3.0 * randn(B, 24))
        if case["masked"]:
            z[torch.rand(B, V, generator=g, device="cuda") < case["masked"]] = float("-inf")
        s["z"] = z.to(_type(case["x"]))
        s["seeds"] = torch.randint(-2 ** 63, 2 ** 63 - 1, (B,), generator=g, device="cuda")
        s["settings"] = _settings(case, g)
        s["ids"] = torch.empty(B, dtype=torch.int32, device="cuda")
        s["logp"] = torch.empty(B, device="cuda")
    elif op == "fp8_store":
        x = randn(case["R"], case["C"])
        if case["blocks"]:
            x.mul_(0.02)
        else:                                          # a residual stream: a few channels twenty times as large
            x.mul_(torch.where(torch.rand(case["C"], generator=g, device="cuda") < 0.01, 20.0, 1.0))
        s["x"] = x.to(_type(case["x"]))
        s["q"], s["scale"] = _room(case["R"], case["C"], case["blocks"])
    elif op == "fp8_matmul":
        T, N, K = case["T"], case["N"], case["K"]
        for name, rows, width, blocks in (("x", T, 1.0, False), ("w", N, 0.02, True)):
            q, scale = _room(rows, K, blocks)
            q[:, :K], scale[:] = _to_fp8(width * randn(rows, K), blocks)
            s[name], s[name + "_scale"] = q, scale
        s["y"] = torch.empty(T, N, dtype=_type(case["y"]), device="cuda")
    else:
        n = _sizes(case)
        s["master"] = [0.02 * randn(k) for k in n]
        s["grad"] = [(1e-3 * randn(k) * torch.exp(randn(k))).to(_type(case["g"])) for k in n]
        m = [1e-4 * randn(k) for k in n]
        r = [1e-3 * torch.exp(0.7 * randn(k)) for k in n]                    # roots of v
        new = lambda t: torch.empty_like(t)
        if case["bits"] == 8:
            held = [_to_fp8(t[None], False) for t in m], [_to_fp8(t[None], False) for t in r]
            s["m"], s["v"] = ([q[0] for q, _ in h] for h in held)
            s["m_scale"], s["v_scale"] = ([a[0] for _, a in h] for h in held)
            s["new_m_scale"], s["new_v_scale"] = ([new(t) for t in s[k]] for k in ("m_scale", "v_scale"))
        else:
            s["m"], s["v"] = m, [t * t for t in r]
        s["new_master"], s["new_m"], s["new_v"] = ([new(t) for t in s[k]] for k in ("master", "m", "v"))
        s["w"] = [torch.empty(k, dtype=torch.bfloat16, device="cuda") for k in n]
        s["clip"] = torch.full((1,), 0.75, device="cuda")                    # factor of the gradients from clipping
        if own:
            _plan(s)
    return s


def _plan(s):
    """The lists of tensors that a program hands to its optimiser once."""
    from paper_2509_08721_b200 import binding as B
    held = s["case"]["bits"] == 8
    state = lambda m, v, a, b: [B.AdamWState(*t) for t in zip(m, v, a if held else [None] * len(m), b if held else [None] * len(m))]
    s["plan"] = B.AdamWTensors(s["master"], state(s["m"], s["v"], s.get("m_scale"), s.get("v_scale")))
    s["plan_out"] = B.AdamWTensors(s["new_master"], state(s["new_m"], s["new_v"], s.get("new_m_scale"), s.get("new_v_scale")), s["w"])


def _room(R, C, blocks):
    """A matrix in 8 bits: rows on 16-byte boundaries, one scale a row (or 128 rows) and 128 columns."""
    q = torch.zeros(R, -(-C // 16) * 16, dtype=F8, device="cuda")
    return q, torch.zeros(-(-R // GROUP) if blocks else R, -(-C // GROUP), device="cuda")


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2509_08721_b200 import binding as B
    op, case = s["op"], s["case"]
    if op == "sample":
        T, k, p, mp = s["settings"]
        B.sapo_sample(s["z"], s["seeds"], s["ids"], s["logp"], s["status"], temperature=T, top_k=k, top_p=p, min_p=mp)
        return {"ids": s["ids"], "logp": s["logp"]}
    if op == "fp8_store":
        B.sapo_fp8_store(s["x"], B.Fp8(s["q"], s["scale"], case["C"], case["blocks"]), s["status"])
        return {"q": s["q"][:, :case["C"]], "scale": s["scale"]}
    if op == "fp8_matmul":
        K = case["K"]
        B.sapo_fp8_matmul(B.Fp8(s["x"], s["x_scale"], K, False), B.Fp8(s["w"], s["w_scale"], K, True), s["y"], s["status"])
        return {"y": s["y"]}
    B.sapo_adamw_step(s["plan"], s["grad"], 10, LR, s["status"], beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                      seed=ADAM_SEED, grad_scale=s["clip"], out=s["plan_out"])
    r = {"master": s["new_master"], "w": s["w"], "m": s["new_m"], "v": s["new_v"]}
    if case["bits"] == 8:
        r.update(m_scale=s["new_m_scale"], v_scale=s["new_v_scale"])
    return _joined(r)


def _joined(r):
    """Large tensors as they are, the small ones of a kind at most four: what is compared stays a short list."""
    return {k: (v if len(v) <= 4 else v[:3] + v[-1:]) for k, v in r.items()}


def _to_fp8(x, blocks):
    """(values in 8 bits, scales) of a 32-bit matrix."""
    R, C = x.shape
    h = GROUP if blocks else 1
    r, c = -(-R // h), -(-C // GROUP)
    t = torch.zeros(r * h, c * GROUP, device=x.device)
    t[:R, :C] = x
    t = t.view(r, h, c, GROUP)
    a = t.abs().amax((1, 3), keepdim=True)
    inv = torch.where(a >= TINY, TOP / a, torch.zeros_like(a))
    scale = torch.where(a >= TINY, a / TOP, torch.zeros_like(a))
    q = (t * inv).clamp_(-TOP, TOP).to(F8)
    return q.view(r * h, c * GROUP)[:R, :C], scale.view(r, c)


def _from_fp8(q, scale, C, blocks):
    x = q[:, :C].float()
    s = scale.repeat_interleave(GROUP, 1)[:, :C]
    return x * (s.repeat_interleave(GROUP, 0)[:len(x)] if blocks else s)


def _philox(c0, c1, c2, c3, k0, k1):
    """Four 32-bit words of the counter-based generator Philox 4x32 with 10 rounds (Salmon et al., 2011), in int64."""
    full = 0xFFFFFFFF

    def wide(mul, c):
        upper = mul * (c >> 16) + ((mul * (c & 0xFFFF)) >> 16)
        return upper >> 16, (mul * c) & full
    for _ in range(10):
        (h0, l0), (h1, l1) = wide(0xD2511F53, c0), wide(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & full, (k1 + 0xBB67AE85) & full
    return c0, c1, c2, c3


def _halves(words):
    """Eight 16-bit numbers from four words, the low half of each first."""
    return torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], -1)


def _exponentials(seeds, V):
    """The unit exponential of each row and token, in 64 bits: 32 random bits of the row's number and the token."""
    k0, k1 = (seeds & 0xFFFFFFFF)[:, None], ((seeds >> 32) & 0xFFFFFFFF)[:, None]
    c = torch.arange(-(-V // 8), device=seeds.device)[None] + 0 * k0
    zero = torch.zeros_like(c)
    high, low = (_halves(_philox(c, zero + j, zero, zero, k0, k1)).flatten(1)[:, :V] for j in (0, 1))
    return -torch.log1p(-(high.mul_(65536).add_(low).double() + 0.5) * 2.0 ** -32)


def _sample_plain(z, seeds, T, k, p, mp):
    B, V = z.shape
    col = lambda v: (v if isinstance(v, torch.Tensor) else torch.full((B,), float(v), device=z.device))[:, None].double()
    T, k, p, mp = col(T), col(k), col(p), col(mp)
    z = z.float()
    vals, order = torch.sort(z, dim=1, descending=True, stable=True)
    d = vals.double() - vals[:, :1].double()
    total = torch.log(torch.exp(d).sum(1))
    w = torch.exp(d / torch.where(T > 0, T, torch.ones_like(T)))
    rank = torch.arange(V, device=z.device)[None]
    keep = (rank < torch.where(k > 0, k, V + 0 * k)) & (rank < torch.where(T > 0, V, 1))
    mass = w * keep
    before = torch.cumsum(mass, 1) - mass
    keep &= (rank == 0) | (before < p * mass.sum(1, keepdim=True)) | (p >= 1)
    keep &= (rank == 0) | (w >= mp)
    race = _exponentials(seeds, V).gather(1, order) / w
    race = torch.where(keep, race, torch.full_like(race, float("inf")))
    best = race.amin(1, keepdim=True)
    ids = torch.where(race == best, order, V).amin(1)
    return ids, z.double().gather(1, ids[:, None])[:, 0] - vals[:, 0].double() - total


def _adamw_plain(i, s):
    case = s["case"]
    theta, g = s["master"][i], s["grad"][i].float() * s["clip"]
    n = len(theta)
    if case["bits"] == 8:
        groups = torch.arange(n, device=theta.device) // GROUP
        m = s["m"][i].float() * s["m_scale"][i][groups]
        root = s["v"][i].float() * s["v_scale"][i][groups]
        v = root * root
    else:
        m, v = s["m"][i], s["v"][i]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * (1 - BETA2)) * g
    root = torch.sqrt(v)
    c1, c2 = 1 / (1 - BETA1 ** 10), 1 / math.sqrt(1 - BETA2 ** 10)
    theta = theta * (1 - LR * DECAY) - LR * ((m * c1) / (root * c2 + EPS))
    r = {"master": theta, "w": theta.to(torch.bfloat16)}
    if case["bits"] == 32:
        return {**r, "m": m, "v": v}
    q, scale = _to_fp8(m[None], False)
    r.update(m=q[0], m_scale=scale[0])
    padded = torch.zeros(-(-n // GROUP) * GROUP, device=theta.device)
    padded[:n] = root
    a = padded.view(-1, GROUP).amax(1, keepdim=True)
    inv = torch.where(a >= TINY, TOP / a, torch.zeros_like(a))
    t = (padded.view(-1, GROUP) * inv).flatten()[:n]
    c = torch.arange(-(-n // 8), device=theta.device)
    bits = _halves(_philox(c & 0xFFFFFFFF, c >> 32, torch.full_like(c, i), torch.full_like(c, 10), ADAM_SEED & 0xFFFFFFFF,
                           ADAM_SEED >> 32)).flatten()[:n].to(torch.int32)
    up = (t.clamp(min=LEAST).view(torch.int32) + bits * 16 + 8) & ~0xFFFFF       # rounded up or down by the random number
    t = torch.where(t > 0, up.view(torch.float32).clamp(max=TOP), torch.zeros_like(t))
    r.update(v=t.to(F8), v_scale=torch.where(a >= TINY, a / TOP, torch.zeros_like(a))[:, 0])
    return r


def _run_plain(s):
    op, case = s["op"], s["case"]
    if op == "sample":
        ids, logp = _sample_plain(s["z"], s["seeds"], *s["settings"])
        return {"ids": ids.to(torch.int32), "logp": logp.float()}
    if op == "fp8_store":
        q, scale = _to_fp8(s["x"].float(), case["blocks"])
        return {"q": q, "scale": scale}
    if op == "fp8_matmul":
        K = case["K"]
        x, w = _from_fp8(s["x"], s["x_scale"], K, False), _from_fp8(s["w"], s["w_scale"], K, True)
        return {"y": (x @ w.T).to(s["y"].dtype)}
    each = [_adamw_plain(i, s) for i in range(len(s["master"]))]
    return _joined({k: [r[k] for r in each] for k in ("master", "w", "m", "v", "m_scale", "v_scale") if k in each[0]})


# ------------------------------------------------------------------------------------------ work
def work(case):
    size = {"bf16": 2, "f32": 4}
    op = case["op"]
    if op == "sample":
        n = case["B"] * case["V"]                      # a random number, an exponential and a comparison a token
        return {"bytes": n * size[case["x"]] + 16 * case["B"], "flops": 8 * n}
    if op == "fp8_store":
        n, c = case["R"] * case["C"], -(-case["C"] // GROUP)
        return {"bytes": n * (size[case["x"]] + 1) + 4 * c * (-(-case["R"] // GROUP) if case["blocks"] else case["R"]), "flops": 3 * n}
    if op == "fp8_matmul":
        T, N, K = case["T"], case["N"], case["K"]
        c = -(-K // GROUP)
        return {"bytes": T * K + N * K + T * N * size[case["y"]] + 4 * c * (T + -(-N // GROUP)), "flops": 2 * T * N * K}
    n, groups = sum(_sizes(case)), sum(-(-k // GROUP) for k in _sizes(case))
    state = 2 * n * 2 * (1 if case["bits"] == 8 else 4) + (16 * groups if case["bits"] == 8 else 0)
    return {"bytes": n * (4 + 4 + 2 + size[case["g"]]) + state, "flops": 14 * n}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "sample":
        return _exact_sample(case, s) if case["B"] * case["V"] <= 1 << 27 else None
    if op == "fp8_store":
        x, h = s["x"].double(), GROUP if case["blocks"] else 1
        q, scale = torch.zeros_like(x), torch.zeros_like(s["scale"], dtype=torch.float64)
        for j in range(scale.shape[1]):
            part = x[:, j * GROUP:(j + 1) * GROUP].abs().amax(1)
            top = torch.nn.functional.pad(part, (0, -len(part) % h)).view(-1, h).amax(1)
            scale[:, j] = torch.where(top >= TINY, top / 448, 0 * top)
            each = scale[:, j].repeat_interleave(h)[:len(x), None]
            q[:, j * GROUP:(j + 1) * GROUP] = _nearest8(x[:, j * GROUP:(j + 1) * GROUP] / torch.where(each > 0, each, 1 + 0 * each)) * (each > 0)
        return {"q": q, "scale": scale}
    if op == "fp8_matmul":
        y = torch.empty(case["T"], case["N"], dtype=torch.float64, device="cuda")
        step, K = 128 * max(1, (1 << 20) // case["K"]), case["K"]
        x = s["x"].double()[:, :K] * s["x_scale"].double().repeat_interleave(GROUP, 1)[:, :K]
        for a in range(0, case["N"], step):
            w = s["w"][a:a + step].double()[:, :K]
            sc = s["w_scale"][a // GROUP:(a + step) // GROUP].double().repeat_interleave(GROUP, 1)[:, :K]
            y[:, a:a + step] = x @ (w * sc.repeat_interleave(GROUP, 0)[:len(w)]).T
        return {"y": y}
    r = {k: [] for k in ("master", "w", "m", "v", "m_scale", "v_scale")}
    for i, theta in enumerate(s["master"]):
        _exact_adamw(s, i, theta.double(), r)
    return _joined({k: v for k, v in r.items() if v})


def _nearest8(t):
    """The nearest value with 3 bits of fraction (ties to even) and an exponent from -6, at most 448."""
    e = torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6)))
    unit = torch.exp2(torch.maximum(torch.where(torch.exp2(e) > t.abs(), e - 1, e), torch.full_like(e, -6.0)) - 3)
    return (torch.round(t / unit) * unit).clamp(-448, 448)


def _philox_numpy(c, key):
    full = np.uint64(0xFFFFFFFF)
    k = [np.uint64(key & 0xFFFFFFFF), np.uint64((key >> 32) & 0xFFFFFFFF)]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & full, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & full]
        k = [(k[0] + np.uint64(0x9E3779B9)) & full, (k[1] + np.uint64(0xBB67AE85)) & full]
    return np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(-1)


def _exact_sample(case, s):
    """Row by row on the host."""
    B, V = case["B"], case["V"]
    Z = s["z"].float().cpu().numpy().astype(np.float64)
    seeds = s["seeds"].cpu().tolist()
    T, K, P, M = ([float(x) for x in v.cpu()] if isinstance(v, torch.Tensor) else [float(v)] * B for v in s["settings"])
    c = np.arange(-(-V // 8), dtype=np.uint64)
    zero = np.zeros_like(c)
    ids, logp = [], []
    for b in range(B):
        d = Z[b] - Z[b].max()
        alive = np.ones(V, bool)
        if T[b] == 0:
            alive[:] = False
            alive[int(np.argmax(d))] = True
        else:
            w = np.exp(d / T[b])
            if 0 < K[b] < V or P[b] < 1:
                order = np.argsort(-d, kind="stable")
                n = int(K[b]) if 0 < K[b] < V else V
                sums = np.cumsum(w[order[:n]])
                if P[b] < 1:
                    n = 1 + int(np.searchsorted(sums, P[b] * sums[-1], side="left"))
                alive[order[n:]] = False
            alive &= (w >= M[b]) | (d == 0)
        at = np.flatnonzero(alive)
        high = _philox_numpy([c, zero, zero, zero], seeds[b])[at].astype(np.float64)
        low = _philox_numpy([c, zero + np.uint64(1), zero, zero], seeds[b])[at].astype(np.float64)
        e = -np.log1p(-(high * 65536 + low + 0.5) / 2.0 ** 32)
        i = int(at[0]) if T[b] == 0 else int(at[np.argmax(d[at] / T[b] - np.log(e))])
        ids.append(i)
        logp.append(d[i] - math.log(np.exp(d).sum()))
    return {"ids": torch.tensor(ids, dtype=torch.int32), "logp": torch.tensor(logp, dtype=torch.float64)}


def _exact_adamw(s, i, theta, r):
    held, n = s["case"]["bits"] == 8, len(theta)
    each = lambda t: t.double().repeat_interleave(GROUP)[:n]
    g = s["grad"][i].double() * s["clip"].double()
    m = s["m"][i].double() * (each(s["m_scale"][i]) if held else 1)
    v = (s["v"][i].double() * each(s["v_scale"][i])) ** 2 if held else s["v"][i].double()
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
    step = m / (1 - BETA1 ** 10) / (torch.sqrt(v / (1 - BETA2 ** 10)) + EPS)
    theta = theta - LR * (step + DECAY * theta)
    r["master"].append(theta)
    r["w"].append(theta)
    if not held:
        r["m"].append(m)
        r["v"].append(v)
        return
    biggest = lambda t: torch.nn.functional.pad(t.abs(), (0, -n % GROUP)).view(-1, GROUP).amax(1) / 448
    sm, sv = biggest(m), biggest(torch.sqrt(v))
    r["m_scale"].append(sm)
    r["v_scale"].append(sv)
    r["m"].append(_nearest8(m / each(sm)))
    c = np.arange(-(-n // 8), dtype=np.uint64)
    word = lambda x: np.full_like(c, x)
    rand = torch.from_numpy(_philox_numpy([c, word(0), word(i), word(10)], ADAM_SEED)[:n].astype(np.float64)).cuda()
    t = (torch.sqrt(v) / each(sv)).clamp(min=2.0 ** -6)
    e = torch.floor(torch.log2(t))
    unit = torch.exp2(torch.where(torch.exp2(e) > t, e - 1, e) - 3)
    r["v"].append((torch.floor(t / unit + (rand + 0.5) / 65536) * unit).clamp(max=448.0))
