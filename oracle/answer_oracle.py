"""Plain float64 definitions of the operators that answer with a policy and update it: drawing tokens from logits, 8-bit
floating point with a scale for each block of 128 and the product of such matrices, AdamW with states in 32 or 8 bits.
numpy only; shares no code with the CUDA path.  What is held in 8 bits depends on single roundings, so those steps are
taken in float32 as the formats define them."""
from __future__ import annotations

from typing import Dict, Tuple

import numpy as np

GROUP = 128
TOP = 448.0
TINY = 2.0 ** -119
_codes = np.arange(127, dtype=np.int64)                       # the 127 codes of values >= 0 (127 is NaN)
_exp, _frac = _codes >> 3, _codes & 7
POSITIVE = np.where(_exp == 0, _frac * 2.0 ** -9, (8 + _frac) * 2.0 ** (_exp.astype(np.float64) - 10))


# ------------------------------------------------------------------------------------------ random numbers
def philox(counter, key) -> np.ndarray:
    """Philox 4x32, 10 rounds: counter a list of four arrays (or numbers), key a pair of numbers; four uint32 arrays."""
    full = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) for v in np.broadcast_arrays(*counter)]
    k = [int(key[0]) & 0xFFFFFFFF, int(key[1]) & 0xFFFFFFFF]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & full, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & full]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c)


def halves(words: np.ndarray, n: int) -> np.ndarray:
    """16-bit numbers 0 .. n-1 from the words of counters 0, 1, ...: eight a counter, the low half of each word first."""
    w = words.T.reshape(-1)
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 1).reshape(-1)[:n].astype(np.int64)


def split_key(seed: int) -> Tuple[int, int]:
    return seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF


# ------------------------------------------------------------------------------------------ drawing
def kept_tokens(z: np.ndarray, temperature: float, top_k: int, top_p: float, min_p: float) -> np.ndarray:
    """Which tokens of a row stay in the draw (at least one is finite)."""
    z = np.asarray(z, np.float64)
    order = np.argsort(-z, kind="stable")
    keep = np.zeros(len(z), bool)
    if temperature == 0 or top_p <= 0:
        keep[order[0]] = True
        return keep
    with np.errstate(over="ignore"):
        w = np.exp(np.maximum((z[order] - z[order[0]]) / temperature, -1e300))
    n = top_k if 0 < top_k < len(z) else len(z)
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:n])])
        n = max(1, int((before[:n] < top_p * before[n]).sum()))
    keep[order[:n]] = w[:n] >= min_p
    keep[order[0]] = True
    return keep


def sample(z, seed: int, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0) -> Tuple[int, float, float]:
    """(id, log-prob at temperature 1, lead): lead is how far behind, in log time, the second token finishes."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all():
        return -1, 0.0, np.inf
    f32 = lambda v: float(np.float32(v))
    temperature, top_p, min_p = f32(temperature), f32(top_p), f32(min_p)
    keep = kept_tokens(z, temperature, int(top_k), top_p, min_p)
    d = z - z.max()
    c = np.arange(-(-len(z) // 8))
    n = halves(philox([c, 0, 0, 0], split_key(seed)), len(z)) * 65536 + halves(philox([c, 1, 0, 0], split_key(seed)), len(z))
    e = -np.log1p(-(n + 0.5) / 2.0 ** 32)
    at = np.flatnonzero(keep & np.isfinite(d))
    if temperature == 0 or len(at) == 1:
        i, lead = int(at[0]), np.inf
    else:
        t = np.log(e[at]) - d[at] / temperature
        first = np.argsort(t, kind="stable")[:2]
        i, lead = int(at[first[0]]), float(t[first[1]] - t[first[0]])
    return i, float(d[i] - np.log(np.exp(d).sum())), lead


# ------------------------------------------------------------------------------------------ 8-bit floating point
def nearest_code(x) -> np.ndarray:
    """Nearest code of float values in [-448, 448]; ties to the even code."""
    a = np.abs(np.asarray(x, np.float64))
    hi = np.clip(np.searchsorted(POSITIVE, a), 1, 126)
    lo = hi - 1
    to_lo, to_hi = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where((to_lo < to_hi) | ((to_lo == to_hi) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def code_values(code) -> np.ndarray:
    code = np.asarray(code).astype(np.int64)
    v = np.append(POSITIVE, np.nan)[code & 127]
    return np.where(code & 128, -v, v)


def fp8_store(x, blocks: bool = False) -> Tuple[np.ndarray, np.ndarray]:
    """(codes uint8 [R, C], scales float32)."""
    x = np.asarray(x, np.float32)
    R, C = x.shape
    h = GROUP if blocks else 1
    codes, scale = np.zeros((R, C), np.uint8), np.zeros((-(-R // h), -(-C // GROUP)), np.float32)
    top = np.float32(TOP)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            where = np.s_[i * h:(i + 1) * h, j * GROUP:(j + 1) * GROUP]
            part = x[where]
            if not np.isfinite(part).all():
                scale[i, j] = np.nan
                continue
            a = np.abs(part).max()
            if a >= TINY:
                scale[i, j] = a * (np.float32(1) / top)
                codes[where] = nearest_code(np.clip(part * (top * (np.float32(1) / a)), -top, top))
    return codes, scale


def fp8_values(codes, scale, blocks: bool = False) -> np.ndarray:
    s = np.repeat(np.asarray(scale, np.float64), GROUP, 1)[:, :codes.shape[1]]
    return code_values(codes) * (np.repeat(s, GROUP, 0)[:codes.shape[0]] if blocks else s)


# ------------------------------------------------------------------------------------------ AdamW
def adamw(master, grad, m, v, step: int, lr: float, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01) -> Dict[str, np.ndarray]:
    """One step in float64; m and v are the moments before it."""
    w, g, m, v = (np.asarray(t, np.float64) for t in (master, grad, m, v))
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    up = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return {"master": w * (1 - lr * decay) - lr * up, "m": m, "v": v, "update": up}


def adamw_moments32(grad, m, v, beta1=0.9, beta2=0.999) -> Tuple[np.ndarray, np.ndarray]:
    """The moments after a step, to the bit: every product and sum rounded to float32."""
    f = np.float32
    g, m, v = (np.asarray(t, f) for t in (grad, m, v))
    with np.errstate(over="ignore"):
        return f(beta1) * m + f(1 - beta1) * g, np.minimum(f(beta2) * v + (f(1 - beta2) * g) * g, np.finfo(f).max)


def _groups(x: np.ndarray) -> np.ndarray:
    return np.pad(x, (0, -len(x) % GROUP)).reshape(-1, GROUP)


def state8(m, v, number: int, step: int, seed: int):
    """(m codes, m_scale, codes of the root of v, v_scale) of float32 moments, to the bit."""
    f = np.float32
    n = len(m)
    top = f(TOP)

    def factors(t):
        a = np.abs(_groups(t)).max(1)
        some = a >= TINY
        safe = np.where(some, a, f(1)).astype(f)
        return np.where(some, a * (f(1) / top), f(0)).astype(f), np.where(some, top * (f(1) / safe), f(0)).astype(f)
    m, root = np.asarray(m, f), np.sqrt(np.asarray(v, f))
    sm, im = factors(m)
    sr, ir = factors(root)
    codes = nearest_code(np.clip(_groups(m) * im[:, None], -top, top)).reshape(-1)[:n]
    c = np.arange(-(-n // 8), dtype=np.uint64)
    r = halves(philox([c & np.uint64(0xFFFFFFFF), c >> np.uint64(32), number, step], split_key(seed)), n)
    t = (_groups(root) * ir[:, None]).astype(f).reshape(-1)[:n]
    bits = (np.maximum(t, f(2.0 ** -6)).view(np.int32).astype(np.int64) + 16 * r + 8) & ~0xFFFFF
    up = np.minimum(bits.astype(np.int32).view(f), top)
    return codes, sm, nearest_code(np.where(t > 0, up, f(0))), sr


def held32(codes, scale) -> np.ndarray:
    """What 8-bit codes stand for, as float32 products."""
    return (_groups(code_values(codes).astype(np.float32)) * np.asarray(scale, np.float32)[:, None]).reshape(-1)[:len(codes)]
