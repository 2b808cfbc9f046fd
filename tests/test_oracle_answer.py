"""Pins of the float64 definitions in oracle/answer_oracle.py: known answers, library routines, statistics, invariants."""
import numpy as np
import pytest
import torch

from oracle import answer_oracle as ao
from oracle import sapo_oracle as orc


def test_philox_is_the_one_of_the_pool_draw():
    for c, k in (((0, 0, 0, 0), (0, 0)), ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2), ((1, 2, 3, 4), (5, 6))):
        assert [int(w) for w in ao.philox(list(c), k)] == list(orc.philox4x32(c, k))
    many = ao.philox([np.arange(5), 1, 0, 0], (7, 8))
    assert [int(w) for w in many[:, 3]] == list(orc.philox4x32((3, 1, 0, 0), (7, 8)))
    assert list(ao.halves(np.array([[0x00020001], [0x00040003], [0x00060005], [0x00080007]], np.uint64), 7)) == [1, 2, 3, 4, 5, 6, 7]


def test_codes_are_those_of_the_torch_type():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ao.code_values(np.arange(256)), every)
    x = np.concatenate([np.linspace(-448, 448, 20011), ao.POSITIVE, (ao.POSITIVE[1:] + ao.POSITIVE[:-1]) / 2]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(ao.nearest_code(x), want)


def test_draws_follow_the_distribution():
    """Frequencies of 20000 draws: chi-square with 5 degrees of freedom, 30.9 is exceeded once in 10^5."""
    z = np.array([0.3, -1.0, 2.0, 0.0, 1.0, -np.inf, 0.5])
    for T in (1.0, 0.5):
        p = np.exp(z / T) / np.exp(z / T).sum()
        ids = np.array([ao.sample(z, s * 0x9E3779B97F4A7C15 % 2 ** 64, T)[0] for s in range(20000)])
        n = np.bincount(ids, minlength=7)
        assert n[5] == 0 and ((n - 20000 * p) ** 2 / np.where(p > 0, 20000 * p, 1)).sum() < 30.9


def test_which_tokens_stay():
    z = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))
    names = lambda **kw: set(np.flatnonzero(ao.kept_tokens(z, **{"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, **kw})))
    assert names() == {0, 1, 2, 3, 4} and names(top_k=4) == {0, 1, 3, 4}           # equal ones: the lower index
    assert names(top_p=0.6) == {1, 3} and names(top_p=0.7) == {1, 3, 4} and names(top_p=0.0) == {1} and names(temperature=0.0) == {1}
    assert names(top_k=2, top_p=0.6) == {1} and names(top_k=2, top_p=0.62) == {1, 3}   # 0.4 of 0.65 is 0.615
    assert names(min_p=0.3) == {1, 3, 4} and names(min_p=1.0) == {1}
    assert names(temperature=0.5, min_p=0.3) == {1, 3}                              # weights squared


def test_stored_values_are_within_half_a_code():
    rng = np.random.default_rng(0)
    for blocks in (False, True):
        x = (rng.normal(size=(130, 300)) * np.exp(3 * rng.normal(size=(130, 300)))).astype(np.float32)
        codes, scale = ao.fp8_store(x, blocks)
        s = np.repeat(np.repeat(scale.astype(np.float64), 128 if blocks else 1, 0)[:130], 128, 1)[:, :300]
        assert np.all(np.abs(ao.fp8_values(codes, scale, blocks) - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 2.0 ** -20))


def test_adamw_is_the_library_optimiser():
    w = torch.randn(50, dtype=torch.float64, generator=torch.Generator().manual_seed(1)).requires_grad_()
    opt = torch.optim.AdamW([w], lr=0.01, weight_decay=0.1)
    mine, m, v = w.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        w.grad = torch.randn(50, dtype=torch.float64, generator=torch.Generator().manual_seed(t))
        r = ao.adamw(mine, w.grad.numpy(), m, v, t, 0.01, decay=0.1)
        mine, m, v = r["master"], r["m"], r["v"]
        opt.step()
        np.testing.assert_allclose(mine, w.detach().numpy(), rtol=1e-12)


def test_the_root_is_right_on_average():
    """10^5 elements with one root, 0.3 of the group's largest: their mean is off by at most 5 standard deviations of
    a rounding to codes 2^5 / 448 apart (uniform to one of two neighbours: at most half of that each)."""
    n = 128 * 800
    root = np.full(n, 0.3, np.float32)
    root[::128] = 1.0
    codes, _, r, scale = ao.state8(np.zeros(n), root * root, 3, 17, 0x123456789ABCDEF)
    held = ao.held32(r, scale)[root < 1].astype(np.float64)
    assert len(np.unique(held)) == 2 and abs(held.mean() - 0.3) < 5 * 0.5 * (16 / 448) / np.sqrt(len(held))
    assert np.all(ao.state8(np.zeros(n), root * 0 + 1e-30 * (root < 1) + (root == 1), 0, 1, 0)[2] > 0)     # no root but 0 becomes 0


@pytest.mark.parametrize("bits", [1, 5])
def test_a_fresh_state_of_zeros(bits):
    codes, sm, r, sr = ao.state8(np.zeros(200), np.zeros(200), 0, bits, 1)
    assert not codes.any() and not r.any() and not sm.any() and not sr.any()
