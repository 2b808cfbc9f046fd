"""Drawing tokens on the device, against the float64 oracle.

The id hangs on which of two tokens finishes first, worked out in 64 bits on both sides: equal.  With top-k and top-p the
device adds the weights up in units of 2^-40 from fp32 exponentials (relative error 2^-21 each), so which token is the last
that stays could differ where the mass comes within 1e-6 of top_p: the rows below keep away from that.
logp: u = 2^-24.  ex2 and its argument: 2^-22 + 48 u at most where the weight matters (above e^-24 of the largest); a
thread's sum of up to 400 terms, then 5 + 16 + 8 partial sums: 429 u; two subtractions and a logarithm: 2 u (|logp| + 30)."""
import numpy as np
import pytest
import torch

from oracle import answer_oracle as ao
from paper_2509_08721_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def logits(B_, V, dtype, seed, ld=None, scale=2.5, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    z = scale * torch.randn(B_, V, generator=g)
    z.scatter_add_(1, torch.randint(0, V, (B_, 8), generator=g), 3 + 2 * torch.randn(B_, 8, generator=g))
    if masked:
        z[torch.rand(B_, V, generator=g) < masked] = float("-inf")
    full = torch.full((B_, ld or V), float("nan"), dtype=dtype)     # nothing between the rows may be read into a result
    full[:, :V] = z.to(dtype)
    return full.cuda()[:, :V]


def numbers(B_, seed):
    return torch.randint(-2 ** 63, 2 ** 63 - 1, (B_,), generator=torch.Generator().manual_seed(seed))


def draw(z, seeds, expect_status=0, **kw):
    ids = torch.full((z.shape[0],), -7, dtype=torch.int32, device="cuda")
    logp, status = torch.full((z.shape[0],), 7.0, device="cuda"), B.new_status()
    B.sapo_sample(z, seeds.cuda(), ids, logp, status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == expect_status, B.decode_status(int(status.item()))
    return ids.cpu().numpy(), logp.cpu().numpy()


def check(z, seeds, **kw):
    ids, logp = draw(z, seeds, **kw)
    host = z.float().cpu().numpy()
    row = lambda v, b: v[b].item() if isinstance(v, torch.Tensor) else v
    for b in range(len(ids)):
        i, lp, lead = ao.sample(host[b], int(seeds[b]) % 2 ** 64, **{k: row(v, b) for k, v in kw.items()})
        assert ids[b] == i, (b, ids[b], i, lead)
        assert abs(logp[b] - lp) <= 2.0 ** -22 + 477 * U + 2 * U * (abs(lp) + 30)
    return ids


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 100, 1001, 4097, 16385, 50001])
def test_own_distribution_at_any_width(V, dtype):
    check(logits(5, V, DT[dtype], V), numbers(5, V))
    check(logits(1, V, DT[dtype], V + 1), numbers(1, V + 1), temperature=0.6)
    ids, _ = draw(z := logits(3, V, DT[dtype], V + 2), numbers(3, 1), temperature=0.0)
    assert np.array_equal(ids, [int(np.argmax(r)) for r in z.float().cpu().numpy()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(top_k=1), dict(top_k=50), dict(top_k=3000), dict(top_p=0.9), dict(top_p=0.37, temperature=0.7),
                                dict(min_p=0.05), dict(top_k=40, top_p=0.8), dict(top_k=2000, top_p=0.95, min_p=0.001, temperature=1.3),
                                dict(top_p=0.999999, temperature=3.0), dict(top_p=0.0), dict(min_p=1.0), dict(top_k=10 ** 9, top_p=5.0)])
def test_filters(kw, dtype):
    for V, rows in ((777, 9), (33001, 6)):
        check(logits(rows, V, DT[dtype], 3 * V, masked=0.2), numbers(rows, V), **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_full_vocabulary_and_a_row_each_its_own(dtype):
    B_, V = 37, 151936
    z = logits(B_, V, DT[dtype], 5, ld=V + 8, masked=0.1)
    g = torch.Generator().manual_seed(6)
    T = torch.where(torch.rand(B_, generator=g) < 0.2, 0.0, 0.3 + torch.rand(B_, generator=g)).cuda()
    k = torch.where(torch.rand(B_, generator=g) < 0.4, 0, torch.randint(1, 400, (B_,), generator=g)).to(torch.int32).cuda()
    p = torch.where(torch.rand(B_, generator=g) < 0.4, 1.0, 0.3 + 0.69 * torch.rand(B_, generator=g)).cuda()
    m = torch.where(torch.rand(B_, generator=g) < 0.5, 0.0, 0.2 * torch.rand(B_, generator=g)).cuda()
    ids = check(z, numbers(B_, 7), temperature=T, top_k=k, top_p=p, min_p=m)
    assert len(set(ids)) > 10
    check(z, numbers(B_, 8), temperature=0.8, top_k=k)                      # one setting a row, the others common


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_logits(dtype):
    """Ties at the cut go to the lower index; a plain of equal logits is one key with as many tokens as the row."""
    for V in (1000, 40000):
        z = torch.full((4, V), 1.5, dtype=DT[dtype]).cuda()
        z[:, 17] = 2.0
        for kw in (dict(), dict(top_k=5), dict(top_k=V - 3), dict(top_p=0.25), dict(top_p=0.75, top_k=V // 2), dict(min_p=0.99)):
            ids = check(z, numbers(4, V), **kw)
            if "top_k" in kw and kw["top_k"] == 5:
                assert set(ids) <= {0, 1, 2, 3, 17}
    z = (torch.randint(0, 3, (6, 30000), generator=torch.Generator().manual_seed(1)).float() * 0.5).to(DT[dtype]).cuda()
    for kw in (dict(top_k=25000), dict(top_k=10500), dict(top_p=0.6), dict(top_p=0.6, top_k=20001)):
        check(z, numbers(6, 2), **kw)


def test_far_apart_and_huge_logits():
    z = torch.zeros(6, 2001)
    z[0] = torch.linspace(-1, 1, 2001) * 3e38                 # differences beyond the fp32 range
    z[1], z[1, 5], z[1, 9] = torch.finfo(torch.float32).min, 1.0, 1.0
    z[2] = torch.finfo(torch.float32).min                    # a mask of the type's lowest value everywhere: all equal
    z[3] = torch.linspace(-80, 0, 2001)
    z[4] = -0.0
    z[4, ::2] = 0.0                                          # both zeros are one value
    z[5] = torch.linspace(-1e-3, 0, 2001)
    for kw in (dict(), dict(top_k=3), dict(top_k=1990), dict(top_p=0.5), dict(min_p=0.5), dict(temperature=1e-30), dict(temperature=1e4)):
        check(z.cuda(), numbers(6, 3), **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_token_and_bad_rows(dtype):
    inf, nan = float("inf"), float("nan")
    V = 5003
    z = logits(6, V, DT[dtype], 1)
    clean = z.clone()
    z[1] = -inf
    z[2, 4000] = nan
    z[3, V - 1] = inf
    z[4] = -inf
    z[4, 77] = -3.0
    for kw in (dict(), dict(top_k=20, top_p=0.9), dict(temperature=0.0)):
        ids, logp = draw(z, numbers(6, 2), expect_status=0x100, **kw)
        assert list(ids[1:4]) == [-1, -1, -1] and list(logp[1:4]) == [0, 0, 0] and ids[4] == 77 and logp[4] == 0
        good, _ = draw(clean, numbers(6, 2), **kw)
        assert ids[0] == good[0] and ids[5] == good[5]
    ids, _ = draw(torch.full((2, 9), -inf, device="cuda"), numbers(2, 0))           # a mask is no fault
    assert list(ids) == [-1, -1]
    T = torch.tensor([1.0, nan, -1.0, inf, 1.0, 1.0]).cuda()
    p = torch.tensor([1.0, 1.0, 1.0, 1.0, nan, 1.0]).cuda()
    m = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.0, -0.1]).cuda()
    ids, _ = draw(clean, numbers(6, 2), expect_status=0x100, temperature=T, top_p=p, min_p=m)
    assert ids[0] >= 0 and list(ids[1:]) == [-1] * 5


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_rows_on_any_boundary(offset):
    for dtype in (torch.bfloat16, torch.float32):
        for V in (40, 3001):
            flat = torch.zeros(4 * (V + offset) + offset, dtype=dtype, device="cuda")
            z = flat[offset:].as_strided((4, V), (V + offset, 1))
            z.copy_(logits(4, V, dtype, V))
            check(z, numbers(4, 1), top_k=30)
            check(z, numbers(4, 2))


def test_the_same_number_draws_the_same_token_and_frequencies_follow_the_weights():
    z = logits(1, 300, torch.float32, 9, scale=1.0).expand(20000, 300)
    seeds = numbers(20000, 4)
    a, _ = draw(z, seeds)
    b, _ = draw(z, seeds.flip(0))
    assert np.array_equal(a, b[::-1])
    p = torch.softmax(z[0].double(), 0).cpu().numpy()
    n = np.bincount(a, minlength=300)
    big = 20000 * p >= 10
    chi = ((n - 20000 * p) ** 2 / (20000 * p))[big].sum()
    k = big.sum()
    assert abs(chi - k) < 6 * np.sqrt(2 * k)                 # mean k, deviation sqrt(2 k)


def test_calls_at_once_on_two_streams_and_replayed():
    z, seeds = logits(8, 20000, torch.bfloat16, 2), numbers(8, 2).cuda()
    want = check(z, seeds.cpu(), top_p=0.9)
    outs = [(torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda"), B.new_status()) for _ in range(3)]
    torch.cuda.synchronize()
    for s, o in zip((torch.cuda.Stream(), torch.cuda.Stream()), outs):
        with torch.cuda.stream(s):
            for _ in range(20):
                B.sapo_sample(z, seeds, *o, top_p=0.9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sapo_sample(z, seeds, *outs[2], top_p=0.9)
    outs[2][0].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(np.array_equal(o[0].cpu().numpy(), want) for o in outs)
    other = numbers(8, 77)
    seeds.copy_(other.cuda())                                # a replayed call reads its random numbers anew
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(outs[2][0].cpu().numpy(), draw(z, other, top_p=0.9)[0])


def test_no_rows_and_the_widest_row():
    assert len(draw(torch.zeros(0, 10, device="cuda"), numbers(0, 0))[0]) == 0
    check(logits(2, 368504, torch.float32, 1), numbers(2, 5), top_k=100)
    with pytest.raises(B.SapoError):
        draw(torch.zeros(1, 368640, device="cuda"), numbers(1, 0))
