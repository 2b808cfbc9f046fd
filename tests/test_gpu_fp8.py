"""8-bit floating point on the device: storing, to the code, and the product of two stored matrices against float64.

Product.  A product of two codes is exact in fp32.  The tensor cores add 128 of them, each addition (or the alignment of
its terms) off by at most 2^-23 of the sum of magnitudes: 128 2^-23 sum |x w|; the scales' product and the fp32 sum over n
blocks add (n + 3) 2^-24 of it.  The output lies between the roundings of both ends of that interval."""
import numpy as np
import pytest
import torch

from oracle import answer_oracle as ao
from paper_2509_08721_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def values(R, C, dtype, seed, ld=None, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    full = torch.full((R, ld or C), float("nan"), dtype=dtype)
    full[:, :C] = (torch.randn(R, C, generator=g) * torch.exp(spread * torch.randn(R, C, generator=g))).to(dtype)
    return full.cuda()[:, :C]


def stored(x, blocks, out=None, expect_status=0):
    out = out or B.alloc_fp8(*x.shape, blocks)
    status = B.new_status()
    B.sapo_fp8_store(x, out, status)
    torch.cuda.synchronize()
    assert int(status.item()) == expect_status
    return out


def host(q):
    return q.data[:, :q.C].view(torch.uint8).cpu().numpy(), q.scale.cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("blocks", [False, True])
@pytest.mark.parametrize("R,C", [(1, 1), (3, 7), (1, 128), (2, 129), (127, 256), (128, 300), (129, 896), (300, 1001), (5, 4864), (1000, 130)])
def test_store_to_the_code(R, C, blocks, dtype):
    x = values(R, C, DT[dtype], R + C)
    if R > 2:
        x[1] = 0                                    # a row of zeros: scale 0
        x[2, :min(C, 128)] = 1e-37                  # below the smallest group
    codes, scale = host(stored(x, blocks))
    want_codes, want_scale = ao.fp8_store(x.float().cpu().numpy(), blocks)
    np.testing.assert_array_equal(scale, want_scale)
    np.testing.assert_array_equal(codes & 127, want_codes & 127)
    assert np.array_equal(codes[(codes & 127) > 0], want_codes[(codes & 127) > 0])        # (the sign of a zero is free)


def test_store_pitches_boundaries_and_what_lies_between_the_rows():
    for blocks in (False, True):
        for dtype, off in ((torch.bfloat16, 1), (torch.float32, 3)):
            flat = values(1, 60 * 530 + off, dtype, 5)[0]
            x = flat[off:].as_strided((60, 517), (523, 1))
            n = 1 if blocks else 60
            data = torch.full((60, 531), 0x33, dtype=torch.uint8, device="cuda")
            scale = torch.full((n, 9), 5.0, device="cuda")
            q = B.Fp8(data.view(torch.float8_e4m3fn)[:, 1:518], scale[:, 2:7], 517, blocks)
            codes, s = host(stored(x, blocks, q))
            want = ao.fp8_store(x.float().cpu().numpy(), blocks)
            assert np.array_equal(codes & 127, want[0] & 127) and np.array_equal(s, want[1])
            assert (data[:, 0] == 0x33).all() and (data[:, 518:] == 0x33).all() and (scale[:, :2] == 5).all() and (scale[:, 7:] == 5).all()


@pytest.mark.parametrize("blocks", [False, True])
def test_store_of_what_is_not_finite(blocks):
    x = values(200, 400, torch.float32, 1)
    x[5, 130], x[150, 399] = float("nan"), float("-inf")
    codes, scale = host(stored(x, blocks, expect_status=0x100))
    want_codes, want_scale = ao.fp8_store(x.cpu().numpy(), blocks)
    np.testing.assert_array_equal(scale, want_scale)
    assert np.isnan(scale).sum() == 2 and np.array_equal(codes & 127, want_codes & 127)


def product(T, N, K, ydt, seed=0, ld_y=None, x=None, w=None):
    x = stored(values(T, K, torch.bfloat16, seed), False) if x is None else x
    w = stored(values(N, K, torch.bfloat16, seed + 1), True) if w is None else w
    full = torch.full((T, ld_y or N), 9.0, dtype=DT[ydt], device="cuda")
    y, status = full[:, :N], B.new_status()
    B.sapo_fp8_matmul(x, w, y, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert (full[:, N:] == 9).all()
    return x, w, y


def check_product(x, w, y):
    K = x.C
    X, W = (torch.from_numpy(ao.fp8_values(*host(m), m.blocks)).cuda() for m in (x, w))
    want, size = X @ W.T, X.abs() @ W.abs().T
    tol = size * (128 * 2.0 ** -23 + (-(-K // 128) + 3) * 2.0 ** -24)
    lo, hi = (v.to(y.dtype).double() for v in (want - tol, want + tol))
    bad = ~((y.double() >= lo) & (y.double() <= hi))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


SIZES = [(1, 1, 1), (1, 128, 128), (1, 1000, 200), (2, 130, 896), (16, 300, 129), (17, 257, 1000), (33, 4864, 256), (64, 1001, 3584),
         (65, 640, 640), (128, 3000, 130), (129, 700, 512), (200, 128, 4000), (300, 9600, 300), (700, 4001, 384), (1500, 2048, 896), (1024, 2500, 100)]


@pytest.mark.parametrize("ydt", ["bf16", "f32"])
@pytest.mark.parametrize("T,N,K", SIZES)
def test_product(T, N, K, ydt):
    check_product(*product(T, N, K, ydt, seed=T + N))
    if T > 1:
        check_product(*product(T, N, K, ydt, seed=T, ld_y=N + 5))


def test_product_of_the_head():
    for T in (1, 40, 300):
        x, w, y = product(T, 20000, 896, "f32", seed=T)
        check_product(x, w, y)


def test_product_where_blocks_differ_by_far():
    """Scales from 1e-30 to 1e30: each block's product is scaled by itself."""
    x, w = B.alloc_fp8(200, 1024), B.alloc_fp8(5000, 1024, True)
    g = torch.Generator().manual_seed(3)
    for m in (x, w):
        m.data.copy_(torch.randn(m.data.shape, generator=g).clamp(-4, 4).cuda().to(torch.float8_e4m3fn))
        m.scale.copy_(10.0 ** (30 * torch.rand(m.scale.shape, generator=g) - 15))
    for T in (200, 30):
        xs = B.Fp8(x.data[:T], x.scale[:T], 1024)
        check_product(xs, w, product(T, 5000, 1024, "f32", x=xs, w=w)[2])


@pytest.mark.parametrize("T", [1, 40, 400])
def test_nan_scales_reach_the_rows_and_columns_that_use_them(T):
    x, w, y = product(T, 6000, 512, "f32")
    good = y.clone()
    x.scale[0, 1], w.scale[2, 3] = float("nan"), float("nan")
    _, _, y = product(T, 6000, 512, "f32", x=x, w=w)
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[0], hit[:, 256:384] = True, True
    assert torch.equal(torch.isnan(y), hit) and torch.equal(y[~hit], good[~hit])


def test_codes_behind_the_last_column_are_not_read():
    for T in (3, 300):
        x, w, y = product(T, 9600, 200, "f32")
        x.data.view(torch.uint8)[:, 200:] = 0x7F              # NaN
        w.data.view(torch.uint8)[:, 200:] = 0x7F
        assert torch.equal(product(T, 9600, 200, "f32", x=x, w=w)[2], y)


def test_same_bits_again_on_two_streams_and_replayed():
    for T, N, K in ((4, 500, 4096), (50, 30000, 256), (600, 5000, 1024)):
        x, w, y = product(T, N, K, "bf16")
        outs = [torch.zeros_like(y) for _ in range(3)]
        st = [B.new_status() for _ in range(3)]
        torch.cuda.synchronize()
        for s, o, f in zip((torch.cuda.Stream(), torch.cuda.Stream()), outs, st):
            with torch.cuda.stream(s):
                for _ in range(10):
                    B.sapo_fp8_matmul(x, w, o, f)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.sapo_fp8_matmul(x, w, outs[2], st[2])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, y) for o in outs) and not any(int(f.item()) for f in st)


def test_no_rows():
    w = B.alloc_fp8(300, 64, True)
    product(0, 300, 64, "f32", x=B.alloc_fp8(0, 64), w=w)
    stored(torch.zeros(0, 64, device="cuda"), False)
