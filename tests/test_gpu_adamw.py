"""AdamW over many tensors on the device: the state to the bit, the weights against float64.

Weights: with u = 2^-24, the decay's factor and product 2 u |w|, the difference u |w'|, and the update.  Its numerator
b1 m + (1 - b1) g may cancel, so its roundings (two factors, two products, a sum) count against the terms: 4 u
(|b1 m| + |(1 - b1) g|), not against the sum.  Root (of v, whose terms do not cancel: 4 u, halved, and its own rounding), two
bias factors and their products, the division (2 ulp), lr and its product: 8 u more.  Together 12 u lr (|b1 m| + |(1 - b1) g|)
/ bias / denominator."""
import numpy as np
import pytest
import torch

from oracle import answer_oracle as ao
from paper_2509_08721_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SEED = 0xFEDCBA9876543210
SIZES = [1, 3, 127, 128, 129, 511, 512, 513, 4095, 4097, 30000]


def setup(sizes, bits, gdt, seed=0, off=0):
    g = torch.Generator().manual_seed(seed)
    put = lambda t: torch.cat([torch.zeros(off, dtype=t.dtype), t]).cuda()[off:]     # off: a boundary of one element
    params = [put(0.1 * torch.randn(n, generator=g)) for n in sizes]
    grads = [put((1e-3 * torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g))).to(gdt)) for n in sizes]
    states = []
    for n in sizes:
        m, v = 1e-3 * torch.randn(n, generator=g), (1e-3 * torch.randn(n, generator=g).abs() * torch.exp(torch.randn(n, generator=g))) ** 2
        v[::17] = 0
        if bits == 32:
            states.append(B.AdamWState(put(m), put(v)))
        else:
            c, sm, r, sr = ao.state8(m.numpy(), v.numpy(), 0, 0, 0)
            code = lambda a: put(torch.from_numpy(a)).view(torch.float8_e4m3fn)
            states.append(B.AdamWState(code(c), code(r), torch.from_numpy(sm).cuda(), torch.from_numpy(sr).cuda()))
    copies = [put(torch.zeros(n, dtype=torch.bfloat16)) for n in sizes]
    return params, grads, states, copies


def moments(st):
    """The moments that a state stands for, as the device forms them in fp32."""
    if st.m_scale is None:
        return st.m.cpu().numpy(), st.v.cpu().numpy()
    m = ao.held32(st.m.view(torch.uint8).cpu().numpy(), st.m_scale.cpu().numpy())
    r = ao.held32(st.v.view(torch.uint8).cpu().numpy(), st.v_scale.cpu().numpy())
    return m, r * r


def check(i, before, after, grad, step, lr, decay, factor=np.float32(1), number=None):
    w0, m0, v0 = before
    g = grad.float().cpu().numpy() * factor
    m1, v1 = ao.adamw_moments32(g, m0, v0)
    st, w1 = after.states[i], after.params[i].cpu().numpy().astype(np.float64)
    if st.m_scale is None:
        np.testing.assert_array_equal(st.m.cpu().numpy(), m1)
        np.testing.assert_array_equal(st.v.cpu().numpy(), v1)
    else:
        c, sm, r, sr = ao.state8(m1, v1, i if number is None else number, step, SEED)
        np.testing.assert_array_equal(st.m_scale.cpu().numpy(), sm)
        np.testing.assert_array_equal(st.v_scale.cpu().numpy(), sr)
        codes = st.m.view(torch.uint8).cpu().numpy()
        assert np.array_equal(codes & 127, c & 127) and np.array_equal(codes[(c & 127) > 0], c[(c & 127) > 0])
        np.testing.assert_array_equal(st.v.view(torch.uint8).cpu().numpy(), r)
    want = ao.adamw(w0, g, m0, v0, step, lr, decay=decay)
    root = np.sqrt(want["v"] / (1 - 0.999 ** step)) + 1e-8
    terms = (0.9 * np.abs(m0.astype(np.float64)) + 0.1 * np.abs(g.astype(np.float64))) / (1 - 0.9 ** step) / root
    tol = U * (2 * np.abs(w0) + np.abs(want["master"]) + 12 * lr * terms)
    assert np.all(np.abs(w1 - want["master"]) <= tol)
    if after.copies[i] is not None:
        assert torch.equal(after.copies[i], after.params[i].bfloat16())


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("gdt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_in_place(bits, gdt, off):
    params, grads, states, copies = setup(SIZES, bits, gdt, 1, off)
    T = B.AdamWTensors(params, states, copies)
    status = B.new_status()
    for step in (1, 2, 3, 900):
        before = [(p.cpu().numpy(), *moments(st)) for p, st in zip(params, states)]
        B.sapo_adamw_step(T, grads, step, 1e-2, status, weight_decay=0.1, seed=SEED)
        torch.cuda.synchronize()
        for i, b in enumerate(before):
            check(i, b, T, grads[i], step, 1e-2, 0.1)
    assert int(status.item()) == 0


def test_a_mixed_list_into_other_arrays_with_factors():
    sizes = [700, 64, 0, 1000, 5000, 896]
    parts = [setup([n], bits, gdt, n, off) for n, bits, gdt, off in zip(sizes, (8, 32, 8, 8, 32, 32), (torch.bfloat16, torch.float32) * 3, (0, 0, 0, 1, 1, 0))]
    params, grads, states, copies = ([p[k][0] for p in parts] for k in range(4))
    copies[1] = None
    new = [setup([n], bits, torch.float32, 9) for n, bits in zip(sizes, (8, 32, 8, 8, 32, 32))]
    lr_factor, decay = [1.0, 0.5, 1.0, 2.0, 1.0, 1.0], [0.1, 0.0, None, 0.3, None, 0.0]
    src = B.AdamWTensors(params, states, lr_factor=lr_factor, weight_decay=decay)
    dst = B.AdamWTensors([p[0][0] for p in new], [p[2][0] for p in new], copies)
    keep = [[t.clone() for t in src.arrays(i) if t is not None] for i in range(6)]
    clip, status = torch.tensor([0.37], device="cuda"), B.new_status()
    for _ in range(2):                                       # the same call again gives the same result
        B.sapo_adamw_step(src, grads, 5, 1e-3, status, weight_decay=0.2, seed=SEED, grad_scale=clip, out=dst)
    torch.cuda.synchronize()
    for i in range(6):
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(keep[i], (t for t in src.arrays(i) if t is not None)))
        check(i, (params[i].cpu().numpy(), *moments(states[i])), dst, grads[i], 5, 1e-3 * lr_factor[i],
              0.2 if decay[i] is None else decay[i], np.float32(0.37))


def test_more_tensors_than_a_launch_takes():
    sizes = [(37 * i) % 900 + 1 for i in range(77)]
    params, grads, states, _ = setup(sizes, 8, torch.float32, 3)
    T, status = B.AdamWTensors(params, states), B.new_status()
    before = [(p.cpu().numpy(), *moments(st)) for p, st in zip(params, states)]
    B.sapo_adamw_step(T, grads, 2, 1e-3, status, seed=SEED)
    torch.cuda.synchronize()
    for i in range(77):
        check(i, before[i], T, grads[i], 2, 1e-3, 0.01)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_finite_leave_their_elements(bits):
    params, grads, states, copies = setup([1000], bits, torch.float32, 5)
    clean = [t.clone() for t in (params[0], grads[0])]
    grads[0][3], grads[0][500], grads[0][999] = float("nan"), float("inf"), float("-inf")
    m0, v0 = moments(states[0])
    T, status = B.AdamWTensors(params, states, copies), B.new_status()
    B.sapo_adamw_step(T, grads, 4, 1e-2, status, seed=SEED)
    torch.cuda.synchronize()
    assert int(status.item()) == 0x100
    hit = ~torch.isfinite(grads[0]).cpu().numpy()
    m1, v1 = ao.adamw_moments32(clean[1].cpu().numpy(), m0, v0)
    m1[hit], v1[hit] = m0[hit], v0[hit]
    assert torch.equal(params[0][torch.from_numpy(hit).cuda()], clean[0][torch.from_numpy(hit).cuda()])
    if bits == 32:
        assert np.array_equal(states[0].m.cpu().numpy(), m1) and np.array_equal(states[0].v.cpu().numpy(), v1)
    else:
        c, sm, r, sr = ao.state8(m1, v1, 0, 4, SEED)
        assert np.array_equal(states[0].m_scale.cpu().numpy(), sm) and np.array_equal(states[0].v.view(torch.uint8).cpu().numpy(), r)


@pytest.mark.parametrize("bits", [32, 8])
def test_huge_and_tiny_gradients(bits):
    """Squares beyond the fp32 range stop at its end; groups of zeros and of the smallest numbers stay finite."""
    n = 128 * 5
    w, g = torch.full((n,), 0.5, device="cuda"), torch.zeros(n, device="cuda")
    g[128:256], g[256:384], g[384:400], g[512] = 1e30, 1e-30, 3e38, 1e-45
    T, status = B.AdamWTensors([w], [B.alloc_adamw_state(n, bits)]), B.new_status()
    for step in (1, 2, 3):
        before = w.cpu().numpy(), *moments(T.states[0])
        B.sapo_adamw_step(T, [g], step, 1e-3, status, seed=SEED, weight_decay=0.0)
        torch.cuda.synchronize()
        m1, v1 = ao.adamw_moments32(g.cpu().numpy(), before[1], before[2])
        if bits == 32:
            assert np.array_equal(T.states[0].m.cpu().numpy(), m1) and np.array_equal(T.states[0].v.cpu().numpy(), v1)
        else:
            c, sm, r, sr = ao.state8(m1, v1, 0, step, SEED)
            assert np.array_equal(T.states[0].m_scale.cpu().numpy(), sm) and np.array_equal(T.states[0].v_scale.cpu().numpy(), sr)
            assert np.array_equal(T.states[0].v.view(torch.uint8).cpu().numpy(), r)
        assert torch.isfinite(w).all()
    assert int(status.item()) == 0


def test_captured_steps_follow_the_counter_and_the_rate_on_the_device():
    sizes = [900, 5000]
    params, grads, states, copies = setup(sizes, 8, torch.bfloat16, 8)
    T, status = B.AdamWTensors(params, states, copies), B.new_status()
    step, lr = torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([0.0], device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        B.sapo_adamw_step(T, grads, step, lr, status, seed=SEED)
    for t in range(1, 5):
        before = [(p.cpu().numpy(), *moments(st)) for p, st in zip(params, states)]
        lr.fill_(1e-3 / t)
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            check(i, before[i], T, grads[i], t, float(np.float32(1e-3 / t)), 0.01)


def test_a_large_tensor():
    """Past 2^31 bytes of one array; only its ends and some places between are looked at."""
    n = (1 << 29) + 4321
    params, st = torch.full((n,), 0.25, device="cuda"), B.alloc_adamw_state(n, 8)
    grad = torch.full((n,), 1e-3, dtype=torch.bfloat16, device="cuda")
    grad[-1] = 0.5
    T, status = B.AdamWTensors([params], [st]), B.new_status()
    B.sapo_adamw_step(T, [grad], 1, 1e-2, status, weight_decay=0.0, seed=SEED)
    torch.cuda.synchronize()
    assert float((params[:-128] - (0.25 - 1e-2)).abs().max()) <= 1e-2 * 12 * U + 2 * U
    c = n // 128 * 128
    m1, v1 = ao.adamw_moments32(grad[c:].float().cpu().numpy(), np.zeros(n - c, np.float32), np.zeros(n - c, np.float32))
    part = np.float32(1) / np.float32(448)
    assert float(st.v_scale[-1]) == np.sqrt(v1).max() * part and float(st.m_scale[-1]) == np.abs(m1).max() * part
    assert int(status.item()) == 0


def test_no_tensors():
    B.sapo_adamw_step(B.AdamWTensors([], []), [], 1, 1e-3, B.new_status())
