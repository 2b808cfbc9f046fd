"""What the binding and the library refuse of the calls that answer and update, before anything is launched: run here on
host tensors that say they are on the GPU (as in test_binding_refusals.py), and on the C entries themselves."""
import pytest
import torch

from paper_2509_08721_b200 import binding as B
from tests.test_binding_refusals import f, gpu, i, lib, refuses  # noqa: F401 (lib is a fixture)

i64 = lambda *n: f(*n, dt=torch.int64)
f8 = lambda *n: gpu(torch.zeros(*n, dtype=torch.uint8).view(torch.float8_e4m3fn))


def fp8(R, K, blocks, **changed):
    a = dict(data=f8(R, -(-K // 16) * 16), scale=f(-(-R // 128) if blocks else R, -(-K // 128)), C=K, blocks=blocks)
    return B.Fp8(**{**a, **changed})


def test_sample_arguments(lib):  # noqa: F811
    good = dict(logits=f(4, 50), seeds=i64(4), ids=i(4), logp=f(4), status=i(1))
    B.sapo_sample(**good)
    B.sapo_sample(**good, temperature=f(4), top_k=i(4), top_p=f(4), min_p=f(4))
    B.sapo_sample(**{**good, "logits": f(1, 50).expand(4, 50)}, top_k=3, temperature=0)
    assert len(lib.calls) == 3
    for change in (dict(logits=torch.zeros(4, 50)), dict(logits=f(4, 100)[:, ::2]), dict(logits=f(4, 50, dt=torch.float16)),
                   dict(seeds=i64(3)), dict(seeds=i(4)), dict(seeds=torch.zeros(4, dtype=torch.int64)), dict(ids=i(3)), dict(ids=i64(4)),
                   dict(logp=f(3)), dict(logp=f(4, dt=torch.bfloat16)), dict(status=i(0)), dict(status=None),
                   dict(temperature=-0.1), dict(temperature=float("nan")), dict(min_p=1.5), dict(min_p=-0.1), dict(top_p=float("nan")),
                   dict(temperature=f(3)), dict(top_k=f(4)), dict(top_k=i64(4)), dict(top_p=f(8)[::2]), dict(min_p=torch.zeros(4))):
        refuses(lib, lambda: B.sapo_sample(**{**good, **change}))


def test_fp8_arguments(lib):  # noqa: F811
    st = i(1)
    B.sapo_fp8_store(f(5, 200), fp8(5, 200, False), st)
    B.sapo_fp8_store(f(300, 200, dt=torch.bfloat16), fp8(300, 200, True), st)
    B.sapo_fp8_matmul(fp8(5, 200, False), fp8(300, 200, True), f(5, 300), st)
    assert len(lib.calls) == 3
    bad = (fp8(4, 200, False), fp8(5, 199, False), fp8(5, 200, False, data=torch.zeros(5, 208, dtype=torch.uint8).view(torch.float8_e4m3fn)),
           fp8(5, 200, False, data=f(5, 208)), fp8(5, 200, False, data=f8(5, 192)), fp8(5, 200, False, data=f8(5, 416)[:, ::2]),
           fp8(5, 200, False, data=f8(1, 208).expand(5, 208)), fp8(5, 200, False, scale=f(5, 1)), fp8(5, 200, False, scale=f(4, 2)),
           fp8(5, 200, False, scale=torch.zeros(5, 2)), fp8(5, 200, False, scale=f(5, 2, dt=torch.bfloat16)),
           fp8(5, 200, False, scale=f(5, 4)[:, ::2]), fp8(5, 200, False, scale=f(1, 2).expand(5, 2)), fp8(5, 200, False, scale=f(10)))
    for q in bad:
        refuses(lib, lambda: B.sapo_fp8_store(f(5, 200), q, st))
        if q.data.shape[0] == 5 and q.C == 200:
            refuses(lib, lambda: B.sapo_fp8_matmul(q, fp8(300, 200, True), f(5, 300), st))
    for x, w, y in ((fp8(5, 200, True), fp8(300, 200, True), f(5, 300)), (fp8(5, 200, False), fp8(300, 200, False), f(5, 300)),
                    (fp8(5, 200, False), fp8(300, 100, True), f(5, 300)), (fp8(5, 200, False), fp8(300, 200, True), f(5, 299)),
                    (fp8(5, 200, False), fp8(300, 200, True), f(4, 300)), (fp8(5, 200, False), fp8(300, 200, True), torch.zeros(5, 300)),
                    (fp8(5, 200, False), fp8(300, 200, True), f(1, 300).expand(5, 300)), (fp8(5, 200, False), fp8(300, 200, True), f(5, 600)[:, ::2])):
        refuses(lib, lambda: B.sapo_fp8_matmul(x, w, y, st))
    for q in (None, i(0), f(1)):
        refuses(lib, lambda: B.sapo_fp8_store(f(5, 200), fp8(5, 200, False), q))
        refuses(lib, lambda: B.sapo_fp8_matmul(fp8(5, 200, False), fp8(300, 200, True), f(5, 300), q))


def state(n, bits):
    if bits == 32:
        return B.AdamWState(f(n), f(n))
    return B.AdamWState(f8(n), f8(n), f(-(-n // 128)), f(-(-n // 128)))


def test_adamw_arguments(lib):  # noqa: F811
    T = B.AdamWTensors([f(200), f(3, 5)], [state(200, 8), state(15, 32)], [f(200, dt=torch.bfloat16), None], 1.0, [0.1, None])
    grads, st = [f(200), f(3, 5, dt=torch.bfloat16)], i(1)
    B.sapo_adamw_step(T, grads, 1, 1e-3, st)
    B.sapo_adamw_step(T, grads, i(1), f(1), st, grad_scale=f(1), out=T)
    assert len(lib.calls) == 2
    for bad in ([grads[0]], [f(199), grads[1]], [f(200, dt=torch.float16), grads[1]], [torch.zeros(200), grads[1]], [f(400)[::2], grads[1]]):
        refuses(lib, lambda: B.sapo_adamw_step(T, bad, 1, 1e-3, st))
    for kw in (dict(step=f(1)), dict(lr=i(1)), dict(grad_scale=f(0)), dict(grad_scale=torch.zeros(1)), dict(status=None),
               dict(out=B.AdamWTensors([f(200), f(15)], [state(200, 32), state(15, 32)])),
               dict(out=B.AdamWTensors([f(201), f(15)], [state(201, 8), state(15, 32)]))):
        refuses(lib, lambda: B.sapo_adamw_step(T, grads, **{**dict(step=1, lr=1e-3, status=st), **kw}))
    one = lambda p, s, **kw: B.AdamWTensors([p], [s], **kw)
    good = state(200, 8)
    for call in (lambda: one(f(200, dt=torch.bfloat16), good), lambda: one(f(400)[::2], good), lambda: one(torch.zeros(200), good),
                 lambda: one(f(201), good), lambda: one(f(200), B.AdamWState(good.m, good.v)), lambda: one(f(200), B.AdamWState(good.m, f(200), good.m_scale, good.v_scale)),
                 lambda: one(f(200), B.AdamWState(good.m, good.v, f(1), good.v_scale)), lambda: one(f(200), good, copies=[f(200)]),
                 lambda: one(f(200), good, copies=[f(199, dt=torch.bfloat16)]), lambda: B.AdamWTensors([f(200)], []),
                 lambda: one(f(200), good, lr_factor=[1.0, 1.0]), lambda: B.alloc_adamw_state(4, 16, "cpu")):
        refuses(lib, call)


def test_tensors_of_another_device(lib, monkeypatch):  # noqa: F811
    """Every tensor of a call is on the device whose stream the kernel goes to."""
    class OnSecond(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 1
    there = lambda t: t.as_subclass(OnSecond)
    monkeypatch.setattr(B, "_raw_device", lambda: 0)
    st = i(1)
    good = dict(logits=f(4, 50), seeds=i64(4), ids=i(4), logp=f(4), status=st, top_p=f(4))
    for k, t in good.items():
        refuses(lib, lambda: B.sapo_sample(**{**good, k: there(t)}))
    refuses(lib, lambda: B.sapo_sample(**{k: there(t) for k, t in good.items()}))          # all on the second, the first is current
    refuses(lib, lambda: B.sapo_fp8_store(there(f(5, 200)), fp8(5, 200, False), st))
    for part in ("data", "scale"):
        q = fp8(5, 200, False)
        setattr(q, part, there(getattr(q, part)))
        refuses(lib, lambda: B.sapo_fp8_store(f(5, 200), q, st))
        refuses(lib, lambda: B.sapo_fp8_matmul(q, fp8(300, 200, True), f(5, 300), st))
    refuses(lib, lambda: B.sapo_fp8_matmul(fp8(5, 200, False), fp8(300, 200, True), there(f(5, 300)), st))
    T = B.AdamWTensors([f(200)], [state(200, 8)])
    refuses(lib, lambda: B.sapo_adamw_step(T, [there(f(200))], 1, 1e-3, st))
    refuses(lib, lambda: B.sapo_adamw_step(T, [f(200)], 1, 1e-3, st, out=B.AdamWTensors([there(f(200))], [state(200, 8)])))
    refuses(lib, lambda: B.sapo_adamw_step(T, [f(200)], there(i(1)), 1e-3, st))
    refuses(lib, lambda: B.AdamWTensors([f(200)], [B.AdamWState(f(200), there(f(200)))]))


X = 0x1000        # any address on a 16-byte boundary: nothing reads it on the host
INVALID, SHAPE = -1, -2


def test_the_sample_entry_refuses():
    lib = B.load()  # noqa: F811

    def call(z=X, dt=1, B_=2, V=100, ld=100, seeds=X, cfg=B.SampleCfgC(1.0, 0, 1.0, 0.0), ids=X, logp=X, status=X):
        return lib.sapo_sample(z, dt, B_, V, ld, seeds, cfg, ids, logp, status, None)
    assert call(B_=0) == 0 and call(B_=0, z=None, seeds=None, ids=None, logp=None) == 0
    for kw in (dict(z=None), dict(seeds=None), dict(ids=None), dict(logp=None), dict(status=None), dict(cfg=None), dict(dt=2), dict(B_=-1), dict(V=0),
               dict(ld=-1), dict(z=X + 2), dict(cfg=B.SampleCfgC(-1.0, 0, 1.0, 0.0)), dict(cfg=B.SampleCfgC(float("nan"), 0, 1.0, 0.0)),
               dict(cfg=B.SampleCfgC(float("inf"), 0, 1.0, 0.0)), dict(cfg=B.SampleCfgC(1.0, 0, float("nan"), 0.0)), dict(cfg=B.SampleCfgC(1.0, 0, 1.0, -1.0))):
        assert call(**kw) == INVALID, kw
    assert call(V=400000, ld=400000) == SHAPE


def test_the_fp8_entries_refuse():
    lib = B.load()  # noqa: F811
    q = lambda blocks=0, data=X, scale=X, ld=208, ld_scale=2: B.Fp8C(data, scale, ld, ld_scale, blocks)

    def store(x=X, dt=0, R=4, C_=200, ld=200, out=q(), status=X):
        return lib.sapo_fp8_store(x, dt, R, C_, ld, out, status, None)
    assert store(R=0, x=None) == 0
    for kw in (dict(x=None), dict(x=X + 1), dict(dt=3), dict(R=-1), dict(C_=0), dict(ld=199), dict(out=None), dict(status=None), dict(out=q(data=None)),
               dict(out=q(scale=None)), dict(out=q(ld=199)), dict(out=q(ld_scale=1)), dict(out=q(2)), dict(out=q(scale=X + 2))):
        assert store(**kw) == INVALID, kw

    def product(x=q(), T=5, w=q(1), N=300, K=200, y=X, dt=1, ld=300, status=X):
        return lib.sapo_fp8_matmul(x, T, w, N, K, y, dt, ld, status, None)
    assert product(T=0, y=None) == 0
    for kw in (dict(x=None), dict(w=None), dict(T=-1), dict(N=0), dict(K=0), dict(y=None), dict(y=X + 2), dict(dt=9), dict(ld=299), dict(status=None),
               dict(x=q(1)), dict(w=q(0)), dict(x=q(data=X + 8)), dict(w=q(1, data=X + 1)), dict(x=q(ld=200)), dict(w=q(1, ld=201)), dict(w=q(1, ld_scale=1)),
               dict(x=q(scale=None)), dict(x=q(data=None))):
        assert product(**kw) == INVALID, kw


def test_the_adamw_entry_refuses():
    lib = B.load()  # noqa: F811
    names = ("master", "master_out", "grad", "m", "v", "m_out", "v_out", "m_scale", "v_scale", "m_scale_out", "v_scale_out", "copy_bf16")

    def call(cfg=None, n=1, status=X, tensors=True, **changed):
        t = dict({k: X for k in names}, n=100, lr_factor=1.0, weight_decay=0.0, grad_dtype=1, state_bits=8)
        t.update(changed)
        c = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, step=1)
        c.update(cfg or {})
        return lib.sapo_adamw_step((B.AdamWTensorC * 1)(B.AdamWTensorC(**t)) if tensors else None, n, B.AdamWCfgC(**c), status, None)
    for k in names[:-1]:
        assert call(**{k: None}) == INVALID, k
    for kw in (dict(n=-1), dict(status=None), dict(tensors=False), dict(state_bits=16), dict(grad_dtype=5), dict(master=X + 2), dict(grad=X + 2),
               dict(grad_dtype=0, grad=X + 1), dict(state_bits=32, m=X + 1), dict(copy_bf16=X + 1), dict(weight_decay=float("nan")),
               dict(lr_factor=float("inf")), dict(cfg=dict(beta1=1.0)), dict(cfg=dict(beta2=-0.1)), dict(cfg=dict(eps=-1.0)), dict(cfg=dict(eps=float("nan"))),
               dict(cfg=dict(lr=float("nan"))), dict(cfg=dict(step=0))):
        assert call(**kw) == INVALID, kw
    c = B.AdamWTensorC(n=-1, state_bits=8, grad_dtype=1)
    assert lib.sapo_adamw_step((B.AdamWTensorC * 1)(c), 1, B.AdamWCfgC(lr=0.1, beta1=0.9, beta2=0.9, eps=0.0, step=1), X, None) == INVALID


def test_the_sample_entry_refuses_rows_of_too_many_tokens():
    lib = B.load()  # noqa: F811
    call = lambda V, dt: lib.sapo_sample(X, dt, 1, V, V, X, B.SampleCfgC(1.0, 0, 1.0, 0.0), X, X, X, None)
    assert call(1 << 19, B.DTYPE_BF16) == SHAPE and call(369000, B.DTYPE_F32) == SHAPE


def test_a_top_k_beyond_32_bits_is_no_small_one(lib):  # noqa: F811
    assert B._sample_cfg(2, 1.0, 2 ** 32 + 5, 1.0, 0.0).top_k == 2 ** 31 - 1
