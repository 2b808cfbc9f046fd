"""The binding refuses arrays that a kernel would read or write out of range, before it calls the library: run here on
host tensors that say they are on the GPU, with a library that only counts its calls."""
import pytest
import torch

from paper_2509_08721_b200 import binding as B


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(t):
    return t.as_subclass(OnGpu)


class Library:
    """Every entry point succeeds and is counted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append(name)
            return 0
        return entry


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B, "_require_cuda", lambda: None)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    return lib


def refuses(lib, call):
    before = len(lib.calls)
    with pytest.raises(B.SapoError):
        call()
    assert len(lib.calls) == before


T, S, Q, H, V = 12, 3, 2, 64, 128
f = lambda *n, dt=torch.float32: gpu(torch.zeros(*n, dtype=dt))
i = lambda *n: f(*n, dt=torch.int32)


def outputs(scores):
    return {k: gpu(v) for k, v in B.alloc_preference_outputs(T, S, Q, device="cpu", scores=scores).items()}


def head_arguments():
    return dict(hidden=f(T, H, dt=torch.bfloat16), W=f(V, H, dt=torch.bfloat16), dhidden=f(T, H), dW=f(V, H),
                ws=f(64, dt=torch.uint8))


def preference(out, status, through_head, **changed):
    """One of the two preference calls; `changed` replaces arguments of the call through the head."""
    if not through_head:
        return B.sapo_preference_loss(f(T), f(T), i(S + 1), f(S), i(Q + 1), 0.1, out, status)
    a = dict(head_arguments(), **changed)
    B.sapo_preference_loss_fwd_bwd(a["hidden"], a["W"], i(T), f(T), i(S + 1), f(S), i(Q + 1), 0.1, out, a["dhidden"], a["dW"],
                                   False, a["ws"], status)


@pytest.mark.parametrize("through_head", [False, True])
def test_preference_outputs_of_the_wrong_length_type_or_place(lib, through_head):
    good = outputs(through_head)
    preference(good, i(1), through_head)
    assert len(lib.calls) == 1
    without = {k: v for k, v in good.items() if k not in ("q_margin", "q_pairs")}        # both are optional
    preference(without, i(1), through_head)
    assert len(lib.calls) == 2
    for key, t in good.items():
        wrong = [t[:-1], t.double(), torch.zeros(len(t), dtype=t.dtype), gpu(torch.zeros(2 * len(t), dtype=t.dtype))[::2]]
        for bad in wrong:
            if bad.is_contiguous() and bad.dtype == t.dtype and bad.is_cuda and len(bad) == len(t):
                continue                                                                  # every other of one element
            refuses(lib, lambda: preference(dict(good, **{key: bad}), i(1), through_head))
    for bad in (i(0), f(1), torch.zeros(1, dtype=torch.int32)):
        refuses(lib, lambda: preference(good, bad, through_head))


@pytest.mark.parametrize("through_head", [False, True])
def test_allocated_outputs_are_checked_once_an_entry_changes(lib, through_head):
    """What alloc_preference_outputs made is only asked for its lengths, until an entry is replaced."""
    def fresh():
        out = B.alloc_preference_outputs(T, S, Q, device="cpu", scores=through_head)
        for k in list(out):
            out[k] = gpu(out[k])
        out.known = tuple(out[k] for k in B._PREF_OUTPUTS)                                # as if they were on the GPU
        return out
    preference(fresh(), i(1), through_head)
    assert lib.calls
    for key in ("gscale", "seq_logratio", "seq_grad", "q_loss", "q_margin", "q_pairs", "loss"):
        out = fresh()
        out[key].resize_(0)
        refuses(lib, lambda: preference(out, i(1), through_head))
        bad = fresh()[key].double()
        for put in (lambda o: o.__setitem__(key, bad), lambda o: o.update({key: bad}), lambda o: o.__ior__({key: bad}),
                    lambda o: (o.pop(key), o.setdefault(key, bad))):
            out = fresh()
            put(out)
            refuses(lib, lambda: preference(out, i(1), through_head))
    out = fresh()
    del out["q_margin"]                                                                   # not asked for any more
    preference(out, i(1), through_head)
    del out["loss"]
    refuses(lib, lambda: preference(out, i(1), through_head))
    out = B.alloc_preference_outputs(T, S, Q, device="cpu", scores=through_head)          # on the host
    refuses(lib, lambda: preference(out, i(1), through_head))


def test_head_operands_with_gaps_between_columns_or_on_the_host(lib):
    good = outputs(True)
    preference(good, i(1), True)
    bf = torch.bfloat16
    for change in (dict(hidden=f(T, 2 * H, dt=bf)[:, ::2]), dict(W=f(V, 2 * H, dt=bf)[:, ::2]), dict(hidden=torch.zeros(T, H, dtype=bf)),
                   dict(W=torch.zeros(V, H, dtype=bf)), dict(dhidden=torch.zeros(T, H)), dict(dW=torch.zeros(V, H))):
        refuses(lib, lambda: preference(good, i(1), True, **change))
    preference(good, i(1), True, hidden=f(T, 2 * H, dt=bf)[:, :H], W=f(V, 2 * H, dt=bf)[:, H:])      # a pitch is fine


def test_checkpoints_with_overlapping_rows_or_on_the_host(lib):
    x, st = f(T, H, dt=torch.bfloat16), i(1)
    data, scale = f(T, H, dt=torch.int8), f(T, 1)
    calls = (lambda c: B.sapo_ckpt8_store(x, c, st), lambda c: B.sapo_ckpt8_restore(c, x),
             lambda c: B.sapo_norm_fwd(x, None, None, 1e-6, "rms", x, None, None, c, st),
             lambda c: B.sapo_norm_bwd(x, c, None, None, f(T), "rms", x, None, None, None),
             lambda c: B.sapo_norm_replay(c, None, None, "rms", None, f(T), x))
    for call in calls:
        call(B.Ckpt8(data, scale, H))
    assert len(lib.calls) == 5
    one_row, one_scale = f(1, H, dt=torch.int8).expand(T, H), f(1, 1).expand(T, 1)
    for bad in (B.Ckpt8(one_row, scale, H), B.Ckpt8(f(2 * T * H, dt=torch.int8).as_strided((T, H), (H // 2, 1)), scale, H),
                B.Ckpt8(data, one_scale, H), B.Ckpt8(torch.zeros(T, H, dtype=torch.int8), scale, H), B.Ckpt8(data, torch.zeros(T, 1), H)):
        for call in calls:
            refuses(lib, lambda: call(bad))
    one = B.Ckpt8(f(1, H, dt=torch.int8).expand(1, H), f(1, 1), H)                        # a single row has no pitch
    B.sapo_ckpt8_restore(one, f(1, H))


def test_workspaces_and_status_words_that_are_not_on_the_gpu(lib):
    x, c = f(T, H, dt=torch.bfloat16), B.Ckpt8(f(T, H, dt=torch.int8), f(T, 1), H)
    back = lambda ws: B.sapo_norm_bwd(x, x, None, None, f(T), "rms", x, f(H), None, ws)
    head = lambda ws: preference(outputs(True), i(1), True, ws=ws)
    for call in (back, head):
        call(f(64, dt=torch.uint8))
        for bad in (torch.zeros(64, dtype=torch.uint8), f(64, dt=torch.uint8)[::2]):
            refuses(lib, lambda: call(bad))
    back(None)                                                    # the library says whether it needs one
    for call in (lambda st: B.sapo_norm_fwd(x, None, None, 1e-6, "rms", x, None, None, c, st), lambda st: B.sapo_ckpt8_store(x, c, st)):
        call(i(1))
        for bad in (None, i(0), f(1), torch.zeros(1, dtype=torch.int32)):
            refuses(lib, lambda: call(bad))
    B.sapo_norm_fwd(x, None, None, 1e-6, "rms", x, None, None)    # without a checkpoint the status is not used
