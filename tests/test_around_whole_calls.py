"""Norms, steps and adapters done whole in native code: plain calls return what the binding's Python returns, everything else is left to it before
anything is launched."""
import os

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_1804_02941_amd import binding as dab
from paper_1804_02941_amd import build

WHOLE = {"rms_norm": 6, "rms_norm_gradient": 7, "adapters": 7, "adapters_gradient": 11, "w4_adapters": 10, "adamw": 9, "state8_restore": 4}
DEV = "cuda:0"


@pytest.fixture(scope="module")
def call():
    if not (os.path.exists(dab.LIB_PATH) and os.path.exists(build.CALL)):
        build.build()
    return dab.native()


@pytest.mark.parametrize("name", WHOLE)
def test_what_is_not_plain_is_left_to_python(call, name):
    f, n = getattr(call, name), WHOLE[name]
    with pytest.raises(TypeError, match=f"takes {n} arguments"):
        f(*[None] * (n + 1))
    for x in (None, 3, 0.5, True, "x", (), torch.zeros(2, 64), torch.zeros(2, 3, 64), torch.zeros(2, 64, dtype=torch.int32), torch.zeros(2, 64, device="meta")):
        assert f(*[x] * n) is None


class Mode(TorchDispatchMode):
    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        return func(*args, **(kwargs or {}))


class Counted:
    """The native half, with the answers of one of its calls noted; python: that call is left to Python."""

    def __init__(self, call, name):
        self.taken, self.python, whole = [], False, getattr(call, name)
        for k in dir(call):
            if not k.startswith("__"):
                setattr(self, k, getattr(call, k))
        setattr(self, name, lambda *a: self.taken.append(None if self.python else whole(*a)) or self.taken[-1])


def tensors(result):
    """The tensors of a result, in order, None among them."""
    return [t for r in result for t in tensors(r)] if isinstance(result, tuple) else [result]


def same(a, b):
    a, b = tensors(a), tensors(b)
    assert len(a) == len(b)
    for s, t in zip(a, b):
        if s is None or t is None:
            assert s is None and t is None
        else:
            assert s.shape == t.shape and s.dtype == t.dtype and s.device == t.device and s.stride() == t.stride() and torch.equal(s, t)


def _calls(dtype):
    """name -> [(call, outputs that it can be given, whether native code takes it)]"""
    g = torch.Generator(device=DEV).manual_seed(5)

    def normal(*shape, t=dtype):
        return torch.randn(shape, generator=g, device=DEV).to(t)

    def wide(t):
        out = torch.full((t.shape[0], t.shape[1] + 5), float("nan"), dtype=t.dtype, device=DEV)
        out[:, :t.shape[1]] = t
        return out[:, :t.shape[1]]
    f32 = torch.float32
    x, r, gain, dy, dh = normal(37, 203), normal(37, 203), normal(203, t=f32), normal(37, 203), normal(37, 203)
    _, h, rstd, _ = dab.dab_rms_norm(x, gain, r)
    many = normal(700, 203)
    some = torch.rand(700, generator=g, device=DEV)
    T, K, F, n, rank = 90, 45, 83, 3, 6
    X, A, B, dY, base, dbase = normal(T, K), normal(n, rank, K), normal(n, rank, F), normal(T, F), normal(T, F), normal(T, K)
    scale, ids = 0.5 + torch.rand(n, generator=g, device=DEV), torch.randint(-1, n, (T,), generator=g, device=DEV).int()
    _, U = dab.dab_adapters(X, ids, A, B, scale)
    Q, S = dab.dab_w4_pack(normal(F, K, t=f32))
    q, s = dab.dab_state8_save(normal(100, t=f32), True)
    norm, grad, forward, backward, served = dab.dab_rms_norm, dab.dab_rms_norm_gradient, dab.dab_adapters, dab.dab_adapters_gradient, dab.dab_w4_adapters
    return {
        "rms_norm": [(lambda **k: norm(x, gain, **k), "Y-r-", True), (lambda **k: norm(wide(x), gain, wide(r), 1e-3, True, **k), "YHrs", True),
                     (lambda **k: norm(x, gain, r, eps=1e-6, **k), "YHr-", True), (lambda **k: norm(x, gain, r, save="only", **k), "-Hrs", False),
                     (lambda **k: norm(x, gain, eps=1, **k), "Y-r-", False)],
        "rms_norm_gradient": [(lambda **k: grad(dy, h, gain, rstd, **k), "yy", True), (lambda **k: grad(wide(dy), wide(h), gain, rstd, wide(dh), **k), "yy", True),
                              (lambda **k: grad(many, many, gain, some, many, **k), "yy", True)],
        "adapters": [(lambda **k: forward(X, ids, A, B, **k), "yy", True), (lambda **k: forward(wide(X), ids, A, B, scale, wide(base), **k), "yy", True),
                     (lambda **k: forward(X[:5], ids[:5], A, B, scale, base[:5].float(), **k), "yy", True)],
        "adapters_gradient": [(lambda **k: backward(dY, X, U, ids, A, B, **k), "yyy", True),
                              (lambda **k: backward(wide(dY), wide(X), U, ids, A, B, scale, wide(dbase), **k), "yyy", True),
                              (lambda **k: backward(dY, X, U, ids, A, B, scale, dbase.float(), **k), "yyy", True),
                              (lambda **k: backward(dY, X, U, ids, A, B, scale, want_dX=False, **k), "-yy", True)],
        "w4_adapters": [(lambda **k: served(X, Q, S, F, ids, A, B, **k), "", True), (lambda **k: served(wide(X[:7]), Q, S, F, ids[:7], A, B, scale, **k), "", True)],
        "state8_restore": [(lambda **k: dab.dab_state8_restore(q, s, True, dtype, **k), "", True), (lambda **k: dab.dab_state8_restore(q, s, False, dtype, **k), "", True),
                           (lambda **k: dab.dab_state8_restore(q, s, True, dtype, n=100, **k), "", None)],
    }


def given(result, kinds):
    """Outputs of a result's shapes, to write into: one tensor, or a tuple with None where there is none to give."""
    if not kinds:
        return torch.zeros_like(result)
    return tuple(None if k == "-" else tuple(torch.zeros_like(t) for t in r) if k == "s" else torch.zeros_like(r) for k, r in zip(kinds, result))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name", [k for k in WHOLE if k != "adamw"])
def test_plain_calls_return_what_python_returns(call, name, dtype, monkeypatch):
    for k, (f, kinds, native) in enumerate(_calls(dtype)[name]):
        proxy = Counted(call, name)
        monkeypatch.setattr(dab, "_native", proxy)
        got = f()
        if native is not None:
            assert (proxy.taken[-1] is got) == native, k            # done whole, or left to Python
        out = given(got, kinds)
        done = f(out=out)
        same(done, got)
        for a, b in zip(tensors(out), tensors(done)):
            assert a is None or a is b
        with Mode():
            moded = f()
        assert not proxy.taken or proxy.taken[-1] is None or native is None           # a mode: left to Python
        same(moded, got)
        proxy.python = True
        same(f(), got)
        out = given(got, kinds)
        done = f(out=out)
        same(done, got)
        for a, b in zip(tensors(out), tensors(done)):
            assert a is None or a is b
        monkeypatch.setattr(dab, "_native", call)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_does_what_python_does(call, bits, monkeypatch):
    proxy = Counted(call, "adamw")
    monkeypatch.setattr(dab, "_native", proxy)
    one = {"lr": torch.full((1,), 0.01, device=DEV), "step": torch.full((1,), 3, dtype=torch.int64, device=DEV)}
    for kind, args in enumerate((dict(lr=0.01, step=3), dict(lr=1, step=1, beta1=0, eps=1e-6, seed=2 ** 40 + 1), one, dict(lr=0.01, step=3, seed=2 ** 63 + 1),
                                 dict(one, grad_scale=torch.full((1,), 0.25, device=DEV), seed=9))):
        sides = []
        for way in ("native", "python", "mode"):
            g = torch.Generator(device=DEV).manual_seed(kind)
            P, G = torch.randn(3001, generator=g, device=DEV), torch.randn(3001, generator=g, device=DEV).bfloat16()
            M, V = dab.adamw_states(P, bits)
            jobs = dab.adamw_jobs([{"P": P, "G": G, "M": M, "V": V, "weight_decay": 0.1}])
            proxy.python = way == "python"
            for _ in range(2):
                if way == "mode":
                    with Mode():
                        dab.dab_adamw(jobs, **args)
                else:
                    dab.dab_adamw(jobs, **args)
            # (a seed that a signed number does not hold is left to Python)
            assert bool(proxy.taken[-1]) == (way == "native" and args.get("seed", 0) < 2 ** 63)
            sides.append((P, M, V))
        same(sides[0], sides[1])
        same(sides[0], sides[2])
        assert not torch.equal(sides[0][0], torch.randn(3001, generator=torch.Generator(device=DEV).manual_seed(kind), device=DEV))


@pytest.mark.gpu
def test_calls_that_need_a_workspace_are_done_whole(call, monkeypatch):
    """Without a workspace, or with one that is too small, the call makes one itself; with one that is large enough it makes none."""
    g = torch.Generator(device=DEV).manual_seed(6)
    X, dY, A, B = (torch.randn(s, generator=g, device=DEV) for s in ((300, 64), (300, 72), (2, 8, 64), (2, 8, 72)))
    ids, rstd, gain = torch.zeros(300, dtype=torch.int32, device=DEV), torch.ones(700, device=DEV), torch.ones(64, device=DEV)
    many = torch.randn((700, 64), generator=g, device=DEV)
    _, U = dab.dab_adapters(X, ids, A, B)
    Q, S = dab.dab_w4_pack(torch.randn((72, 64), generator=g, device=DEV))
    calls = {"rms_norm_gradient": (lambda ws: dab.dab_rms_norm_gradient(many, many, gain, rstd, ws=ws), 2),
             "adapters_gradient": (lambda ws: dab.dab_adapters_gradient(dY, X, U, ids, A, B, ws=ws), 3),
             "w4_adapters": (lambda ws: dab.dab_w4_adapters(X, Q, S, 72, ids, A, B, ws=ws), 1)}
    small, large = torch.empty(1, dtype=torch.uint8, device=DEV), torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    for name, (f, outputs) in calls.items():
        want = f(None)
        for ws, made in ((None, 1), (small, 1), (large, 0)):
            for python in (False, True):
                proxy = Counted(call, name)
                proxy.python = python
                monkeypatch.setattr(dab, "_native", proxy)
                before = torch.cuda.memory_stats()["allocation.all.allocated"]
                got = f(ws)
                assert torch.cuda.memory_stats()["allocation.all.allocated"] - before == outputs + made, (name, made, python)
                assert (proxy.taken[-1] is not None) != python
                same(got, want)
                monkeypatch.setattr(dab, "_native", call)
