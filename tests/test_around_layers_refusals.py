"""What the C entry points of norms, steps and adapters refuse, before any HIP call (no GPU needed)."""
import ctypes
import os

import pytest

from paper_1804_02941_amd import binding, build

NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 5
F32, BF16, F16 = binding.DAB_F32, binding.DAB_BF16, binding.DAB_F16
p = ctypes.c_void_p(4096)              # never dereferenced
odd = ctypes.c_void_p(4098)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def test_norm(lib):
    ok = dict(X=p, t=BF16, ldx=40, R=p, ldr=40, g=p, eps=1e-5, rows=4, cols=40, H=p, Y=p, Q=p, S=p, rstd=p)

    def call(**k):
        return lib.dab_rms_norm(*{**ok, **k}.values(), None)
    for k in ("X", "g", "H", "Q", "S", "rstd"):
        assert call(**{k: None}) == NULL
    assert call(Y=None, Q=None, S=None) == NULL
    assert call(rows=0) == SHAPE and call(cols=0) == SHAPE and call(ldx=39) == SHAPE and call(ldr=39) == SHAPE and call(eps=-1.0) == SHAPE
    assert call(eps=float("nan")) == SHAPE and call(t=9) == UNSUPPORTED and call(cols=(1 << 26) + 1, ldx=1 << 27, ldr=1 << 27) == UNSUPPORTED
    for k in ("X", "R", "H", "Y", "Q", "g", "rstd"):
        assert call(**{k: odd}) == ALIGN
    # an output over an input: only element by element
    for k, ld in (("X", "ldx"), ("R", "ldr")):
        for out in ("H", "Y"):
            apart = {"X": 1 << 20, "R": 1 << 21, "H": 1 << 22, "Y": 1 << 23}
            for shift in (-16, 16, 3 * 40 * 2 + 64):
                assert call(**{**apart, out: apart[k] + shift}) == UNSUPPORTED
            assert call(**{**apart, out: apart[k], ld: 48}) == UNSUPPORTED


def test_norm_gradient(lib):
    need = lib.dab_rms_norm_gradient_workspace_bytes(1000, 40)
    assert need >= 160 and lib.dab_rms_norm_gradient_workspace_bytes(0, 40) == 0
    assert lib.dab_rms_norm_gradient_workspace_bytes(2, 4096) == 0                 # few rows: nothing to join
    assert lib.dab_rms_norm_gradient_workspace_bytes(512, 4096) == 0 and lib.dab_rms_norm_gradient_workspace_bytes(513, 4096) > 0
    # parts for what the chip holds at once, not for every row
    assert lib.dab_rms_norm_gradient_workspace_bytes(1 << 24, 4096) < 1 << 27
    ok = dict(dY=p, lddy=40, H=p, ldh=40, t=F32, g=p, rstd=p, dH=p, lddh=40, rows=1000, cols=40, dX=p, dg=p, ws=p, n=need)

    def call(**k):
        return lib.dab_rms_norm_gradient(*{**ok, **k}.values(), None)
    for k in ("dY", "H", "g", "rstd", "dX", "dg"):
        assert call(**{k: None}) == NULL
    for k in ("lddy", "ldh", "lddh"):
        assert call(**{k: 39}) == SHAPE
    assert call(t=-1) == UNSUPPORTED and call(dX=odd) == ALIGN and call(dH=odd) == ALIGN
    for k, ld in (("dY", "lddy"), ("H", "ldh"), ("dH", "lddh")):
        apart = {"dY": 1 << 20, "H": 1 << 21, "dH": 1 << 22, "dX": 1 << 23, "ws": None}
        assert call(**{**apart, "dX": apart[k]}) == WORKSPACE and call(**{**apart, "dX": apart[k], ld: 41}) == UNSUPPORTED
        assert call(**{**apart, "dX": apart[k] + 16}) == UNSUPPORTED and call(**{**apart, "dX": apart[k] - 16}) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(n=need - 1) == WORKSPACE and call(ws=ctypes.c_void_p(4096 + 16)) == WORKSPACE


def test_adamw_jobs(lib):
    def call(count=1, **k):
        job = binding.dab_adamw_job(4096, 4096, 4096, 4096, 4096, 4096, 4096, 100, 64, F32, BF16, 8, 0.1)
        for name, v in k.items():
            setattr(job, name, v)
        plan = binding.dab_adamw_plan()
        rc = lib.dab_adamw_plan_of((binding.dab_adamw_job * 1)(job), count, ctypes.byref(plan))
        return rc if rc else plan
    assert lib.dab_adamw_plan_of(None, 1, ctypes.byref(binding.dab_adamw_plan())) == NULL and call(count=0) == SHAPE
    for k in ("P", "G", "M", "V", "MS", "VS"):
        assert call(**{k: None}) == NULL
    assert call(n=0) == SHAPE and call(place=33) == SHAPE and call(weight_decay=float("inf")) == SHAPE
    assert call(grad_dtype=3) == UNSUPPORTED and call(copy_dtype=F32) == UNSUPPORTED and call(bits=16) == UNSUPPORTED and call(n=(1 << 34) + 1) == UNSUPPORTED
    for k in ("P", "G", "M", "V", "copy"):
        assert call(**{k: 4098}) == ALIGN
    plan = call()
    assert plan.n_jobs == 1 and plan.workgroups == 1 and plan.table_bytes >= 100
    job = (binding.dab_adamw_job * 1)(binding.dab_adamw_job(4096, 4096, 4096, 4096, 4096, 4096, 4096, 100, 64, F32, BF16, 8, 0.1))
    table = lib.dab_adamw_table
    assert table(None, ctypes.byref(plan), p, 4096, None) == NULL and table(job, ctypes.byref(plan), None, 4096, None) == NULL
    assert table(job, ctypes.byref(plan), p, plan.table_bytes - 1, None) == WORKSPACE and table(job, ctypes.byref(plan), odd, 4096, None) == WORKSPACE
    other = call(n=100000)
    assert table(job, ctypes.byref(other), p, 1 << 20, None) == SHAPE


def test_adamw(lib):
    plan = binding.dab_adamw_plan(1, 1, 1, 256)

    def call(table=p, size=4096, plan=plan, **k):
        s = binding.dab_adamw_step(1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None, None)
        for name, v in k.items():
            setattr(s, name, v)
        return lib.dab_adamw(table, size, ctypes.byref(plan), ctypes.byref(s), None)
    assert lib.dab_adamw(p, 4096, ctypes.byref(plan), None, None) == NULL and call(table=None) == NULL and call(table=odd) == WORKSPACE
    assert call(size=100) == WORKSPACE and call(plan=binding.dab_adamw_plan(0, 1, 1, 256)) == SHAPE and call(plan=binding.dab_adamw_plan(2, 1, 1, 256)) == SHAPE
    for bad in (dict(lr=float("nan")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")), dict(step=0)):
        assert call(**bad) == SHAPE
    assert call(lr_dev=4097) == ALIGN and call(step_dev=4100) == ALIGN and call(grad_scale=4097) == ALIGN


def test_states(lib):
    back, save = lib.dab_state8_restore, lib.dab_state8_save
    assert back(None, p, 5, 1, p, F32, None) == NULL and back(p, p, 0, 1, p, F32, None) == SHAPE and back(p, p, 5, 1, p, 4, None) == UNSUPPORTED
    assert back(odd, p, 5, 1, p, F32, None) == ALIGN and save(p, 5, 0, odd, p, None) == ALIGN and save(p, 5, 0, p, None, None) == NULL
    assert save(p, (1 << 34) + 1, 0, p, p, None) == UNSUPPORTED


def test_adapters(lib):
    ok = dict(X=p, t=BF16, ldx=40, ids=p, A=p, B=p, s=p, T=5, K=40, F=24, n=2, r=3, base=p, bt=BF16, ldb=24, Y=p, U=p)

    def call(**k):
        return lib.dab_adapters(*{**ok, **k}.values(), None)
    for k in ("X", "ids", "A", "B", "Y", "U"):
        assert call(**{k: None}) == NULL
    for k in ("T", "K", "F", "n", "r"):
        assert call(**{k: 0}) == SHAPE
    assert call(ldx=39) == SHAPE and call(ldb=23) == SHAPE and call(t=5) == UNSUPPORTED and call(bt=F16) == UNSUPPORTED
    assert call(r=257) == UNSUPPORTED and call(n=65536) == UNSUPPORTED and call(T=(1 << 25) + 1) == UNSUPPORTED
    for k in ("X", "A", "B", "base", "Y", "U", "ids", "s"):
        assert call(**{k: odd}) == ALIGN
    # X is read for other columns of Y
    assert call() == UNSUPPORTED and call(Y=ctypes.c_void_p(4096 + 4 * 40 * 2 + 64)) == UNSUPPORTED


def test_adapters_gradient(lib):
    size = lib.dab_adapters_gradient_workspace_bytes
    need = size(5, 40, 24, 2, 3)
    assert need > 0 and size(0, 40, 24, 2, 3) == 0 and size(5, 40, 24, 2, 257) == 0
    assert size(8192, 4096, 4096, 4, 16) < 1 << 27
    q = ctypes.c_void_p(1 << 20)
    ok = dict(dY=p, lddy=24, X=p, t=BF16, ldx=40, U=p, ids=p, A=p, B=p, s=p, T=5, K=40, F=24, n=2, r=3, base=p, bt=F32, ldb=40, dX=q, dA=p, dB=p, ws=p, nb=need)

    def call(**k):
        return lib.dab_adapters_gradient(*{**ok, **k}.values(), None)
    for k in ("dY", "X", "U", "ids", "A", "B", "dX", "dA", "dB"):
        assert call(**{k: None}) == NULL
    # X and dY are read again behind dX
    assert call(dX=p) == UNSUPPORTED and call(dX=ctypes.c_void_p(4096 + 4 * 24 * 2 + 16)) == UNSUPPORTED and call(X=q) == UNSUPPORTED
    assert call(X=q, dX=ctypes.c_void_p((1 << 20) + 400), ws=None) == WORKSPACE              # right behind X
    assert call(lddy=23) == SHAPE and call(ldb=39) == SHAPE and call(bt=F16) == UNSUPPORTED and call(dY=odd) == ALIGN and call(dA=odd) == ALIGN
    assert call(ws=None) == WORKSPACE and call(nb=need - 1) == WORKSPACE and call(ws=ctypes.c_void_p(4096 + 16)) == WORKSPACE


def test_served(lib):
    size = lib.dab_w4_adapters_workspace_bytes
    need = size(5, 40, 24, 3, BF16, 40)
    assert need > 0 and size(0, 40, 24, 3, BF16, 40) == 0 and size(5, 40, 24, 3, 8, 40) == 0
    ok = dict(X=p, t=BF16, ldx=40, Q=p, S=p, ids=p, A=p, B=p, s=p, T=5, K=40, F=24, n=2, r=3, Y=p, ws=p, nb=need)

    def call(**k):
        return lib.dab_w4_adapters(*{**ok, **k}.values(), None)
    for k in ("X", "Q", "S", "ids", "A", "B", "Y"):
        assert call(**{k: None}) == NULL
    assert call(F=0) == SHAPE and call(r=257) == UNSUPPORTED and call(T=65536) == UNSUPPORTED and call(F=65536 * 16) == UNSUPPORTED
    assert call(Q=odd) == ALIGN and call(Y=odd) == ALIGN and call(ws=None) == WORKSPACE and call(nb=need - 1) == WORKSPACE
    assert call() == UNSUPPORTED                                   # Y over X
