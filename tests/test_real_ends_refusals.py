"""What the C entry points of the real-valued ends refuse, before any HIP call (no GPU needed)."""
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


def test_save_and_restore(lib):
    save, back = lib.dab_ckpt8_save, lib.dab_ckpt8_restore
    assert save(None, F32, 4, 4, 4, p, p, None) == NULL and save(p, F32, 4, 4, 4, None, p, None) == NULL
    assert save(p, F32, 0, 4, 4, p, p, None) == SHAPE and save(p, F32, 4, 0, 4, p, p, None) == SHAPE
    assert save(p, F32, 4, 4, 3, p, p, None) == SHAPE and save(p, F32, -1, 4, 4, p, p, None) == SHAPE
    assert save(p, 7, 4, 4, 4, p, p, None) == UNSUPPORTED and save(odd, F32, 4, 4, 4, p, p, None) == ALIGN
    assert save(p, F32, 4, 4, 4, odd, p, None) == ALIGN
    assert back(None, p, 4, 4, p, F32, 4, None) == NULL and back(p, p, 4, 4, odd, F32, 4, None) == ALIGN
    assert back(p, p, 4, 4, p, 3, 4, None) == UNSUPPORTED and back(p, p, 4, 4, p, F32, 2, None) == SHAPE


def test_weight_gradient(lib):
    f, ws = lib.dab_ckpt8_weight_gradient, lib.dab_ckpt8_weight_gradient_workspace_bytes
    need = ws(100, 60, 30, F32, 30)
    assert need > 0 and ws(0, 60, 30, F32, 30) == 0 and ws(100, 60, 30, 9, 30) == 0
    assert f(None, F32, 30, p, p, 100, 60, 30, p, p, need, None) == NULL
    assert f(p, F32, 29, p, p, 100, 60, 30, p, p, need, None) == SHAPE
    assert f(p, F32, 30, p, p, 100, 60, 0, p, p, need, None) == SHAPE
    assert f(p, 5, 30, p, p, 100, 60, 30, p, p, need, None) == UNSUPPORTED
    assert f(p, F32, 1 << 23, p, p, 100, 60, 30, p, p, need, None) == UNSUPPORTED
    assert f(odd, F32, 30, p, p, 100, 60, 30, p, p, need, None) == ALIGN
    assert f(p, F32, 30, p, p, 100, 60, 30, p, p, need - 1, None) == WORKSPACE
    assert f(p, F32, 30, p, p, 100, 60, 30, p, None, need, None) == WORKSPACE
    assert f(p, F32, 30, p, p, 100, 60, 30, p, ctypes.c_void_p(4096 + 16), need, None) == WORKSPACE


def test_head(lib):
    loss, ws = lib.dab_head_loss, lib.dab_head_loss_workspace_bytes
    need = ws(10, 16, 100, BF16, 16, 16)
    assert need > 0 and ws(10, 16, 100, F16, 16, 16) == 0 and ws(10, 16, 0, BF16, 16, 16) == 0
    ok = dict(H=p, ldh=16, W=p, ldw=16, t=BF16, y=p, i=-100, T=10, D=16, V=100, a=p, b=p, ws=p, n=need)

    def call(**k):
        return loss(*{**ok, **k}.values(), None)
    for k in ("H", "W", "y", "a", "b"):
        assert call(**{k: None}) == NULL
    for k in ("T", "D", "V"):
        assert call(**{k: 0}) == SHAPE
    assert call(ldh=15) == SHAPE and call(ldw=15) == SHAPE
    assert call(t=F16) == UNSUPPORTED and call(t=4) == UNSUPPORTED and call(ldw=1 << 23) == UNSUPPORTED
    assert call(H=odd) == ALIGN and call(W=odd) == ALIGN and call(y=odd) == ALIGN and call(a=odd) == ALIGN
    assert call(ws=None) == WORKSPACE and call(n=need - 1) == WORKSPACE and call(ws=ctypes.c_void_p(4096 + 128)) == WORKSPACE


def test_head_gradient(lib):
    f, ws = lib.dab_head_loss_gradient, lib.dab_head_loss_gradient_workspace_bytes
    need = ws(10, 16, 100, F32, 16, 16)
    ok = dict(H=p, ldh=16, W=p, ldw=16, t=F32, y=p, i=-100, l=p, g=None, T=10, D=16, V=100, dH=p, dW=p, ws=p, n=need)

    def call(**k):
        return f(*{**ok, **k}.values(), None)
    for k in ("H", "W", "y", "l", "dH", "dW"):
        assert call(**{k: None}) == NULL
    assert call(V=0) == SHAPE and call(ldw=8) == SHAPE and call(t=F16) == UNSUPPORTED
    assert call(g=odd) == ALIGN and call(dW=odd) == ALIGN and call(n=need - 1) == WORKSPACE
    # the workspace of a piece of the vocabulary, not of all logits
    assert ws(8192, 2048, 131072, BF16, 2048, 2048) < 2 * 8192 * 131072 / 4


def test_4_bit_weights(lib):
    pack, back, mul, ws = lib.dab_w4_pack, lib.dab_w4_unpack, lib.dab_w4_matvec, lib.dab_w4_matvec_workspace_bytes
    assert pack(None, F32, 4, 4, 4, p, p, None) == NULL and pack(p, F32, 4, 4, 3, p, p, None) == SHAPE
    assert pack(p, F32, 0, 4, 4, p, p, None) == SHAPE and pack(p, 3, 4, 4, 4, p, p, None) == UNSUPPORTED
    assert pack(odd, F32, 4, 4, 4, p, p, None) == ALIGN and pack(p, F32, 65536 * 16, 4, 4, p, p, None) == UNSUPPORTED
    assert back(p, p, 4, 4, None, None) == NULL and back(p, p, 4, 0, p, None) == SHAPE and back(odd, p, 4, 4, p, None) == ALIGN
    assert ws(1, 4096, 64, BF16, 4096) == 0 and ws(1, 4096, 64, F32, 4096) > 0 and ws(1, 4095, 64, BF16, 4095) > 0
    assert mul(None, F32, 64, p, p, 1, 64, 8, p, p, 1 << 20, None) == NULL
    assert mul(p, F32, 63, p, p, 1, 64, 8, p, p, 1 << 20, None) == SHAPE and mul(p, F32, 64, p, p, 0, 64, 8, p, p, 1 << 20, None) == SHAPE
    assert mul(p, F32, 64, p, p, 70000, 64, 8, p, p, 1 << 30, None) == UNSUPPORTED
    assert mul(p, F32, 64, p, odd, 1, 64, 8, p, p, 1 << 20, None) == ALIGN
    assert mul(p, F32, 64, p, p, 1, 64, 8, p, None, 0, None) == WORKSPACE
