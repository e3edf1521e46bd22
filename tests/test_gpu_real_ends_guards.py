"""Calls of the real-valued ends whose workspace and outputs lie in front of (and behind) bytes of somebody else's, which stay as they are.

Results are compared with float64 as tests/test_gpu_real_ends.py does over whole tensors (bf16 4e-3: P, dH and dW are rounded to 8 bits, about
2^-9 each in the mean; fp32 2e-6 times the largest logit), and bit for bit with the same call's where the binding allocates.
"""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PATTERN = 0xA5


class Guarded:
    """Tensors cut out of the middle of filled buffers."""

    def __init__(self, behind):
        self.behind, self.buffers = behind, []

    def tensor(self, shape, dtype):
        n = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
        front = 4096
        raw = torch.full((front + n + self.behind,), PATTERN, dtype=torch.uint8, device=DEV)
        self.buffers.append((raw, front, n))
        return raw[front:front + n].view(dtype).view(shape)

    def workspace(self, nbytes):
        """A workspace of which the call may use nbytes (the binding hands over as many as the call asks for)."""
        raw = torch.full((4096 + nbytes + self.behind,), PATTERN, dtype=torch.uint8, device=DEV)
        self.buffers.append((raw, 4096, nbytes))
        return raw[4096:]

    def untouched(self):
        torch.cuda.synchronize()
        return all(bool((raw[:front] == PATTERN).all()) and bool((raw[front + n:] == PATTERN).all()) for raw, front, n in self.buffers)


def head_case(T, D, V, dtype, seed=3):
    g = torch.Generator(device=DEV).manual_seed(seed)
    H = torch.randn((T, D), generator=g, device=DEV).to(dtype)
    W = (torch.randn((V, D), generator=g, device=DEV) * (2.0 / D ** 0.5)).to(dtype)
    t = torch.randint(0, V, (T,), generator=g, device=DEV)
    t[::7] = -100
    return H, W, t, 0.5 + torch.rand((T,), generator=g, device=DEV)


# Large tiles with a last round that is not full, where the workspace has no room for shares: of bf16 the first piece, the last of several, up to 128
# tokens, few words; fp32 planes; and sizes with room, small heads, fp32 operands as they are.
HEADS = [(1632, 3796, 6071, torch.bfloat16), (8192, 2048, 50257, torch.bfloat16), (65, 8256, 4097, torch.bfloat16), (215, 4071, 1024, torch.bfloat16),
         (2048, 6144, 128000, torch.float32), (2048, 4096, 32768, torch.bfloat16), (4000, 2050, 40001, torch.bfloat16), (299, 1504, 628, torch.float32),
         (75, 931, 901, torch.bfloat16), (33, 500, 20000, torch.float32), (1, 2083, 256, torch.bfloat16), (2, 2083, 256, torch.bfloat16)]


@pytest.mark.parametrize("T,D,V,dtype", HEADS)
def test_head_keeps_to_its_workspace_and_outputs(T, D, V, dtype):
    H, W, t, g = head_case(T, D, V, dtype)
    code = dab.DAB_BF16 if dtype == torch.bfloat16 else dab.DAB_F32
    G = Guarded(192 << 20)
    loss, lse = dab.dab_head_loss(H, W, t, out=(G.tensor((T,), torch.float32), G.tensor((T,), torch.float32)),
                                  ws=G.workspace(dab.lib().dab_head_loss_workspace_bytes(T, D, V, code, D, D)))
    dH, dW = dab.dab_head_loss_gradient(H, W, t, lse, g, out=(G.tensor((T, D), dtype), G.tensor((V, D), dtype)),
                                        ws=G.workspace(dab.lib().dab_head_loss_gradient_workspace_bytes(T, D, V, code, D, D)))
    assert G.untouched()
    again = dab.dab_head_loss(H, W, t)
    assert torch.equal(loss, again[0]) and torch.equal(lse, again[1])
    again = dab.dab_head_loss_gradient(H, W, t, lse, g)
    assert torch.equal(dH, again[0]) and torch.equal(dW, again[1])
    del again
    live = t != -100
    L = H[live].double() @ W.double().t()
    most = float(L.abs().max()) if L.numel() else 0.0             # (a lone token may be ignored: no rows)
    ref = torch.logsumexp(L, 1)
    assert bool(((lse[live].double() - ref).abs() <= 2e-6 * max(1.0, most) * 8).all())
    assert bool(((loss[live].double() - ref + L.gather(1, t[live][:, None])[:, 0]).abs() <= 2e-6 * max(1.0, most) * 8).all())
    P = L.sub_(ref[:, None]).exp_()
    P[torch.arange(P.shape[0], device=DEV), t[live]] -= 1
    P *= g[live].double()[:, None]
    limit = 4e-3 if dtype == torch.bfloat16 else 2e-6 * max(1.0, most)
    want = P @ W.double()
    assert float((dH[live].double() - want).norm()) <= limit * float(want.norm()) and not bool(dH[~live].any())
    want = P.t().contiguous() @ H[live].double()
    assert float((dW.double() - want).norm()) <= limit * float(want.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,F", [(1, 1, 1), (65, 100, 127), (8191, 777, 301), (1030, 520, 300), (300, 4100, 4100)])
def test_weight_gradient_keeps_to_its_workspace_and_outputs(dtype, rows, cols, F):
    g = torch.Generator(device=DEV).manual_seed(rows)
    X = torch.randint(-60, 61, (rows, cols), generator=g, device=DEV).float()
    X[:, ::32] = 64                                                # (steps of one: nothing is lost)
    Y = torch.randint(-3, 4, (rows, F), generator=g, device=DEV).to(dtype)
    code = {torch.float32: dab.DAB_F32, torch.bfloat16: dab.DAB_BF16, torch.float16: dab.DAB_F16}[dtype]
    G, n = Guarded(64 << 20), (cols + 31) // 32
    Q, S = dab.dab_ckpt8_save(X, out=(G.tensor((rows, 32 * n), torch.int8), G.tensor((rows, n), torch.uint8)))
    dW = dab.dab_ckpt8_weight_gradient(Y, Q, S, cols, out=G.tensor((F, cols), torch.float32),
                                       ws=G.workspace(dab.lib().dab_ckpt8_weight_gradient_workspace_bytes(rows, cols, F, code, F)))
    back = dab.dab_ckpt8_restore(Q, S, cols, dtype, out=G.tensor((rows, cols), dtype))
    assert G.untouched()
    assert torch.equal(back.float(), X) and torch.equal(dW.double(), Y.double().t().contiguous() @ X.double())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,K,F", [(1, 1, 1), (7, 1111, 1099), (17, 136, 31), (200, 160, 35)])
def test_4_bit_weights_keep_to_their_workspace_and_outputs(dtype, B, K, F):
    g = torch.Generator(device=DEV).manual_seed(B)
    W = torch.randint(-4, 5, (F, K), generator=g, device=DEV).float()
    W[:, ::32] = 6                                                 # (steps of one: 5 alone is no level, and not among them)
    X = torch.randint(-2, 3, (B, K), generator=g, device=DEV).to(dtype)
    code = {torch.float32: dab.DAB_F32, torch.bfloat16: dab.DAB_BF16, torch.float16: dab.DAB_F16}[dtype]
    G = Guarded(1 << 20)
    Q, S = dab.dab_w4_pack(W, out=(G.tensor(((F + 15) // 16, (K + 127) // 128, 64, 16), torch.uint8),
                                   G.tensor(((F + 15) // 16, (K + 511) // 512, 64, 4), torch.uint8)))
    back = dab.dab_w4_unpack(Q, S, F, K, out=G.tensor((F, K), torch.float32))
    Y = dab.dab_w4_matvec(X, Q, S, F, out=G.tensor((B, F), dtype), ws=G.workspace(dab.lib().dab_w4_matvec_workspace_bytes(B, K, F, code, K)))
    assert G.untouched()
    assert torch.equal(back, W) and torch.equal(Y, (X.double() @ W.double().t()).to(dtype))
