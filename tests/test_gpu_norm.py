"""The root-mean-square norm and its gradients through the C ABI, against float64 (oracle/around_layers.py).

u = 2^-24 is half a step of fp32; a value rounded to bf16 is off by 2^-8 of itself at most, to f16 by 2^-11.  A row's sum adds every term at most D
times: eight values of up to four vectors a lane (or more in long rows), six steps within a wavefront, sixteen wavefronts.
"""
import numpy as np
import pytest
import torch

from oracle import around_layers as oa
from oracle import real_ends as oe
from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# rows and columns of every form: four lanes to a workgroup for a row, short last vectors, rows that no workgroup holds
SIZES = [(1, 1), (3, 7), (1, 32), (70, 33), (5, 64), (9, 100), (65, 200), (33, 500), (2, 777), (4, 1003), (3, 2000), (257, 4096), (2, 5000), (3, 8200), (1, 16384),
         (2, 20001), (2, 32769), (3, 70000)]


def additions(cols):
    return 8 * max(4, -(-cols // 8192)) + 22


def f64(t):
    return t.double().cpu().numpy()


def strided(t, extra, lead):
    rows, cols = t.shape
    wide = torch.full((rows, cols + extra + lead), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, lead:lead + cols] = t
    return wide[:, lead:lead + cols]


def inputs(rows, cols, dtype, seed=0):
    rng = np.random.default_rng(1000 * rows + cols + seed)
    gain = np.exp(0.5 * rng.standard_normal(cols))
    x, r, dy, dh = (torch.from_numpy(rng.standard_normal((rows, cols)) * gain * k).to(dtype).to(DEV) for k in (1, 1, 0.1, 0.1))
    return x, r, torch.from_numpy(1 + 0.3 * rng.standard_normal(cols)).float().to(DEV), dy, dh


def check_norm(x, r, gain, eps, got):
    Y, H, rstd, saved = got
    dtype, (rows, cols) = x.dtype, x.shape
    h = x if r is None else (x.float() + r.float()).to(dtype)
    assert torch.equal(H, h) and H.dtype == dtype
    y, s = oa.rms_norm(f64(h), f64(gain), eps)
    # sum and square: D + 1 roundings of positive terms; mean, eps: 2 more; half of them through the root, then the root and the quotient
    off = ((additions(cols) + 3) / 2 + 2) * U
    assert np.all(np.abs(f64(rstd) - s) <= off * s * 1.01)
    off = (off + 2 * U) * 1.01 * np.abs(y)
    if Y is not None:
        assert Y.dtype == dtype
        assert np.all(np.abs(f64(Y) - y) <= off + HALF[dtype] * (np.abs(y) + off) + 2.0 ** -25 * (dtype == torch.float16))
    if saved is not None:
        Q, S = saved[0].cpu().numpy(), saved[1].cpu().numpy().astype(int)
        groups = -(-cols // 32)
        assert Q.shape == (rows, 32 * groups) and not Q[:, cols:].any()
        Qo, So = oe.save8(y)
        # the exponent is the definition's, but where the largest value lies within its error of the next one
        assert np.all(np.abs(S - So) <= 1) and np.mean(S != So) < 0.02
        back = oe.restore8(Q, S, cols)
        half = np.repeat(np.ldexp(0.5, S - 127), 32, axis=1)[:, :cols]
        assert np.all(np.abs(back - y) <= half + off)
        assert np.mean(Q != Qo) < 0.02


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_norm(dtype, rows, cols):
    x, r, gain, _, _ = inputs(rows, cols, dtype)
    for X, R, save in ((x, None, False), (x, r, True), (strided(x, 3, 0), strided(r, 5, 8), True), (x, strided(r, 1, 16), "only")):
        got = dab.dab_rms_norm(X, gain, residual=R, eps=1e-5, save=save)
        assert (got[0] is None) == (save == "only") and (got[3] is None) == (save is False)
        check_norm(X, R, gain, 1e-5, got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_norm_gradient(dtype, rows, cols):
    x, _, gain, dy, dh = inputs(rows, cols, dtype)
    _, _, rstd, _ = dab.dab_rms_norm(x, gain, eps=1e-3)
    for DY, H, DH in ((dy, x, None), (strided(dy, 3, 0), strided(x, 1, 8), strided(dh, 5, 0))):
        dX, dgain = dab.dab_rms_norm_gradient(DY, H, gain, rstd, dH=DH)
        assert dX.dtype == dtype and dgain.dtype == torch.float32
        s, n, w = f64(rstd)[:, None], f64(x) * f64(rstd)[:, None], f64(dy) * f64(gain)[None, :]
        want, wgain = oa.rms_norm_gradient(f64(dy), f64(x), f64(gain), f64(rstd), None if DH is None else f64(dh))
        size = np.mean(np.abs(w * n), axis=1, keepdims=True)
        off = s * U * (3 * np.abs(w) + np.abs(n) * size * (additions(cols) + 8)) + 2 * U * np.abs(want) + (0 if DH is None else U * np.abs(f64(dh)))
        assert np.all(np.abs(f64(dX) - want) <= 1.01 * off + HALF[dtype] * (np.abs(want) + off) + 2.0 ** -25 * (dtype == torch.float16))
        assert np.all(np.abs(f64(dgain) - wgain) <= (rows + 3) * U * np.abs(f64(dy) * n).sum(axis=0) * 1.01 + 1e-30)


# more rows than one launch with whole columns takes: parts of dgain, of every form
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(513, 1), (600, 7), (2100, 33), (1031, 64), (777, 100), (530, 200), (2050, 500), (520, 777), (1999, 1003), (523, 2000), (600, 4096),
                                       (420, 5000), (257, 8200), (129, 16384)])
def test_norm_gradient_of_many_rows(dtype, rows, cols):
    test_norm_gradient(dtype, rows, cols)


def test_many_rows():
    """More rows than the chip holds at once, so that workgroups take several, and rows of few values."""
    for rows, cols in ((40000, 40), (9001, 520), (70001, 8)):
        x, r, gain, dy, dh = inputs(rows, cols, torch.float32)
        got = dab.dab_rms_norm(x, gain, residual=r, save=True)
        check_norm(x, r, gain, 1e-5, got)
        dX, dgain = dab.dab_rms_norm_gradient(dy, got[1], gain, got[2], dH=dh)
        want, wgain = oa.rms_norm_gradient(f64(dy), f64(got[1]), f64(gain), f64(got[2]), f64(dh))
        n = np.abs(f64(got[1])) * f64(got[2])[:, None]
        assert np.all(np.abs(f64(dgain) - wgain) <= (rows + 3) * U * (np.abs(f64(dy)) * n).sum(axis=0) * 1.01)
        np.testing.assert_allclose(f64(dX), want, rtol=0, atol=60 * U * np.max(np.abs(want)))
        again = dab.dab_rms_norm_gradient(dy, got[1], gain, got[2], dH=dh)
        assert torch.equal(again[0], dX) and torch.equal(again[1], dgain)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(dtype):
    for rows, cols in ((5, 100), (5, 4096), (5, 40000), (600, 93)):
        x, r, gain, dy, dh = inputs(rows, cols, dtype)
        Y, H, rstd, _ = dab.dab_rms_norm(x, gain, residual=r)
        a, b = x.clone(), r.clone()
        Y2, H2, _, _ = dab.dab_rms_norm(a, gain, residual=b, out=(a, b, None, None))      # the sum over the residual, the output over the input
        assert Y2 is a and H2 is b and torch.equal(a, Y) and torch.equal(b, H)
        a = x.clone()
        assert torch.equal(dab.dab_rms_norm(a, gain, residual=r, out=(None, a, None, None))[0], Y) and torch.equal(a, H)
        a = x.clone()
        assert torch.equal(dab.dab_rms_norm(a, gain, out=(a, None, None, None))[0], dab.dab_rms_norm(x, gain)[0])
        dX, dgain = dab.dab_rms_norm_gradient(dy, H, gain, rstd, dH=dh)
        for i in range(2):
            p, q = dy.clone(), dh.clone()
            got = dab.dab_rms_norm_gradient(p, H, gain, rstd, dH=q, out=((p, q)[i], None))
            assert torch.equal(got[0], dX) and torch.equal(got[1], dgain)
        p = H.clone()
        got = dab.dab_rms_norm_gradient(dy, p, gain, rstd, dH=dh, out=(p, None))
        assert torch.equal(got[0], dX) and torch.equal(got[1], dgain)


def test_values_at_the_edges():
    gain = torch.ones(64, device=DEV)
    x = torch.zeros((8, 64), device=DEV)
    x[1, 3], x[2, 5], x[3, 0] = float("inf"), float("nan"), -float("inf")
    x[4] = 1e25                                                    # its squares pass fp32's range
    x[5, 63] = 1e-30
    x[6] = torch.arange(64, device=DEV) - 32.0
    Y, _, rstd, (Q, S) = dab.dab_rms_norm(x, gain, eps=1e-6, save=True)
    assert not Y[0].any() and abs(float(rstd[0]) - 1000.0) < 1e-3 and bool((S[0] == 17).all())
    for row in (1, 2, 3):
        bad = torch.zeros(64, dtype=torch.bool, device=DEV)
        bad[{1: 3, 2: 5, 3: 0}[row]] = True
        # an infinity: rstd 0, its own output undefined, the others 0; a NaN: all undefined
        assert bool(Y[row].isnan().eq(bad).all()) if row != 2 else bool(Y[row].isnan().all())
        assert S[row].tolist() == ([255, 17] if row != 2 else [255, 255])
    assert float(rstd[4]) == 0 and not Y[4].any() and not Y[7].any()
    assert abs(float(Y[5, 63]) - 1e-27) < 1e-33
    # one row's values do not reach another's
    assert torch.equal(Y[6], dab.dab_rms_norm(x[6:7], gain, eps=1e-6)[0][0])
    zero = dab.dab_rms_norm(torch.zeros((2, 40), device=DEV), torch.ones(40, device=DEV), eps=0.0)
    assert bool(zero[2].isinf().all()) and bool(zero[0].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(5, 9), (5, 37), (5, 131), (5, 515), (5, 4097), (5, 33003), (600, 37), (600, 515), (530, 4097)])
def test_what_the_last_columns_neighbours_hold(dtype, rows, cols):
    """A row's last few columns are read with those before them, whose infinities and NaN stay where they are."""
    x, r, gain, dy, dh = inputs(rows, cols, dtype, 3)
    at, own = cols - 8, cols % 8                                    # read again; columns of the last lane
    Y, H, rstd, (q, s) = dab.dab_rms_norm(x, gain, r, save=True)
    dX, dgain = dab.dab_rms_norm_gradient(dy, H, gain, rstd, dh)
    group = at // 32
    for bad in (float("inf"), float("nan")):
        wrong = gain.clone()
        wrong[at] = bad
        Yb, Hb, rb, (qb, sb) = dab.dab_rms_norm(x, wrong, r, save=True)
        rest = [c for c in range(cols) if c != at]
        assert torch.equal(Hb, H) and torch.equal(rb, rstd) and torch.equal(Yb[:, rest], Y[:, rest]) and not torch.isfinite(Yb[:, at].float()).any()
        groups = [g for g in range(s.shape[1]) if g != group]
        assert torch.all(sb[:, group] == 255) and torch.equal(sb[:, groups], s[:, groups])
        for g in groups:
            assert torch.equal(qb[:, 32 * g:32 * g + 32], q[:, 32 * g:32 * g + 32])
        far = dy.clone()
        far[2, at] = bad                                            # the whole row's dX, but one column's dgain
        dXb, dgb = dab.dab_rms_norm_gradient(far, H, gain, rstd, dh)
        others = [row for row in range(rows) if row != 2]
        assert torch.equal(dXb[others], dX[others]) and torch.isnan(dXb[2].float()).any()
        assert torch.equal(dgb[rest], dgain[rest]) and not torch.isfinite(dgb[at])
    assert own != 0


def test_nothing_behind_the_outputs_is_written():
    rows, cols = 3, 45
    x, r, gain, dy, dh = inputs(rows, cols, torch.bfloat16)
    big = [torch.full((rows * cols + 64,), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    part = [b[:rows * cols].view(rows, cols) for b in big]
    rstd, dgain = torch.full((rows + 8,), 7.0, device=DEV), torch.full((cols + 8,), 7.0, device=DEV)
    Q, S = torch.full((rows * 64 + 64,), 7, dtype=torch.int8, device=DEV), torch.full((rows * 2 + 9,), 7, dtype=torch.uint8, device=DEV)
    dab.dab_rms_norm(x, gain, residual=r, save=True, out=(part[0], part[1], rstd[:rows], (Q[:rows * 64].view(rows, 64), S[:rows * 2].view(rows, 2))))
    dab.dab_rms_norm_gradient(dy, part[1], gain, rstd[:rows], dH=dh, out=(part[2], dgain[:cols]))
    for b in big:
        assert bool((b[rows * cols:] == 7).all())
    assert bool((rstd[rows:] == 7).all()) and bool((dgain[cols:] == 7).all()) and bool((Q[rows * 64:] == 7).all()) and bool((S[rows * 2:] == 7).all())


def test_offsets_past_32_bits():
    rows, ld, cols = 70000, 32768, 40                              # 2.3e9 elements between the first row and the last
    wide = torch.empty((rows, ld), dtype=torch.bfloat16, device=DEV)
    x = wide[:, 64:64 + cols]
    x.normal_()
    gain = torch.ones(cols, device=DEV)
    a, b = dab.dab_rms_norm(x, gain), dab.dab_rms_norm(x.contiguous(), gain)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
    dy = torch.randn((rows, cols), device=DEV).bfloat16()
    p, q = dab.dab_rms_norm_gradient(dy, x, gain, a[2]), dab.dab_rms_norm_gradient(dy, x.contiguous(), gain, a[2])
    assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])


@pytest.mark.parametrize("rows", [300, 900])
def test_captured_and_on_another_stream(rows):
    x, r, gain, dy, dh = inputs(rows, 1000, torch.bfloat16)
    outs = [torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=DEV), dab.ckpt8_outputs(rows, 1000, torch.device(DEV))]
    grads = [torch.empty_like(x), torch.empty(1000, device=DEV)]
    ws = torch.empty(dab.lib().dab_rms_norm_gradient_workspace_bytes(rows, 1000), dtype=torch.uint8, device=DEV)

    def work():
        dab.dab_rms_norm(x, gain, residual=r, save=True, out=tuple(outs))
        dab.dab_rms_norm_gradient(dy, outs[1], gain, outs[2], dH=dh, out=tuple(grads), ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        x.normal_()
        dy.normal_()
        graph.replay()
        got = [t.clone() for t in (*outs[:3], *outs[3], *grads)]
        Y, H, rstd, saved = dab.dab_rms_norm(x, gain, residual=r, save=True)
        dX, dgain = dab.dab_rms_norm_gradient(dy, H, gain, rstd, dH=dh)
        for a, b in zip(got, (Y, H, rstd, *saved, dX, dgain)):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_saved_output_is_what_the_weight_gradient_takes():
    x, r, gain, _, _ = inputs(130, 300, torch.bfloat16)
    dY = torch.randn((130, 70), device=DEV).bfloat16()
    Y, _, _, (Q, S) = dab.dab_rms_norm(x, gain, residual=r, save=True)
    dW = dab.dab_ckpt8_weight_gradient(dY, Q, S, 300)
    kept = f64(dab.dab_ckpt8_restore(Q, S, 300))
    assert np.all(np.abs(f64(dW) - f64(dY).T @ kept) <= 140 * U * (np.abs(f64(dY)).T @ np.abs(kept)))
    assert np.all(np.abs(kept - f64(Y)) <= np.abs(f64(Y)) * 2.0 ** -8 + np.max(np.abs(f64(Y))) / 126)


def test_refusals():
    x, r, gain, dy, _ = inputs(4, 40, torch.float32)
    rstd = torch.ones(4, device=DEV)
    for bad, error in ((dict(X=x.cpu()), TypeError), (dict(X=x.double()), TypeError), (dict(X=x[:, ::2]), ValueError), (dict(gain=gain[:39]), ValueError),
                       (dict(gain=gain.double()), TypeError), (dict(residual=r.bfloat16()), TypeError), (dict(residual=r[:3]), ValueError),
                       (dict(eps=-1.0), dab.DabError), (dict(eps=float("nan")), dab.DabError), (dict(X=x[:, 1:], gain=gain[1:]), dab.DabError),
                       (dict(out=(torch.empty(4, 41, device=DEV), None, None, None)), ValueError)):
        with pytest.raises(error):
            dab.dab_rms_norm(**{**dict(X=x, gain=gain), **bad})
    for bad, error in ((dict(dY=dy.bfloat16()), TypeError), (dict(dY=None), TypeError), (dict(rstd=rstd[:3]), ValueError), (dict(dH=dy[:, :39]), ValueError),
                       (dict(H=x[:0], dY=dy[:0], rstd=rstd[:0]), dab.DabError)):
        with pytest.raises(error):
            dab.dab_rms_norm_gradient(**{**dict(dY=dy, H=x, gain=gain, rstd=rstd), **bad})
    small = torch.empty(16, dtype=torch.uint8, device=DEV)          # a workspace that is too small: a new one is taken
    assert torch.equal(dab.dab_rms_norm_gradient(dy, x, gain, rstd, ws=small)[1], dab.dab_rms_norm_gradient(dy, x, gain, rstd)[1])
