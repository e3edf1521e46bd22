"""Operators of large language models that stand around the binarized and the 4-bit layers: what is timed of them, and their plain forms.

Between its layers a network normalizes, behind its gradients it steps, and where one set of 4-bit weights serves many requests each
brings a correction of its own:

  norm      the root-mean-square norm with the residual's addition, whose output is also kept in 8 bits for the next layer's
            weight gradient, and its gradients with respect to the input and the gain
  adamw     a step of Adam with decoupled weight decay over many tensors at once, its two states in 32 bits or in 8
  adapters  products of low rank, one pair of matrices per request, beside a shared projection: with the 4-bit weights for the few tokens that
            are served, and for the many tokens of a training step with the gradients

Kinds of work (a case's "kind"), each over a range of sizes that draw() covers: "norm" (a forward pass; "saved": its output in 8 bits
too), "norm_grad", "adamw" ("bits" of the states), "serve" (tokens through 4-bit weights with their adapters), "adapt" (adapters
forward beside a given product, then all gradients).

Formats (include/dab.h).  Saved outputs and 4-bit weights are those of perf/operators.py.  A state in 8 bits: groups of 32 share
a power of two 2^f, the least that makes the last code no smaller than the largest magnitude, f within -100 .. 120; a first moment is a sign,
four bits of exponent and three of significand, the root of a second moment four bits of exponent and four of significand, both below
2^(f+1); they are rounded up or down by chance, with the probabilities that keep the mean, by a number that depends on (seed, step, place) alone.
"""
import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GROUP = 32                                  # values that share a scale
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-5                                  # of the norm
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.01, 7, 20180402941
LAYERS = "128x64x5x5 256x128x3x3 256x256x3x3 256x256x3x3 512x256x7x7 512x512 250x512"    # the sketch network's trunk and its classes


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token between two layers while serving: latency
        {"name": "norm_token", "kind": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "residual": True, "saved": False},
        # a training batch in front of a layer whose weight gradient reads the output back from 8 bits (bandwidth)
        {"name": "norm_saved_16384x4096", "kind": "norm", "rows": 16384, "cols": 4096, "dtype": "bf16", "residual": True, "saved": True},
        # its backward pass, with the gradient that arrives on the residual's side
        {"name": "norm_grad_16384x4096", "kind": "norm_grad", "rows": 16384, "cols": 4096, "dtype": "bf16", "residual": True},
        # nothing fits a vector or a wavefront, this package's own type
        {"name": "norm_grad_ragged", "kind": "norm_grad", "rows": 1999, "cols": 1003, "dtype": "f32", "residual": False},
        # the step behind the weight side of the sketch network's training iteration, gradients and states in this package's own type
        {"name": "adamw_trunk_f32", "kind": "adamw", "sizes": LAYERS, "grad": "f32", "bits": 32, "copy": ""},
        # a large bf16 head, projections and gains, kept in fp32 with the bf16 copies that the products read
        {"name": "adamw8_head", "kind": "adamw", "sizes": "65536x1024" + " 1024x1024" * 8 + " 1024" * 17, "grad": "bf16", "bits": 8, "copy": "bf16"},
        # adapters alone are trained: many small tensors of odd sizes (launches)
        {"name": "adamw8_small", "kind": "adamw", "sizes": " ".join(str(1 + (7919 * i) % 4099) for i in range(96)), "grad": "f32", "bits": 8, "copy": ""},
        # one token of one request through the square layer (latency)
        {"name": "serve_4096_b1", "kind": "serve", "B": 1, "K": 4096, "F": 4096, "n": 8, "r": 16, "dtype": "bf16"},
        # thirty-two requests at once, nearly each with its own adapter
        {"name": "serve_16384_b32", "kind": "serve", "B": 32, "K": 4096, "F": 16384, "n": 64, "r": 16, "dtype": "bf16"},
        # a few requests, sizes that fit no tile, this package's own type
        {"name": "serve_ragged_b7", "kind": "serve", "B": 7, "K": 9111, "F": 4099, "n": 3, "r": 8, "dtype": "f32"},
        # a training step of four adapters over a long batch of tokens beside the square layer
        {"name": "adapt_8192x4096", "kind": "adapt", "T": 8192, "K": 4096, "F": 4096, "n": 4, "r": 16, "dtype": "bf16"},
        # tokens, channels and rank that fit no tile, some tokens without an adapter
        {"name": "adapt_ragged", "kind": "adapt", "T": 1999, "K": 777, "F": 301, "n": 3, "r": 5, "dtype": "f16"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm; often a round one, often not."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 32:
        v = 16 * ((v + 8) // 16)
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "adamw", "adamw", "serve", "serve", "adapt", "adapt"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("norm", "norm_grad"):
        while True:
            c = {"kind": kind, "rows": _log(rng, 1, 65536), "cols": _log(rng, 32, 16384), "dtype": dtype, "residual": rng.random() < 0.7}
            if kind == "norm":
                c["saved"] = rng.random() < 0.5
            if c["rows"] * c["cols"] <= 16384 * 4096 // (2 if dtype == "f32" else 1):
                return c
    if kind == "adamw":
        bits = rng.choice([8, 32])
        count, most = _log(rng, 1, 150), _log(rng, 100, 32 * 1024 * 1024)
        sizes = [_log(rng, 1, max(2, most // count)) for _ in range(count)]
        return {"kind": kind, "sizes": " ".join(map(str, sizes)), "grad": rng.choice(["f32", "bf16", "f16"]), "bits": bits,
                "copy": rng.choice(["", "bf16", "f16"])}
    while True:
        c = {"kind": kind, "K": _log(rng, 64, 16384 if kind == "serve" else 9216), "F": _log(rng, 16, 131072 if kind == "serve" else 9216),
             "n": _log(rng, 1, 64 if kind == "serve" else 16), "r": _log(rng, 1, 64), "dtype": dtype}
        if kind == "serve":
            c["B"] = _log(rng, 1, 64)
            if c["F"] * c["K"] <= 16384 * 8192 and c["n"] * c["r"] * (c["F"] + c["K"]) <= 64 * 16 * 65536:
                return c
        else:
            c["T"] = _log(rng, 1, 8192)
            if c["T"] * (c["K"] + c["F"]) <= 8192 * 4096 and c["T"] * (c["K"] + c["F"]) * c["n"] * c["r"] <= 8192 * 8192 * 256:
                return c


def _sizes(text):
    return [math.prod(int(v) for v in s.split("x")) for s in text.split()]


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 29)


def _normal(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _hidden(rows, cols, g):
    """A layer's input: normal, some channels larger than the others."""
    return _normal((rows, cols), g).mul_(torch.exp(0.5 * _normal((1, cols), g)))


def _gradient(n, g):
    """Gradients of a flat run of weights: magnitudes of their own in every stretch of 1024, a few per cent of them zero."""
    size = torch.exp(_normal((-(-n // 1024), 1), g)).mul_(1e-3).expand(-1, 1024).reshape(-1)[:n]
    return _normal((n,), g).mul_(size).mul_((torch.rand((n,), generator=g, device=DEV) > 0.03).float())


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(c)
    if c["kind"] in ("norm", "norm_grad"):
        dt = DTYPES[c["dtype"]]
        s["X"] = _hidden(c["rows"], c["cols"], g).to(dt)
        s["gain"] = 1.0 + 0.2 * _normal((c["cols"],), g)
        s["R"] = _hidden(c["rows"], c["cols"], g).to(dt) if c["residual"] else None
        if c["kind"] == "norm_grad":
            s["dY"] = _normal((c["rows"], c["cols"]), g).mul_(0.01).to(dt)
            s["rstd"] = torch.rsqrt(s["X"].double().square().mean(dim=1) + EPS).float()
        return s
    if c["kind"] == "adamw":
        return _prepare_adamw(s, g)
    dt = DTYPES[c["dtype"]]
    n, r, K, F = c["n"], c["r"], c["K"], c["F"]
    s["A"] = _normal((n, r, K), g).mul_(1.0 / math.sqrt(K)).to(dt)
    s["Bt"] = _normal((n, r, F), g).mul_(0.2).to(dt)
    s["scale"] = 0.5 + torch.rand((n,), generator=g, device=DEV)
    if c["kind"] == "serve":
        w = _normal((F, K), g).mul_(1.0 / math.sqrt(K))
        s["Q"], s["S"] = _tiles(*_quantize4(w))
        s["X"] = _normal((c["B"], K), g).to(dt)
        # requests in any order, one in ten without an adapter
        s["ids"] = torch.where(torch.rand((c["B"],), generator=g, device=DEV) < 0.1, -1, torch.randint(0, n, (c["B"],), generator=g, device=DEV)).int()
        return s
    T = c["T"]
    s["X"] = _normal((T, K), g).to(dt)
    s["base"] = _normal((T, F), g).to(dt)
    s["dY"] = _normal((T, F), g).mul_(0.01).to(dt)
    s["dbase"] = _normal((T, K), g).mul_(0.01).to(dt)
    # sequences of up to 128 tokens, each with its adapter or, one in ten, with none
    runs = -(-T // 128)
    who = torch.where(torch.rand((runs,), generator=g, device=DEV) < 0.1, -1, torch.randint(0, n, (runs,), generator=g, device=DEV))
    s["ids"] = who.repeat_interleave(128)[:T].int().contiguous()
    return s


def _prepare_adamw(s, g):
    """One run of memory for each kind of tensor, every tensor from a multiple of 32 on: what lies between two of them is zero."""
    sizes = _sizes(s["sizes"])
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += GROUP * -(-n // GROUP)
    at = torch.tensor(starts, device=DEV)
    ends = at + torch.tensor(sizes, device=DEV)
    place = torch.arange(total, device=DEV)
    inside = place < ends[torch.searchsorted(at, place, right=True) - 1]
    del place
    s["P"] = _normal((total,), g).mul_(0.05).mul_(inside)
    s["G"] = _gradient(total, g).mul_(inside).to(DTYPES[s["grad"]])
    m = _gradient(total, g).mul_(0.3).mul_(inside)
    root = _gradient(total, g).abs_().add_(3e-5).mul_(0.1).mul_(inside)
    if s["bits"] == 8:
        zero = torch.full((total,), 1 << 15, dtype=torch.int64, device=DEV)               # to the nearest: half of a step
        s["M"], s["V"] = _code(m, zero, 3), _code(root, zero, 4)
    else:
        s["M"], s["V"] = m, root.square_()
    s["copy16"] = torch.zeros(total, dtype=DTYPES[s["copy"]], device=DEV) if s["copy"] else None
    s["grad_scale"] = torch.full((1,), 0.8, device=DEV)
    # the tensors, as a program has them; their parts of the states, and each one's place in the sequence of random numbers
    s["items"] = []
    for n, a in zip(sizes, starts):
        groups = slice(a // GROUP, (a + n + GROUP - 1) // GROUP)
        part = slice(a, a + n)
        state = [(s[k][0][a:groups.stop * GROUP], s[k][1][groups]) if s["bits"] == 8 else s[k][part] for k in ("M", "V")]
        s["items"].append({"P": s["P"][part], "G": s["G"][part], "M": state[0], "V": state[1],
                           "copy": s["copy16"][part] if s["copy"] else None, "weight_decay": DECAY, "place": a})
    return s


# ------------------------------------------------------------------------------------------ formats, in plain operations
def _pow2(e):
    """2^e as fp32, exactly, for whole e of -126 .. 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _restore8(x):
    """What a tensor saved in 8 bits stands for, fp32."""
    rows, cols = x.shape
    n = -(-cols // GROUP)
    v = torch.nn.functional.pad(x.float(), (0, n * GROUP - cols)).reshape(rows, n, GROUP)
    e, v = _exponent(v, 6, lambda a: a >= 127.5)
    return (torch.round(v).clamp(-127, 127) * _pow2(e)).reshape(rows, -1)[:, :cols]


def _exponent(v, top, over):
    """floor(log2(largest magnitude)) - top of each group, one more where the largest would be `over`; and the values scaled."""
    big = v.abs().amax(dim=2, keepdim=True)
    e = (torch.frexp(big)[1] - 1 - top).clamp(-110, 120)
    at = big * _pow2(-e)
    e = torch.where(over(at), e + 1, e)
    e = torch.where(big == 0, torch.full_like(e, -110), e)
    return e, v * _pow2(-e)


def _quantize4(w):
    """Codes 0..15 [rows, K'] and scale bytes [rows, K'/32] of weights, K' a multiple of 128."""
    F, K = w.shape
    K1 = 128 * -(-K // 128)
    e, v = _exponent(torch.nn.functional.pad(w, (0, K1 - K)).reshape(F, K1 // GROUP, GROUP), 2, lambda a: a > 7.0)
    a = v.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
            + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
    code = code + 8 * torch.signbit(v).to(torch.uint8)
    return code.reshape(F, -1), (e + 127).to(torch.uint8).squeeze(2)


def _tiles(code, scale):
    """The layout of include/dab.h: per 16 rows and 128 weights 64 pieces of 16 bytes, piece l of row l % 16 and group l / 16; scales likewise,
    four steps of 128 weights side by side."""
    F, K = code.shape
    Ft, Kt = (F + 15) // 16, K // 128
    code = torch.nn.functional.pad(code, (0, 0, 0, Ft * 16 - F))
    K4 = (Kt + 3) // 4
    scale = torch.nn.functional.pad(scale, (0, 4 * (K4 * 4 - Kt), 0, Ft * 16 - F), value=17)
    pair = code.reshape(Ft, 16, Kt, 4, 16, 2)
    Q = (pair[..., 0] | (pair[..., 1] << 4)).permute(0, 2, 3, 1, 4).contiguous()      # [Ft][Kt][group][row][byte]
    S = scale.reshape(Ft, 16, K4, 4, 4).permute(0, 2, 4, 1, 3).contiguous()           # [Ft][K4][group][row][step]
    return Q.reshape(Ft, Kt, 64, 16), S.reshape(Ft, K4, 64, 4)


def _untile(Q, S, F, K):
    """The weights that a layout stands for, fp32 [F, K]."""
    Ft, Kt = Q.shape[:2]
    b = Q.reshape(Ft, Kt, 4, 16, 16).permute(0, 3, 1, 2, 4)                           # [Ft][row][Kt][group][byte]
    code = torch.stack([b & 15, b >> 4], dim=-1).reshape(Ft * 16, Kt * 128)
    scale = S.reshape(Ft, S.shape[1], 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(Ft * 16, -1)[:, :Kt * 4]
    levels = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=Q.device)
    v = levels[code.long()].reshape(Ft * 16, -1, GROUP) * _pow2(scale.int() - 127).unsqueeze(2)
    return v.reshape(Ft * 16, -1)[:F, :K]


def _mix(x):
    """32 bits, mixed; x: int64 of 0 .. 2^32 - 1, or a Python int."""
    x = x ^ (x >> 16)
    x = (x * 0x85A308D3) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x9E3779B1) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _chance(total):
    """The 32 random bits of every place."""
    key = _mix((SEED & 0xFFFFFFFF) + _mix((SEED >> 32) + _mix(STEP) & 0xFFFFFFFF) & 0xFFFFFFFF)
    place = torch.arange(total, device=DEV)
    return _mix((place + _mix(key)) & 0xFFFFFFFF)                 # (places here are below 2^32: their upper half is 0)


def _code(x, chance, bits):
    """(codes uint8, scale bytes) of values in groups of 32, rounded by 16 bits of chance; bits: of the significand (3: with a sign above it)."""
    v = x.reshape(-1, GROUP)
    big = v.abs().amax(dim=1, keepdim=True)
    drop = 23 - bits
    f = (((big.view(torch.int32) + ((1 << drop) - 1)) >> 23) - 127).clamp(-100, 120)
    y = v.abs() * _pow2(-f)
    whole = torch.where(y >= 2.0 ** -14, y.view(torch.int32) - (112 << 23), (y * 2.0 ** 37).to(torch.int32))
    code = ((whole + (chance.reshape(-1, GROUP).to(torch.int32) << (drop - 16))) >> drop).clamp(max=(16 << bits) - 1)
    if bits == 3:
        code = code + 128 * torch.signbit(v)
    else:
        code = torch.where(v > 0, code.clamp(min=1), code)
    return code.to(torch.uint8).reshape(-1), (f + 127).to(torch.uint8).reshape(-1)


def _value(code, scale, bits):
    """What codes stand for, fp32."""
    c = code.reshape(-1, GROUP).to(torch.int32)
    a = c & 127 if bits == 3 else c
    e, low = a >> bits, (a & ((1 << bits) - 1)).float()
    v = torch.where(e == 0, low * 2.0 ** (-14 - bits), (low * 2.0 ** -bits + 1.0) * _pow2(e - 15))
    v = v * _pow2(scale.int() - 127).unsqueeze(1)
    return (torch.where(c >= 128, -v, v) if bits == 3 else v).reshape(-1)


# ------------------------------------------------------------------------------------------ plain forms
def _plain_norm(s):
    dt = s["X"].dtype
    H = s["X"] if s["R"] is None else (s["X"].float() + s["R"].float()).to(dt)
    h = H.float()
    rstd = torch.rsqrt(h.square().mean(dim=1) + EPS)
    y = h * rstd.unsqueeze(1) * s["gain"]
    out = {"Y": y.to(dt), "rstd": rstd}
    if s["R"] is not None:
        out["H"] = H
    if s["saved"]:
        out["saved"] = _restore8(y).to(torch.bfloat16)
    return out


def _plain_norm_grad(s):
    h, rstd, dy = s["X"].float(), s["rstd"].unsqueeze(1), s["dY"].float()
    n = h * rstd
    w = dy * s["gain"]
    dx = (w - n * (w * n).mean(dim=1, keepdim=True)) * rstd
    if s["R"] is not None:
        dx = dx + s["R"].float()
    return {"dX": dx.to(s["X"].dtype), "dgain": (dy * n).sum(dim=0)}


def _plain_adamw(s):
    g = s["G"].float() * s["grad_scale"]
    m = s["M"] if s["bits"] == 32 else _value(*s["M"], 3)
    v = s["V"] if s["bits"] == 32 else _value(*s["V"], 4).square()
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + ((1.0 - BETA2) * g) * g
    root = v.sqrt()
    step = (LR / (1.0 - BETA1 ** STEP)) * m / (root * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + ADAM_EPS)
    s["P"].copy_(s["P"] * (1.0 - LR * DECAY) - step)
    out = {"P": s["P"]}
    if s["bits"] == 32:
        s["M"].copy_(m), s["V"].copy_(v)
        out.update(M=s["M"], V=s["V"])
    else:
        chance = _chance(m.numel())
        for k, x, bits, part in (("M", m, 3, chance & 0xFFFF), ("V", root, 4, chance >> 16)):
            q, e = _code(x, part, bits)
            s[k][0].copy_(q), s[k][1].copy_(e)
            out[k] = _value(q, e, bits).to(torch.bfloat16)
    if s["copy"]:
        s["copy16"].copy_(s["P"])
        out["copy"] = s["copy16"]
    return out


def _flat(s):
    """Every adapter's rows under one another, fp32, and which of them a token takes, times its scale."""
    n, r = s["n"], s["r"]
    A, Bt = s["A"].float().reshape(n * r, -1), s["Bt"].float().reshape(n * r, -1)
    takes = s["ids"].long().unsqueeze(1) == torch.arange(n, device=DEV).unsqueeze(0)
    return A, Bt, takes.float().repeat_interleave(r, dim=1), s["scale"].repeat_interleave(r)


def _plain_serve(s):
    A, Bt, takes, scale = _flat(s)
    x = s["X"].float()
    return {"Y": (x @ _untile(s["Q"], s["S"], s["F"], s["K"]).t() + ((x @ A.t()) * takes * scale) @ Bt).to(s["X"].dtype)}


def _plain_adapt(s):
    A, Bt, takes, scale = _flat(s)
    dt, T, n, r = s["X"].dtype, s["T"], s["n"], s["r"]
    x, dy = s["X"].float(), s["dY"].float()
    U = (x @ A.t()) * takes
    Y = s["base"].float() + (U * scale) @ Bt
    V = (dy @ Bt.t()) * takes * scale
    dX = s["dbase"].float() + V @ A
    return {"Y": Y.to(dt), "U": U.reshape(T, n, r).sum(dim=1), "dX": dX.to(dt), "dA": (V.t() @ x).reshape(n, r, -1),
            "dBt": ((U * scale).t() @ dy).reshape(n, r, -1)}


def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "adamw": _plain_adamw, "serve": _plain_serve, "adapt": _plain_adapt}[s["kind"]](s)


def _run_own(s):
    from paper_1804_02941_amd import binding as dab
    kind = s["kind"]
    if kind == "norm":
        Y, H, rstd, saved = dab.dab_rms_norm(s["X"], s["gain"], residual=s["R"], eps=EPS, save=s["saved"])
        out = {"Y": Y, "rstd": rstd}
        if s["R"] is not None:
            out["H"] = H
        if s["saved"]:
            out["saved"] = dab.dab_ckpt8_restore(*saved, s["cols"], torch.bfloat16)
        return out
    if kind == "norm_grad":
        dX, dgain = dab.dab_rms_norm_gradient(s["dY"], s["X"], s["gain"], s["rstd"], dH=s["R"])
        return {"dX": dX, "dgain": dgain}
    if kind == "adamw":
        if "jobs" not in s:
            s["jobs"] = dab.adamw_jobs(s["items"])
        dab.dab_adamw(s["jobs"], LR, STEP, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, grad_scale=s["grad_scale"], seed=SEED)
        out = {"P": s["P"]}
        for k, signed in (("M", True), ("V", False)):
            out[k] = s[k] if s["bits"] == 32 else dab.dab_state8_restore(*s[k], signed, torch.bfloat16)
        if s["copy"]:
            out["copy"] = s["copy16"]
        return out
    if kind == "serve":
        return {"Y": dab.dab_w4_adapters(s["X"], s["Q"], s["S"], s["F"], s["ids"], s["A"], s["Bt"], s["scale"])}
    Y, U = dab.dab_adapters(s["X"], s["ids"], s["A"], s["Bt"], s["scale"], base=s["base"])
    dX, dA, dBt = dab.dab_adapters_gradient(s["dY"], s["X"], U, s["ids"], s["A"], s["Bt"], s["scale"], base=s["dbase"])
    return {"Y": Y, "U": U, "dX": dX, "dA": dA, "dBt": dBt}


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "norm":        # the input in, the output out; a residual in and their sum out; the 8-bit output out and in, its values out
        e = SIZE[c["dtype"]] * (4 if c["residual"] else 2) + (2 * (1 + 1 / GROUP) + 2 if c["saved"] else 0)
        return {"bytes": c["rows"] * (c["cols"] * e + 4) + 4 * c["cols"], "flops": 0}
    if c["kind"] == "norm_grad":
        return {"bytes": c["rows"] * (c["cols"] * SIZE[c["dtype"]] * (4 if c["residual"] else 3) + 4) + 8 * c["cols"], "flops": 0}
    if c["kind"] == "adamw":       # weights and states in and out, gradients in, copies out; 8-bit states are read once more, as values
        state = 16 if c["bits"] == 32 else 4 * (1 + 1 / GROUP) + 2 * (1 + 1 / GROUP + 2)
        return {"bytes": sum(_sizes(c["sizes"])) * (8 + SIZE[c["grad"]] + state + (2 if c["copy"] else 0)), "flops": 0}
    size, n, r, K, F = SIZE[c["dtype"]], c["n"], c["r"], c["K"], c["F"]
    if c["kind"] == "serve":       # adapters of at most B requests
        return {"bytes": F * K * (0.5 + 1 / GROUP) + size * (c["B"] * (K + F) + min(n, c["B"]) * r * (K + F)), "flops": 2 * c["B"] * (F * K + r * (K + F))}
    T = c["T"]
    return {"bytes": 3 * size * T * (K + F) + n * r * (K + F) * (size + 4) + 4 * T * r, "flops": 6 * T * r * (K + F)}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def _levels64(x):
    """Each weight's nearest 4-bit level times its group's scale."""
    rows, cols = x.shape
    n = -(-cols // GROUP)
    big = torch.zeros((rows, n * GROUP), dtype=torch.float64, device=x.device)
    big[:, :cols] = x.double().abs()
    big = big.reshape(rows, n, GROUP).amax(dim=2)
    scale = torch.exp2((torch.floor(torch.log2(big.clamp(min=2.0 ** -120))) - 2).clamp(-110, 120).round())
    scale = torch.where(big / scale > 7.0, 2 * scale, scale).repeat_interleave(GROUP, dim=1)[:, :cols]
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    a = x.double().abs() / scale
    lo = (torch.searchsorted(levels, a.contiguous(), right=True) - 1).clamp(0, 6)
    below, above = a - levels[lo], levels[lo + 1] - a
    up = (above < below) | ((above == below) & (lo % 2 == 1))
    return torch.sign(x.double()) * levels[torch.where(up, lo + 1, lo)] * scale


def _bytes64(y):
    """Values y (float64) rounded to bytes with a power of two per 32 of a row."""
    rows, cols = y.shape
    out = torch.empty_like(y)
    for a in range(0, cols, GROUP):
        part = y[:, a:a + GROUP]
        big = part.abs().amax(dim=1, keepdim=True)
        _, e = torch.frexp(torch.where(big > 0, big, torch.full_like(big, 2.0 ** -200)))
        scale = torch.ldexp(torch.ones_like(big), (e - 7).clamp(-110, 120))
        scale = torch.where(big / scale >= 127.5, 2 * scale, scale)
        out[:, a:a + GROUP] = torch.round(part / scale) * scale
    return out


def _by_chance64(x, chance, bits):
    """A multiple of the step of its binade below or above each value, the upper one where the rest and the chance make up a step."""
    v = x.reshape(-1, GROUP)
    big = v.abs().amax(dim=1, keepdim=True).clamp(min=2.0 ** -100)
    top = torch.frexp(big)[1] - 1
    top = torch.where(big > torch.ldexp(torch.full_like(big, 2.0 - 2.0 ** -bits), top), top + 1, top)
    own_binade = torch.frexp(v.abs().clamp(min=2.0 ** -300))[1] - 1
    step = torch.ldexp(torch.ones_like(v), torch.maximum(own_binade, top - 14) - bits)
    code = torch.floor(v.abs() / step + chance.reshape(-1, GROUP).double() / 65536.0)
    if bits == 4:
        code = torch.where(v != 0, code.clamp(min=1.0), code)
    most = torch.ldexp(torch.full_like(big, 2.0 - 2.0 ** -bits), top)
    return (torch.minimum(code * step, most) * torch.sign(v)).reshape(-1)


def _exact_adamw(case, s):
    P, M, V, copy = [], [], [], []
    chance = _chance(s["P"].numel()) if case["bits"] == 8 else None
    part = 16 * 1024 * 1024
    keep, first = 1.0 - LR * DECAY, LR / (1.0 - BETA1 ** STEP)
    for a in range(0, s["P"].numel(), part):
        at = slice(a, a + part)
        g = s["G"][at].double() * float(s["grad_scale"])
        if case["bits"] == 8:
            groups = slice(a // GROUP, (a + part) // GROUP)
            m, v = _value(s["M"][0][at], s["M"][1][groups], 3).double(), _value(s["V"][0][at], s["V"][1][groups], 4).double() ** 2
        else:
            m, v = s["M"][at].double(), s["V"][at].double()
        m, v = BETA1 * m + (1.0 - BETA1) * g, BETA2 * v + (1.0 - BETA2) * g * g
        P.append(s["P"][at].double() * keep - first * m / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + ADAM_EPS))
        if case["bits"] == 8:
            m, v = _by_chance64(m, chance[at] & 0xFFFF, 3), _by_chance64(torch.sqrt(v), chance[at] >> 16, 4)
        M.append(m), V.append(v)
    out = {"P": torch.cat(P), "M": torch.cat(M), "V": torch.cat(V)}
    if case["copy"]:
        out["copy"] = out["P"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        # the norm is that of the sum as it is kept
        total = s["X"].double() if s["R"] is None else s["X"].double() + s["R"].double()
        h = s["X"].double() if s["R"] is None else total.float().to(s["X"].dtype).double()
        rstd = 1.0 / torch.sqrt((h * h).sum(dim=1) / case["cols"] + EPS)
        y = h * rstd[:, None] * s["gain"].double()[None, :]
        out = {"Y": y, "rstd": rstd}
        if s["R"] is not None:
            out["H"] = total
        if case["saved"]:
            out["saved"] = _bytes64(y)
        return out
    if kind == "norm_grad":
        # y_j = gain_j x_j / q with q^2 = mean(x^2) + eps:  dx_i = gain_i dy_i / q - x_i sum_j(gain_j dy_j x_j) / (cols q^3)
        x, dy, gain = s["X"].double(), s["dY"].double(), s["gain"].double()
        q = 1.0 / s["rstd"].double()[:, None]
        dot = (dy * gain * x).sum(dim=1, keepdim=True)
        dx = dy * gain / q - x * dot / (case["cols"] * q ** 3)
        if s["R"] is not None:
            dx += s["R"].double()
        return {"dX": dx, "dgain": (dy * (x / q)).sum(dim=0)}
    if kind == "adamw":
        return _exact_adamw(case, s)
    X, ids, scale = s["X"].double(), s["ids"].long(), s["scale"].double()
    A, Bt = s["A"].double(), s["Bt"].double()
    if kind == "serve":
        g = _gen(seed)                                             # prepare()'s draws up to the weights
        _normal((case["n"], case["r"], case["K"]), g), _normal((case["n"], case["r"], case["F"]), g)
        torch.rand((case["n"],), generator=g, device=DEV)
        Y = torch.mm(X, _levels64(_normal((case["F"], case["K"]), g).mul_(1.0 / math.sqrt(case["K"]))).t())
        for b, i in enumerate(ids.tolist()):
            if i >= 0:
                Y[b] += scale[i] * torch.mv(Bt[i].t(), torch.mv(A[i], X[b]))
        return {"Y": Y}
    dY, Y, dX = s["dY"].double(), s["base"].double(), s["dbase"].double()
    U = torch.zeros((case["T"], case["r"]), dtype=torch.float64, device=DEV)
    dA, dBt = torch.zeros_like(A), torch.zeros_like(Bt)
    for i in range(case["n"]):
        at = torch.nonzero(ids == i).squeeze(1)
        if at.numel():
            U[at] = torch.mm(X[at], A[i].t())
            Y[at] += scale[i] * torch.mm(U[at], Bt[i])
            V = scale[i] * torch.mm(dY[at], Bt[i].t())
            dX[at] += torch.mm(V, A[i])
            dA[i], dBt[i] = torch.mm(V.t(), X[at]), scale[i] * torch.mm(U[at].t(), dY[at])
    return {"Y": Y, "U": U, "dX": dX, "dA": dA, "dBt": dBt}
