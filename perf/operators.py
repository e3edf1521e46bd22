"""Operators of large language models around the binarized layers: what is timed of them, and their plain forms.

A network whose body is binarized keeps real-valued ends.  Three sets of operators serve them, from a
training step to the answer to one token:

  head      the loss at the end of the network: softmax cross entropy of H W^T over a large vocabulary, in pieces of
            the vocabulary, without the logits, and its gradients with respect to H and W
  ckpt      what a layer's backward pass reads, held in 8 bits: a real input saved as bytes with one power of two per
            32 channels, and the product dW = dY^T X with what was saved (the upstream gradient of the binarized
            weights)
  w4        the layers that stay real (the head above all), served with 4-bit weights and one power of two per 32
            weights: the weights laid out once, and products of one token or a few with them

Kinds of work (a case's "kind"), each over a range of sizes that draw() covers: "head" (loss and both gradients), "save"
(save and restore), "grad" (save, then the weight gradient), "pack" (lay weights out and read them back), "matvec".

Formats (include/dab.h).  A group is 32 values that share a scale 2^(s-127), s one byte.  ckpt: signed bytes of -127 .. 127.
w4: sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6.  With f = floor(log2(largest magnitude)) the exponent is f - 6 (ckpt) or f - 2
(w4), one more where the largest would then lie at or above 127.5 (ckpt) or above 7 (w4); values are rounded to the nearest, ties to even.
"""
import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GROUP = 32                                  # values that share a scale
IGNORE = -100                               # target of a token that has no loss
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the last layer of a language model in training: a long batch of tokens, a large vocabulary
        {"name": "head_t8192_v131072", "kind": "head", "T": 8192, "D": 2048, "V": 131072, "dtype": "bf16", "ignored": 0.1},
        # a smaller vocabulary behind a layer as wide as the fully-connected ones of this package's benchmark
        {"name": "head_t2048_v32768", "kind": "head", "T": 2048, "D": 4096, "V": 32768, "dtype": "bf16", "ignored": 0.0},
        # fine tuning on answers: half of the tokens carry no loss; nothing fits a tile
        {"name": "head_ragged", "kind": "head", "T": 1999, "D": 1000, "V": 50021, "dtype": "bf16", "ignored": 0.5},
        # the classes behind the sketch network's last binarized layer, its training batch, in its own type
        {"name": "head_classes_f32", "kind": "head", "T": 256, "D": 512, "V": 250, "dtype": "f32", "ignored": 0.0},
        # a layer's input kept for the backward pass and read back (bandwidth)
        {"name": "save_65536x4096", "kind": "save", "rows": 65536, "cols": 4096, "dtype": "bf16"},
        # the weight gradient of the square fully-connected layer over a long batch of tokens
        {"name": "grad_16384x4096", "kind": "grad", "rows": 16384, "cols": 4096, "F": 4096, "dtype": "bf16"},
        # the wide fully-connected layer at its training batch, in this package's own type
        {"name": "grad_9216_f32", "kind": "grad", "rows": 1024, "cols": 9216, "F": 4096, "dtype": "f32"},
        # few filters, a long sum, nothing fits a tile
        {"name": "grad_ragged", "kind": "grad", "rows": 8191, "cols": 777, "F": 301, "dtype": "f16"},
        # one token through the square layer (latency), and through the head (bandwidth)
        {"name": "matvec_4096_b1", "kind": "matvec", "B": 1, "K": 4096, "F": 4096, "dtype": "bf16"},
        {"name": "matvec_head_b1", "kind": "matvec", "B": 1, "K": 4096, "F": 131072, "dtype": "bf16"},
        # a few requests served together, sizes that fit no tile, in this package's own type
        {"name": "matvec_ragged_b7", "kind": "matvec", "B": 7, "K": 9111, "F": 4099, "dtype": "f32"},
        # the wide layer's weights laid out
        {"name": "pack_4096x9216", "kind": "pack", "F": 4096, "K": 9216, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm; often a round one, often not."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 32:
        v = 16 * ((v + 8) // 16)
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["head", "head", "save", "grad", "grad", "matvec", "matvec", "pack"])
    if kind == "head":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = (8192 * 2048 * 131072) // (16 if dtype == "f32" else 2)
        while True:
            c = {"kind": kind, "T": _log(rng, 1, 8192), "D": _log(rng, 64, 4096), "V": _log(rng, 100, 131072), "dtype": dtype,
                 "ignored": rng.choice([0.0, 0.1, 0.5])}
            if c["T"] * c["D"] * c["V"] <= most:
                return c
    if kind in ("save", "grad"):
        while True:
            c = {"kind": kind, "rows": _log(rng, 1, 65536), "cols": _log(rng, 32, 9216), "dtype": rng.choice(["bf16", "f16", "f32"])}
            if kind == "grad":
                c["F"] = _log(rng, 32, 4096)
            if c["rows"] * c["cols"] <= 65536 * 4096 and c["rows"] * c["cols"] * c.get("F", 1) <= 65536 * 4096 * 1024:
                return c
    while True:
        c = {"kind": kind, "F": _log(rng, 16, 131072), "K": _log(rng, 64, 16384), "dtype": rng.choice(["bf16", "f16", "f32"])}
        if kind == "matvec":
            c["B"] = _log(rng, 1, 32)
        if c["F"] * c["K"] <= (131072 * 4096 if kind == "matvec" else 8192 * 8192):
            return c


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)


def _normal(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _activations(rows, cols, g):
    """A layer's input: normal, some channels much larger than the others, one row in a hundred zero."""
    gain = torch.exp(0.7 * _normal((1, cols), g))
    live = (torch.rand((rows, 1), generator=g, device=DEV) > 0.01).float()
    return _normal((rows, cols), g).mul_(gain).mul_(live)


def prepare(case, seed):
    c, g = case, _gen(seed)
    dt = DTYPES[c["dtype"]]
    s = dict(c)
    if c["kind"] == "head":
        s["H"] = _normal((c["T"], c["D"]), g).to(dt)
        # logits of a few units: peaked, but with a tail that counts
        s["W"] = _normal((c["V"], c["D"]), g).mul_(2.5 / math.sqrt(c["D"])).to(dt)
        t = torch.randint(0, c["V"], (c["T"],), generator=g, device=DEV)
        dead = torch.rand((c["T"],), generator=g, device=DEV) < c["ignored"]
        s["targets"] = torch.where(dead, torch.full_like(t, IGNORE), t)
        # every token its own weight (packed sequences of several lengths), about one over their number
        s["g"] = (0.5 + torch.rand((c["T"],), generator=g, device=DEV)) / c["T"]
    elif c["kind"] == "save":
        s["X"] = _activations(c["rows"], c["cols"], g).to(dt)
    elif c["kind"] == "grad":
        s["X"] = _activations(c["rows"], c["cols"], g).to(dt)
        s["dY"] = _normal((c["rows"], c["F"]), g).mul_(0.01).to(dt)
    elif c["kind"] == "pack":
        s["W"] = _normal((c["F"], c["K"]), g).mul_(1.0 / math.sqrt(c["K"])).to(dt)
    else:
        w = _normal((c["F"], c["K"]), g).mul_(1.0 / math.sqrt(c["K"]))
        s["Q"], s["S"] = _tiles(*_quantize4(w))
        s["X"] = _normal((c["B"], c["K"]), g).to(dt)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _groups(x, pad_to=GROUP):
    """x [rows, cols] as fp32 [rows, groups, 32], the last group filled with zeros."""
    rows, cols = x.shape
    full = pad_to * ((cols + pad_to - 1) // pad_to)
    x = x.float()
    if full != cols:
        x = torch.cat([x, torch.zeros((rows, full - cols), device=x.device)], dim=1)
    return x.reshape(rows, full // GROUP, GROUP)


def _pow2(e):
    """2^e as fp32, exactly, for whole e of -126 .. 127 (an exp2 that is off by a last bit would turn ties into other values)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(v, top, over):
    """floor(log2(largest magnitude)) - top of each group, one more where the largest would be `over` or more; and the values scaled."""
    big = v.abs().amax(dim=2, keepdim=True)
    e = (torch.frexp(big)[1] - 1 - top).clamp(-110, 120)
    at = big * _pow2(-e)
    e = torch.where(over(at), e + 1, e)
    e = torch.where(big == 0, torch.full_like(e, -110), e)
    return e, v * _pow2(-e)


def _restore8(x):
    """What a saved tensor stands for, fp32."""
    rows, cols = x.shape
    e, v = _exponent(_groups(x), 6, lambda a: a >= 127.5)
    return (torch.round(v).clamp(-127, 127) * _pow2(e)).reshape(rows, -1)[:, :cols]


def _quantize4(w):
    """Codes 0..15 [rows, K'] and scale bytes [rows, K'/32] of weights, K' a multiple of 128."""
    e, v = _exponent(_groups(w, 128), 2, lambda a: a > 7.0)
    a = v.abs()
    # magnitudes between two levels go to the nearer one, those in the middle to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
            + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
    code = code + 8 * torch.signbit(v).to(torch.uint8)
    return code.reshape(w.shape[0], -1), (e + 127).to(torch.uint8).squeeze(2)


def _value4(code, scale):
    levels = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=code.device)
    v = levels[code.long()].reshape(code.shape[0], -1, GROUP) * _pow2(scale.int() - 127).unsqueeze(2)
    return v.reshape(code.shape[0], -1)


def _tiles(code, scale):
    """The layout of include/dab.h: per 16 rows and 128 weights 64 pieces of 16 bytes, piece l of row l % 16 and group l / 16; scales likewise,
    four steps of 128 weights side by side."""
    F, K = code.shape
    Ft, Kt = (F + 15) // 16, K // 128
    if Ft * 16 != F:
        code = torch.cat([code, code.new_zeros((Ft * 16 - F, K))])
        scale = torch.cat([scale, scale.new_full((Ft * 16 - F, K // GROUP), 17)])
    pair = code.reshape(Ft, 16, Kt, 4, 16, 2)
    Q = (pair[..., 0] | (pair[..., 1] << 4)).permute(0, 2, 3, 1, 4).contiguous()      # [Ft][Kt][group][row][byte]
    K4 = (Kt + 3) // 4
    if K4 * 4 != Kt:
        scale = torch.cat([scale, scale.new_full((Ft * 16, 4 * (K4 * 4 - Kt)), 17)], dim=1)
    S = scale.reshape(Ft, 16, K4, 4, 4).permute(0, 2, 4, 1, 3).contiguous()           # [Ft][K4][group][row][step]
    return Q.reshape(Ft, Kt, 64, 16), S.reshape(Ft, K4, 64, 4)


def _untile(Q, S, F, K):
    """The weights that a layout stands for, fp32 [F, K]."""
    Ft, Kt = Q.shape[:2]
    b = Q.reshape(Ft, Kt, 4, 16, 16).permute(0, 3, 1, 2, 4)                           # [Ft][row][Kt][group][byte]
    code = torch.stack([b & 15, b >> 4], dim=-1).reshape(Ft * 16, Kt * 128)
    scale = S.reshape(Ft, S.shape[1], 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(Ft * 16, -1)[:, :Kt * 4]
    return _value4(code, scale)[:F, :K]


def _plain_head(s):
    H, W, t, dt = s["H"].float(), s["W"].float(), s["targets"], s["H"].dtype
    live = t != IGNORE
    H = torch.where(live.unsqueeze(1), H, torch.zeros_like(H))
    at = torch.where(live, t, torch.zeros_like(t)).unsqueeze(1)
    L = H @ W.t()
    m = L.amax(dim=1, keepdim=True)
    target = L.gather(1, at)
    P = L.sub_(m).exp_()
    z = P.sum(dim=1, keepdim=True)
    loss = torch.where(live, (m + z.log() - target).squeeze(1), torch.zeros_like(s["g"]))
    P.div_(z)
    P.scatter_add_(1, at, torch.full_like(target, -1.0))
    P.mul_(torch.where(live, s["g"], torch.zeros_like(s["g"])).unsqueeze(1))
    return {"loss": loss, "dH": (P @ W).to(dt), "dW": (P.t() @ H).to(dt)}


def run(s):
    if own:
        return _run_own(s)
    kind = s["kind"]
    if kind == "head":
        return _plain_head(s)
    if kind == "save":
        return {"X": _restore8(s["X"]).to(s["X"].dtype)}
    if kind == "grad":
        return {"dW": s["dY"].float().t() @ _restore8(s["X"])}
    if kind == "pack":
        code, scale = _quantize4(s["W"])
        return {"W": _value4(code, scale)[:, :s["K"]]}
    return {"Y": (s["X"].float() @ _untile(s["Q"], s["S"], s["F"], s["K"]).t()).to(s["X"].dtype)}


def _run_own(s):
    from paper_1804_02941_amd import binding as dab
    kind = s["kind"]
    if kind == "head":
        loss, lse = dab.dab_head_loss(s["H"], s["W"], s["targets"], ignore_index=IGNORE)
        dH, dW = dab.dab_head_loss_gradient(s["H"], s["W"], s["targets"], lse, s["g"], ignore_index=IGNORE)
        return {"loss": loss, "dH": dH, "dW": dW}
    if kind == "save":
        Q, S = dab.dab_ckpt8_save(s["X"])
        return {"X": dab.dab_ckpt8_restore(Q, S, s["cols"], s["X"].dtype)}
    if kind == "grad":
        Q, S = dab.dab_ckpt8_save(s["X"])
        return {"dW": dab.dab_ckpt8_weight_gradient(s["dY"], Q, S, s["cols"])}
    if kind == "pack":
        Q, S = dab.dab_w4_pack(s["W"])
        return {"W": dab.dab_w4_unpack(Q, S, s["F"], s["K"])}
    return {"Y": dab.dab_w4_matvec(s["X"], s["Q"], s["S"], s["F"])}


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    size = {"f32": 4, "bf16": 2, "f16": 2}[c["dtype"]]
    if c["kind"] == "head":
        T, D, V = c["T"], c["D"], c["V"]
        return {"bytes": 2 * size * (T * D + V * D) + 20 * T, "flops": 6 * T * D * V}
    if c["kind"] == "save":        # in, bytes out, bytes in, out
        return {"bytes": c["rows"] * c["cols"] * (2 * size + 2 * (1 + 1 / GROUP)), "flops": 0}
    if c["kind"] == "grad":
        rows, cols, F = c["rows"], c["cols"], c["F"]
        return {"bytes": rows * cols * (size + 2 * (1 + 1 / GROUP)) + rows * F * size + 4 * F * cols, "flops": 2 * rows * cols * F}
    if c["kind"] == "pack":
        return {"bytes": c["F"] * c["K"] * (size + 4 + 2 * (0.5 + 1 / GROUP)), "flops": 0}
    return {"bytes": c["F"] * c["K"] * (0.5 + 1 / GROUP) + size * c["B"] * (c["K"] + c["F"]), "flops": 2 * c["B"] * c["F"] * c["K"]}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def _scale64(x, levels_top, limit, include):
    """Per value: the group's scale in float64, from the definition."""
    rows, cols = x.shape
    n = -(-cols // GROUP)
    big = torch.zeros((rows, n * GROUP), dtype=torch.float64, device=x.device)
    big[:, :cols] = x.double().abs()
    big = big.reshape(rows, n, GROUP).max(dim=2).values
    safe = torch.where(big > 0, big, torch.ones_like(big))
    _, f = torch.frexp(safe)
    scale = (((f - 1 - levels_top).clamp(-110, 120).long() + 1023) << 52).view(torch.float64)
    up = safe / scale >= limit if include else safe / scale > limit
    return torch.where(up, 2 * scale, scale).repeat_interleave(GROUP, dim=1)[:, :cols]


def _levels64(x):
    """Each weight's nearest level times its group's scale."""
    scale = _scale64(x, 2, 7.0, False)
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    a = x.double().abs() / scale
    lo = (torch.searchsorted(levels, a.contiguous(), right=True) - 1).clamp(0, 6)
    hi = lo + 1
    below, above = a - levels[lo], levels[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return torch.sign(x.double()) * levels[torch.where(up, hi, lo)] * scale


def _bytes64(x):
    scale = _scale64(x, 6, 127.5, True)
    return torch.round(x.double() / scale) * scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "head":
        # every token's softmax in turns of a few thousand tokens, so that 64 bits fit
        T, V, t = case["T"], case["V"], s["targets"]
        W = s["W"].double()
        loss, dH = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros((T, case["D"]), dtype=torch.float64, device=DEV)
        dW = torch.zeros((V, case["D"]), dtype=torch.float64, device=DEV)
        for at in torch.nonzero(t != IGNORE).squeeze(1).split(2048):
            h = s["H"][at].double()
            z = torch.mm(h, W.t())
            lse = torch.logsumexp(z, dim=1)
            rows = torch.arange(at.numel(), device=DEV)
            loss[at] = lse - z[rows, t[at]]
            p = torch.exp(z - lse[:, None])
            p[rows, t[at]] -= 1
            p *= s["g"][at].double()[:, None]
            dH[at] = torch.mm(p, W)
            dW += torch.mm(p.t(), h)
        return {"loss": loss, "dH": dH, "dW": dW}
    if case["kind"] == "save":
        return {"X": _bytes64(s["X"])}
    if case["kind"] == "grad":
        return {"dW": torch.mm(s["dY"].double().t(), _bytes64(s["X"]))}
    if case["kind"] == "pack":
        return {"W": _levels64(s["W"])}
    w = _normal((case["F"], case["K"]), _gen(seed)).mul_(1.0 / math.sqrt(case["K"]))    # prepare()'s first draw
    return {"Y": torch.mm(s["X"].double(), _levels64(w).t())}
