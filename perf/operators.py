"""The work that the operators around the activation are measured by.

A transformer block trained with few-bit activations spends what is left of its
memory and time in three more places, and a case is one pass of a user's program
through one of them:

  op "attention"     mode "layer": the differentiable call and the gradients of q, k and v;
                     mode "calls": forward and backward called directly;
                     mode "fwd":   the forward alone (prompts in chunks, single tokens over a cache)
  op "qk_norm_rope"  RMS norm of every query and key head and its rotary position, in one
                     pass; modes as above
  op "adamw"         one optimizer step over all tensors of a model, moments in 32 bits or in 8

Where `own` is false a pass is computed in its plain form: elementary torch
operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch
import torch.nn.functional as F

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6                      # of the norms
BLOCK = 256                     # elements of a tensor that share one scale in 8-bit moments
BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.95, 1e-8, 3e-4, 0.1


# ---------------------------------------------------------------- the cases
def _attn(name, mode, dtype, b, sq, sk, hq, hkv, d, causal, window=0, lens="full"):
    c = {"op": "attention", "mode": mode, "dtype": dtype, "b": b, "sq": sq, "sk": sk, "hq": hq,
         "hkv": hkv, "d": d, "causal": causal, "window": window, "lens": lens}
    return c if name is None else {"name": name, **c}


def _qk(name, mode, dtype, b, s, hq, hkv, d, rot, interleaved):
    c = {"op": "qk_norm_rope", "mode": mode, "dtype": dtype, "b": b, "s": s, "hq": hq, "hkv": hkv,
         "d": d, "rot": rot, "interleaved": interleaved}
    return c if name is None else {"name": name, **c}


def _adamw(name, dtype, bits, master, layers, d, ff, count=0, most=0):
    c = {"op": "adamw", "dtype": dtype, "bits": bits, "master": master, "layers": layers, "d": d,
         "ff": ff, "count": count, "most": most}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one token over a short cache, one sequence: host work and launches only
        _attn("decode_bf16_1x777_h12_d64", "fwd", "bf16", 1, 1, 777, 12, 12, 64, True),
        # a served batch of single tokens over caches of very different lengths
        _attn("decode_bf16_64x8192_h16_4_d128", "fwd", "bf16", 64, 1, 8192, 16, 4, 128, True, lens="cache"),
        # a chunk of a long prompt behind a sliding window
        _attn("chunk_f16_1x1000_16384_h16_4_w4096", "fwd", "f16", 1, 1000, 16384, 16, 4, 128, True, window=4096),
        # BERT-base's attention at 8 x 512 tokens, both directions
        _attn("calls_f16_8x512_h12_d64", "calls", "f16", 8, 512, 512, 12, 12, 64, False),
        # documents of ragged lengths packed without padding, shared key heads
        _attn("calls_bf16_packed_24x1500_h16_4", "calls", "bf16", 24, 1500, 1500, 16, 4, 128, True, lens="packed"),
        # the attention beside the benchmark's feed-forward: 16 x 2048 tokens of width 2048
        _attn("layer_bf16_16x2048_h16_d128", "layer", "bf16", 16, 2048, 2048, 16, 16, 128, True),
        # one token for each of 64 sequences, before it is written to the cache
        _qk("qk_fwd_bf16_64x1_h16_4_d128", "fwd", "bf16", 64, 1, 16, 4, 128, 128, False),
        # adjacent pairs, half of the head rotated, an odd number of tokens
        _qk("qk_calls_f16_3x509_h12_d64", "calls", "f16", 3, 509, 12, 12, 64, 32, True),
        # 16 x 2048 tokens of width 2048 with shared key heads
        _qk("qk_layer_bf16_16x2048_h16_4_d128", "layer", "bf16", 16, 2048, 16, 4, 128, 128, False),
        # adapters and norms: many small tensors of odd sizes, a master copy
        _adamw("adamw_bf16_8bit_master_200_odd", "bf16", 8, True, 0, 0, 0, count=200, most=50001),
        # BERT-base's layers in fp32 with moments in 32 bits
        _adamw("adamw_f32_32bit_12x768", "f32", 32, False, 12, 768, 3072),
        # eight layers of width 2048 with moments in 8 bits
        _adamw("adamw_bf16_8bit_8x2048", "bf16", 8, False, 8, 2048, 8192),
    ]


_MOST_PAIRS = 16 * 16 * 2048 * 2048          # scores that the plain form of the largest listed case writes
_MOST_CACHE = 64 * 8192 * 4 * 128            # elements of the largest listed cache
_MOST_QK = 16 * 2048 * 20 * 128
_MOST_PARAMS = 8 * (4 * 2048 * 2048 + 2 * 2048 * 8192)


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "qk_norm_rope", "adamw"))
    if op == "attention":
        mode = rng.choice(("fwd", "calls", "calls", "layer"))
        dtype = rng.choice(("bf16", "bf16", "f16"))
        d = rng.choice((64, 64, 128, 128, 128, 32, 80, 96))
        hkv, g = rng.choice((1, 2, 3, 4, 8, 12, 16)), rng.choice((1, 1, 2, 4, 8))
        b, sq = _log(rng, 1, 32), _log(rng, 16, 4096)
        sk, lens, causal, window = sq, "full", rng.random() < 0.7, 0
        if mode == "fwd":
            sk, lens = _log(rng, 16, 16384), rng.choice(("full", "cache"))
            sq = min(sk, rng.choice((1, 1, 1, _log(rng, 2, 1024))))
            b = _log(rng, 1, 64)
        elif rng.random() < 0.4:
            lens = "packed"
        if causal and rng.random() < 0.3:
            window = _log(rng, 8, 2048)
        while b * hkv * g * sq * sk > _MOST_PAIRS or b * sk * hkv * d > _MOST_CACHE:
            if b > 1:
                b = b // 2
            elif g > 1:
                g = g // 2
            else:
                hkv = max(1, hkv // 2)
        return _attn(None, mode, dtype, b, sq, sk, hkv * g, hkv, d, causal, window, lens)
    if op == "qk_norm_rope":
        mode = rng.choice(("fwd", "calls", "layer"))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        d = rng.choice((64, 128, 128, 96, 256))
        rot = rng.choice((d, d, d // 2))
        hkv, g = rng.choice((1, 2, 4, 8, 12)), rng.choice((1, 2, 4))
        b, s = _log(rng, 1, 64), _log(rng, 1, 4096)
        while b * s * (hkv * g + hkv) * d * SIZE[dtype] > 2 * _MOST_QK:
            b, s = (b // 2, s) if b > 1 else (1, s // 2)
        return _qk(None, mode, dtype, b, s, hkv * g, hkv, d, rot, rng.random() < 0.4)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    bits, master = rng.choice((8, 8, 32)), dtype != "f32" and rng.random() < 0.4
    if rng.random() < 0.4:
        count, most = _log(rng, 3, 400), _log(rng, 100, 200000)
        return _adamw(None, dtype, bits, master, 0, 0, 0, count=count, most=most)
    d = 8 * _log(rng, 16, 256)
    layers = rng.choice((2, 4, 8, 12))
    while sum(_sizes(_adamw(None, dtype, bits, master, layers, d, 4 * d))) * (1 if bits == 8 else 4) > _MOST_PARAMS:
        layers -= 1
        if layers == 0:
            layers, d = 1, d // 2
    return _adamw(None, dtype, bits, master, layers, d, 4 * d)


# ---------------------------------------------------------------- sizes that follow from a case
def _lengths(case):
    """Queries and keys of each sequence (lists): all of them alike, or spread as documents and
    caches are, the same for every seed."""
    b, sq, sk = case["b"], case["sq"], case["sk"]
    if case["lens"] == "full":
        return [sq] * b, [sk] * b
    r = random.Random(1000003 * b + 31 * sk + sq)
    if case["lens"] == "cache":
        return [sq] * b, [sk] + [r.randint(1, sk) for _ in range(b - 1)]
    lens = [sq] + [r.randint(1, sq) for _ in range(b - 1)]
    return lens, lens


def _pairs(case):
    """(Query, key) pairs that the mask lets through, for one head, and the keys that any of them reads."""
    pairs = keys = 0
    for nq, nk in zip(*_lengths(case)):
        hi = np.minimum(nk, np.arange(nq) + nk - nq + 1) if case["causal"] else np.full(nq, nk)
        hi = np.maximum(hi, 0)
        lo = np.maximum(0, np.arange(nq) + nk - nq + 1 - case["window"]) if case["window"] else np.zeros(nq, dtype=int)
        n = np.maximum(0, hi - lo)
        pairs += int(n.sum())
        seen = n > 0
        keys += int(hi[seen].max() - lo[seen].min()) if seen.any() else 0
    return pairs, keys


def _sizes(case):
    """Elements of every tensor that the optimizer steps."""
    if case["count"]:
        r = random.Random(17 * case["count"] + case["most"])
        return [case["most"], 1] + [_log(r, 1, case["most"]) for _ in range(case["count"] - 2)]
    d, ff = case["d"], case["ff"]
    layer = [3 * d * d, 3 * d, d * d, d, ff * d, ff, d * ff, d, d, d, d, d]
    return layer * case["layers"]


def _blocks(n):
    return -(-n // BLOCK)


# ---------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _prepare_attention(case, gen):
    dt = DTYPES[case["dtype"]]
    b, sq, sk, hq, hkv, d = (case[k] for k in ("b", "sq", "sk", "hq", "hkv", "d"))
    nq, nk = _lengths(case)
    state = {"nq": torch.tensor(nq, device="cuda"), "nk": torch.tensor(nk, device="cuda"), "k_len": None, "cu": None}
    q_rows, k_rows = ((sum(nq),), (sum(nk),)) if case["lens"] == "packed" else ((b, sq), (b, sk))
    state["q"] = _randn(gen, *q_rows, hq, d).to(dt)
    if case["mode"] == "fwd":                            # a cache: keys and values each in their own buffer
        state["k"], state["v"] = _randn(gen, *k_rows, hkv, d).to(dt), _randn(gen, *k_rows, hkv, d).to(dt)
    else:                                                # keys from the norm, values a view of the projection
        state["k"] = _randn(gen, *k_rows, hkv, d).to(dt)
        state["v"] = _randn(gen, *k_rows, hq + 2 * hkv, d).to(dt)[..., hq + hkv:, :]
        state["dout"] = _randn(gen, *q_rows, hq, d).to(dt)
    if case["lens"] == "cache":
        state["k_len"] = torch.tensor(nk, dtype=torch.int32, device="cuda")
    elif case["lens"] == "packed":
        cu = [0]
        for n in nq:
            cu.append(cu[-1] + n)
        state["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    if case["mode"] == "layer":
        for name in ("q", "k", "v"):
            state[name].requires_grad_()
    return state


def _prepare_qk(case, gen):
    dt = DTYPES[case["dtype"]]
    b, s, hq, hkv, d, rot = (case[k] for k in ("b", "s", "hq", "hkv", "d", "rot"))
    qkv = _randn(gen, b, s, hq + 2 * hkv, d)
    qkv = (qkv * torch.rand(b, s, 1, 1, generator=gen, device="cuda").mul_(4.0).add_(0.1)).to(dt)
    state = {"q": qkv[:, :, :hq], "k": qkv[:, :, hq:hq + hkv]}
    for name in ("wq", "wk"):
        state[name] = (1.0 + 0.2 * _randn(gen, d)).to(dt)
    most = 8192
    first = torch.randint(0, most - s + 1, (b, 1), generator=gen, device="cuda")
    state["positions"] = first + torch.arange(s, device="cuda")
    angle = torch.arange(most, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda").double() / rot)
    state["cos"], state["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    if case["mode"] != "fwd":
        state["dq"], state["dk"] = _randn(gen, b, s, hq, d).to(dt), _randn(gen, b, s, hkv, d).to(dt)
    if case["mode"] == "layer":
        for name in ("q", "k", "wq", "wk"):
            state[name].requires_grad_()
    return state


def _prepare_adamw(case, gen):
    dt, sizes = DTYPES[case["dtype"]], _sizes(case)
    total = sum(_blocks(n) for n in sizes) * BLOCK
    at = [0]
    for n in sizes:
        at.append(at[-1] + _blocks(n) * BLOCK)
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for n, a in zip(sizes, at):
        inside[a:a + n] = True
    spread = torch.exp(1.5 * _randn(gen, total // BLOCK, 1))             # rows of very different size

    def values(scale):
        return (_randn(gen, total // BLOCK, BLOCK).mul_(spread).mul_(scale).view(-1)).mul_(inside)

    weights = _randn(gen, total).mul_(0.02).mul_(inside)
    state = {"bits": case["bits"], "sizes": sizes, "t": 100, "flat": weights.to(dt), "master": weights if case["master"] else None}
    grads = values(1e-3).to(dt)
    state["params"] = [state["flat"][a:a + n] for n, a in zip(sizes, at)]
    state["grads"] = [grads[a:a + n] for n, a in zip(sizes, at)]
    m, v = values(3e-4), values(1e-3).square_()
    if case["bits"] == 32:
        return {**state, "m": m, "v": v, "ms": None, "vs": None}
    for name, x in (("m", m), ("v", v)):
        x = x.view(-1, BLOCK)
        scale = _scale(x.abs().amax(1, keepdim=True))
        state[name] = (x / scale).to(torch.float8_e4m3fn).view(-1)
        state[name + "s"] = scale.view(-1)
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    make = {"attention": _prepare_attention, "qk_norm_rope": _prepare_qk, "adamw": _prepare_adamw}[case["op"]]
    return {"case": case, **make(case, gen)}


# ---------------------------------------------------------------- attention, plain
def _heads(x, state, case, n, lens):
    """[b, kv heads, head's share of the q heads x tokens, d] in 32 bits of a padded or packed tensor."""
    x = x.float()
    if case["lens"] == "packed":
        x = F.pad(x, (0, 0, 0, 0, 0, 1))
        at = state["cu"][:-1, None] + torch.arange(n, device="cuda")
        x = x[torch.where(torch.arange(n, device="cuda") < lens[:, None], at, x.shape[0] - 1)]
    x = x.unflatten(2, (case["hkv"], -1)).permute(0, 2, 3, 1, 4)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[4])


def _rows(x, state, case, n, lens, dtype):
    """_heads' way back, rounded."""
    x = x.unflatten(2, (-1, n)).permute(0, 3, 1, 2, 4).flatten(2, 3).to(dtype)
    return x[torch.arange(n, device="cuda") < lens[:, None]] if case["lens"] == "packed" else x.contiguous()


def _plain_attention(state):
    case, nq, nk = state["case"], state["nq"], state["nk"]
    sq, sk, dt = case["sq"], case["sk"], state["q"].dtype
    q, k, v = (_heads(state[n], state, case, s, c) for n, s, c in (("q", sq, nq), ("k", sk, nk), ("v", sk, nk)))
    i = torch.arange(sq, device="cuda")[:, None] + (nk - nq)[:, None, None]      # the key that stands where a query does
    j = torch.arange(sk, device="cuda")
    hidden = (j >= nk[:, None, None]).expand(-1, sq, -1)
    if case["causal"]:
        hidden = hidden | (j > i)
    if case["window"]:
        hidden = hidden | (j <= i - case["window"])
    scale = 1.0 / math.sqrt(case["d"])
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).unflatten(2, (-1, sq))
    s = s.masked_fill_(hidden[:, None, None], -math.inf).flatten(2, 3)
    most = s.amax(3, keepdim=True)
    p = s.sub_(most.clamp(min=-1e30)).exp_()
    total = p.sum(3, keepdim=True)
    lse = (most + torch.log(total)).squeeze(3).unflatten(2, (-1, sq)).flatten(1, 2)
    p = p.div_(torch.where(total > 0, total, 1.0))
    out = torch.matmul(p, v)
    r = {"out": _rows(out, state, case, sq, nq, dt)}
    if case["mode"] != "layer":
        r["lse"] = lse.transpose(1, 2)[torch.arange(sq, device="cuda") < nq[:, None]].t().contiguous() if case["lens"] == "packed" else lse
    if case["mode"] == "fwd":
        return r
    do = _heads(state["dout"], state, case, sq, nq)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * out).sum(3, keepdim=True)).mul_(p).mul_(scale)
    r["dq"] = _rows(torch.matmul(ds, k), state, case, sq, nq, dt)
    r["dk"] = _rows(torch.matmul(ds.transpose(2, 3), q), state, case, sk, nk, dt)
    r["dv"] = _rows(dv, state, case, sk, nk, dt)
    return r


# ---------------------------------------------------------------- norm and rotation, plain
def _rotate(x, cos, sin, interleaved):
    """The first 2 * cos.shape[-1] of the last axis turned by the angles, the others as they are."""
    half = cos.shape[-1]
    a, b = (x[..., :2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_norm(state, name):
    """One of q and k: its output and, in training, its gradient and its weight's."""
    case, x, w = state["case"], state[name].float(), state["w" + name].float()
    cos, sin = state["cos"][state["positions"]].unsqueeze(2), state["sin"][state["positions"]].unsqueeze(2)
    dt, turn = state[name].dtype, case["interleaved"]
    size = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    unit = x * size
    y = _rotate(unit * w, cos, sin, turn).to(dt)
    if case["mode"] == "fwd":
        return {name: y}
    g = _rotate(state["d" + name].float(), cos, -sin, turn)
    dw = (g * unit).sum((0, 1, 2))
    g = g * w
    dx = (g - unit * (g * unit).mean(-1, keepdim=True)) * size
    # the layer's weight is an ordinary parameter: its gradient has its type
    return {name: y, "d" + name: dx.to(dt), "dw" + name: dw.to(dt) if case["mode"] == "layer" else dw}


# ---------------------------------------------------------------- optimizer step, plain
def _scale(most):
    """The least power of two that takes a block's largest magnitude to at most 448, the largest number of
    the 8-bit format, and no less than 2^-125."""
    f, e = torch.frexp(most.clamp(min=2.0 ** -117))
    return torch.ldexp(torch.ones_like(most), e - 9 + (f > 0.875))


def _dither(n, seed):
    """Two numbers of 16 bits for every element, in [0, 1): the seed's and the element's place."""
    word = 0xFFFFFFFF
    x = torch.arange(n, device="cuda") * 0x9E3779B1 + ((seed * 0x6A09E667 + 0x3C6EF372) & word)
    x = x & word
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & word
    x = x ^ (x >> 13)
    return (x >> 16).float() * 2.0 ** -16, (x & 0xFFFF).float() * 2.0 ** -16


def _to_8_bits(x, u):
    """The codes and scales of blocks, each value rounded down or up at random (u) so that its mean is kept."""
    x = x.view(-1, BLOCK)
    scale = _scale(x.abs().amax(1, keepdim=True))
    y = x / scale
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), e.clamp(min=-5) - 4)       # 3 bits after the leading one
    return torch.copysign(torch.floor(y.abs() / step + u.view(-1, BLOCK)) * step, y), scale.view(-1)


def _plain_adamw(state):
    b1, b2, t = BETA1, BETA2, state["t"]
    pads = [_blocks(n) * BLOCK - n for n in state["sizes"]]
    g = torch.cat([F.pad(x.float(), (0, n)) for x, n in zip(state["grads"], pads)])
    w = state["master"] if state["master"] is not None else torch.cat([F.pad(x.float(), (0, n)) for x, n in zip(state["params"], pads)])
    m, v = state["m"].float(), state["v"].float()
    if state["bits"] == 8:
        m = (m.view(-1, BLOCK) * state["ms"][:, None]).view(-1)
        v = (v.view(-1, BLOCK) * state["vs"][:, None]).view(-1)
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * g) * (1.0 - b2)
    w = w * (1.0 - LR * DECAY) - (LR / (1.0 - b1 ** t)) * (m / (torch.sqrt(v) / math.sqrt(1.0 - b2 ** t) + ADAM_EPS))
    torch._foreach_copy_(state["params"], [x[:n] for x, n in zip(torch.split(w, [n + p for n, p in zip(state["sizes"], pads)]), state["sizes"])])
    if state["master"] is not None:
        state["master"].copy_(w)
    if state["bits"] == 8:
        um, uv = _dither(m.numel(), t)
        codes, scale = _to_8_bits(m, um)
        state["m"].copy_(codes.view(-1))
        state["ms"].copy_(scale)
        codes, scale = _to_8_bits(v, uv)
        codes = torch.where(v.view(-1, BLOCK) > 0, codes.clamp(min=2.0 ** -9), codes)      # none becomes 0
        state["v"].copy_(codes.view(-1))
        state["vs"].copy_(scale)
    else:
        state["m"].copy_(m)
        state["v"].copy_(v)


# ---------------------------------------------------------------- the framework's calls
def _own_attention(state):
    import paper_2202_00441_amd as P
    case = state["case"]
    mask = {"causal": case["causal"], "window": case["window"], "k_len": state["k_len"], "cu_q": state["cu"], "cu_k": state["cu"]}
    q, k, v = state["q"], state["k"], state["v"]
    if case["mode"] == "layer":
        out = P.attention(q, k, v, **mask)
        dq, dk, dv = torch.autograd.grad(out, (q, k, v), state["dout"])
        return {"out": out, "dq": dq, "dk": dk, "dv": dv}
    out, lse = P.attention_fwd(q, k, v, **mask)
    if case["mode"] == "fwd":
        return {"out": out, "lse": lse}
    dq, dk, dv = P.attention_bwd(state["dout"], q, k, v, out, lse, **mask)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_qk(state):
    import paper_2202_00441_amd as P
    case = state["case"]
    x = (state["q"], state["k"], state["wq"], state["wk"])
    rest = (state["cos"], state["sin"], state["positions"], EPS, case["interleaved"])
    if case["mode"] == "layer":
        q, k = P.qk_norm_rope(*x, *rest)
        dq, dk, dwq, dwk = torch.autograd.grad((q, k), x, (state["dq"], state["dk"]))
    else:
        q, k = P.qk_norm_rope_fwd(*x, *rest)
        if case["mode"] == "fwd":
            return {"q": q, "k": k}
        dq, dk, dwq, dwk = P.qk_norm_rope_bwd(state["dq"], state["dk"], *x, *rest)
    return {"q": q, "dq": dq, "dwq": dwq, "k": k, "dk": dk, "dwk": dwk}


def _own_adamw(state):
    import paper_2202_00441_amd as P
    P.adamw_step(state["params"], state["grads"], state["m"], state["v"], state["ms"], state["vs"], state["master"],
                 lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY, step=state["t"], seed=state["t"])


# ---------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if op == "adamw":
        (_own_adamw if own else _plain_adamw)(state)
        state["t"] += 1
        return {k: state[k] for k in ("flat", "m", "v", "ms", "vs", "master") if state[k] is not None}
    if own:
        return _own_attention(state) if op == "attention" else _own_qk(state)
    with torch.no_grad():                                # the gradients are written out
        return _plain_attention(state) if op == "attention" else {**_plain_norm(state, "q"), **_plain_norm(state, "k")}


# ---------------------------------------------------------------- what a pass needs
def work(case):
    op = case["op"]
    if op == "attention":
        s, d = SIZE[case["dtype"]], case["d"]
        pairs, keys = _pairs(case)
        rows = sum(_lengths(case)[0]) * case["hq"]
        forward = 2 * rows * d * s + 2 * keys * case["hkv"] * d * s
        flops = 4 * pairs * case["hq"] * d
        if case["mode"] == "fwd":
            return {"bytes": forward + 4 * rows, "flops": flops}
        # backward: q, out, dout and lse are read and dq written; k, v and their gradients
        return {"bytes": forward + 4 * rows * d * s + 8 * rows + 4 * keys * case["hkv"] * d * s, "flops": flops + 10 * pairs * case["hq"] * d}
    if op == "qk_norm_rope":
        tokens = case["b"] * case["s"]
        n = tokens * (case["hq"] + case["hkv"]) * case["d"]
        table = tokens * (8 + 4 * case["rot"])
        one = 2 * n * SIZE[case["dtype"]] + table
        back = 3 * n * SIZE[case["dtype"]] + table
        return {"bytes": one if case["mode"] == "fwd" else one + back, "flops": n * (9 if case["mode"] == "fwd" else 26)}
    n, s = sum(_sizes(case)), SIZE[case["dtype"]]
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (2 * s + moments + (8 if case["master"] else s)), "flops": n * (18 if case["bits"] == 32 else 40)}


# ---------------------------------------------------------------- reference values
def _exact_attention(case, state):
    """Head by head, from softmax's definition; the gradients are autograd's of that definition."""
    packed, train = case["lens"] == "packed", case["mode"] != "fwd"
    g = case["hq"] // case["hkv"]
    outs = {n: torch.zeros(state[s].shape, dtype=torch.float64, device="cuda") for n, s in (("out", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    rows = state["q"].shape[:-2]
    lse = torch.zeros((case["hq"], *rows) if packed else (rows[0], case["hq"], *rows[1:]), dtype=torch.float64, device="cuda")
    at = 0
    for b, (nq, nk) in enumerate(zip(*_lengths(case))):
        qi, ki = (slice(at, at + nq), slice(at, at + nk)) if packed else ((b, slice(0, nq)), (b, slice(0, nk)))
        at += nq
        back = torch.arange(nq, device="cuda").unsqueeze(1) + (nk - nq) - torch.arange(nk, device="cuda")   # how far behind a key is
        seen = torch.ones(nq, nk, dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen &= back >= 0
        if case["window"]:
            seen &= back < case["window"]
        some = seen.any(1)
        for h in range(case["hkv"]):
            kk, vv = state["k"][ki][:, h].detach().double(), state["v"][ki][:, h].detach().double()
            for x in (kk, vv):
                x.requires_grad_(train)
            for f in range(h * g, h * g + g):
                qq = state["q"][qi][:, f].detach().double().requires_grad_(train)
                score = (qq @ kk.t()) / case["d"] ** 0.5
                weight = torch.where(seen, torch.exp(score - torch.where(seen, score, -1e300).amax(1, keepdim=True).detach()), 0.0)
                out = (weight / torch.where(some, weight.sum(1), 1.0).unsqueeze(1)) @ vv
                outs["out"][qi][:, f] = out.detach()
                value = torch.logsumexp(torch.where(seen, score.detach(), -math.inf), 1)
                if packed:
                    lse[f, qi] = value
                else:
                    lse[b, f] = value
                if train:
                    grads = torch.autograd.grad(out, (qq, kk, vv), state["dout"][qi][:, f].double())
                    outs["dq"][qi][:, f] = grads[0]
                    outs["dk"][ki][:, h] += grads[1]
                    outs["dv"][ki][:, h] += grads[2]
    keep = {"fwd": ("out", "lse"), "layer": ("out", "dq", "dk", "dv"), "calls": ("out", "lse", "dq", "dk", "dv")}[case["mode"]]
    return {k: v for k, v in {**outs, "lse": lse}.items() if k in keep}


def _exact_qk(case, state):
    """Rotations as products of complex numbers; the gradients are autograd's."""
    half, r = case["rot"] // 2, {}
    turn = torch.complex(state["cos"].double(), state["sin"].double())[state["positions"]].unsqueeze(2)
    for name in ("q", "k"):
        x, w = state[name].detach().double(), state["w" + name].detach().double()
        if case["mode"] != "fwd":
            x.requires_grad_()
            w.requires_grad_()
        y = w * x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / case["d"] + EPS)
        pairs = y[..., :case["rot"]].unflatten(-1, (half, 2)) if case["interleaved"] else y[..., :case["rot"]].unflatten(-1, (2, half)).transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y = torch.cat(((pairs if case["interleaved"] else pairs.transpose(-1, -2)).flatten(-2), y[..., case["rot"]:]), -1)
        r[name] = y.detach()
        if case["mode"] != "fwd":
            r["d" + name], r["dw" + name] = torch.autograd.grad(y, (x, w), state["d" + name].double())
    return r


def _exact_adamw(case, state):
    """Piece by piece of the flat buffers; the 8-bit values by their distance from the numbers below and above."""
    t, total, piece = state["t"], state["flat"].numel(), 1 << 24
    grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()      # all numbers from 0 to 448
    grad = torch.zeros(total, dtype=state["flat"].dtype, device="cuda")
    at = 0
    for x in state["grads"]:
        grad[at:at + x.numel()] = x
        at += _blocks(x.numel()) * BLOCK
    r = {k: [] for k in ("flat", "m", "v", "ms", "vs", "master")}
    for a in range(0, total, piece):
        part = slice(a, min(total, a + piece))
        blocks = slice(a // BLOCK, -(-part.stop // BLOCK))
        g, m, v = grad[part].double(), state["m"][part].double(), state["v"][part].double()
        if case["bits"] == 8:
            m = (m.view(-1, BLOCK) * state["ms"][blocks].double().unsqueeze(1)).flatten()
            v = (v.view(-1, BLOCK) * state["vs"][blocks].double().unsqueeze(1)).flatten()
        m, v = torch.lerp(g, m, BETA1), torch.lerp(g ** 2, v, BETA2)
        w = (state["flat"] if state["master"] is None else state["master"])[part].double()
        step = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
        w = w - LR * DECAY * w - LR * step
        r["flat"].append(w)
        r["master"].append(w)
        if case["bits"] == 32:
            r["m"].append(m)
            r["v"].append(v)
            continue
        place = np.arange(a, part.stop, dtype=np.uint64) * np.uint64(0x9E3779B1) + np.uint64((t * 0x6A09E667 + 0x3C6EF372) % 2 ** 32)
        h = place.astype(np.uint32)
        h = (h ^ (h >> np.uint32(15))) * np.uint32(0xBB67AE85)
        h = h ^ (h >> np.uint32(13))
        for name, x, u in (("m", m, h >> np.uint32(16)), ("v", v, h & np.uint32(0xFFFF))):
            x, u = x.view(-1, BLOCK), torch.from_numpy((u / 65536.0).reshape(-1, BLOCK)).cuda()
            scale = 2.0 ** torch.ceil(torch.log2(x.abs().amax(1, keepdim=True).clamp(min=2.0 ** -117) / 448.0))
            y = x.abs() / scale
            low = (torch.searchsorted(grid, y, right=True) - 1).clamp(max=125)
            up = (y - grid[low]) / (grid[low + 1] - grid[low]) + u >= 1.0
            code = grid[low + up.long()]
            if name == "v":
                code = torch.where(x > 0, code.clamp(min=grid[1].item()), code)
            r[name].append((torch.sign(x) * code).flatten())
            r[name + "s"].append(scale.flatten())
    return {k: torch.cat(x) for k, x in r.items() if x and not (k == "master" and state["master"] is None)}


def exact(case, seed):
    state = prepare(case, seed)
    return {"attention": _exact_attention, "qk_norm_rope": _exact_qk, "adamw": _exact_adamw}[case["op"]](case, state)
