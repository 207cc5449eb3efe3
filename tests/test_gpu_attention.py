"""Attention and its gradient against the formulas in 64 bits.

Tolerances, element by element, follow from the roundings the kernels make, with
u half a unit in the last place of the storage type (2^-8 bf16, 2^-11 fp16, which
have 8 and 11 significant bits) and a = 2^-25 the absolute error below fp16's normal range:
  out   P is rounded before P V, and out itself:   u P|V| + a 1|V| + u |out|
  dV    likewise:                                  u P^T|dO| + a 1|dO| + u |dV|
  dS    = P (dP - delta), delta from the rounded out, dS rounded:
        E = u |dS| + a + P (|dO| |out error|),  dQ: scale E|K| + u|dQ|, dK alike
each doubled for the fp32 sums and the exponentials under them, plus 1e-6 of the
largest magnitude of the row's terms.  lse is a sum of fp32 terms: 1e-5.
"""
import math
import random

import pytest
import torch

import paper_2202_00441_amd as P

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def make(dtype, b, sq, sk, hq, hkv, d, seed=0, packed=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    lead = () if packed else (b,)

    def one(rows, heads):
        return torch.randn(*lead, rows, heads, d, generator=g, device="cuda").to(dtype)

    return one(sq, hq), one(sk, hkv), one(sk, hkv), one(sq, hq)


def reference(q, k, v, dout, causal, window, scale, nk=None):
    """One sequence [rows, heads, d]: outputs, gradients and bounds of their errors, in 64 bits."""
    dt = q.dtype
    u, a = U[dt], TINY[dt]
    g = q.shape[1] // k.shape[1]
    nk = k.shape[0] if nk is None else nk
    kk, vv = k[:nk].repeat_interleave(g, 1).double().transpose(0, 1), v[:nk].repeat_interleave(g, 1).double().transpose(0, 1)
    qq, do = q.double().transpose(0, 1), dout.double().transpose(0, 1)
    nq = q.shape[0]
    behind = torch.arange(nq, device=q.device)[:, None] + nk - nq - torch.arange(nk, device=q.device)
    seen = torch.ones(nq, nk, dtype=torch.bool, device=q.device)
    if causal:
        seen &= behind >= 0
    if window:
        seen &= behind < window
    s = (qq @ kk.transpose(1, 2) * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 2) if nk else torch.full((qq.shape[0], nq), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(seen, torch.exp(s - lse.clamp(min=-1e300)[:, :, None]), 0.0)
    out = p @ vv
    one = seen.double().expand(p.shape)
    e_out = u * (p @ vv.abs()) + a * (one @ vv.abs()) + u * out.abs()
    dv = p.transpose(1, 2) @ do
    e_dv = u * (p.transpose(1, 2) @ do.abs()) + a * (one.transpose(1, 2) @ do.abs())
    ds = p * (do @ vv.transpose(1, 2) - (do * out).sum(2, keepdim=True))
    e_ds = u * ds.abs() + a * one + p * (do.abs() * (2 * e_out)).sum(2, keepdim=True)
    dq, dk = scale * ds @ kk, scale * ds.transpose(1, 2) @ qq
    e_dq, e_dk = scale * e_ds @ kk.abs(), scale * e_ds.transpose(1, 2) @ qq.abs()

    def shared(x, e):            # heads that share a key head
        x, e = (y.unflatten(0, (-1, g)).sum(1) for y in (x, e))
        pad = torch.zeros(x.shape[0], k.shape[0] - nk, x.shape[2], dtype=x.dtype, device=x.device)
        return torch.cat((x, pad), 1).transpose(0, 1), torch.cat((e, pad), 1).transpose(0, 1)

    dk, e_dk = shared(dk, e_dk)
    dv, e_dv = shared(dv, e_dv)
    r = {"out": (out.transpose(0, 1), e_out.transpose(0, 1)), "dq": (dq.transpose(0, 1), e_dq.transpose(0, 1)),
         "dk": (dk, e_dk), "dv": (dv, e_dv)}
    return {n: (x, 2 * (e + u * x.abs()) + a + 1e-6 * (x.abs().amax() if x.numel() else 0.0)) for n, (x, e) in r.items()}, lse


def near(x, ref, what):
    want, tol = ref
    assert x.shape == want.shape, what
    off = (x.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((off - tol).max()):.3g}"


def check(q, k, v, dout, causal=False, window=0, scale=None, k_len=None, back=True):
    kw = {"causal": causal, "window": window, "scale": scale}
    lens = None if k_len is None else torch.tensor(k_len, dtype=torch.int32, device="cuda")
    out, lse = P.attention_fwd(q, k, v, k_len=lens, **kw)
    grads = P.attention_bwd(dout, q, k, v, out, lse, k_len=lens, **kw) if back else ()
    for b in range(q.shape[0]):
        ref, want = reference(q[b], k[b], v[b], dout[b], causal, window, scale or 1 / math.sqrt(q.shape[-1]),
                              None if k_len is None else min(max(k_len[b], 0), k.shape[1]))
        assert torch.equal(torch.isinf(want), torch.isinf(lse[b])), "empty rows"
        fine = ~torch.isinf(want)
        assert torch.allclose(lse[b].double()[fine], want[fine], rtol=1e-5, atol=1e-5)
        near(out[b], ref["out"], f"out of {b}")
        for x, n in zip(grads, ("dq", "dk", "dv")):
            near(x[b], ref[n], f"{n} of {b}")
    return (out, lse, *grads)


BF16, F16 = torch.bfloat16, torch.float16
CASES = [
    # dtype, b, sq, sk, hq, hkv, d, causal, window
    (BF16, 1, 1, 1, 1, 1, 64, False, 0), (F16, 2, 1, 1, 3, 3, 8, True, 0), (BF16, 2, 1, 33, 4, 1, 128, True, 0),
    (F16, 1, 31, 31, 2, 2, 64, True, 0), (BF16, 1, 32, 64, 2, 1, 128, False, 0), (F16, 1, 33, 65, 3, 1, 72, True, 0),
    (BF16, 2, 127, 127, 2, 2, 64, True, 0), (BF16, 1, 129, 129, 8, 2, 128, True, 0), (F16, 3, 64, 63, 1, 1, 40, False, 0),
    (BF16, 1, 200, 333, 6, 2, 96, True, 50), (F16, 1, 257, 257, 2, 1, 128, True, 1), (BF16, 1, 130, 500, 2, 2, 80, True, 131),
    (BF16, 1, 97, 40, 4, 2, 64, True, 0), (F16, 1, 300, 1, 2, 2, 128, True, 0), (F16, 1, 70, 64, 2, 1, 32, True, 5),
    (BF16, 1, 640, 640, 1, 1, 128, False, 0), (BF16, 5, 65, 190, 12, 12, 64, False, 0), (F16, 1, 3, 4097, 8, 1, 128, True, 0),
]


@pytest.mark.parametrize("dtype,b,sq,sk,hq,hkv,d,causal,window", CASES)
def test_against_the_formula(dtype, b, sq, sk, hq, hkv, d, causal, window):
    check(*make(dtype, b, sq, sk, hq, hkv, d), causal=causal, window=window)


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("d", (64, 128))
def test_large_scores(dtype, d):
    """Scores of some hundreds: one key takes all of a row's weight, the others underflow."""
    q, k, v, do = make(dtype, 1, 150, 150, 2, 2, d)
    check(q * 8, k * 8, v, do, causal=True)


@pytest.mark.parametrize("b,sq,sk,hq,hkv,d,causal,window", [
    (1, 2048, 2048, 2, 2, 64, False, 0), (2, 700, 900, 4, 2, 128, True, 0), (9, 70, 300, 16, 16, 40, False, 0), (1, 1500, 1500, 1, 1, 80, True, 300)])
@pytest.mark.parametrize("size", (1.0, 1e-3, 1e-4, 1e-5))
def test_small_gradients_in_fp16(b, sq, sk, hq, hkv, d, causal, window, size):
    """Gradients of small dO, as without a loss scale: dS lies below fp16's normal range, the results need not.  In norm an
    error of at most u = 2^-11 of the whole each from P, dS and delta, beside the rounding of the exact gradient, which at
    these sizes is the largest part (a quarter more for it falls on other numbers)."""
    q, k, v, do = make(F16, b, sq, sk, hq, hkv, d)
    do = (do.float() * size).to(F16)
    kw = {"causal": causal, "window": window}
    out, lse = P.attention_fwd(q, k, v, **kw)
    grads = dict(zip(("dq", "dk", "dv"), P.attention_bwd(do, q, k, v, out, lse, **kw)))
    refs = [reference(q[i], k[i], v[i], do[i], causal, window, 1 / math.sqrt(d))[0] for i in range(b)]
    for name, got in grads.items():
        want = torch.stack([r[name][0] for r in refs])
        rounding = (want.to(F16).double() - want).norm()
        assert (got.double() - want).norm() <= 1.25 * rounding + 3 * 2.0 ** -11 * want.norm(), name


def test_gradients_of_rows_of_different_sizes_in_fp16():
    """Each row's dQ by itself, in norm, dO falling from row to row and values growing from key to key."""
    q, k, v, do = make(F16, 1, 500, 900, 2, 1, 64)
    do = (do.float() * 10.0 ** -(torch.arange(500, device="cuda") % 4)[:, None, None]).to(F16)
    v = (v.float() * 2.0 ** (torch.arange(900, device="cuda") // 100 - 4)[:, None, None]).to(F16)
    out, lse = P.attention_fwd(q, k, v)
    dq = P.attention_bwd(do, q, k, v, out, lse)[0][0].double()
    want = reference(q[0], k[0], v[0], do[0], False, 0, 1 / 8)[0]["dq"][0]
    rounding = (want.to(F16).double() - want).norm(dim=-1)
    assert ((dq - want).norm(dim=-1) <= 1.5 * rounding + 6 * 2.0 ** -11 * want.norm(dim=-1)).all()


@pytest.mark.parametrize("sq,sk,d,causal", [(40, 16, 64, False), (200, 200, 128, True), (333, 33, 40, False)])
def test_large_gradients_in_fp16(sq, sk, d, causal):
    """dS past fp16's largest number, dQ and dK within it."""
    q, k, v, do = make(F16, 1, sq, sk, 2, 1, d)
    check(q * 0.01, k * 0.01, v * 100, do * 2000, causal=causal)


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("b,sq,sk,hq,hkv,d,causal,window", [
    (2, 30, 1, 2, 1, 64, False, 0), (1, 300, 300, 4, 2, 128, True, 1), (3, 70, 70, 8, 1, 40, True, 0), (1, 50, 20, 2, 2, 80, True, 0),
    (1, 2100, 2100, 1, 1, 64, True, 0)])
def test_gradient_of_rows_that_see_one_key(dtype, b, sq, sk, hq, hkv, d, causal, window):
    """Softmax over one key is 1 whatever the scores: such a row gives queries and keys no gradient.  dP and delta are fp32
    sums of d terms and P is off by what lse is, so 1e-5 of the sum of their terms' magnitudes."""
    q, k, v, do = make(dtype, b, sq, sk, hq, hkv, d)
    kw = {"causal": causal, "window": window}
    out, lse = P.attention_fwd(q, k, v, **kw)
    i = torch.arange(sq, device="cuda") + sk - sq                     # the key where a query stands
    last = i.clamp(max=sk - 1) if causal else torch.full_like(i, sk - 1)
    one = last == (i - window + 1).clamp(min=0) if window else last == 0
    assert one.any()
    do = do * one[None, :, None, None].to(dtype)                      # the other rows have none to give
    dq, dk, _ = P.attention_bwd(do, q, k, v, out, lse, **kw)
    most = [x.double().abs().amax() for x in (q, k)]
    terms = float(do.double().abs().sum(-1).amax() * v.double().abs().amax()) / math.sqrt(d)
    assert float(dq.double().abs().amax()) <= 1e-5 * terms * float(most[1])
    assert float(dk.double().abs().amax()) <= 1e-5 * terms * float(most[0]) * int(one.sum()) * (hq // hkv)


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("b,n,hq,hkv,d,window", [(16, 16, 8, 8, 64, 0), (8, 24, 16, 4, 128, 0), (8, 40, 16, 16, 80, 8), (2, 200, 16, 16, 64, 2)])
def test_gradients_of_rows_that_see_few_keys(dtype, b, n, hq, hkv, d, window):
    """In norm, dQ is rounded twice, in dS and itself, by the same relative amount, and dK in fp16 a third time, in the P
    that dS is formed from: sqrt(2) and sqrt(3) of the exact gradient's own rounding, and 6% for what fp32 adds.  Delta
    from the rounded output would be another, the larger the fewer keys a row sees."""
    q, k, v, do = make(dtype, b, n, n, hq, hkv, d)
    kw = {"causal": True, "window": window}
    out, lse = P.attention_fwd(q, k, v, **kw)
    grads = P.attention_bwd(do, q, k, v, out, lse, **kw)
    refs = [reference(q[i], k[i], v[i], do[i], True, window, 1 / math.sqrt(d))[0] for i in range(b)]
    for name, got, roundings in (("dq", grads[0], 2), ("dk", grads[1], 3 if dtype is F16 else 2)):
        want = torch.stack([r[name][0] for r in refs])
        rounding = (want.to(dtype).double() - want).norm()
        assert (got.double() - want).norm() <= 1.06 * math.sqrt(roundings) * rounding, name


def test_scale():
    q, k, v, do = make(BF16, 1, 70, 90, 2, 2, 64)
    check(q, k, v, do, scale=0.7)
    check(q, k, v, do, scale=1e-4)


# single tokens and few rows over caches: the forward that splits keys
@pytest.mark.parametrize("dtype,b,sq,hq,hkv,d,sk,lens", [
    (BF16, 4, 1, 8, 2, 128, 1000, (1000, 1, 0, 513)), (F16, 3, 1, 12, 12, 64, 777, (777, 128, 129)),
    (BF16, 1, 1, 16, 1, 96, 9001, (8999,)), (F16, 2, 3, 6, 2, 128, 5000, (2, 4999)),
    (BF16, 2, 7, 4, 4, 64, 4096, (4096, 3)), (BF16, 1, 1, 32, 1, 128, 130, (130,)), (F16, 1, 40, 4, 1, 128, 3000, (2900,)),
    (BF16, 3, 1, 2, 1, 8, 300, (-5, 400, 7)), (BF16, 1, 600, 1, 1, 128, 20000, (20000,))])
@pytest.mark.parametrize("window", (0, 200))
def test_cache(dtype, b, sq, hq, hkv, d, sk, lens, window):
    q, k, v, do = make(dtype, b, sq, sk, hq, hkv, d)
    there = torch.arange(sk, device="cuda") < torch.tensor(lens, device="cuda")[:, None]
    k[~there], v[~there] = math.nan, math.inf               # a cache's free part is never read
    for x in (k, v):
        x[~there] = math.nan
    check(q, k, v, do, causal=True, window=window, k_len=list(lens))


@pytest.mark.parametrize("dtype,b,hq,hkv,d,sq,window", [(BF16, 70, 32, 16, 128, 1, 0), (F16, 90, 12, 12, 40, 1, 50), (BF16, 130, 16, 8, 64, 3, 0)])
def test_many_caches(dtype, b, hq, hkv, d, sq, window):
    """Enough caches of different lengths, some of them empty, to give every CU several."""
    sk = 200
    q, k, v, do = make(dtype, b, sq, sk, hq, hkv, d)
    lens = [(37 * i) % (sk + 1) for i in range(b)]
    there = torch.arange(sk, device="cuda") < torch.tensor(lens, device="cuda")[:, None]
    for x in (k, v):
        x[~there] = math.nan
    check(q, k, v, do, causal=True, window=window, k_len=lens, back=False)


@pytest.mark.parametrize("lens", (False, True))
def test_many_short_sequences(lens):
    """Windows of a few rows: 2^24 rows of a sequence and key head, more than a launch has workgroups."""
    b, n, h, d = 65536, 16, 16, 8
    q, k, v, do = make(BF16, b, n, n, h, h, d)
    k_len = torch.arange(b, dtype=torch.int32, device="cuda") % (n + 1) if lens else None
    out, lse = P.attention_fwd(q, k, v, k_len=k_len)
    dq, dk, dv = P.attention_bwd(do, q, k, v, out, lse, k_len=k_len)
    for i in (0, 1, 7, 16, 17, 255, 4097, 32767, 32768, 65534, 65535):
        ref, want = reference(q[i], k[i], v[i], do[i], False, 0, 1 / math.sqrt(d), i % (n + 1) if lens else None)
        assert torch.equal(torch.isinf(want), torch.isinf(lse[i]))
        for x, name in ((out, "out"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
            near(x[i], ref[name], f"{name} of {i}")
    few = slice(60000, 60100)
    o, _ = P.attention_fwd(q[few], k[few], v[few], k_len=None if k_len is None else k_len[few])
    assert ((o.float() - out[few].float()).abs() <= 2.0 ** -6 * v[few].float().abs().amax((1, 3))[:, None, :, None]).all()


@pytest.mark.parametrize("dtype,lens,extra,hq,hkv,d,causal,window", [
    (BF16, (5, 1, 0, 130, 64), 0, 4, 2, 64, True, 0), (F16, (129,), 7, 2, 2, 128, False, 0), (BF16, (0, 0), 3, 2, 1, 64, True, 0),
    (BF16, (300, 1, 255, 2), 5, 8, 1, 128, True, 100), (F16, tuple(range(90)), 0, 2, 2, 32, True, 0), (BF16, (), 9, 2, 2, 64, True, 0)])
def test_packed(dtype, lens, extra, hq, hkv, d, causal, window):
    total = sum(lens) + extra                               # rows past the last belong to no sequence
    q, k, v, do = make(dtype, 1, total, total, hq, hkv, d, packed=True)
    cu = torch.tensor([0, *torch.tensor(lens, dtype=torch.int64).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    kw = {"causal": causal, "window": window, "cu_q": cu, "cu_k": cu}
    out, lse = P.attention_fwd(q, k, v, **kw)
    grads = P.attention_bwd(do, q, k, v, out, lse, **kw)
    assert lse.shape == (hq, total)
    at = 0
    for n in lens:
        i = slice(at, at + n)
        at += n
        ref, want = reference(q[i], k[i], v[i], do[i], causal, window, 1 / math.sqrt(d))
        assert torch.allclose(lse[:, i].double(), want, rtol=1e-5, atol=1e-5)
        near(out[i], ref["out"], "out")
        for x, name in zip(grads, ("dq", "dk", "dv")):
            near(x[i], ref[name], name)
    assert torch.all(lse[:, at:] == -math.inf)
    for x in (out, *grads):
        assert not x[at:].any()


# heads of at most 64 in many workgroups: the kernel for dK and dV takes 256 keys in each
@pytest.mark.parametrize("dtype,b,sq,sk,hq,hkv,d,causal,window", [
    (F16, 6, 65, 300, 24, 12, 64, True, 0), (BF16, 9, 70, 257, 16, 16, 40, False, 0), (BF16, 12, 190, 130, 12, 12, 64, True, 33)])
def test_many_workgroups(dtype, b, sq, sk, hq, hkv, d, causal, window):
    check(*make(dtype, b, sq, sk, hq, hkv, d), causal=causal, window=window)


# few workgroups and long walks: the walks are divided and joined, forward, dQ and dK with dV
@pytest.mark.parametrize("dtype,b,sq,sk,hq,hkv,d,causal,window,k_len", [
    (BF16, 1, 700, 1500, 2, 1, 128, False, 0, None), (F16, 1, 1500, 1500, 1, 1, 64, True, 0, None),
    (BF16, 2, 1400, 650, 2, 2, 80, True, 0, None), (F16, 1, 1900, 1999, 1, 1, 40, True, 700, None),
    (BF16, 4, 900, 1100, 3, 1, 128, False, 0, (1100, 0, 1, 64)), (F16, 3, 333, 1777, 2, 1, 72, True, 0, (1000, 300, 5)),
    (BF16, 1, 128, 2047, 8, 8, 128, True, 1200, None)])
def test_walks_in_parts(dtype, b, sq, sk, hq, hkv, d, causal, window, k_len):
    check(*make(dtype, b, sq, sk, hq, hkv, d), causal=causal, window=window, k_len=k_len)


@pytest.mark.parametrize("dtype,causal,d", [(BF16, True, 128), (F16, False, 64)])
def test_walks_in_parts_packed(dtype, causal, d):
    lens = (1700, 0, 1, 900, 64, 65)
    q, k, v, do = make(dtype, 1, sum(lens), sum(lens), 2, 1, d, packed=True)
    cu = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    out, lse = P.attention_fwd(q, k, v, cu_q=cu, cu_k=cu, causal=causal)
    grads = P.attention_bwd(do, q, k, v, out, lse, cu_q=cu, cu_k=cu, causal=causal)
    for i in range(len(lens)):
        at = slice(int(cu[i]), int(cu[i + 1]))
        ref, want = reference(q[at], k[at], v[at], do[at], causal, 0, 1 / math.sqrt(d))
        assert torch.allclose(lse[:, at].double(), want, rtol=1e-5, atol=1e-5)
        for x, n in zip((out, *grads), ("out", "dq", "dk", "dv")):
            near(x[at], ref[n], f"{n} of {i}")


def test_packed_with_other_keys():
    """Queries and keys of different lengths: some sequences have no keys, or no queries."""
    nq, nk = (10, 0, 70, 3, 200), (64, 5, 0, 300, 130)
    q, _, _, do = make(BF16, 1, sum(nq), 0, 4, 2, 64, packed=True)
    k, v = (make(BF16, 1, 0, sum(nk), 4, 2, 64, seed=s, packed=True)[1] for s in (1, 2))
    cu_q, cu_k = (torch.tensor([0, *torch.tensor(n).cumsum(0).tolist()], dtype=torch.int32, device="cuda") for n in (nq, nk))
    for causal in (False, True):
        kw = {"causal": causal, "cu_q": cu_q, "cu_k": cu_k}
        out, lse = P.attention_fwd(q, k, v, **kw)
        grads = P.attention_bwd(do, q, k, v, out, lse, **kw)
        for b in range(len(nq)):
            i, j = slice(sum(nq[:b]), sum(nq[:b + 1])), slice(sum(nk[:b]), sum(nk[:b + 1]))
            ref, want = reference(q[i], k[j], v[j], do[i], causal, 0, 1 / 8)
            assert torch.equal(torch.isinf(want), torch.isinf(lse[:, i]))
            near(out[i], ref["out"], "out")
            for x, name, rows in zip(grads, ("dq", "dk", "dv"), (i, j, j)):
                near(x[rows], ref[name], name)


def test_packed_bounds_are_clamped():
    """Whatever the offsets say, nothing outside the tensors is read or written."""
    q, k, v, do = make(BF16, 1, 100, 100, 2, 2, 64, packed=True)
    for cu in ([0, 1000, 50, -3], [7, 7, 7, 7], [0, 100, 2 ** 31 - 1, -2 ** 31], [90, 10, 40, 20]):
        cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        out, lse = P.attention_fwd(q, k, v, causal=True, cu_q=cu, cu_k=cu)
        P.attention_bwd(do, q, k, v, out, lse, causal=True, cu_q=cu, cu_k=cu)
    torch.cuda.synchronize()


def effective(cu, rows):
    """Where sequences begin: the first at 0, bounds inside the tensor, none before one ahead of it."""
    r = [0]
    for x in cu[1:]:
        r.append(max(r[-1], min(max(x, 0), rows)))
    return r


@pytest.mark.parametrize("heads,d,causal,window", [((2, 2), 64, True, 0), ((8, 2), 128, False, 0), ((3, 1), 40, True, 17)])
@pytest.mark.parametrize("cu_q,cu_k", [
    ([90, 10, 40, 20], [90, 10, 40, 20]), ([0, 1000, 50, -3], [0, 3, 2, 290]), ([0, 60, 10, 60, 5, 200], [0, 10, 300, 20, 4, 1]),
    ([7, 7, 7, 7], [300, 200, 100, 0]), (None, None)])
def test_packed_offsets_out_of_order(heads, d, causal, window, cu_q, cu_k):
    """An offset below one before it counts as that one: the same bits as with those offsets, and no row left out."""
    nq, nk = 250, 300
    if cu_q is None:                                        # more sequences than a wave looks at together
        r = random.Random(3)
        cu_q, cu_k = ([max(0, min(n, 2 * i + r.randint(-40, 40))) for i in range(140)] for n in (nq, nk))
    q, _, _, do = make(BF16, 1, nq, 0, *heads, d, packed=True)
    k, v = (make(BF16, 1, 0, nk, *heads, d, seed=s, packed=True)[1] for s in (1, 2))
    results = []
    for bounds in ((cu_q, cu_k), (effective(cu_q, nq), effective(cu_k, nk))):
        bounds = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in bounds]
        kw = {"causal": causal, "window": window, "cu_q": bounds[0], "cu_k": bounds[1]}
        out, lse = P.attention_fwd(q, k, v, **kw)
        results.append((out, lse, *P.attention_bwd(do, q, k, v, out, lse, **kw)))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    at_q, at_k = effective(cu_q, nq), effective(cu_k, nk)
    for b in range(len(at_q) - 1):
        i, j = slice(at_q[b], at_q[b + 1]), slice(at_k[b], at_k[b + 1])
        ref, want = reference(q[i], k[j], v[j], do[i], causal, window, 1 / math.sqrt(d))
        assert torch.equal(torch.isinf(want), torch.isinf(results[0][1][:, i]))
        for x, name, rows in zip((results[0][0], *results[0][2:]), ("out", "dq", "dk", "dv"), (i, i, j, j)):
            near(x[rows], ref[name], f"{name} of {b}")


def test_no_keys_and_no_rows():
    q, k, v, do = make(BF16, 2, 40, 0, 4, 2, 64)
    out, lse = P.attention_fwd(q, k, v)
    dq, dk, dv = P.attention_bwd(do, q, k, v, out, lse)
    assert not out.any() and not dq.any() and torch.all(lse == -math.inf) and dk.shape == dv.shape == k.shape
    q, k, v, do = make(BF16, 2, 0, 40, 4, 2, 64)
    out, lse = P.attention_fwd(q, k, v)
    dq, dk, dv = P.attention_bwd(do, q, k, v, out, lse)
    assert out.shape == dq.shape == q.shape and not dk.any() and not dv.any()
    q, k, v, do = make(BF16, 0, 4, 4, 4, 2, 64)
    assert P.attention_fwd(q, k, v)[0].shape == q.shape


def test_layouts():
    """Views of one projection, heads before rows, a key head for all, one batch entry for all."""
    g = torch.Generator(device="cuda").manual_seed(3)
    qkv = torch.randn(2, 90, 8, 64, generator=g, device="cuda").to(BF16)
    do = torch.randn(2, 4, 90, 64, generator=g, device="cuda").to(BF16).transpose(1, 2)
    check(qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:], do, causal=True)
    heads = torch.randn(2, 4, 90, 64, generator=g, device="cuda").to(BF16).transpose(1, 2)
    check(heads, heads, heads, do, causal=True)
    one = torch.randn(1, 90, 1, 64, generator=g, device="cuda").to(BF16)
    check(heads, one.expand(2, 90, 4, 64), one.expand(2, 90, 4, 64), do)


def test_differentiable_call_takes_any_layout():
    g = torch.Generator(device="cuda").manual_seed(4)
    base = torch.randn(2, 50, 3, 2, 67, generator=g, device="cuda").to(BF16).requires_grad_()
    q, k, v = (base[:, :, i, :, 3:67] for i in range(3))            # rows that start off any 16 bytes
    out = P.attention(q, k, v, causal=True)
    do = torch.randn(64, 2, 50, 2, generator=g, device="cuda").to(BF16).permute(1, 2, 3, 0)
    (grad,) = torch.autograd.grad(out, base, do)
    x = [t.detach().contiguous() for t in (q, k, v)]
    o, lse = P.attention_fwd(*x, causal=True)
    want = P.attention_bwd(do.contiguous(), *x, o, lse, causal=True)
    assert torch.equal(out, o)
    for i in range(3):
        assert torch.equal(grad[:, :, i, :, 3:], want[i]) and not grad[:, :, i, :, :3].any()


def test_gradient_of_a_shared_input():
    """Keys broadcast over the batch: their gradient is the sum over it."""
    q, k, v, do = make(BF16, 3, 40, 50, 2, 2, 64)
    k1, v1 = k[:1].clone().requires_grad_(), v[:1].clone().requires_grad_()
    out = P.attention(q, k1.expand(3, -1, -1, -1), v1.expand(3, -1, -1, -1))
    dk, dv = torch.autograd.grad(out, (k1, v1), do)
    ks, vs = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)
    o, lse = P.attention_fwd(q, ks, vs)
    _, each_k, each_v = P.attention_bwd(do, q, ks, vs, o, lse)
    assert torch.allclose(dk.float(), each_k.float().sum(0, keepdim=True), rtol=2.0 ** -7, atol=1e-3)
    assert torch.allclose(dv.float(), each_v.float().sum(0, keepdim=True), rtol=2.0 ** -7, atol=1e-3)


@pytest.mark.parametrize("name", ("q", "k", "v"))
def test_gradient_against_differences(name):
    """<gradient, direction> against central differences of the loss in 64 bits.  With h = 1e-4 the differences are
    exact to 1e-7 of the loss's scale; the gradient's roundings (2^-8 each, of random signs, over 2 * 60 * 64 terms)
    leave less than 1 % of the product of norms over the root of the number of terms, times ten."""
    x = dict(zip("qkv", make(BF16, 1, 60, 60, 2, 2, 64)))
    do = make(BF16, 1, 60, 60, 2, 2, 64, seed=9)[3]
    out, lse = P.attention_fwd(x["q"], x["k"], x["v"], causal=True)
    grads = dict(zip("qkv", P.attention_bwd(do, x["q"], x["k"], x["v"], out, lse, causal=True)))
    direction = torch.randn(x[name].shape, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))

    def loss(h):
        y = {n: t[0].double().transpose(0, 1) for n, t in x.items()}
        y[name] = y[name] + h * direction[0].transpose(0, 1)
        s = y["q"] @ y["k"].transpose(1, 2) / 8
        s = s.masked_fill(torch.ones(60, 60, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        return float((torch.softmax(s, 2) @ y["v"] * do[0].double().transpose(0, 1)).sum())

    want = (loss(1e-4) - loss(-1e-4)) / 2e-4
    got = float((grads[name].double() * direction).sum())
    norms = float(grads[name].double().norm() * direction.norm())
    assert abs(got - want) <= 0.1 * norms / math.sqrt(direction.numel())


def test_same_inputs_same_bits():
    q, k, v, do = make(BF16, 2, 300, 300, 8, 2, 128)
    first = None
    for _ in range(3):
        out, lse = P.attention_fwd(q, k, v, causal=True)
        r = (out, lse, *P.attention_bwd(do, q, k, v, out, lse, causal=True))
        first = first or r
        assert all(torch.equal(a, b) for a, b in zip(first, r))


def test_rows_past_32_bits():
    """A cache whose rows lie more than 2^31 elements apart from its first."""
    stride, rows, d = 1 << 24, 150, 64                    # 2.5e9 elements
    big = torch.empty(rows * stride, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    q, do = (torch.randn(1, rows, 2, d, generator=g, device="cuda").to(BF16) for _ in range(2))
    k, v = (big.as_strided((1, rows, 2, d), (0, stride, d, 1), at) for at in (0, 4096))
    for x in (k, v):
        x.copy_(torch.randn(1, rows, 2, d, generator=g, device="cuda"))
    check(q, k, v, do, causal=True)
    check(q[:, :1], k, v, do[:, :1], causal=True, back=False)
    check(k, q, q, v, causal=True)


def test_stream_and_graph():
    q, k, v, do = make(BF16, 1, 200, 5000, 4, 2, 128)
    want = P.attention_fwd(q[:, :1], k, v)
    full = P.attention_fwd(q, k, v, causal=True)
    full = (*full, *P.attention_bwd(do, q, k, v, *full, causal=True))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = P.attention_fwd(q[:, :1], k, v)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token = P.attention_fwd(q[:, :1], k, v)
        out = P.attention_fwd(q, k, v, causal=True)
        grads = P.attention_bwd(do, q, k, v, *out, causal=True)
    for _ in range(3):
        for x in (*token, *out, *grads):
            x.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*want, *full), (*token, *out, *grads)))
        P.attention_fwd(q, k, v)


def test_nan_stays_in_its_row():
    q, k, v, do = make(BF16, 1, 100, 100, 2, 2, 64)
    q[0, 17, 1, 3] = math.nan
    out, _ = P.attention_fwd(q, k, v)
    bad = torch.isnan(out).any(-1)
    assert bad[0, 17, 1] and int(bad.sum()) == 1
    q, k, v, do = make(BF16, 1, 100, 100, 2, 2, 64)
    k[0, 60, 0] = math.nan                                 # a key that rows before it do not see
    out, _ = P.attention_fwd(q, k, v, causal=True)
    bad = torch.isnan(out).any(-1)[0]
    assert bad[60:, 0].all() and not bad[:60].any() and not bad[:, 1].any()


def test_refusals():
    q, k, v, do = make(BF16, 2, 10, 12, 4, 2, 64)
    out, lse = P.attention_fwd(q, k, v)
    i32 = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in ((q.float(), k.float(), v.float()), (q, k.half(), v), (q.double(), k, v)):
        with pytest.raises(TypeError):
            P.attention_fwd(*bad)
    for bad, kw in (((q[0], k[0], v[0]), {}), ((q, k[:1], v[:1]), {}), ((q, k, v[:, :5]), {}), ((q, k[..., :32], v[..., :32]), {}),
                    ((q[:, :, :3], k, v), {}), ((q, k[:, :, :0], v[:, :, :0]), {}), ((q[..., :12], k[..., :12], v[..., :12]), {}),
                    ((q[..., 1:9], k[..., :8], v[..., :8]), {}), ((q[..., ::2], k[..., ::2], v[..., ::2]), {}),
                    ((q, k, v), {"window": 3}), ((q, k, v), {"window": -1, "causal": True}), ((q, k, v), {"scale": 0.0}),
                    ((q, k, v), {"scale": math.nan}), ((q, k, v), {"k_len": i32[:1]}), ((q, k, v), {"k_len": i32.long()}),
                    ((q, k, v), {"k_len": i32.cpu()}), ((q, k, v), {"cu_q": i32}), ((q, k, v), {"cu_q": i32, "cu_k": i32}),
                    ((q[0], k[0], v[0]), {"cu_q": i32, "cu_k": i32[:1]}), ((q.cpu(), k, v), {})):
        with pytest.raises(ValueError):
            P.attention_fwd(*bad, **kw)
    with pytest.raises(ValueError):
        P.attention_bwd(do[:, :5], q, k, v, out, lse)
    with pytest.raises(ValueError):
        P.attention_bwd(do, q, k, v, out.transpose(1, 2).contiguous().transpose(1, 2), lse)
    with pytest.raises(ValueError):
        P.attention_bwd(do, q, k, v, out, lse.half())
    with pytest.raises(ValueError):
        P.attention_bwd(do, q, k, v, out, lse[:, :2])
    with pytest.raises(TypeError):
        P.attention_bwd(do.half(), q, k, v, out, lse)
