"""The norm and rotary position of query and key heads, and the gradients, against
the formulas in 64 bits.

Tolerances: everything is formed in fp32 from the inputs and rounded once, so an
element is off by at most u of its size (2^-8 bf16, 2^-11 fp16, nothing for fp32)
plus the fp32 steps': at most 20 roundings of 2^-24 of the largest magnitudes met
on the way, which are bounded by |w| sqrt(d) for the outputs and by the formula's
terms taken absolutely for the gradients: 20 * 2^-24 < 1.2e-6 of those.  The
weights' gradients add n terms in fp32 in pairs or runs of at most some hundred:
1e-5 of the sum of magnitudes.
"""
import math

import pytest
import torch

import paper_2202_00441_amd as P

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}


def inputs(dtype, b, s, hq, hkv, d, rot, seed=0, rows=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, dq, dk = (torch.randn(b, s, h, d, generator=g, device="cuda").to(dtype) for h in (hq, hkv, hq, hkv))
    qw, kw = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype) for _ in range(2))
    cos, sin = P.rope_tables(rows or max(s, 1), rot)
    return q, k, qw, kw, dq, dk, cos, sin


def turn(x, c, s, inter):
    h = c.shape[-1]
    a, b = (x[..., :2 * h:2], x[..., 1:2 * h:2]) if inter else (x[..., :h], x[..., h:2 * h])
    y = torch.empty_like(x)
    y[..., 2 * h:] = x[..., 2 * h:]
    (y[..., :2 * h:2] if inter else y[..., :h]).copy_(a * c - b * s)
    (y[..., 1:2 * h:2] if inter else y[..., h:2 * h]).copy_(b * c + a * s)
    return y


def reference(x, w, dy, cos, sin, pos, eps, inter):
    c, s = cos.double()[pos].unsqueeze(-2), sin.double()[pos].unsqueeze(-2)
    x, w, dy = x.double(), w.double(), dy.double()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    u = x * r
    y = turn(u * w, c, s, inter)
    g = turn(dy, c, -s, inter)
    dx = r * (g * w - u * (g * w * u).mean(-1, keepdim=True))
    size = r * ((g * w).abs() + u.abs() * (g * w * u).abs().mean(-1, keepdim=True))
    lead = tuple(range(x.dim() - 1))
    return (y, (u * w).abs().amax(-1, keepdim=True)), (dx, size.amax(-1, keepdim=True)), ((g * u).sum(lead), (g * u).abs().sum(lead))


def near(x, want, size, dtype, what):
    tol = U[dtype] * want.abs() + 1.2e-6 * size + (2.0 ** -25 if dtype is F16 else 0.0)
    off = (x.double() - want).abs()
    assert x.shape == want.shape and not (~(off <= tol)).any(), f"{what}: worst {float((off - tol).max()):.3g}"


def check(q, k, qw, kw, dq, dk, cos, sin, pos=None, eps=1e-6, inter=False):
    rest = (cos, sin, pos, eps, inter)
    outs = P.qk_norm_rope_fwd(q, k, qw, kw, *rest)
    gq, gk, gqw, gkw = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, *rest)
    at = torch.arange(q.shape[-3], device="cuda") if pos is None else pos
    for x, w, dy, y, gx, gw, name in ((q, qw, dq, outs[0], gq, gqw, "q"), (k, kw, dk, outs[1], gk, gkw, "k")):
        ry, rx, rw = reference(x, w, dy, cos, sin, at, eps, inter)
        near(y, *ry, x.dtype, name)
        near(gx, *rx, x.dtype, "d" + name)
        assert gw.dtype == F32 and not (~((gw.double() - rw[0]).abs() <= 1e-5 * rw[1])).any(), "weight of " + name


CASES = [(BF16, 2, 5, 4, 2, 128, 128), (F16, 1, 1, 1, 1, 64, 64), (F32, 3, 7, 2, 2, 64, 32), (BF16, 1, 33, 12, 12, 64, 16),
         (F32, 1, 9, 3, 1, 256, 256), (F16, 2, 17, 8, 1, 96, 96), (BF16, 1, 3, 5, 3, 80, 80), (F32, 1, 4, 2, 1, 16, 16),
         (BF16, 1, 2, 1, 40, 160, 32), (F16, 4, 257, 4, 4, 112, 48), (BF16, 2, 1000, 16, 4, 128, 64), (F32, 1, 3, 2, 2, 128, 0)]


@pytest.mark.parametrize("inter", (False, True))
@pytest.mark.parametrize("dtype,b,s,hq,hkv,d,rot", CASES)
def test_against_the_formula(dtype, b, s, hq, hkv, d, rot, inter):
    check(*inputs(dtype, b, s, hq, hkv, d, rot), inter=inter)


@pytest.mark.parametrize("shape", ((3, 10), (1, 10), (10,)))
def test_positions(shape):
    x = inputs(BF16, 3, 10, 4, 2, 64, 64, rows=5000)
    pos = torch.randint(0, 5000, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    check(*x, pos=pos)
    check(*x, pos=pos.expand(3, 10).t().contiguous().t())


def test_positions_outside_the_tables():
    q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, 1, 6, 2, 1, 64, 32, rows=100)
    pos = torch.tensor([0, -1, 99, 100, 2 ** 62, -2 ** 63], device="cuda")
    bad = torch.tensor([False, True, False, True, True, True], device="cuda")
    for y in P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin, pos):
        assert torch.equal(torch.isnan(y[0, :, :, :32]).all(-1).all(-1), bad) and not torch.isnan(y[0, ~bad]).any()
        assert not torch.isnan(y[..., 32:]).any()
    gq, gk, _, _ = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin, pos)
    for g in (gq, gk):
        assert torch.isnan(g[0, bad]).any(-1).all() and not torch.isnan(g[0, ~bad]).any()


def test_layouts():
    g = torch.Generator(device="cuda").manual_seed(2)
    cos, sin = P.rope_tables(50, 64)
    w = torch.ones(64, device="cuda").to(BF16)
    qkv = torch.randn(2, 50, 8, 64, generator=g, device="cuda").to(BF16)
    do = torch.randn(2, 8, 50, 64, generator=g, device="cuda").to(BF16).transpose(1, 2)
    check(qkv[:, :, :4], qkv[:, :, 4:6], w, w, do[:, :, :4], do[:, :, 4:6], cos, sin)
    heads = torch.randn(2, 4, 50, 64, generator=g, device="cuda").to(BF16).transpose(1, 2)
    check(heads, heads[:, :, :1], w, w, do[:, :, :4], do[:, :, :1], cos, sin)
    check(qkv[0, :, :4], qkv[0, :, 4:6], w, w, do[0, :, :4], do[0, :, 4:6], cos, sin)           # tokens without a batch
    odd = torch.randn(2, 50, 4, 67, generator=g, device="cuda").to(BF16)[..., 3:]
    with pytest.raises(ValueError):
        P.qk_norm_rope_fwd(odd, odd, w, w, cos, sin)
    a = P.qk_norm_rope(odd, odd, w, w, cos, sin)[0]
    assert torch.equal(a, P.qk_norm_rope_fwd(odd.contiguous(), odd.contiguous(), w, w, cos, sin)[0])


def test_differentiable_call():
    q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, 2, 30, 4, 2, 128, 128)
    x = [t.clone().requires_grad_() for t in (q, k, qw, kw)]
    y = P.qk_norm_rope(*x, cos, sin)
    grads = torch.autograd.grad(y, x, (dq, dk))
    want = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin)
    assert all(torch.equal(a, b.to(BF16)) for a, b in zip(grads, want))
    # a loss that only the queries enter
    y = P.qk_norm_rope(*x, cos, sin)
    grads = torch.autograd.grad(y[0], x, dq)
    assert torch.equal(grads[0], want[0]) and not grads[1].any() and not grads[3].any()


def test_differentiable_call_takes_weights_anywhere():
    """Weights that are views into one flat buffer, off any 16 bytes, or strided."""
    q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, 2, 30, 4, 2, 128, 128)
    flat = torch.zeros(300, dtype=BF16, device="cuda")
    flat[3:131], flat[131:259] = qw, kw
    flat.requires_grad_()
    wide = torch.stack((qw, kw), 1).requires_grad_()
    want = P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin)
    grads = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin)[2:]
    for base, a, b in ((flat, flat[3:131], flat[131:259]), (wide, wide[:, 0], wide[:, 1])):
        y = P.qk_norm_rope(q, k, a, b, cos, sin)
        assert all(torch.equal(s, t) for s, t in zip(y, want))
        (g,) = torch.autograd.grad(y, base, (dq, dk))
        got = (g[3:131], g[131:259]) if base is flat else (g[:, 0], g[:, 1])
        assert all(torch.equal(s, t.to(BF16)) for s, t in zip(got, grads))


@pytest.mark.parametrize("inter", (False, True))
def test_gradient_against_differences(inter):
    """fp32, central differences of the formula in 64 bits along a random direction: exact to 1e-8 with h = 1e-5; the
    gradient's roundings are 1e-6 of it."""
    q, k, qw, kw, dq, dk, cos, sin = inputs(F32, 1, 20, 3, 2, 64, 32)
    gq, gk, gqw, gkw = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin, None, 1e-6, inter)
    pos = torch.arange(20, device="cuda")
    for x, w, dy, gx, gw in ((q, qw, dq, gq, gqw), (k, kw, dk, gk, gkw)):
        ex, ew = torch.randn_like(x, dtype=torch.float64), torch.randn_like(w, dtype=torch.float64)

        def loss(h):
            y = reference(x.double() + h * ex, w.double() + h * ew, dy, cos, sin, pos, 1e-6, inter)[0][0]
            return float((y * dy.double()).sum())

        want = (loss(1e-5) - loss(-1e-5)) / 2e-5
        got = float((gx.double() * ex).sum() + (gw.double() * ew).sum())
        size = float((gx.double() * ex).abs().sum() + (gw.double() * ew).abs().sum())
        assert abs(got - want) <= 1e-5 * size


def test_zeros_and_extremes():
    q, k, qw, kw, dq, dk, cos, sin = inputs(F32, 1, 8, 2, 1, 64, 64)
    q[0, 0], q[0, 1] = 0.0, q[0, 1] * 1e-20                # a zero row is left at 0; eps keeps a tiny one small
    q[0, 2] *= 1e18                                        # squares to 1e36
    check(q, k, qw, kw, dq, dk, cos, sin)
    y = P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin)[0]
    assert not y[0, 0].any() and torch.isfinite(y).all()
    q[0, 3, 1, 5] = math.nan
    y = P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin)[0]
    assert torch.isnan(y[0, 3, 1]).all() and int(torch.isnan(y).any(-1).sum()) == 1


def test_nothing():
    for shape in ((0, 4), (2, 0)):
        q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, *shape, 4, 2, 64, 64)
        assert P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin)[0].shape == q.shape
        r = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin)
        assert not r[2].any() and not r[3].any()
    q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, 2, 5, 4, 0, 64, 64)
    r = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin)
    assert r[1].shape == k.shape and r[2].any() and not r[3].any()


def test_same_inputs_same_bits_on_any_stream_and_in_a_graph():
    q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, 4, 700, 8, 2, 128, 128)
    want = (*P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin), *P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want[2:], got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (*P.qk_norm_rope_fwd(q, k, qw, kw, cos, sin), *P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin))
    for _ in range(3):
        for x in got:
            x.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        P.qk_norm_rope_bwd(dq, dk, q, k, qw, kw, cos, sin)


def test_refusals():
    q, k, qw, kw, dq, dk, cos, sin = inputs(BF16, 2, 10, 4, 2, 64, 64)
    for bad in ((q, k.half(), qw, kw, cos, sin), (q, k, qw.float(), kw, cos, sin), (q, k, qw, kw, cos.half(), sin.half()),
                (q.double(), k.double(), qw, kw, cos, sin), (q, k, qw, kw, cos, sin, torch.zeros(10, dtype=torch.int32, device="cuda"))):
        with pytest.raises(TypeError):
            P.qk_norm_rope_fwd(*bad)
    for bad in ((q, k[:1], qw, kw, cos, sin), (q, k[:, :5], qw, kw, cos, sin), (q[..., :40], k[..., :40], qw[:40], kw[:40], cos, sin),
                (q, k, qw[:32], kw, cos, sin), (q, k, qw, kw, cos[:, :20], sin[:, :20]), (q, k, qw, kw, cos[:5], sin[:5]),
                (q, k, qw, kw, cos, sin[:9]), (q[..., :32], k[..., :32], qw[:32], kw[:32], cos, sin), (q, k, qw, kw, cos.cpu(), sin.cpu()),
                (q, k, qw, kw, cos, sin, torch.zeros(9, dtype=torch.int64, device="cuda")), (q, k, qw, kw, cos, sin, None, -1.0),
                (q[..., ::2], k[..., ::2], qw[::2], kw[::2], cos[:, ::2], sin[:, ::2]), (q[0, 0], k[0, 0], qw, kw, cos, sin)):
        with pytest.raises(ValueError):
            P.qk_norm_rope_fwd(*bad)
    with pytest.raises(ValueError):
        P.qk_norm_rope_bwd(dq[:, :5], dk, q, k, qw, kw, cos, sin)
