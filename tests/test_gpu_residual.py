"""Dropout from a counter, the residual addition with its norm (in 16, 32 and 8 bits) and
the product in 8-bit integers, and their gradients, against the formulas in 64 bits.

Tolerances.  u is half a step of the type: 2^-8 bf16, 2^-11 fp16, 2^-24 fp32; fp16 results
below its normal range are off by at most 2^-25 besides.

  dropout   one product in fp32, rounded once: equal to the same steps in torch, bit for bit.
  h         a sum of two, rounded: in fp32 one rounding of the (scaled) sum, with the scaled
            branch's own before it: u of it and 2 * 2^-24 of both terms' magnitudes.
  y         of the kernel's own h: a sum of squares of w elements is added in runs of at most
            32 in a lane, 6 steps across lanes and 16 across waves: 54 roundings and one of
            the square, halved by the root; with the root, two divisions and two products
            60 / 2 + 5 < 36 roundings of 2^-24 of y, and u of it.
  dresidual 36 such roundings of r in each term, the same number for the mean of products
            (three roundings each): 100 * 2^-24 of |dh| + r (|g| + |h r| mean|g h r|), and u
            of the result.  dx: of it before it is rounded, times the scale.
  dw        n rows are added in runs of at most n / 512 + 3 in a workgroup, of the workgroups' sums
            (at most 512) 16 and then 5: below 80 roundings with r's 36 for the n here, 1e-5 > 80 *
            2^-24 of the sum of magnitudes.
  codes     equal, everything between h, w and a code being exact here (64 bits hold
            254 |h w| of 16-bit storage and, but for the last of its 56 bits, of fp32).
  scale     36 roundings for r, three for the rest: 40 * 2^-24.
  product   the sum is exact; it becomes fp32 (one rounding), two products and one addition:
            4 * 2^-24 of |scaled sum| + |bias| =: d before the activation, u after it.  The
            activation adds 1.2 d (its derivative is below 1.13) and, of its own, on the
            tail |z| Q(|z|) that it subtracts 1.9e-4 (bf16), 5.5e-5 (fp16), 1.3e-6 (fp32) by
            its fit, which SiLU does not have, and 2^-18 for the exponential of a rounded
            argument (|argument| < 21 where the tail exceeds 2^-24 of anything here).
"""
import math

import numpy as np
import pytest
import torch

import paper_2202_00441_amd as P
from paper_2202_00441_amd import transformer as TR

import dropout_ref as R

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
LOW = {BF16: 0.0, F16: 2.0 ** -25, F32: 0.0}
TYPES = (BF16, F16, F32)
STEP = 2.0 ** -24


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def near(x, want, tol, what):
    off = (x.double() - want).abs()
    assert x.shape == want.shape and not (~(off <= tol)).any(), f"{what}: worst {float((off - tol).max()):.3g}"


def mask(shape, p, seed, site=0):
    m, scale = R.kept(math.prod(shape), p, seed, site)
    return torch.from_numpy(m).cuda().view(shape), scale


def dropped(x, p, seed, site=0):
    """The same steps in torch: a product in fp32, rounded."""
    m, scale = mask(x.shape, p, seed, site)
    return torch.where(m, x.float() * scale, 0.0).to(x.dtype)


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", (1, 7, 8, 9, 15, 511, 512, 2047, 2048, 2049, 8192, 8197, 100003))
def test_dropout_of_every_length(n, dtype):
    x = randn(gen(n), n + 24, dtype=dtype)
    buffer = torch.full((n + 64,), 7.0, dtype=dtype, device="cuda")
    for p, seed, site in ((0.1, 12345, 0), (0.5, -1, 3), (0.999, 2 ** 62 + 5, 2 ** 32 - 1)):
        y = P.dropout_fwd(x[:n], p, seed, site)
        assert torch.equal(y, dropped(x[:n], p, seed, site)), p
        assert torch.equal(P.dropout_bwd(x[:n], p, seed, site), y)
    # nothing past the end is written: into a buffer, by the C call on its own memory
    view = buffer[:n]
    view.copy_(x[:n])
    drop_in_place(view, 0.1, 12345)
    assert torch.equal(view, dropped(x[:n], 0.1, 12345)) and (buffer[n:] == 7.0).all()


@pytest.mark.parametrize("dtype", (BF16, F16))
def test_dropout_of_every_pattern(dtype):
    """The product in fp32 and then its rounding: not the exact product's, which differs where the first lies on a border
    of the second."""
    x = torch.arange(65536, device="cuda").to(torch.int32).to(torch.int16).view(dtype)
    x = torch.where(x.isnan(), torch.zeros_like(x), x).repeat(3)[:-5]          # and single elements at the end
    for p in (0.05, 0.1, 0.3, 0.3851085064129369, 0.6, 0.9):
        assert torch.equal(P.dropout_fwd(x, p, 7), dropped(x, p, 7)), p


def drop_in_place(x, p, seed):
    import ctypes as C
    from test_residual_host import LIB, Drop
    d = Drop(p=p, seed=seed)
    dt = {F32: P.F32, F16: P.F16, BF16: P.BF16}[x.dtype]
    at = C.c_void_p(x.data_ptr())
    assert LIB.fewbit_dropout(C.byref(d), dt, C.c_int64(x.numel()), at, at, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_of_none_all_and_of_values_that_are_not_finite(dtype):
    x = randn(gen(1), 5000, dtype=dtype)
    x[::3] = math.nan
    x[1::3] = math.inf
    assert torch.equal(P.dropout_fwd(x, 0.0, 1).isnan(), x.isnan()) and torch.equal(P.dropout_fwd(x, 2.0 ** -18, 1)[1::3], x[1::3])
    assert (P.dropout_fwd(x, 1.0, 1) == 0).all()
    m, _ = mask(x.shape, 0.5, 9)
    y = P.dropout_fwd(x, 0.5, 9)
    assert (y[~m] == 0).all() and torch.equal(y[m].isnan(), x[m].isnan()) and torch.equal(y[m].isinf(), x[m].isinf())


def test_dropout_far_into_a_tensor():
    """Offsets past 2^32 bytes."""
    n = (1 << 31) + 4099
    x = torch.ones(n, dtype=F16, device="cuda")
    y = P.dropout_fwd(x, 0.25, 77, 5)
    for first in (0, (1 << 28) - 100, n // 8 - 1000):
        m, scale = R.kept(min(8192, n - 8 * first), 0.25, 77, 5, first=first)
        part = y[8 * first:8 * first + m.size].float().cpu().numpy()
        assert np.array_equal(part != 0, m) and np.all(part[m] == np.float32(np.float16(scale)))
    del x, y
    torch.cuda.empty_cache()


def test_dropout_differentiable_with_any_layout_and_broadcast_gradients():
    x = randn(gen(2), 33, 70).t().requires_grad_()
    y = P.dropout(x, 0.3, 11, 2)
    assert torch.equal(y, dropped(x.detach().contiguous(), 0.3, 11, 2))
    dx, = torch.autograd.grad(y.sum(), x)
    m, scale = mask(x.shape, 0.3, 11, 2)
    assert torch.equal(dx, torch.where(m, torch.full_like(dx, scale), 0.0))
    odd = randn(gen(3), 1001, dtype=BF16)[1:].requires_grad_()             # starts off 16 bytes
    assert torch.equal(P.dropout(odd, 0.3, 11), dropped(odd.detach().clone(), 0.3, 11))
    assert P.dropout(torch.empty(0, 8, device="cuda"), 0.3, 1).shape == (0, 8)


@pytest.mark.parametrize("strided", (False, True))
def test_layers_differentiated_twice(strided):
    """Dropout's gradient is dropout again, to any order; the norm's raises.  By both of the layers' paths."""
    g = gen(12)
    x = (randn(g, 24, 40).t() if strided else randn(g, 40, 24)).requires_grad_()
    y = P.dropout(x, 0.5, 3)
    dx, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    m, k = mask(x.shape, 0.5, 3)
    assert torch.equal(dx, torch.where(m, 2 * k * k * x, 0.0))
    ddx, = torch.autograd.grad(dx.sum(), x)
    assert torch.equal(ddx, torch.where(m, torch.full_like(ddx, 2 * k * k), 0.0))
    w = torch.ones(24, device="cuda", requires_grad=True)
    h, y = P.residual_norm(x, None if strided else x.detach(), w, p=0.0 if strided else 0.5, seed=1)
    dx, dw = torch.autograd.grad((y * y * y).sum(), (x, w), create_graph=True)
    with pytest.raises(RuntimeError, match="twice|cannot be differentiated"):
        (dx.sum() + dw.sum()).backward()


def test_layers_without_gradients_and_with_some_wanted():
    x, res, w, dh, dy = norm_inputs(BF16, 30, 72)
    want = P.residual_norm_fwd(x, res, w, p=0.3, seed=2)
    for t in (x, res, w):
        t.requires_grad_()
        h, y = P.residual_norm(x, res, w, p=0.3, seed=2)
        assert torch.equal(h, want[0]) and torch.equal(y, want[1]) and h.requires_grad and y.requires_grad
        g, = torch.autograd.grad((h, y), t, (dh, dy))
        all_ = P.residual_norm_bwd(dh, dy, want[0], w.detach(), p=0.3, seed=2)
        assert torch.equal(g, all_[0 if t is x else 1 if t is res else 2].to(BF16))
        h, y = P.residual_norm(x, None, w, p=0.3, seed=2)
        if t is not res:
            g, = torch.autograd.grad((h, y), t, (dh, dy))
            all_ = P.residual_norm_bwd(dh, dy, h.detach(), w.detach(), p=0.3, seed=2)
            assert torch.equal(g, all_[0 if t is x else 2].to(BF16))
        with torch.no_grad():
            h, y = P.residual_norm(x, res, w, p=0.3, seed=2)
            assert not h.requires_grad and not P.dropout(x, 0.5, 1).requires_grad
        t.requires_grad_(False)
    with torch.inference_mode():
        h, y = P.residual_norm(x, res, w, p=0.3, seed=2)
        assert torch.equal(y, want[1]) and P.dropout(h, 0.5, 1).is_inference()


def test_dropout_keeps_nothing_and_the_norm_its_sum():
    kept = []
    x, res, w, _, _ = norm_inputs(BF16, 20, 64)
    x, res = x.requires_grad_(), res.requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        P.dropout(x, 0.5, 1)
        assert kept == []
        h, y = P.residual_norm(x, res, w, p=0.5, seed=1)
    assert {t.data_ptr() for t in kept} == {h.data_ptr(), w.data_ptr()}


def test_saved_tensors_kept_on_the_host():
    x, res, w, dh, dy = (t.requires_grad_() for t in norm_inputs(BF16, 20, 64))
    seed = torch.tensor([4], device="cuda")
    with torch.autograd.graph.save_on_cpu():
        h, y = P.residual_norm(x, res, w, p=0.25, seed=seed)
        z = P.dropout(y, 0.5, seed, 1)
    got = torch.autograd.grad((h, z), (x, res, w), (dh.detach(), dy.detach()))
    want = P.residual_norm_bwd(dh.detach(), P.dropout_bwd(dy.detach(), 0.5, 4, 1), h.detach(), w.detach(), p=0.25, seed=4)
    assert all(torch.equal(a, b.to(BF16)) for a, b in zip(got, want))


@pytest.mark.parametrize("change,kind", ((lambda t: t.cpu(), ValueError), (lambda t: t.float(), TypeError), (lambda t: t.half(), TypeError),
                                         (lambda t: t.flatten()[:8].clone(), ValueError)))
def test_saved_tensors_that_a_hook_replaced(change, kind):
    """On the host, of another type or shape: refused before anything is launched, one of them alone too."""
    x, res, w, dh, dy = norm_inputs(BF16, 20, 64)
    leaves = [t.requires_grad_() for t in (x, res, w)]
    for which in (lambda t: True, lambda t: t.dim() == 2, lambda t: t.dim() == 1):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: change(t) if t.is_floating_point() and which(t) else t, lambda t: t):
            h, y = P.residual_norm(x, res, w, p=0.25, seed=5)
        for grads in ((dh.detach(), dy.detach()), (dh.detach(), None), (None, dy.detach())):
            outs, grads = zip(*((o, g) for o, g in zip((h, y), grads) if g is not None))
            with pytest.raises((kind, ValueError)):
                torch.autograd.grad(outs, leaves, grads, retain_graph=True)


@pytest.mark.parametrize("change,kind", ((lambda t: t.cpu(), ValueError), (lambda t: t.int(), TypeError), (lambda t: t.expand(2).clone(), ValueError)))
@pytest.mark.parametrize("create_graph", (False, True))
def test_saved_seeds_that_a_hook_replaced(change, kind, create_graph):
    x, res, w, dh, dy = norm_inputs(BF16, 20, 64)
    seed = torch.tensor([5], device="cuda")
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t if t.is_floating_point() else change(t), lambda t: t):
        h, _ = P.residual_norm(x.requires_grad_(), res, w, p=0.25, seed=seed)
        z = P.dropout(x, 0.5, seed)
    for t, g in ((h, dh), (z, dy)):
        with pytest.raises(kind):
            torch.autograd.grad(t, x, g, create_graph=create_graph)


def test_seeds_of_64_bits():
    x = randn(gen(9), 1000)
    assert torch.equal(P.dropout_fwd(x, 0.5, 2 ** 64 - 3), P.dropout_fwd(x, 0.5, -3))
    assert torch.equal(P.dropout_fwd(x, 0.5, torch.tensor(-3, device="cuda")), P.dropout_fwd(x, 0.5, -3))
    assert torch.equal(P.dropout_fwd(x, 0.5, -2 ** 63), P.dropout_fwd(x, 0.5, 2 ** 63))
    for bad in (2 ** 64, -2 ** 63 - 1):
        with pytest.raises(TypeError):
            P.dropout_fwd(x, 0.5, bad)


def test_dropout_module():
    d = P.Dropout(0.4, site=3)
    x = randn(gen(4), 64, 40)
    torch.manual_seed(0)
    a, b = d(x), d(x)
    torch.manual_seed(0)
    assert torch.equal(a, d(x)) and not torch.equal(a, b)
    assert torch.equal(d(x, seed=5), dropped(x, 0.4, 5, 3)) and d.eval()(x) is x


@pytest.mark.parametrize("reentrant", (False, True))
def test_dropout_in_a_checkpoint(reentrant):
    """What is computed again in the backward draws the same seed and so the same mask."""
    from torch.utils.checkpoint import checkpoint
    net = torch.nn.Sequential(torch.nn.Linear(32, 64), P.Dropout(0.4), torch.nn.ReLU(), P.Dropout(0.2, site=1), torch.nn.Linear(64, 8)).cuda()
    x = randn(gen(15), 20, 32).requires_grad_()
    torch.manual_seed(3)
    want = torch.autograd.grad(net(x).square().sum(), [x, *net.parameters()])
    torch.manual_seed(3)
    checkpoint(net, x, use_reentrant=reentrant).square().sum().backward()
    for t, g in zip([x, *net.parameters()], want):
        assert torch.equal(t.grad, g)


def test_seed_on_the_device_in_a_replayed_graph():
    """Forward and backward captured once; every replay draws by what the seed is then."""
    x = randn(gen(5), 3000, dtype=BF16)
    dy = randn(gen(6), 3000, dtype=BF16)
    seed = torch.tensor([5], device="cuda")
    for _ in range(2):
        P.dropout_fwd(x, 0.2, seed, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = P.dropout_fwd(x, 0.2, seed, 1), P.dropout_bwd(dy, 0.2, seed, 1)
        seed.add_(1 << 40)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        now = 5 + (i << 40)
        assert torch.equal(y, dropped(x, 0.2, now, 1)) and torch.equal(dx, dropped(dy, 0.2, now, 1))
        assert torch.equal(P.dropout_fwd(x, 0.2, seed, 1), dropped(x, 0.2, now + (1 << 40), 1))


# ---------------------------------------------------------------- residual and norm
WIDTHS = (8, 16, 504, 512, 520, 768, 1024, 1032, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 32768)


def norm_inputs(dtype, rows, width, seed=0):
    g = gen(seed + width)
    x, res, dh, dy = (randn(g, rows, width, dtype=dtype) for _ in range(4))
    return x * 3, res, (1 + 0.3 * randn(g, width)).to(dtype), dh, dy


def check_norm(x, res, w, dh, dy, p, seed, site, eps=1e-6, got=None):
    dtype = x.dtype
    u, low = U[dtype], LOW[dtype]
    m, scale = mask(x.shape, p, seed, site) if p else (torch.ones_like(x, dtype=torch.bool), 1.0)
    h, y = P.residual_norm_fwd(x, res, w, eps, p, seed, site)
    branch = torch.where(m, x.double() * scale, 0.0)
    total = branch + (0.0 if res is None else res.double())
    near(h, total, u * total.abs() + 2 * STEP * (branch.abs() + (0.0 if res is None else res.double().abs())) + low, "h")
    hd, wd = h.double(), w.double()
    r = (hd.square().mean(-1, keepdim=True) + eps).rsqrt()
    want = hd * r * wd
    near(y, want, (u + 36 * STEP) * want.abs() + low, "y")
    if dy is None:
        return h, y
    dx, dres, dw = P.residual_norm_bwd(dh, dy, h, w, eps, p, seed, site)
    g, hu = dy.double() * wd, hd * r
    zero = 0.0 if dh is None else dh.double()
    grad = zero + r * (g - hu * (g * hu).mean(-1, keepdim=True))
    size = (zero if dh is None else zero.abs()) + r * (g.abs() + hu.abs() * (g * hu).abs().mean(-1, keepdim=True))
    near(dres, grad, u * grad.abs() + 100 * STEP * size + low, "dresidual")
    near(dx, torch.where(m, grad * scale, 0.0), torch.where(m, scale * (u * grad.abs() + 101 * STEP * size), 0.0) + low, "dx")
    rows = tuple(range(h.dim() - 1))
    near(dw, (dy.double() * hu).sum(rows), 1e-5 * (dy.double() * hu).abs().sum(rows), "dw")
    return h, y, dx, dres, dw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_of_every_width(width, dtype):
    for rows in (1, 3, 70):
        for p, residual in ((0.0, True), (0.1, True), (0.0, False), (0.4, False)):
            x, res, w, dh, dy = norm_inputs(dtype, rows, width, rows)
            check_norm(x, res if residual else None, w, dh, dy, p, 99 + rows, 4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", ((1027, 8), (4099, 768), (1500, 2048), (1025, 2056), (1030, 8192), (1030, 16384)))
def test_norm_of_many_rows(rows, width, dtype):
    x, res, w, dh, dy = norm_inputs(dtype, rows, width)
    a = check_norm(x, res, w, dh, dy, 0.1, -5, 0)
    b = check_norm(x, res, w, dh, dy, 0.1, -5, 0)
    assert all(torch.equal(s, t) for s, t in zip(a, b))          # equal inputs give equal bits
    check_norm(x, res, w, None, dy, 0.0, 0, 0)


def test_norm_returns_its_input_where_nothing_is_added():
    x, res, w, dh, dy = norm_inputs(BF16, 5, 64)
    h, y = P.residual_norm_fwd(x, None, w)
    assert h.data_ptr() == x.data_ptr()
    assert P.residual_norm_int8(x, None, w)[0].data_ptr() == x.data_ptr()
    assert P.residual_norm(x, None, w)[0].data_ptr() == x.data_ptr()
    dx, dres, _ = P.residual_norm_bwd(dh, dy, h, w)
    assert dx.data_ptr() == dres.data_ptr()
    assert P.residual_norm_bwd(dh, dy, h, w, p=0.5, seed=1, residual=False)[1] is None


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_strided_rows(dtype):
    """Rows of a projection, part of a sequence, one row for all, axes before the last two."""
    g = gen(8)
    wide = randn(g, 4, 9, 3, 96, dtype=dtype)
    w = randn(g, 96, dtype=dtype)
    x, res = wide[:, 2:7, 1], wide[:, :5, 2]
    dh, dy = randn(g, 96, dtype=dtype).expand(4, 5, 96), wide[:, 4:, 0]
    check_norm_views(x, res, w, dh, dy)
    check_norm_views(wide[:, -1:, 0], wide[:, :1, 1], w, None, wide[:, 3:4, 2])
    check_norm_views(wide.unflatten(0, (2, 2))[:, :, 3, 1], wide.unflatten(0, (2, 2))[:, :, 0, 2], w, None, wide.unflatten(0, (2, 2))[:, :, 1, 0])
    check_norm_views(wide[0, 0, 0], wide[1, 1, 1], w, None, wide[2, 2, 2])
    check_norm_views(wide[:, :, 0].transpose(0, 1), wide[:, :, 1].transpose(0, 1), w, None, wide[:, :, 2].transpose(0, 1))


def check_norm_views(x, res, w, dh, dy):
    dense = [None if t is None else t.contiguous() for t in (x, res, dh, dy)]
    for p in (0.0, 0.3):
        h, y = P.residual_norm_fwd(x, res, w, p=p, seed=3)
        h1, y1 = P.residual_norm_fwd(dense[0], dense[1], w, p=p, seed=3)
        assert torch.equal(h, h1) and torch.equal(y, y1) and h.is_contiguous()
        for a, b in zip(P.residual_norm_bwd(dh, dy, h, w, p=p, seed=3), P.residual_norm_bwd(dense[2], dense[3], h, w, p=p, seed=3)):
            assert torch.equal(a, b)
    for a, b in zip(P.residual_norm_int8(x, res, w), P.residual_norm_int8(dense[0], dense[1], w)):
        assert torch.equal(a, b)
    for a, b in zip(P.quantize_rows(x), P.quantize_rows(dense[0])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("p,residual", ((0.0, True), (0.3, True), (0.3, False), (0.0, False)))
def test_norm_gradients_by_the_layer_and_against_differences(p, residual):
    """The layer's gradients are the raw call's, with any layout; and along a direction they are the central
    difference of the loss, in fp32: the loss is of order sqrt(n) with terms rounded to about 40 * 2^-24, which the
    step of 2^-6 divides, and the third derivative leaves 2^-12 of the same order."""
    g = gen(21)
    x, res = randn(g, 6, 5, 64).transpose(0, 1).requires_grad_(), randn(g, 5, 64, 6).transpose(1, 2).requires_grad_()
    w = (1 + 0.3 * randn(g, 64)).requires_grad_()
    dh, dy = randn(g, 5, 6, 64), randn(g, 64, 6, 5).permute(2, 1, 0)
    leaves = (x, w, res) if residual else (x, w)

    def loss(*t):
        h, y = P.residual_norm(t[0], t[2] if residual else None, t[1], 1e-6, p, 17, 3)
        return h, y, (h.double() * dh).sum() + (y.double() * dy).sum()

    h, y, total = loss(*leaves)
    grads = torch.autograd.grad((h, y), leaves, (dh, dy))
    dx, dres, dw = P.residual_norm_bwd(dh, dy.contiguous(), h.detach().contiguous(), w.detach(), 1e-6, p, 17, 3)
    assert torch.equal(grads[0], dx) and torch.equal(grads[1], dw) and (not residual or torch.equal(grads[2], dres))
    way = [randn(g, *t.shape) for t in leaves]
    e = 2.0 ** -6
    with torch.no_grad():
        up, down = (loss(*(t + s * e * d for t, d in zip(leaves, way)))[2] for s in (1, -1))
    slope = sum((a.double() * d).sum() for a, d in zip(grads, way))
    scale = sum(a.double().norm() * d.double().norm() for a, d in zip(grads, way))
    assert abs(float((up - down) / (2 * e) - slope)) < 2e-3 * float(scale)


def test_norm_layer_with_one_of_its_results_unused():
    x, res, w, dh, dy = (t.requires_grad_() for t in norm_inputs(BF16, 9, 128))
    for p in (0.0, 0.2):
        h, y = P.residual_norm(x, res, w, p=p, seed=8)
        want = P.residual_norm_bwd(None, dy.detach(), h.detach(), w.detach(), p=p, seed=8)
        got = torch.autograd.grad(y, (x, res, w), dy.detach())
        assert all(torch.equal(a, b.to(BF16)) for a, b in zip(got, want))
        h, y = P.residual_norm(x, res, w, p=p, seed=8)
        got = torch.autograd.grad(h, (x, res, w), dh.detach())
        assert torch.equal(got[1], dh) and torch.equal(got[0], dropped(dh.detach(), p, 8) if p else dh) and (got[2] == 0).all()
    seed = torch.tensor(8, device="cuda")
    h, y = P.residual_norm(x, res, w, p=0.2, seed=seed)
    assert torch.equal(torch.autograd.grad(y, x, dy.detach(), retain_graph=True)[0], want[0])
    seed.add_(1)                        # the backward would draw another mask
    with pytest.raises(RuntimeError, match="modified"):
        torch.autograd.grad(y, x, dy.detach())


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_no_rows(dtype):
    w = torch.ones(64, dtype=dtype, device="cuda")
    x = torch.empty(2, 0, 64, dtype=dtype, device="cuda")
    h, y = P.residual_norm_fwd(x, x, w)
    assert h.shape == y.shape == x.shape
    dx, dres, dw = P.residual_norm_bwd(None, x, x, w)
    assert dx.shape == x.shape and dw.shape == (64,) and (dw == 0).all()
    assert [t.shape for t in P.residual_norm_int8(x, x, w)] == [x.shape, x.shape, (2, 0)]


# ---------------------------------------------------------------- 8 bits
def codes_of(a):
    """Codes and m of rows a in 64 bits: 127 a / m to the nearest whole number, halves to the even."""
    m = a.abs().amax(-1, keepdim=True)
    return torch.round(127.0 * a / torch.where(m > 0, m, 1.0)).to(torch.int8), m.squeeze(-1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_codes_of_every_width(width, dtype):
    for rows in (1, 5, 1100 if width <= 4104 else 33):
        x, res, w, _, _ = norm_inputs(dtype, rows, width, 7)
        for residual in (res, None):
            h, codes, scale = P.residual_norm_int8(x, residual, w)
            assert torch.equal(h, x if residual is None else P.residual_norm_fwd(x, residual, w)[0])
            want, m = codes_of(h.double() * w.double())
            assert torch.equal(codes, want)
            size = (h.double().square().mean(-1) + 1e-6).rsqrt() * m / 127
            near(scale, size, 40 * STEP * size, "scale")
        codes, scale = P.quantize_rows(x)
        want, m = codes_of(x.double())
        assert torch.equal(codes, want)
        near(scale, m / 127, 2 * STEP * m, "scale of rows")


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_halfway_between(dtype):
    """Whole numbers up to 254 in a row whose largest is 254: every odd one lies on a border, and so it does
    when the row is scaled by a power of two, or the weights bring the factor in."""
    ticks = torch.arange(-254, 255, device="cuda")
    ticks = torch.cat((ticks, ticks[:3])).view(1, -1).to(dtype)                  # 512
    want = torch.round(ticks.double() / 2).to(torch.int8)
    for power in (0, -8, 6 if dtype is F16 else 100, -20 if dtype is F16 else -118, -20 if dtype is F16 else -126):
        x = (ticks.double() * 2.0 ** power).to(dtype)
        if bool((x.double() == ticks.double() * 2.0 ** power).all()):
            assert torch.equal(P.quantize_rows(x)[0], want), power
    w = torch.where(torch.arange(512, device="cuda") % 2 == 0, 2.0, 0.5).to(dtype)
    x = (ticks.double() / w.double()).to(dtype)
    assert bool((x.double() * w.double() == ticks.double()).all())
    assert torch.equal(P.residual_norm_int8(x, None, w)[1], want)


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_of_rows_without_numbers(dtype):
    x = randn(gen(3), 6, 1032, dtype=dtype)
    x[0] = 0.0
    x[1, 700] = math.nan
    x[2, 5] = math.inf
    x[3, 1031] = -math.inf
    x[4] = 0.0
    x[4, 77] = torch.finfo(dtype).smallest_normal
    w = torch.ones(1032, dtype=dtype, device="cuda")
    w[3] = 0.0
    for codes, scale in (P.quantize_rows(x), P.residual_norm_int8(x, None, w)[1:]):
        assert (codes[:4] == 0).all() and scale[0] == 0 and scale[1:4].isnan().all()
        assert codes[4, 77] == 127 and int(codes[4].abs().sum()) == 127 and scale[4] > 0 and int(codes[5].abs().amax()) == 127
    w[9] = math.nan
    assert P.residual_norm_int8(x, None, w)[2].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", (8, 2048, 4104, 32768))
def test_rows_of_zeros_without_epsilon(width, dtype):
    """Codes and scale 0, and the product of such a row its bias."""
    x, res, w, _, _ = norm_inputs(dtype, 3, width)
    x[1], res[1] = 0.0, 0.0
    for residual in (res, None):
        h, codes, scale = P.residual_norm_int8(x, residual, w, 0.0)
        want, m = codes_of(h.double() * w.double())
        size = h.double().square().mean(-1).rsqrt() * m / 127
        size[1] = 0.0
        assert torch.equal(codes, want) and scale[1] == 0
        near(scale, size, 40 * STEP * size, "scale")
    if width % 16 == 0:
        bias = randn(gen(1), 16, dtype=dtype)
        ones = torch.ones(16, width, dtype=torch.int8, device="cuda")
        assert torch.equal(P.int8_linear(codes, scale, ones, torch.ones(16, device="cuda"), bias, dtype=dtype)[1], bias)


@pytest.mark.parametrize("width", (16, 512, 2056, 8200))
def test_codes_of_products_below_fp32s_range(width):
    """Of 32-bit storage products of 64 bits count: signs, codes and scales where fp32's products would be subnormal or 0.
    Squares vanish beside eps here, so r = eps^-1/2; the scale's roundings, and 2^-149 where it is subnormal itself."""
    g = gen(width)
    x = torch.randn(7, width, generator=g, device="cuda") * torch.exp2(torch.tensor([-80.0, -90, -100, -110, -120, -80, -100], device="cuda"))[:, None]
    w = torch.randn(width, generator=g, device="cuda") * 2.0 ** -50
    x[5] *= torch.exp2(-20 * torch.rand(width, generator=g, device="cuda"))
    x[6, 3:] = 0.0
    for eps in (1e-6, 1e-20):
        h, codes, scale = P.residual_norm_int8(x, None, w, eps)
        a = x.double() * w.double()
        want, m = codes_of(a)
        assert torch.equal(codes, want) and (want.abs().amax(1) == 127).all()
        size = m / 127 * float(torch.tensor(eps)) ** -0.5
        near(scale, size, 40 * STEP * size + 2.0 ** -149, "scale")


ACTS = {None: lambda z: z, "gelu": lambda z: z * torch.special.ndtr(z), "silu": lambda z: z * torch.sigmoid(z)}
FIT = {"gelu": {BF16: 1.9e-4, F16: 5.5e-5, F32: 1.3e-6}, "silu": {BF16: 0.0, F16: 0.0, F32: 0.0}}


def check_product(x, xs, w, ws, bias, act, dtype):
    y = P.int8_linear(x, xs, w, ws, bias, act, dtype)
    z = torch.matmul(x.double(), w.double().t()) * xs.double()[..., None] * ws.double()
    b = 0.0 if bias is None else bias.double()
    d = 4 * STEP * (z.abs() + (0.0 if bias is None else b.abs()))
    z = z + b
    want = ACTS[act](z)
    tol = d
    if act:
        tol = 1.2 * d + (FIT[act][dtype] + 2.0 ** -18) * ACTS[act](-z.abs()).abs()
    near(y, want, U[dtype] * want.abs() + tol + LOW[dtype], f"{tuple(x.shape)} x {tuple(w.shape)} {act}")
    return y


def product_inputs(rows, out, width, dtype, seed=0, bias=True):
    g = gen(seed + rows + out + width)
    x, w = (torch.randint(-127, 128, (n, width), generator=g, device="cuda", dtype=torch.int8) for n in (rows, out))
    xs, ws = (0.01 * torch.rand(n, generator=g, device="cuda") + 1e-4 for n in (rows, out))
    xs = xs * (3.0 / math.sqrt(width))
    return x, xs, w, ws, randn(g, out, dtype=dtype) if bias else None


@pytest.mark.parametrize("act", (None, "gelu", "silu"))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", (1, 2, 15, 16, 17, 31, 33, 64, 65, 129, 300))
def test_product_of_every_number_of_rows(rows, dtype, act):
    for out, width in ((1, 16), (5, 32), (16, 112), (33, 128), (127, 144), (128, 1040), (130, 96), (132, 272), (257, 256), (1000, 4096), (64, 8208)):
        check_product(*product_inputs(rows, out, width, dtype, bias=out % 3 != 1), act, dtype)


@pytest.mark.parametrize("rows,out,width", ((1, 8192, 2048), (64, 2048, 8192), (777, 1001, 1040), (2048, 2000, 528), (1000, 4100, 2048), (4097, 520, 144),
                                            (2600, 3002, 160), (5000, 4098, 144), (9001, 2052, 160), (2819, 6871, 272), (13, 228, 15280)))
def test_product_of_larger_sizes(rows, out, width):
    check_product(*product_inputs(rows, out, width, BF16), None, BF16)
    a = check_product(*product_inputs(rows, out, width, F16), "gelu", F16)
    assert torch.equal(a, check_product(*product_inputs(rows, out, width, F16), "gelu", F16))


def half_step(want, dtype):
    """Half the distance between neighbours of dtype where want lies."""
    e = torch.frexp(want).exponent - 1
    return torch.ldexp(torch.full_like(want, torch.finfo(dtype).eps / 2), e).clamp_min(LOW[dtype])


@pytest.mark.parametrize("act", ("gelu", "silu"))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,width", ((1, 8192, 256), (64, 500, 4096), (300, 520, 160), (1500, 1500, 144)))
def test_activations_of_products_are_formed_in_fp32(rows, out, width, dtype, act):
    """Whatever the result's type: off by half a step of that type where it lies, and else by fp32's figures alone."""
    x, xs, w, ws, bias = product_inputs(rows, out, width, dtype)
    y = P.int8_linear(x, xs, w, ws, bias, act, dtype)
    z = torch.matmul(x.double(), w.double().t()) * xs.double()[:, None] * ws.double()
    d = 4 * STEP * (z.abs() + bias.double().abs())
    z = z + bias.double()
    want = ACTS[act](z)
    near(y, want, half_step(want, dtype) + 1.2 * d + (FIT[act][F32] + 2.0 ** -18) * ACTS[act](-z.abs()).abs(), act)


@pytest.mark.parametrize("act", (None, "gelu", "silu"))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,width", ((1500, 1500, 144), (1025, 2004, 272), (2600, 3002, 160), (1000, 4100, 400), (4100, 4100, 160), (7001, 4099, 144),
                                            (5003, 4104, 272), (64, 1001, 4112), (200, 260, 8192), (20, 250, 16400)))
def test_product_of_every_tile_and_type(rows, out, width, dtype, act):
    """Tiles of 128 (one and two workgroups a CU) and of 256, and shares of the width; rows that end inside a tile, results
    whose rows are aligned to 2, 4, 8 and 16 bytes."""
    x, xs, w, ws, bias = product_inputs(rows, out, width, dtype)
    y = check_product(x, xs, w, ws, bias, act, dtype)
    assert torch.equal(y, P.int8_linear(x, xs, w, ws, bias, act, dtype))


@pytest.mark.parametrize("act", (None, "gelu", "silu"))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,width", ((1, 2048, 8192), (8, 1000, 4096), (5, 1600, 8176), (7, 333, 272), (4, 500, 8192), (1, 100, 2048), (2, 900, 16368),
                                            (3, 300, 16384), (3, 17, 1040), (1, 5, 400)))
def test_product_of_few_rows_with_places_of_the_width(rows, out, width, dtype, act):
    """Two and four places in an operand's rows, each with codes of its own, some past its first run or cut short."""
    check_product(*product_inputs(rows, out, width, dtype), act, dtype)


@pytest.mark.parametrize("rows", (1, 20, 64, 300))
def test_product_sums_are_exact(rows):
    """The largest sums that there are: every product of two codes of -128, and the widest row."""
    width = 131056
    x = torch.full((rows, width), -128, dtype=torch.int8, device="cuda")
    w = torch.full((35, width), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    one = torch.ones(rows, device="cuda"), torch.ones(35, device="cuda")
    y = P.int8_linear(x, one[0], w, one[1], dtype=F32)
    want = torch.tensor([128 * 128 * width, -128 * 127 * width], device="cuda").float()      # each rounded once
    assert torch.equal(y, want[torch.arange(35, device="cuda") % 2].expand(rows, 35))


@pytest.mark.parametrize("rows", (1, 3, 40, 200))
def test_product_of_strided_rows(rows):
    x, xs, w, ws, b = product_inputs(rows, 70, 160, BF16)
    want = P.int8_linear(x, xs, w, ws, b)
    wide = torch.full((rows, 3, 192), 99, dtype=torch.int8, device="cuda")
    wide[:, 1, 16:176] = x
    many = torch.full((70, 2, 176), -99, dtype=torch.int8, device="cuda")
    many[:, 0, :160] = w
    assert torch.equal(P.int8_linear(wide[:, 1, 16:176], xs, many[:, 0, :160], ws, b), want)
    assert torch.equal(P.int8_linear(x.view(1, rows, 160), xs.view(1, rows), w, ws, b), want.view(1, rows, 70))
    if rows % 2 == 0:
        assert torch.equal(P.int8_linear(x.view(2, rows // 2, 160), xs.view(2, -1), w, ws, b), want.view(2, rows // 2, 70))
    same = x[:1].expand(rows, 160)
    assert torch.equal(P.int8_linear(same, xs, w, ws, b), P.int8_linear(same.contiguous(), xs, w, ws, b))
    assert torch.equal(P.int8_linear(x, xs, w[:1].expand(70, 160), ws, b), P.int8_linear(x, xs, w[:1].repeat(70, 1), ws, b))
    assert torch.equal(P.int8_linear(x[0], xs[0], w, ws, b), want[0])


@pytest.mark.parametrize("rows", (3, 8, 260))
def test_product_of_rows_far_apart(rows):
    """As far as a tile's rows may be, of both operands; further ones are refused."""
    x, xs, w, ws, b = product_inputs(rows, 40, 64, BF16)
    want = P.int8_linear(x, xs, w, ws, b)
    for far in (x, w):
        wide = torch.empty(far.shape[0], 1 << 23, dtype=torch.int8, device="cuda")
        wide[:, :64] = far
        y = P.int8_linear(wide[:, :64], xs, w, ws, b) if far is x else P.int8_linear(x, xs, wide[:, :64], ws, b)
        assert torch.equal(y, want)
    wide = torch.empty(2, (1 << 23) + 16, dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError, match="apart"):
        P.int8_linear(wide[:, :64], xs[:2], w, ws, b)
    with pytest.raises(ValueError, match="apart"):
        P.int8_linear(x, xs, wide[:, :64], ws[:2], b[:2])
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,width", ((1, 100, 2048), (5, 100, 2048), (64, 500, 4096), (300, 520, 160), (1500, 1500, 144)))
def test_scales_of_any_size(rows, out, width, dtype):
    """Small ones whose product is below fp32's range while the result is not, large ones whose product is above it, and
    sums of 0 by those: the bias."""
    x, _, w, _, bias = product_inputs(rows, out, width, dtype)
    x[-1] = 0
    z = torch.matmul(x.double(), w.double().t())
    g = gen(rows)
    low = F16 if dtype is F16 else F32
    for xs, ws in ((1e-20, 1e-21), (2.0 ** -126, 0.5), (1e-22, 1e-17), (1e28, 1e-30), (1e-30, 1e28), (1e-37, 1e30)):
        xs, ws = xs * (1 + torch.rand(rows, generator=g, device="cuda")), ws * (1 + torch.rand(out, generator=g, device="cuda"))
        y = P.int8_linear(x, xs, w, ws, None, None, dtype)
        want = z * xs.double()[:, None] * ws.double()
        small = {BF16: 2.0 ** -134, F16: LOW[F16], F32: 2.0 ** -150}[dtype] + 2.0 ** -149      # where results are subnormal
        most = torch.finfo(dtype).max
        fits = want.abs() < 0.99 * most
        near(torch.where(fits, y, 0.0), torch.where(fits, want, 0.0), (U[dtype] + 4 * STEP) * want.abs() + small, f"{float(xs[0])} {float(ws[0])}")
        assert (y[want.abs() > 1.01 * most].isinf()).all()
    large = torch.full((rows,), 1e29, device="cuda"), torch.full((out,), 1e30, device="cuda")
    y = P.int8_linear(x, large[0], w, large[1], bias, None, dtype)
    assert torch.equal(y[z == 0], bias.expand_as(y)[z == 0])


def test_product_of_nothing_and_of_scales_that_are_not_numbers():
    x, xs, w, ws, b = product_inputs(20, 40, 64, BF16)
    assert P.int8_linear(x[:0], xs[:0], w, ws, b).shape == (0, 40)
    assert P.int8_linear(x, xs, w[:0], ws[:0], b[:0]).shape == (20, 0)
    xs[3], ws[7] = math.nan, math.nan
    for act in (None, "gelu", "silu"):
        y = P.int8_linear(x, xs, w, ws, b, act)
        bad = torch.zeros(20, 40, dtype=torch.bool, device="cuda")
        bad[3], bad[:, 7] = True, True
        assert torch.equal(y.isnan(), bad)


def test_refusals_on_the_device():
    x, w = torch.ones(4, 64, dtype=BF16, device="cuda"), torch.ones(64, dtype=BF16, device="cuda")
    q, s = torch.ones(4, 64, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    wide = torch.ones(4, 4, 3, 64, dtype=BF16, device="cuda")
    for kind, call in ((ValueError, lambda: P.dropout_fwd(x.t(), 0.1, 1)), (ValueError, lambda: P.dropout_fwd(x, 1.5, 1)),
                       (ValueError, lambda: P.dropout_fwd(x, math.nan, 1)), (TypeError, lambda: P.dropout_fwd(x, 0.1, 1.5)),
                       (TypeError, lambda: P.dropout_fwd(x, 0.1, s)), (ValueError, lambda: P.dropout_fwd(x, 0.1, torch.tensor(1))),
                       (ValueError, lambda: P.dropout_fwd(x, 0.1, torch.ones(2, dtype=torch.int64, device="cuda"))),
                       (ValueError, lambda: P.dropout_fwd(x, 0.1, 1, -1)), (ValueError, lambda: P.dropout_fwd(x, 0.1, 1, 1 << 32)),
                       (TypeError, lambda: P.dropout_fwd(q, 0.1, 1)), (TypeError, lambda: P.dropout_fwd(x, 0.1, 1 << 64)),
                       (ValueError, lambda: P.residual_norm_fwd(x[:, :60], None, w[:60])), (ValueError, lambda: P.residual_norm_fwd(x, x[:3], w)),
                       (TypeError, lambda: P.residual_norm_fwd(x, x.float(), w)), (TypeError, lambda: P.residual_norm_fwd(x, x, w.float())),
                       (ValueError, lambda: P.residual_norm_fwd(x, x, w[:32])), (ValueError, lambda: P.residual_norm_fwd(x[:, 4:60], None, w[:56])),
                       (ValueError, lambda: P.residual_norm_fwd(x, x, w, -1.0)), (ValueError, lambda: P.residual_norm_fwd(wide[:, :2, :, :], None, w)),
                       (ValueError, lambda: P.residual_norm_bwd(None, x, x.t().contiguous().t(), w)), (ValueError, lambda: P.quantize_rows(x.t())),
                       (ValueError, lambda: P.int8_linear(q, s, q[:, :32], s)), (TypeError, lambda: P.int8_linear(q, s, x, s)),
                       (TypeError, lambda: P.int8_linear(q, s.double(), q, s)), (ValueError, lambda: P.int8_linear(q, s[:3], q, s)),
                       (ValueError, lambda: P.int8_linear(q[:, :24], s, q[:, :24], s)), (ValueError, lambda: P.int8_linear(q[:, 8:56], s, q[:, 8:56], s)),
                       (TypeError, lambda: P.int8_linear(q, s, q, s, s)), (ValueError, lambda: P.int8_linear(q, s, q, s, w[:3])),
                       (ValueError, lambda: P.int8_linear(q.view(2, 2, 64).transpose(0, 1), s.view(2, 2), q, s))):
        with pytest.raises(kind):
            call()


def test_on_another_stream():
    x, res, w, dh, dy = norm_inputs(BF16, 300, 768)
    want = *P.residual_norm_fwd(x, res, w, p=0.1, seed=1), *P.residual_norm_int8(x, res, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        x2 = x * 1.0                          # not ready on the other stream
        got = *P.residual_norm_fwd(x2, res, w, p=0.1, seed=1), *P.residual_norm_int8(x2, res, w)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_far_into_tensors():
    """Offsets past 2^32 bytes: the last rows are those of a call on them alone."""
    rows, width = 270001, 8192
    x = torch.full((rows, width), 0.5, dtype=BF16, device="cuda")
    x[-3:] = randn(gen(1), 3, width, dtype=BF16)
    w = randn(gen(2), width, dtype=BF16)
    h, y = P.residual_norm_fwd(x, x, w)
    assert torch.equal(h[-3:], 2 * x[-3:]) and torch.equal(y[-3:], P.residual_norm_fwd(x[-3:], x[-3:], w)[1])
    h, codes, scale = P.residual_norm_int8(x, x, w)
    small = P.residual_norm_int8(x[-3:], x[-3:], w)
    assert torch.equal(codes[-3:], small[1]) and torch.equal(scale[-3:], small[2])
    dx, dres, _ = P.residual_norm_bwd(x, x, h, w, p=0.25, seed=9)
    small = P.residual_norm_bwd(x[-3:], x[-3:], h[-3:], w, p=0.25, seed=9)
    m, k = R.kept(3 * width, 0.25, 9, 0, first=(rows - 3) * width // 8)
    m = torch.from_numpy(m).cuda().view(3, width)
    assert torch.equal(dres[-3:], small[1]) and (dx[-3:][~m] == 0).all() and (dx[-3:][m] != 0).float().mean() > 0.99
    del x, h, y, codes, dx, dres
    rows, out = 70001, 32768
    x, xs, w, ws, b = product_inputs(rows, out, 32, BF16)
    y = P.int8_linear(x, xs, w, ws, b)
    assert torch.equal(y[-200:], P.int8_linear(x[-200:].clone(), xs[-200:].clone(), w, ws, b))
    del y
    torch.cuda.empty_cache()


def test_two_streams_at_once():
    """Products with workspaces and backward passes of two streams, a few after one another on each."""
    a, b = (product_inputs(64, 512, 8192, BF16, seed) for seed in (0, 1))
    x, res, w, dh, dy = norm_inputs(BF16, 700, 1024)
    want = [P.int8_linear(*t) for t in (a, b)], [P.residual_norm_bwd(dh, t, x, w) for t in (dy, dh)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((P.int8_linear(*(a, b)[i]), P.residual_norm_bwd(dh, (dy, dh)[i], x, w)))
    torch.cuda.synchronize()
    for i in range(2):
        for product, grads in got[i]:
            assert torch.equal(product, want[0][i]) and all(torch.equal(s, t) for s, t in zip(grads, want[1][i]))


# ---------------------------------------------------------------- together
def test_layers_of_8_bits():
    """A linear layer and its 8-bit form, and that of codes that come with their scales."""
    g = gen(31)
    lin = torch.nn.Linear(512, 200).cuda().bfloat16()
    x = randn(g, 3, 7, 512, dtype=BF16)
    q = P.Int8Linear(lin, "gelu")
    y = q(x)
    codes, scale = P.quantize_rows(x)
    assert torch.equal(y, q(codes, scale)) and y.shape == (3, 7, 200)
    wq, ws = P.quantize_rows(lin.weight.detach())
    assert torch.equal(y, check_product(codes, scale, wq, ws, lin.bias.detach(), "gelu", BF16))
    assert set(q.state_dict()) == {"weight", "weight_scale", "bias"}
    assert torch.equal(q(x.transpose(0, 1)), y.transpose(0, 1))


@pytest.mark.parametrize("bias", (True, False))
def test_layer_of_8_bits_converted(bias):
    """Scales stay fp32, whatever the module becomes; the result's type follows, and so do copies and devices."""
    import copy
    lin = torch.nn.Linear(64, 48, bias=bias).cuda().bfloat16()
    q = P.Int8Linear(lin, "silu")
    x = randn(gen(61), 5, 64, dtype=BF16)
    codes, scale = P.quantize_rows(x)
    kept = q.weight_scale.clone()
    for convert, dtype in ((lambda m: m.half(), F16), (lambda m: m.to(F32), F32), (lambda m: m.bfloat16(), BF16),
                           (lambda m: torch.nn.Sequential(m).to(F16)[0], F16), (lambda m: copy.deepcopy(m).cpu().cuda().float(), F32)):
        q = convert(q)
        assert q.weight_scale.dtype is F32 and torch.equal(q.weight_scale, kept) and q.weight.dtype is torch.int8
        b = None if not bias else lin.bias.detach().to(dtype)
        y = q(codes, scale)
        assert y.dtype is dtype and torch.equal(y, P.int8_linear(codes, scale, q.weight, kept, b, "silu", dtype))
        assert q(x.to(dtype)).dtype is dtype
    assert q.cpu().weight_scale.device.type == "cpu" and q.to("meta").weight_scale.is_meta
    assert q.to_empty(device="cuda").weight_scale.dtype is F32
    with pytest.raises(TypeError, match="dtype"):
        q.double()(codes, scale)


def stack(p, **more):
    torch.manual_seed(3)
    return TR.Transformer(50, 256, 2, 4, 2, 512, most=128, dropout=p, **more).cuda()


def test_stack_without_dropping_is_the_plain_stack():
    """dropout=0.0 goes through the fused norms, None through torch's: the same numbers but for bf16's roundings,
    about ten in a row in each of two layers."""
    a, b = stack(0.0).bfloat16(), stack(None).bfloat16()
    b.load_state_dict(a.state_dict())
    tokens = torch.randint(0, 50, (3, 70), device="cuda", generator=gen(1))
    ya, yb = a(tokens), b(tokens)
    assert float((ya - yb).float().norm() / yb.float().norm()) < 0.03
    ga, gb = (torch.autograd.grad(y.float().square().sum(), list(m.parameters())) for y, m in ((ya, a), (yb, b)))
    for s, t in zip(ga, gb):
        assert float((s.double() - t.double()).norm() / t.double().norm()) < 0.06


@pytest.mark.parametrize("dtype", TYPES)
def test_epsilon_of_norms_without_one(dtype):
    """The fused passes take the one that torch's norm takes: of rows whose mean square is near it, the same numbers.
    Each side is off by half a step and 36 roundings."""
    norm = torch.nn.RMSNorm(256).cuda().to(dtype)
    x = torch.cat([randn(gen(51), 8, 256) * s for s in (1.0, 0.02, 1e-3, 1e-4)]).to(dtype)
    want = norm(x).detach().double()
    near(P.residual_norm_fwd(x, None, norm.weight.detach(), TR._eps(norm))[1], want, 2 * (U[dtype] + 36 * STEP) * want.abs() + 2 * LOW[dtype], "y")


def small_stack(p):
    """Embeddings as small as they usually are: rows whose mean square is 4e-4."""
    model = stack(p)
    with torch.no_grad():
        model.embed.weight.mul_(0.02)
    return model.bfloat16().eval()


def test_stack_of_small_embeddings():
    """The fused passes (dropout=0.0), torch's norms (None), serving from a cache and serving in 8 bits are one function:
    the bounds of test_stack_without_dropping_is_the_plain_stack and test_serving_in_8_bits."""
    a, b = small_stack(0.0), small_stack(None)
    b.load_state_dict(a.state_dict())
    tokens = torch.randint(0, 50, (3, 60), device="cuda", generator=gen(9))
    with torch.no_grad():
        want = b(tokens).float()
        fused = a(tokens).float()
    off = lambda y: float((y.float() - want).norm() / want.norm())
    assert off(fused) < 0.03
    assert off(a.extend(tokens, a.cache(3, 100))) < 0.03 and off(b.extend(tokens, b.cache(3, 100))) < 0.03
    served = TR.Int8Transformer(a)
    assert off(served.extend(tokens, served.cache(3, 100))) < 0.06


def test_stack_with_dropout_against_plain_formulas():
    """Gradients of the whole stack with the masks formed apart: in fp64 on the same weights, bf16's roundings of about
    ten tensors in a row in each of two layers between the two, with random signs."""
    p, seed = 0.2, 4242
    model = stack(p, bits=None).bfloat16()
    tokens = torch.randint(0, 50, (2, 60), device="cuda", generator=gen(2))
    dy = randn(gen(3), 2, 60, 50, dtype=BF16)
    y = model(tokens, seed=seed)
    params = list(model.parameters())
    grads = torch.autograd.grad(y, params, dy)
    exact = stack(p, bits=None).double()
    exact.load_state_dict({k: v.double() for k, v in model.state_dict().items()})

    def drop(x, site):
        m, scale = mask(x.shape, p, seed, site)
        return torch.where(m, x * scale, 0.0)

    def norm(x, w, eps):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w

    def turn(x, cos, sin):
        h = cos.shape[-1]
        c, s = cos[:x.shape[1]].double().unsqueeze(1), sin[:x.shape[1]].double().unsqueeze(1)
        return torch.cat((x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s), -1)

    eps = torch.finfo(BF16).eps
    cos, sin = model.tables(tokens.device)
    h, x = 0.0, exact.embed(tokens)
    for i, b in enumerate(exact.blocks):
        h = h + drop(x, 2 * i)
        q, k, v = b.qkv(norm(h, b.norm1.weight, eps)).unflatten(-1, (-1, b.head_dim)).split((b.heads, b.kv_heads, b.kv_heads), -2)
        q, k = turn(norm(q, b.q_norm, 1e-6), cos, sin), turn(norm(k, b.k_norm, 1e-6), cos, sin)
        q, k, v = (t.transpose(1, 2) for t in (q, k.repeat_interleave(2, 2), v.repeat_interleave(2, 2)))
        s = (q @ k.transpose(2, 3) / math.sqrt(b.head_dim)).masked_fill(torch.ones(60, 60, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        h = h + drop(b.out((torch.softmax(s, -1) @ v).transpose(1, 2).flatten(-2)), 2 * i + 1)
        x = b.down(b.act(b.up(norm(h, b.norm2.weight, eps))))
    want = exact.head(norm(h + drop(x, 4), exact.norm.weight, eps))
    assert float((y.double() - want).norm() / want.norm()) < 0.04
    for got, g in zip(grads, torch.autograd.grad(want, list(exact.parameters()), dy.double())):
        assert float((got.double() - g).norm() / g.norm()) < 0.06


def test_stack_with_dropout_in_a_captured_step():
    """Forward and backward captured with the seed on the device: each replay's gradients are the eager ones of that
    seed, bit for bit."""
    model = stack(0.1).bfloat16()
    params = list(model.parameters())
    tokens = torch.randint(0, 50, (2, 40), device="cuda", generator=gen(5))
    dy = randn(gen(6), 2, 40, 50, dtype=BF16)
    seed = torch.tensor([100], device="cuda")
    model.tables(tokens.device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(model(tokens, seed=seed), params, dy)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = model(tokens, seed=seed)
        grads = torch.autograd.grad(y, params, dy)
    for i in range(3):
        seed.fill_(100 + i)
        graph.replay()
        torch.cuda.synchronize()
        eager = model(tokens, seed=100 + i)
        assert torch.equal(y, eager), i
        # the embedding's and the products' gradients are the library's; those of the norms are this framework's
        for (name, _), a, b in zip(model.named_parameters(), grads, torch.autograd.grad(eager, params, dy)):
            assert float((a.double() - b.double()).norm()) <= 1e-2 * float(b.double().norm()), name
    eval_y = model.eval()(tokens)
    assert torch.equal(eval_y, model(tokens))


def test_training_with_dropout_runs():
    r = TR.train(steps=3, layers=2, width=256, heads=4, kv_heads=2, batch=4, length=64, tokens=32, dropout=0.1)
    assert all(math.isfinite(v) for v in r["losses"])


@pytest.mark.parametrize("bits,act", ((3, "gelu"), (None, "silu")))
def test_serving_in_8_bits(bits, act):
    """Logits from products in 8 bits against the model's own.  A code is off by half of 1/127 of its row's largest,
    about 1/300 of the values' size (rows of 256 normal values reach three times it): times sqrt(2) for both operands
    1.5 % of a product's size at most (uniform errors: / sqrt 3 gives 0.8 %), four products in a row in each of two
    layers on branches of the stream: below 6 % together."""
    model = stack(None, bits=bits, act=act).bfloat16().eval()
    served = TR.Int8Transformer(model)
    tokens = torch.randint(0, 50, (3, 60), device="cuda", generator=gen(7))
    with torch.no_grad():
        want = model(tokens).float()
    cache = served.cache(3, 100)
    parts = [served.extend(tokens[:, a:b], cache).float() for a, b in ((0, 33), (33, 34), (34, 35), (35, 60))]
    got = torch.cat(parts, 1)
    assert float((got - want).norm() / want.norm()) < 0.06
    out = served.generate(tokens[:, :20], 4)
    assert out.shape == (3, 4)
    with pytest.raises(RuntimeError):
        served(tokens)


def test_stack_in_8_bits_converted():
    """Another type for the served stack, and the model that it was made of as it was."""
    model = stack(None).bfloat16().eval()
    tokens = torch.randint(0, 50, (2, 30), device="cuda", generator=gen(10))
    with torch.no_grad():
        want = model(tokens)
    served = TR.Int8Transformer(model).half()
    got = served.extend(tokens, served.cache(2, 40))
    assert got.dtype is F16 and float((got.float() - want.float()).norm() / want.float().norm()) < 0.06
    with torch.no_grad():
        assert all(t.dtype is BF16 for t in model.parameters()) and torch.equal(model(tokens), want)
    served.cpu()
    assert all(t.is_cuda for t in model.parameters())
    # one memory all the same: a step of training is served
    served = TR.Int8Transformer(model)
    with torch.no_grad():
        model.head.weight.mul_(2.0)
    assert torch.equal(served.head.weight, model.head.weight) and served.embed.weight.data_ptr() == model.embed.weight.data_ptr()


def test_serving_step_in_a_replayed_graph():
    """A norm, a product, an activation, another layout and product, captured together."""
    g = gen(41)
    up, down = torch.nn.Linear(512, 1024).cuda().bfloat16(), torch.nn.Linear(1024, 512).cuda().bfloat16()
    up, down = P.Int8Linear(up, "gelu"), P.Int8Linear(down)
    w = (1 + 0.2 * randn(g, 512)).to(BF16)
    for rows in (1, 48, 300):
        x, res = randn(g, rows, 512, dtype=BF16), randn(g, rows, 512, dtype=BF16)

        def serve():
            h, codes, scale = P.residual_norm_int8(x, res, w)
            return P.residual_norm_fwd(down(up(codes, scale)), h, w)

        serve()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h, y = serve()
        for i in range(3):
            x.copy_(randn(g, rows, 512, dtype=BF16))
            res.mul_(0.9)
            graph.replay()
            eager = serve()
            torch.cuda.synchronize()
            assert torch.equal(h, eager[0]) and torch.equal(y, eager[1])
