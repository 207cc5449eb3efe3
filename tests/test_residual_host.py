"""Host-side checks of the C ABI and the calls of the operators between a block's
products (no GPU, nothing is launched), and of the dropout generator's definition.
"""
import ctypes as C
import os
import re
import shutil
import subprocess
import tempfile

import pytest
import torch

import paper_2202_00441_amd as P
from paper_2202_00441_amd import transformer
from paper_2202_00441_amd._lib import E_ALIGN, E_DTYPE, E_INVALID, E_NULL, OK

import dropout_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fewbit_residual.h")
LIB = C.CDLL(P.LIB_PATH)
LIB.fewbit_rnorm_workspace.restype = LIB.fewbit_mm8_workspace.restype = C.c_int64
A = C.c_void_p(16)           # aligned and never read: every call here ends before a launch
ODD = C.c_void_p(24)


class Drop(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_int64), ("seed_at", C.c_void_p), ("site", C.c_uint32), ("reserved", C.c_uint32)]


class Rnorm(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("width", C.c_int32), ("outer", C.c_int64), ("rows", C.c_int64),
                ("x_stride", C.c_int64 * 2), ("residual_stride", C.c_int64 * 2), ("dh_stride", C.c_int64 * 2),
                ("dy_stride", C.c_int64 * 2), ("eps", C.c_float), ("dw_dtype", C.c_int32), ("drop", Drop)]


class Mm8(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("rows", C.c_int64), ("out", C.c_int64), ("width", C.c_int32),
                ("reserved", C.c_int32), ("x_stride", C.c_int64), ("w_stride", C.c_int64)]


def test_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(fewbit_\w+)\s*\(", src)))
    assert names == ["fewbit_dropout", "fewbit_mm8_fwd", "fewbit_mm8_workspace", "fewbit_rnorm_bwd", "fewbit_rnorm_fwd",
                     "fewbit_rnorm_int8", "fewbit_rnorm_workspace", "fewbit_rows8"]
    for name in names:
        assert hasattr(LIB, name), name


def test_header_is_plain_c():
    src = '#include "fewbit_residual.h"\nint main(void) { return sizeof(fewbit_rnorm) + sizeof(fewbit_mm8) > 0 ? 0 : 1; }\n'
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-fsyntax-only", "-I", os.path.dirname(HEADER), "-x", "c", "-"],
                       input=src, text=True, capture_output=True)
    assert r.returncode == 0, r.stderr


def test_structures_are_the_headers():
    """Sizes as the compiler lays them out."""
    src = '#include <stdio.h>\n#include "fewbit_residual.h"\nint main(void) { printf("%zu %zu %zu", sizeof(fewbit_drop), sizeof(fewbit_rnorm), sizeof(fewbit_mm8)); return 0; }\n'
    with tempfile.TemporaryDirectory() as d:
        subprocess.run(["gcc", "-I", os.path.dirname(HEADER), "-x", "c", "-", "-o", os.path.join(d, "sizes")], input=src, text=True, check=True)
        out = subprocess.run([os.path.join(d, "sizes")], capture_output=True, text=True, check=True).stdout
    assert out.split() == [str(C.sizeof(t)) for t in (Drop, Rnorm, Mm8)]


# ---------------------------------------------------------------- the generator
@pytest.mark.parametrize("counter,key,want", (
    ((0, 0, 0, 0), (0, 0), (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
    ((R.WORD,) * 4, (R.WORD,) * 2, (0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0x4DFCCABA, 0x190A87F0, 0xC47362BA, 0xB6B5242A))))
def test_generator_gives_its_authors_answers(counter, key, want):
    assert tuple(R.philox(counter, key, 7)) == want


def test_elements_take_halves_of_blocks():
    seed, site = -7 * 10 ** 17, 0xFFFFFFF0
    u, scale = R.kept(37, 0.5, seed, site, first=(1 << 32) - 2)
    assert scale == 2.0
    for e in range(37):
        block = (1 << 32) - 2 + e // 8
        word = R.philox((block & R.WORD, block >> 32, site, 0), (seed & R.WORD, (seed >> 32) & R.WORD), 7)[e % 8 // 2]
        assert u[e] == ((word >> 16 if e % 2 else word & 0xFFFF) >= 32768)


def test_share_of_dropped_elements():
    """Of n independent numbers with chance p: within five standard deviations, whatever the site and the seed."""
    n = 1 << 18
    for p in (0.1, 0.5):
        masks = [R.kept(n, p, seed, site)[0] for seed in (0, 1) for site in (0, 1)]
        for m in masks:
            assert abs((~m).sum() - n * p) < 5 * (n * p * (1 - p)) ** 0.5
        for i in range(4):
            for j in range(i):
                both = p * p
                assert abs((~masks[i] & ~masks[j]).sum() - n * both) < 5 * (n * both * (1 - both)) ** 0.5


# ---------------------------------------------------------------- dropout
def drop(**changes):
    return Drop(**{"p": 0.1, "seed": 3, **changes})


def dropout(d, dtype=P.BF16, n=100, x=A, y=A):
    return LIB.fewbit_dropout(C.byref(d) if d else None, dtype, C.c_int64(n), x, y, None)


@pytest.mark.parametrize("changes,status", (({"p": -0.1}, E_INVALID), ({"p": 1.1}, E_INVALID), ({"p": float("nan")}, E_INVALID),
                                            ({"reserved": 1}, E_INVALID), ({"seed_at": 20}, E_ALIGN)))
def test_dropout_refusals(changes, status):
    assert dropout(drop(**changes)) == status
    for f in (fwd, bwd):
        assert f(rnorm(drop=drop(**changes))) == status


def test_dropout_arguments():
    assert dropout(None) == E_NULL and dropout(drop(), dtype=9) == E_DTYPE
    assert dropout(drop(), n=-1) == dropout(drop(), n=1 << 37) == E_INVALID
    assert dropout(drop(), x=None) == dropout(drop(), y=None) == E_NULL
    assert dropout(drop(), x=ODD) == dropout(drop(), y=ODD) == E_ALIGN
    assert dropout(drop(), n=0, x=None, y=None) == OK


def test_dropout_of_more_than_a_launch_takes():
    """256 threads for 8192 elements: at 2^37 - 8191 they would be 2^32.  (Without a device a call that is not refused
    ends at the stream.)"""
    assert dropout(drop(), n=(1 << 37) - 8191) == dropout(drop(), n=(1 << 37) - 1) == E_INVALID
    assert dropout(drop(), n=(1 << 37) - 8192, x=None) == E_NULL


# ---------------------------------------------------------------- residual and norm
def rnorm(**changes):
    a = Rnorm(dtype=P.BF16, width=64, outer=2, rows=5, eps=1e-6, drop=drop(p=0.0))
    for s in ("x_stride", "residual_stride", "dh_stride", "dy_stride"):
        setattr(a, s, (C.c_int64 * 2)(320, 64))
    for k, v in changes.items():
        setattr(a, k, (C.c_int64 * 2)(*v) if k.endswith("stride") else v)
    return a


def fwd(a, x=A, res=A, w=A, h=A, y=A):
    return LIB.fewbit_rnorm_fwd(C.byref(a) if a else None, x, res, w, h, y, None)


def int8(a, x=A, res=A, w=A, h=A, codes=A, scale=A):
    return LIB.fewbit_rnorm_int8(C.byref(a) if a else None, x, res, w, h, codes, scale, None)


def rows8(a, x=A, codes=A, scale=A):
    return LIB.fewbit_rows8(C.byref(a) if a else None, x, codes, scale, None)


def bwd(a, dh=A, dy=A, h=A, w=A, dx=A, dres=None, dw=A, work=A, size=1 << 40):
    return LIB.fewbit_rnorm_bwd(C.byref(a) if a else None, dh, dy, h, w, dx, dres, dw, work, C.c_int64(size), None)


@pytest.mark.parametrize("changes,status", (
    ({"dtype": 3}, E_DTYPE), ({"dtype": -1}, E_DTYPE), ({"width": 0}, E_INVALID), ({"width": 12}, E_INVALID), ({"width": 32776}, E_INVALID),
    ({"outer": -1}, E_INVALID), ({"rows": -1}, E_INVALID), ({"rows": 1 << 31}, E_INVALID), ({"outer": 1 << 16, "rows": 1 << 15}, E_INVALID),
    ({"eps": -1.0}, E_INVALID), ({"eps": float("inf")}, E_INVALID), ({"eps": float("nan")}, E_INVALID), ({"dw_dtype": P.F16}, E_INVALID), ({"dw_dtype": 3}, E_INVALID)))
def test_norm_refusals(changes, status):
    a = rnorm(**changes)
    assert fwd(a) == int8(a) == rows8(a) == bwd(a) == LIB.fewbit_rnorm_workspace(C.byref(a)) == status


def test_norm_arguments():
    a, p = rnorm(), rnorm(drop=drop())
    for f, names in ((fwd, ("x", "w", "h", "y")), (int8, ("x", "w", "h", "codes", "scale")), (rows8, ("x", "codes", "scale")),
                     (bwd, ("dy", "h", "w", "dx", "dw", "work"))):
        assert f(None) == E_NULL
        for name in names:
            assert f(a, **{name: None}) == E_NULL, name
            if name not in ("scale", "dw"):          # written an element at a time
                assert f(a, **{name: ODD}) == E_ALIGN, name
    assert fwd(a, res=ODD) == int8(a, res=ODD) == bwd(a, dh=ODD) == bwd(p, dres=ODD) == E_ALIGN
    assert fwd(p, res=None, h=None) == E_NULL            # the sum of dropout alone is written
    assert fwd(rnorm(x_stride=(320, 68))) == rows8(rnorm(x_stride=(324, 64))) == E_ALIGN
    assert fwd(rnorm(residual_stride=(320, 4))) == bwd(rnorm(dy_stride=(4, 64))) == bwd(rnorm(dh_stride=(4, 64))) == E_ALIGN
    assert int8(p) == E_INVALID                          # no dropout there
    assert bwd(a, dres=A) == E_INVALID                   # dx is it
    need = LIB.fewbit_rnorm_workspace(C.byref(a))
    assert need > 0 and need % (64 * 4) == 0 and bwd(a, size=need - 1) == E_INVALID
    none = rnorm(rows=0)
    assert fwd(none, *[None] * 5) == int8(none, *[None] * 6) == rows8(none, *[None] * 3) == OK
    assert LIB.fewbit_rnorm_workspace(C.byref(none)) == 0 and bwd(none, dw=None) == E_NULL


# ---------------------------------------------------------------- product in 8 bits
def mm8(**changes):
    return Mm8(**{"dtype": P.BF16, "act": -1, "rows": 3, "out": 40, "width": 64, "x_stride": 64, "w_stride": 64, **changes})


def product(a, x=A, xs=A, w=A, ws=A, bias=None, y=A, work=A, size=1 << 40):
    return LIB.fewbit_mm8_fwd(C.byref(a) if a else None, x, xs, w, ws, bias, y, work, C.c_int64(size), None)


@pytest.mark.parametrize("changes,status", (
    ({"dtype": 3}, E_DTYPE), ({"act": 2}, E_INVALID), ({"act": -2}, E_INVALID), ({"rows": -1}, E_INVALID), ({"out": -1}, E_INVALID),
    ({"rows": 1 << 31}, E_INVALID), ({"out": 1 << 31}, E_INVALID), ({"width": 0}, E_INVALID), ({"width": 24}, E_INVALID),
    ({"width": 131072}, E_INVALID), ({"reserved": 1}, E_INVALID), ({"x_stride": -64}, E_INVALID), ({"w_stride": -64}, E_INVALID),
    ({"x_stride": (1 << 23) + 16}, E_INVALID), ({"w_stride": (1 << 23) + 16}, E_INVALID)))
def test_product_refusals(changes, status):
    a = mm8(**changes)
    assert product(a) == LIB.fewbit_mm8_workspace(C.byref(a)) == status


def test_product_arguments():
    a = mm8()
    assert product(None) == E_NULL and LIB.fewbit_mm8_workspace(None) == E_NULL
    for name in ("x", "xs", "w", "ws", "y"):
        assert product(a, **{name: None}) == E_NULL, name
        assert product(a, **{name: ODD}) == E_ALIGN, name
    assert product(a, bias=ODD) == product(a, work=ODD) == E_ALIGN
    assert product(mm8(x_stride=72)) == product(mm8(w_stride=72)) == E_ALIGN
    assert LIB.fewbit_mm8_workspace(C.byref(a)) >= 0
    for none in (mm8(rows=0), mm8(out=0)):
        assert product(none, *[None] * 7) == OK and LIB.fewbit_mm8_workspace(C.byref(none)) == 0


@pytest.mark.parametrize("rows", (1, 2, 16, 17, 64, 65, 200, 512, 4096))
@pytest.mark.parametrize("out,width", ((1, 16), (64, 4096), (2048, 8192), (8192, 2048), (777, 131056)))
def test_product_workspace_is_asked_for_and_checked(rows, out, width):
    a = mm8(rows=rows, out=out, width=width, x_stride=width, w_stride=width)
    need = LIB.fewbit_mm8_workspace(C.byref(a))
    assert 0 <= need <= 256 << 20
    if need:
        assert product(a, work=None) == E_NULL and product(a, size=need - 1) == E_INVALID


@pytest.mark.skipif(shutil.which("nm") is None, reason="needs nm")
def test_library_holds_the_kernels_that_a_product_may_take():
    """Shares of the width are offered for tiles of 64 alone (the last argument: whether there are shares)."""
    names = subprocess.run(["nm", "-C", P.LIB_PATH], capture_output=True, text=True, check=True).stdout
    tiles = {tuple(t.replace(" ", "").split(",")) for t in re.findall(r"::tile_kernel<([^>]*)>", names)}
    assert {t[2] for t in tiles if t[-1] == "false"} == {"64", "128", "256"}
    assert {t[2] for t in tiles if t[-1] == "true"} == {"64"}


# ---------------------------------------------------------------- the package's calls
def test_calls_take_device_tensors_alone():
    x, w = torch.ones(4, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    q, s = torch.ones(4, 64, dtype=torch.int8), torch.ones(4)
    for call in (lambda: P.dropout_fwd(x, 0.1, 1), lambda: P.dropout_bwd(x, 0.1, 1), lambda: P.dropout(x, 0.1, 1),
                 lambda: P.residual_norm_fwd(x, x, w), lambda: P.residual_norm(x, x, w), lambda: P.residual_norm_bwd(x, x, x, w),
                 lambda: P.residual_norm_int8(x, x, w), lambda: P.quantize_rows(x), lambda: P.int8_linear(q, s, q, s)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    for call in (lambda: P.dropout_fwd(None, 0.1, 1), lambda: P.residual_norm_fwd(3, x, w), lambda: P.quantize_rows([1.0])):
        with pytest.raises(TypeError, match="must be a tensor"):
            call()
    with pytest.raises(ValueError, match="act"):
        P.int8_linear(q, s, q, s, act="tanh")
    with pytest.raises(TypeError, match="dtype"):
        P.int8_linear(q, s, q, s, dtype=torch.float64)


def test_modules_check_their_arguments():
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ValueError):
            P.Dropout(p)
        with pytest.raises(ValueError):
            transformer.Transformer(10, 32, 1, 2, 1, bits=None, dropout=p)
    with pytest.raises(ValueError, match="multiple of 16"):
        P.Int8Linear(torch.nn.Linear(24, 8))
    with pytest.raises(ValueError, match="act"):
        P.Int8Linear(torch.nn.Linear(32, 8), act="relu")
    x = torch.ones(3)
    assert P.Dropout(0.5).eval()(x) is x and P.Dropout(0.0)(x) is x


@pytest.mark.parametrize("width", (0, 32784, 131056))
def test_layer_of_8_bits_takes_rows_that_are_laid_out(width):
    with pytest.raises(ValueError, match="in_features must be a multiple of 16 up to 32768"):
        P.Int8Linear(torch.nn.Linear(width, 4, device="meta"))


def test_host_seed_follows_torchs_generator():
    from paper_2202_00441_amd.residual import draw_seed
    torch.manual_seed(5)
    a = [draw_seed() for _ in range(3)]
    torch.manual_seed(5)
    assert a == [draw_seed() for _ in range(3)] and len(set(a)) == 3 and all(-2 ** 63 <= v < 2 ** 63 for v in a)


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16, torch.float32, torch.float64))
def test_epsilon_of_norms_without_one(dtype):
    """What torch's norm takes: a value so small that the mean square hardly counts beside it gives it away.
    2^-14 squared is 1/32 of fp32's step: half a step of the type and a few roundings of 32 bits (or 64)."""
    norm = torch.nn.RMSNorm(64).to(dtype)
    x = torch.full((64,), 2.0 ** -14, dtype=dtype)
    want = 2.0 ** -14 * (2.0 ** -28 + transformer._eps(norm)) ** -0.5
    assert abs(float(norm(x)[0].detach()) / want - 1) < max(torch.finfo(dtype).eps / 2, 2.0 ** -24) + 8 * 2.0 ** -24
    norm.eps = 0.25
    assert transformer._eps(norm) == 0.25
