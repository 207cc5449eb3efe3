"""Host-side checks of the block operators' C ABI and calls (no GPU, nothing is
launched): the library exports what include/fewbit_block.h declares, every
argument error comes back before a launch, and the package's calls refuse
tensors that are not on a device.
"""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2202_00441_amd as P
from paper_2202_00441_amd import _lib, transformer
from paper_2202_00441_amd._lib import E_ALIGN, E_BITS, E_DTYPE, E_INVALID, E_NULL, OK

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fewbit_block.h")
LIB = C.CDLL(P.LIB_PATH)
LIB.fewbit_attn_workspace.restype = LIB.fewbit_qk_workspace.restype = C.c_int64
A = C.c_void_p(16)           # aligned and never read: every call here ends before a launch
ODD = C.c_void_p(24)


class Attn(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads_q", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32),
                ("causal", C.c_int32), ("window", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32),
                ("batch", C.c_int64), ("rows_q", C.c_int64), ("rows_k", C.c_int64), ("cu_q", C.c_void_p),
                ("cu_k", C.c_void_p), ("k_len", C.c_void_p), ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("dout_stride", C.c_int64 * 3)]


class Qk(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads_q", C.c_int32), ("heads_k", C.c_int32), ("head_dim", C.c_int32),
                ("rot", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32),
                ("batch", C.c_int64), ("tokens", C.c_int64), ("table_rows", C.c_int64), ("q_stride", C.c_int64 * 3),
                ("k_stride", C.c_int64 * 3), ("dq_stride", C.c_int64 * 3), ("dk_stride", C.c_int64 * 3),
                ("position_stride", C.c_int64 * 2)]


class AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("n", C.c_int64)]


class Adamw(C.Structure):
    _fields_ = [("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("state_bits", C.c_int32), ("reserved", C.c_int32),
                ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("step", C.c_int64), ("seed", C.c_int64)]


def test_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(fewbit_\w+)\s*\(", src)))
    assert names == ["fewbit_adamw_step", "fewbit_attn_bwd", "fewbit_attn_fwd", "fewbit_attn_workspace",
                     "fewbit_qk_bwd", "fewbit_qk_fwd", "fewbit_qk_workspace"]
    for name in names:
        assert hasattr(LIB, name), name


# ---------------------------------------------------------------- attention
def attn(**changes):
    a = Attn(dtype=P.BF16, heads_q=8, heads_kv=2, head_dim=64, scale=0.125, batch=2, rows_q=10, rows_k=12)
    for s in ("q_stride", "k_stride", "v_stride", "dout_stride"):
        setattr(a, s, (C.c_int64 * 3)(5120, 512, 64))
    for k, v in changes.items():
        setattr(a, k, (C.c_int64 * 3)(*v) if k.endswith("stride") else v)
    return a


def attn_fwd(a, q=A, k=A, v=A, out=A, lse=A, work=A, size=1 << 40):
    return LIB.fewbit_attn_fwd(C.byref(a) if a else None, q, k, v, out, lse, work, C.c_int64(size), None)


def attn_bwd(a, *p, work=A, size=1 << 40):
    p = list(p) + [A] * (9 - len(p))
    return LIB.fewbit_attn_bwd(C.byref(a) if a else None, *p, work, C.c_int64(size), None)


BAD_ATTN = [({"dtype": P.F32}, E_DTYPE), ({"dtype": 7}, E_DTYPE), ({"heads_q": 7}, E_INVALID), ({"heads_q": 0}, E_INVALID),
            ({"heads_kv": 0}, E_INVALID), ({"head_dim": 0}, E_INVALID), ({"head_dim": 12}, E_INVALID),
            ({"head_dim": 136}, E_INVALID), ({"causal": 2}, E_INVALID), ({"window": -1, "causal": 1}, E_INVALID),
            ({"window": 4}, E_INVALID), ({"scale": 0.0}, E_INVALID), ({"scale": -1.0}, E_INVALID),
            ({"scale": float("inf")}, E_INVALID), ({"scale": float("nan")}, E_INVALID), ({"reserved": 1}, E_INVALID),
            ({"batch": -1}, E_INVALID), ({"rows_q": -1}, E_INVALID), ({"rows_k": -1}, E_INVALID),
            ({"rows_q": 1 << 30}, E_INVALID), ({"rows_k": 1 << 30}, E_INVALID), ({"cu_q": 16}, E_INVALID),
            ({"cu_q": 16, "cu_k": 16, "k_len": 16}, E_INVALID)]


@pytest.mark.parametrize("changes,status", BAD_ATTN)
def test_attention_refusals(changes, status):
    a = attn(**changes)
    assert attn_fwd(a) == attn_bwd(a) == status
    assert LIB.fewbit_attn_workspace(C.byref(a), 0) == LIB.fewbit_attn_workspace(C.byref(a), 1) == status


def test_attention_pointers_strides_and_workspace():
    a = attn()
    assert attn_fwd(None) == attn_bwd(None) == E_NULL
    for i in range(5):
        p = [A] * 5
        p[i] = None
        assert attn_fwd(a, *p) == E_NULL
    for i in range(4):
        p = [A] * 5
        p[i] = ODD
        assert attn_fwd(a, *p) == E_ALIGN
    for i in range(9):
        p = [A] * 9
        p[i] = None
        assert attn_bwd(a, *p) == E_NULL
        if i != 5:           # lse is read a float at a time
            p[i] = ODD
            assert attn_bwd(a, *p) == E_ALIGN
    for name in ("q_stride", "k_stride", "v_stride"):
        assert attn_fwd(attn(**{name: (5120, 516, 64)})) == attn_bwd(attn(**{name: (5120, 516, 64)})) == E_ALIGN
    assert attn_bwd(attn(dout_stride=(5120, 512, 4))) == E_ALIGN
    # numbers for every row and head; a long cache needs room for every share of a sequence
    need = LIB.fewbit_attn_workspace(C.byref(a), 1)
    assert need > 0 and need % (2 * 10 * 8 * 4) == 0
    assert attn_bwd(a, work=None) == E_NULL and attn_bwd(a, size=need - 1) == E_INVALID
    long = attn(rows_q=1, rows_k=100000)
    need = LIB.fewbit_attn_workspace(C.byref(long), 0)
    assert need > 0 and need % (8 * 65 * 4) == 0
    assert attn_fwd(long, work=None) == E_NULL and attn_fwd(long, size=need - 1) == E_INVALID
    assert attn_fwd(long, work=ODD) == E_ALIGN


def test_attention_strides_are_not_negative():
    """A lane's offset inside a load is a number without a sign: rows in reverse order would be read far ahead."""
    for i in range(3):
        for name in ("q_stride", "k_stride", "v_stride", "dout_stride"):
            stride = [5120, 512, 64]
            stride[i] = -stride[i]
            assert attn_bwd(attn(**{name: stride})) == E_INVALID, (name, i)
            if name != "dout_stride":
                assert attn_fwd(attn(**{name: stride})) == E_INVALID, (name, i)


def test_packed_attention_has_no_stride_of_sequences():
    """The first stride is not used then, whatever it is: the call ends at the next check, the workspace's size."""
    names = ("q_stride", "k_stride", "v_stride", "dout_stride")
    for first in (3, -8):
        odd = {name: (first, 512, 64) for name in names}
        assert attn_bwd(attn(cu_q=16, cu_k=16, **odd), size=0) == E_INVALID
        assert attn_bwd(attn(**odd), size=0) == (E_ALIGN if first == 3 else E_INVALID)
    assert attn_bwd(attn(cu_q=16, cu_k=16, q_stride=(0, 516, 64)), size=0) == E_ALIGN


def test_many_caches_are_not_divided():
    """Shares of many caches with lengths of their own would have to be found from all lengths by each workgroup: where
    every CU has several caches they are left whole, and need no room for joins."""
    few, many = attn(batch=16, rows_q=1, rows_k=4096, k_len=16), attn(batch=4096, rows_q=1, rows_k=4096, k_len=16)
    assert LIB.fewbit_attn_workspace(C.byref(few), 0) > 0 == LIB.fewbit_attn_workspace(C.byref(many), 0)


def test_attention_grids_past_a_launch():
    """A launch has fewer than 2^32 threads.  The kernel for dK and dV has 512 to a workgroup, here of one key head
    each, 2^23 of them: refused before the kernel for dQ, of 256 threads, is launched.  Sizes whose products pass 64
    bits are refused too."""
    a = attn(batch=1 << 20, heads_q=8, heads_kv=8, head_dim=128, rows_q=1, rows_k=1)
    assert attn_bwd(a) == E_INVALID
    for most in ({"batch": (1 << 30) - 1, "rows_q": (1 << 30) - 1, "heads_q": 1 << 18, "heads_kv": 1 << 18},
                 {"batch": 1 << 29, "rows_q": 1 << 29, "rows_k": 1 << 29, "heads_q": 1 << 19, "heads_kv": 1 << 19}):
        assert attn_fwd(attn(**most), size=(1 << 63) - 1) == attn_bwd(attn(**most), size=(1 << 63) - 1) == E_INVALID


def test_attention_of_nothing():
    assert attn_fwd(attn(batch=0)) == attn_bwd(attn(batch=0)) == OK
    assert attn_fwd(attn(rows_q=0)) == OK
    assert attn_bwd(attn(rows_q=0, rows_k=0)) == OK


# ---------------------------------------------------------------- norm and rotation
def qk(**changes):
    a = Qk(dtype=P.BF16, heads_q=4, heads_k=2, head_dim=64, rot=64, eps=1e-6, batch=2, tokens=10, table_rows=100)
    for s in ("q_stride", "k_stride", "dq_stride", "dk_stride"):
        setattr(a, s, (C.c_int64 * 3)(5120, 512, 64))
    for k, v in changes.items():
        setattr(a, k, (C.c_int64 * 3)(*v) if k.endswith("stride") else v)
    return a


def qk_fwd(a, *p):
    p = list(p) + [A] * (9 - len(p))
    return LIB.fewbit_qk_fwd(C.byref(a) if a else None, *p, None)


def qk_bwd(a, *p, work=A, size=1 << 40):
    p = list(p) + [A] * (13 - len(p))
    return LIB.fewbit_qk_bwd(C.byref(a) if a else None, *p, work, C.c_int64(size), None)


BAD_QK = [({"dtype": 3}, E_DTYPE), ({"dtype": -1}, E_DTYPE), ({"heads_q": -1}, E_INVALID), ({"heads_k": -1}, E_INVALID),
          ({"head_dim": 24}, E_INVALID), ({"head_dim": 0}, E_INVALID), ({"head_dim": 272}, E_INVALID),
          ({"rot": 8}, E_INVALID), ({"rot": 80}, E_INVALID), ({"rot": -16}, E_INVALID), ({"interleaved": 2}, E_INVALID),
          ({"eps": -1.0}, E_INVALID), ({"eps": float("nan")}, E_INVALID), ({"reserved": 1}, E_INVALID),
          ({"batch": -1}, E_INVALID), ({"tokens": -1}, E_INVALID), ({"table_rows": -1}, E_INVALID),
          ({"tokens": 1 << 31}, E_INVALID), ({"batch": 1 << 30, "tokens": 1 << 30}, E_INVALID)]


@pytest.mark.parametrize("changes,status", BAD_QK)
def test_qk_refusals(changes, status):
    a = qk(**changes)
    assert qk_fwd(a) == qk_bwd(a) == LIB.fewbit_qk_workspace(C.byref(a)) == status


def test_qk_pointers_strides_and_workspace():
    a = qk()
    assert qk_fwd(None) == qk_bwd(None) == LIB.fewbit_qk_workspace(None) == E_NULL
    for i in range(9):
        if i == 6:           # positions may be missing
            continue
        p = [A] * 9
        p[i] = None
        assert qk_fwd(a, *p) == E_NULL, i
        p[i] = ODD
        assert qk_fwd(a, *p) == E_ALIGN, i
    for i in range(13):
        if i == 8:
            continue
        p = [A] * 13
        p[i] = None
        assert qk_bwd(a, *p) == E_NULL, i
        if i < 11:           # the weights' gradients are written a float at a time
            p[i] = ODD
            assert qk_bwd(a, *p) == E_ALIGN, i
    assert qk_fwd(qk(q_stride=(5120, 516, 64))) == qk_bwd(qk(dk_stride=(5120, 512, 4))) == E_ALIGN
    need = LIB.fewbit_qk_workspace(C.byref(a))
    assert need > 0 and need % (64 * 4) == 0
    assert qk_bwd(a, work=None) == E_NULL and qk_bwd(a, size=need - 1) == E_INVALID
    assert qk_fwd(qk(tokens=0)) == qk_fwd(qk(batch=0)) == qk_bwd(qk(heads_q=0, heads_k=0), *[None] * 13) == OK


# ---------------------------------------------------------------- AdamW
def adamw(**changes):
    a = Adamw(param_dtype=P.BF16, grad_dtype=P.BF16, state_bits=8, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8,
              weight_decay=0.1, step=1)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


def step(a, tensors=((16, 16, 100),), m=A, v=A, ms=A, vs=A, master=None, count=None):
    list_ = (AdamwTensor * max(1, len(tensors)))(*[AdamwTensor(*t) for t in tensors])
    return LIB.fewbit_adamw_step(C.byref(a) if a else None, list_, len(tensors) if count is None else count, m, v, ms, vs,
                                 master, None)


@pytest.mark.parametrize("changes,status", [
    ({"param_dtype": 3}, E_DTYPE), ({"grad_dtype": P.F16}, E_DTYPE), ({"param_dtype": P.F32}, E_DTYPE),
    ({"state_bits": 16}, E_BITS), ({"reserved": 1}, E_INVALID), ({"step": 0}, E_INVALID), ({"lr": -1.0}, E_INVALID),
    ({"lr": float("nan")}, E_INVALID), ({"beta1": 1.0}, E_INVALID), ({"beta1": -0.1}, E_INVALID),
    ({"beta2": 1.0}, E_INVALID), ({"eps": -1.0}, E_INVALID), ({"weight_decay": float("inf")}, E_INVALID)])
def test_adamw_refusals(changes, status):
    assert step(adamw(**changes)) == status


def test_adamw_lists_and_pointers():
    a = adamw()
    assert step(None) == E_NULL
    assert step(a, count=-1) == E_INVALID
    assert step(a, ()) == step(a, ((16, 16, 0),)) == OK
    assert step(a, ((16, 16, -1),)) == E_INVALID
    assert step(a, ((None, 16, 5),)) == E_NULL
    for name in ("m", "v", "ms", "vs"):
        assert step(a, **{name: None}) == E_NULL
        assert step(a, **{name: ODD}) == E_ALIGN
    assert step(a, master=ODD) == E_ALIGN
    assert step(adamw(param_dtype=P.F32, grad_dtype=P.F32), master=A) == E_INVALID


# ---------------------------------------------------------------- the package's calls
def test_calls_refuse_tensors_that_are_not_on_a_device():
    x = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    w, table = torch.ones(64, dtype=torch.bfloat16), torch.ones(8, 32)
    with pytest.raises(ValueError, match="device tensor"):
        P.attention_fwd(x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        P.attention(x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        P.attention_bwd(x, x, x, x, x, torch.zeros(1, 2, 4))
    with pytest.raises(ValueError, match="device tensor"):
        P.qk_norm_rope(x, x, w, w, table, table)
    with pytest.raises(ValueError, match="device tensor"):
        P.adamw_step([x], [x], x, x, lr=0.1, step=1)
    with pytest.raises(TypeError, match="must be a tensor"):
        P.attention_fwd(None, x, x)
    with pytest.raises(TypeError, match="sequence"):
        P.adamw_step(None, [x], x, x, lr=0.1, step=1)
    with pytest.raises(ValueError, match="same length"):
        P.adamw_step([x], [], x, x, lr=0.1, step=1)
    P.adamw_step([], [], x, x, lr=0.1, step=1)


def test_generation_stays_inside_the_cache_and_the_tables():
    """A token past a cache, or past the positions there are angles for, is refused on the host."""
    model = transformer.Transformer(10, 64, 1, 2, 1, bits=None, most=20)
    tokens = torch.zeros(2, 6, dtype=torch.long)
    with pytest.raises(ValueError, match="the cache holds 5 tokens"):
        model.extend(tokens, model.cache(2, 5))
    cache = model.cache(2, 9)
    cache.used = 4                                          # as after four tokens
    with pytest.raises(ValueError, match="the cache holds 9 tokens"):
        model.extend(tokens, cache)
    with pytest.raises(ValueError, match="the model has 20 positions"):
        model.extend(torch.zeros(1, 21, dtype=torch.long), model.cache(1, 30))
    with pytest.raises(ValueError, match="the model has 20 positions"):
        model.generate(tokens, 16)                          # the last token has no position yet: 21 are needed
    with pytest.raises(ValueError, match="the model has 20 positions"):
        model(torch.zeros(1, 21, dtype=torch.long))
    with pytest.raises(ValueError, match="sequences"):
        model.extend(tokens, model.cache(3, 9))


def test_generation_of_nothing():
    model = transformer.Transformer(10, 64, 1, 2, 1, bits=None, most=20)
    out = model.generate(torch.zeros(2, 6, dtype=torch.long), 0)
    assert out.shape == (2, 0) and out.dtype == torch.long


def test_blocks():
    assert [P.adamw_blocks(n) for n in (0, 1, 256, 257)] == [0, 1, 1, 2]
    assert _lib.strerror(E_ALIGN)
