"""The operators' C ABI (include/paraanya_ops.h) on the CPU: every declared entry point is exported,
the binding's structures match the header's, arguments are refused before any HIP call; and the 64-bit
formulas that the device tests compare with agree with differences."""
import ctypes as C
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

import ops_reference as R
from paper_2609_36522_amd import binding as B
from paper_2609_36522_amd import ops as O

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include")
PTR = C.c_void_p(4096)                  # never dereferenced: the calls fail before any launch


def test_library_exports_every_declared_symbol():
    src = open(os.path.join(INCLUDE, "paraanya_ops.h")).read()
    names = sorted(set(re.findall(r"PA_API\s+[\w\s\*]*?\b(paraanya_\w+)\s*\(", src)))
    assert sorted(O.EXPORTED) == names
    lib = B.load_library()
    for n in names:
        assert hasattr(lib, n), n


def test_struct_layouts_and_constants_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    structs = {"pa_norm_t": O.Norm, "pa_cross_t": O.Cross, "pa_cross_grad_t": O.CrossGrad, "pa_lora_t": O.Lora}
    consts = ["PA_F32", "PA_BF16", "PA_F16", "PA_MASK_NONE", "PA_MASK_BOOL", "PA_MASK_ADD", "PA_NORM_MAX_COLS", "PA_LORA_MAX_RANK"]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "paraanya_ops.h"', "int main(void) {"]
    for st, cls in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({st}));')
        lines += [f'printf("%zu\\n", offsetof({st}, {f}));' for f, _ in cls._fields_]
    lines += [f'printf("%d\\n", (int){c});' for c in consts]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run([cc, "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    it = iter(int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    for st, cls in structs.items():
        assert next(it) == C.sizeof(cls), st
        for f, _ in cls._fields_:
            assert next(it) == getattr(cls, f).offset, f"{st}.{f}"
    for c in consts:
        assert next(it) == getattr(O, c), c


def _refused(rc, code, frag):
    msg = B.load_library().paraanya_last_error().decode()
    assert rc == code, (rc, msg)
    assert frag in msg, msg


NORM = dict(rows=4, cols=64, dtype=O.PA_BF16, param_dtype=O.PA_BF16, eps=1e-5, x_stride=64, y_stride=64, dx_stride=64)


@pytest.mark.parametrize("kw,frag", [
    (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(cols=(1 << 20) + 1), "cols"), (dict(dtype=3), "dtype"),
    (dict(param_dtype=O.PA_F16), "param_dtype"), (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(eps=math.inf), "eps"),
    (dict(x_stride=63), "strides"), (dict(y_stride=1), "strides"),
])
def test_layer_norm_refuses(kw, frag):
    lib, p = O._library(), O.Norm(**{**NORM, **kw})
    _refused(lib.paraanya_layer_norm(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, None), B.PA_ERR_INVALID_ARG, frag)
    n = C.c_size_t(7)
    _refused(lib.paraanya_layer_norm_backward_workspace(C.byref(p), C.byref(n)), B.PA_ERR_INVALID_ARG, frag)
    _refused(lib.paraanya_layer_norm_backward(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None),
             B.PA_ERR_INVALID_ARG, frag)


def test_layer_norm_refuses_pointers_and_workspaces():
    lib, p = O._library(), O.Norm(**NORM)
    I = B.PA_ERR_INVALID_ARG
    _refused(lib.paraanya_layer_norm(None, PTR, None, None, PTR, None, None, None), I, "NULL")
    _refused(lib.paraanya_layer_norm(C.byref(p), None, None, None, PTR, None, None, None), I, "NULL")
    _refused(lib.paraanya_layer_norm(C.byref(p), C.c_void_p(4097), None, None, PTR, None, None, None), I, "aligned")
    _refused(lib.paraanya_layer_norm(C.byref(p), PTR, None, None, PTR, C.c_void_p(4098), None, None), I, "aligned")
    bwd = lib.paraanya_layer_norm_backward
    _refused(bwd(C.byref(p), PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None), I, "NULL")
    _refused(bwd(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, 0, None), I, "workspace")
    _refused(bwd(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, C.c_void_p(4100), 1 << 30, None), I, "workspace")
    n = C.c_size_t(0)
    assert lib.paraanya_layer_norm_backward_workspace(C.byref(p), C.byref(n)) == B.PA_OK and n.value > 0
    _refused(bwd(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, n.value - 1, None), I, "too small")
    _refused(lib.paraanya_layer_norm_backward_workspace(C.byref(p), None), I, "NULL")
    q = O.Norm(**{**NORM, "dx_stride": 3})
    _refused(bwd(C.byref(q), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None), I, "strides")
    z = O.Norm(**{**NORM, "rows": 0})
    assert lib.paraanya_layer_norm(C.byref(z), None, None, None, None, None, None, None) == B.PA_OK
    assert bwd(C.byref(p), PTR, PTR, PTR, PTR, PTR, None, None, None, None, 0, None) == B.PA_OK


def _cross(**kw):
    d = dict(batch=2, q_len=5, kv_len=9, q_heads=4, kv_heads=2, head_dim=64, dtype=O.PA_BF16, scale=0.125,
             q_stride=(5 * 256, 256, 64), k_stride=(9 * 128, 128, 64), v_stride=(9 * 128, 128, 64), o_stride=(5 * 256, 256, 64))
    d.update(kw)
    for s in ("q_stride", "k_stride", "v_stride", "o_stride"):
        d[s] = (C.c_int64 * 3)(*d[s])
    return O.Cross(**d)


@pytest.mark.parametrize("kw,code,frag", [
    (dict(batch=-1), -1, "batch"), (dict(batch=65536), -1, "batch"), (dict(q_len=-1), -1, "q_len"), (dict(kv_len=-2), -1, "kv_len"),
    (dict(kv_len=(1 << 30) + 1), -1, "kv_len"), (dict(q_heads=0), -1, "heads"), (dict(q_heads=3), -1, "heads"),
    (dict(kv_heads=0), -1, "heads"), (dict(q_len=1 << 29), -1, "2^30"), (dict(head_dim=0), -1, "head_dim"),
    (dict(head_dim=129), -6, "head_dim"), (dict(dtype=O.PA_F32), -6, "fp32"), (dict(dtype=9), -1, "dtype"),
    (dict(scale=math.inf), -1, "scale"), (dict(scale=math.nan), -1, "scale"), (dict(mask_kind=3), -1, "mask_kind"),
    (dict(mask_kind=1), -1, "mask"), (dict(mask=4096), -1, "mask"), (dict(mask=4098, mask_kind=2), -1, "aligned"),
    (dict(mask=4096, mask_kind=2, mask_stride=-1), -1, "mask_stride"), (dict(kv_lens=4097), -1, "aligned"),
    (dict(q_stride=(-1, 256, 64)), -1, "stride"), (dict(o_stride=(0, 256, 64)), -1, "overlaps"),
    (dict(o_stride=(1280, 32, 64)), -1, "overlaps"), (dict(o_stride=(1280, 256, 0)), -1, "overlaps"),
    (dict(batch=60000, kv_len=1 << 20), -6, "keys"), (dict(batch=60000, q_len=1 << 20), -6, "rows"),
])
def test_cross_attention_refuses(kw, code, frag):
    lib, p = O._library(), _cross(**kw)
    n = C.c_size_t(0)
    g = O.CrossGrad(*[(C.c_int64 * 3)(1 << 20, 256, 64)] * 4)
    _refused(lib.paraanya_cross_attention(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, 1 << 40, None), code, frag)
    _refused(lib.paraanya_cross_attention_workspace(C.byref(p), C.byref(n)), code, frag)
    _refused(lib.paraanya_cross_attention_backward(C.byref(p), C.byref(g), PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 40, None),
             code, frag)


def test_cross_attention_refuses_pointers_and_workspaces():
    lib, p, I = O._library(), _cross(), B.PA_ERR_INVALID_ARG
    fwd, bwd = lib.paraanya_cross_attention, lib.paraanya_cross_attention_backward
    _refused(fwd(None, PTR, PTR, PTR, PTR, None, None, 0, None), I, "NULL")
    _refused(fwd(C.byref(p), None, PTR, PTR, PTR, None, None, 0, None), I, "NULL")
    _refused(fwd(C.byref(p), PTR, PTR, None, PTR, None, None, 0, None), I, "NULL")
    _refused(fwd(C.byref(p), PTR, C.c_void_p(4097), PTR, PTR, None, None, 0, None), I, "aligned")
    n = C.c_size_t(0)
    long = _cross(batch=1, q_len=1, kv_len=100000, o_stride=(256, 256, 64))
    assert lib.paraanya_cross_attention_workspace(C.byref(long), C.byref(n)) == B.PA_OK and n.value > 0
    _refused(fwd(C.byref(long), PTR, PTR, PTR, PTR, None, PTR, n.value - 1, None), I, "too small")
    _refused(fwd(C.byref(long), PTR, PTR, PTR, PTR, None, None, 0, None), I, "workspace")
    g = O.CrossGrad(*[(C.c_int64 * 3)(1 << 20, 256, 64)] * 4)
    args = [C.byref(p), C.byref(g), PTR, PTR, PTR, PTR, PTR, PTR]
    _refused(bwd(C.byref(p), None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None), I, "NULL")
    _refused(bwd(*args, PTR, PTR, None, PTR, 1 << 30, None), I, "together")
    _refused(bwd(*args, PTR, PTR, PTR, None, 0, None), I, "workspace")
    _refused(bwd(*args[:2], None, *args[3:], PTR, PTR, PTR, PTR, 1 << 30, None), I, "NULL")
    bad = O.CrossGrad(*[(C.c_int64 * 3)(1 << 20, 256, 64)] * 2, (C.c_int64 * 3)(0, 256, 64), (C.c_int64 * 3)(1 << 20, 256, 64))
    _refused(bwd(C.byref(p), C.byref(bad), *args[2:], PTR, PTR, PTR, PTR, 1 << 30, None), I, "dk overlaps")
    z = _cross(batch=0)
    assert fwd(C.byref(z), None, None, None, None, None, None, 0, None) == B.PA_OK
    assert bwd(*args, None, None, None, None, 0, None) == B.PA_OK


LORA = dict(rows=8, in_features=64, out_features=32, rank=8, adapters=2, requests=1, dtype=O.PA_BF16, x_stride=64, w_stride=64,
            y_stride=32, offsets=4096, ids=4096, scales=4096)


@pytest.mark.parametrize("kw,code,frag", [
    (dict(rows=-1), -1, "rows"), (dict(in_features=0), -1, "in_features"), (dict(out_features=(1 << 20) + 1), -1, "out_features"),
    (dict(rank=0), -1, "rank"), (dict(rank=129), -6, "rank"), (dict(adapters=-1), -1, "adapters"), (dict(requests=-1), -1, "requests"),
    (dict(requests=65536), -1, "requests"), (dict(dtype=O.PA_F32), -6, "fp32"), (dict(dtype=5), -1, "dtype"),
    (dict(x_stride=63), -1, "strides"), (dict(w_stride=0), -1, "strides"), (dict(y_stride=31), -1, "strides"),
    (dict(offsets=None), -1, "offsets"), (dict(ids=None), -1, "ids"), (dict(offsets=4097), -1, "aligned"),
    (dict(rows=1 << 30, out_features=1 << 20, y_stride=1 << 20), -6, "outputs"),
])
def test_lora_linear_refuses(kw, code, frag):
    lib, p = O._library(), O.Lora(**{**LORA, **kw})
    n = C.c_size_t(0)
    _refused(lib.paraanya_lora_linear(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 40, None), code, frag)
    _refused(lib.paraanya_lora_linear_workspace(C.byref(p), C.byref(n)), code, frag)


def test_lora_linear_refuses_pointers_and_workspaces():
    lib, p, I = O._library(), O.Lora(**LORA), B.PA_ERR_INVALID_ARG
    f = lib.paraanya_lora_linear
    _refused(f(None, PTR, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None), I, "NULL")
    _refused(f(C.byref(p), None, PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None), I, "NULL")
    _refused(f(C.byref(p), PTR, PTR, PTR, None, PTR, PTR, PTR, 1 << 30, None), I, "NULL")
    _refused(f(C.byref(p), PTR, PTR, C.c_void_p(4097), PTR, PTR, PTR, PTR, 1 << 30, None), I, "aligned")
    _refused(f(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, None, 0, None), I, "workspace")
    z = O.Lora(**{**LORA, "rows": 0})
    assert f(C.byref(z), None, None, None, None, None, None, None, 0, None) == B.PA_OK


# ------------------------------------------------------------------ the formulas against differences
def _slope(f, args, which, direction, h=1e-5):
    up, dn = list(args), list(args)
    up[which], dn[which] = args[which] + h * direction, args[which] - h * direction
    return float((f(*up) - f(*dn)) / (2 * h))


def test_layer_norm_formula_against_differences():
    g = torch.Generator().manual_seed(0)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((5, 13), (13,), (13,), (5, 13)))
    R.U[torch.float64] = R.TINY[torch.float64] = 0.0
    ref = R.layer_norm(x, w, b, 1e-3, dy)
    for which, name in enumerate(("dx", "dw", "db")):
        e = torch.randn((x, w, b)[which].shape, generator=g, dtype=torch.float64)
        got = _slope(lambda *a: (R.layer_norm(*a, 1e-3)["y"][0] * dy).sum(), (x, w, b), which, e)
        assert abs(got - float((ref[name][0] * e).sum())) < 1e-7, name


@pytest.mark.parametrize("Hq,Hk", [(2, 2), (4, 2), (3, 1)])
def test_cross_attention_formula_against_differences(Hq, Hk):
    g = torch.Generator().manual_seed(1)
    q, k, v, do = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 4, Hq, 6), (3, 7, Hk, 6), (3, 7, Hk, 6), (3, 4, Hq, 6)))
    R.U[torch.float64] = R.TINY[torch.float64] = 0.0
    mask = torch.randn(3, 7, generator=g)
    mask[1, 2:5] = -math.inf
    mask[2] = -math.inf
    kw = dict(mask=mask, kv_lens=torch.tensor([7, 6, 7]))
    ref = R.cross_attention(q, k, v, do, **kw)
    assert not ref["o"][0][2].any() and not ref["dk"][0][2].any() and not ref["dk"][0][1, 2:5].any()
    for which, name in enumerate(("dq", "dk", "dv")):
        e = torch.randn((q, k, v)[which].shape, generator=g, dtype=torch.float64)
        got = _slope(lambda *a: (R.cross_attention(*a, **kw)["o"][0] * do).sum(), (q, k, v), which, e)
        assert abs(got - float((ref[name][0] * e).sum())) < 1e-7, name


# ------------------------------------------------------------------ autograd, on formulas in the kernels' place
def _norm_formula(x, w, b, eps):
    mean = x.mean(-1)
    rstd = 1 / torch.sqrt(x.var(-1, unbiased=False) + eps)
    xh = (x - mean[..., None]) * rstd[..., None]
    return xh * w + b, mean, rstd


def _norm_formula_backward(dy, x, mean, rstd, w, param_dtype=None):
    xh = (x - mean[..., None]) * rstd[..., None]
    g = dy * w
    return (rstd[..., None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True)), (dy * xh).sum(0), dy.sum(0))


def test_layer_norm_refuses_second_derivatives(monkeypatch):
    """The backward pass has no derivative of its own: a gradient's gradient is refused, not taken as zero."""
    monkeypatch.setattr(O, "layer_norm_forward", _norm_formula)
    monkeypatch.setattr(O, "layer_norm_backward", _norm_formula_backward)
    g = torch.Generator().manual_seed(2)
    x, w, b = (torch.randn(s, generator=g, dtype=torch.float64).requires_grad_() for s in ((4, 9), (9,), (9,)))
    loss = O.layer_norm(x, w, b).pow(3).sum() + x.square().sum()
    want, = torch.autograd.grad(torch.nn.functional.layer_norm(x, (9,), w, b).pow(3).sum() + x.square().sum(), x)
    grad, = torch.autograd.grad(loss, x, create_graph=True)
    assert torch.allclose(grad, want)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.square().sum().backward()


def test_cross_attention_refuses_second_derivatives(monkeypatch):
    def formula(q, k, v, *, kv_lens=None, mask=None, scale=None):
        return R.cross_attention(q, k, v)["o"][0], torch.zeros(1)

    def backward(do, q, k, v, o, stats, *, kv_lens=None, mask=None, scale=None):
        ref = R.cross_attention(q, k, v, do)
        return tuple(ref[n][0] for n in ("dq", "dk", "dv"))

    monkeypatch.setitem(R.U, torch.float64, 0.0)
    monkeypatch.setitem(R.TINY, torch.float64, 0.0)
    monkeypatch.setattr(O, "cross_attention_forward", formula)
    monkeypatch.setattr(O, "cross_attention_backward", backward)
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((1, n, 2, 6), generator=g, dtype=torch.float64).requires_grad_() for n in (4, 7, 7))
    loss = O.cross_attention(q, k, v).pow(3).sum() + q.square().sum()
    grad, = torch.autograd.grad(loss, q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.square().sum().backward()


def test_cross_attention_refuses_a_learned_mask(monkeypatch):
    """An additive mask gets no gradient: one that asks for it is refused where gradients are recorded."""
    monkeypatch.setattr(O, "cross_attention_forward", lambda q, k, v, *, kv_lens=None, mask=None, scale=None: (q * 1, torch.zeros(1)))
    q, k, v = (torch.zeros(1, n, 2, 8, dtype=torch.bfloat16) for n in (3, 5, 5))
    mask = torch.zeros(1, 5, requires_grad=True)
    for first in (q, q.clone().requires_grad_()):
        with pytest.raises(ValueError, match="mask"):
            O.cross_attention(first, k, v, mask=mask)
        assert O.cross_attention(first, k, v, mask=mask.detach()).shape == q.shape
        with torch.no_grad():
            assert O.cross_attention(first, k, v, mask=mask).shape == q.shape


def test_cross_attention_refuses_heads_without_elements():
    """The default scale of a head width of 0 is no error of its own: the library refuses the width."""
    q = torch.zeros(1, 2, 2, 0, dtype=torch.bfloat16)
    with pytest.raises(B.PAError, match="head_dim"):
        O._cross_args(q, q, q, None, None, None, q)


@pytest.mark.parametrize("kw", [dict(q_len=0, o_stride=(0, 256, 64)), dict(batch=0, o_stride=(0, 0, 0)),
                                dict(q_len=0, kv_len=0, o_stride=(0, 0, 0))])
def test_cross_attention_outputs_without_elements_overlap_nothing(kw):
    """Strides of an output that has no elements are not looked at: a dense one without tokens has a stride of 0."""
    lib, p, n = O._library(), _cross(**kw), C.c_size_t(0)
    assert lib.paraanya_cross_attention_workspace(C.byref(p), C.byref(n)) == B.PA_OK, lib.paraanya_last_error()
    assert lib.paraanya_cross_attention(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, 1 << 30, None) == B.PA_OK
    none = O.CrossGrad(*[(C.c_int64 * 3)(0, 0, 0)] * 4)
    if kw.get("batch") == 0:
        assert lib.paraanya_cross_attention_backward(C.byref(p), C.byref(none), *[PTR] * 10, 1 << 30, None) == B.PA_OK
