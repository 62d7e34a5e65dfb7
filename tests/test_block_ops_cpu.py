"""Group norm, the feed-forward block and the 8-bit projection (include/paraanya_ops.h) on the CPU: the binding's
structures match the header's, arguments are refused before any HIP call; and the 64-bit formulas that the device
tests compare with agree with differences."""
import ctypes as C
import math
import os
import shutil
import subprocess

import pytest
import torch

import block_ops_reference as R
import ops_reference
from paper_2609_36522_amd import binding as B
from paper_2609_36522_amd import ops as O

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include")
PTR = C.c_void_p(4096)                  # never dereferenced: the calls fail before any launch
I, BIG = B.PA_ERR_INVALID_ARG, 1 << 50


def test_struct_layouts_and_constants_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    structs = {"pa_group_norm_t": O.GroupNorm, "pa_feed_t": O.Feed, "pa_feed_grad_t": O.FeedGrad, "pa_quantize_t": O.Quantize,
               "pa_int8_linear_t": O.Int8Linear}
    consts = ["PA_ACT_NONE", "PA_ACT_SILU", "PA_ACT_GELU", "PA_GROUP_MAX_CHANNELS", "PA_INT8_MAX_IN"]
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


# ------------------------------------------------------------------ group norm
def _group(**kw):
    d = dict(batch=2, pixels=100, channels=64, groups=4, dtype=O.PA_BF16, param_dtype=O.PA_BF16, activation=O.PA_ACT_SILU, eps=1e-5,
             x_stride=(6400, 64), y_stride=(6400, 64), dx_stride=(6400, 64))
    d.update(kw)
    for s in ("x_stride", "y_stride", "dx_stride"):
        d[s] = (C.c_int64 * 2)(*d[s])
    return O.GroupNorm(**d)


def _group_calls(p, bytes_=BIG):
    lib = O._library()
    return (lib.paraanya_group_norm(C.byref(p), PTR, PTR, PTR, PTR, PTR, PTR, PTR, bytes_, None),
            lib.paraanya_group_norm_backward(C.byref(p), *[PTR] * 9, PTR, bytes_, None))


@pytest.mark.parametrize("kw,code,frag", [
    (dict(batch=-1), -1, "batch"), (dict(batch=65536), -1, "batch"), (dict(pixels=-1), -1, "pixels"), (dict(pixels=(1 << 30) + 1), -1, "pixels"),
    (dict(channels=0), -1, "channels"), (dict(channels=(1 << 20) + 4), -1, "channels"), (dict(groups=0), -1, "groups"),
    (dict(groups=5), -1, "groups"), (dict(channels=4097, groups=1, x_stride=(BIG >> 12, 5000), y_stride=(BIG >> 12, 5000)), -6, "channels in a group"),
    (dict(dtype=7), -1, "dtype"), (dict(param_dtype=O.PA_F16), -1, "param_dtype"), (dict(activation=3), -1, "activation"),
    (dict(eps=-1.0), -1, "eps"), (dict(eps=math.nan), -1, "eps"), (dict(eps=math.inf), -1, "eps"),
    (dict(x_stride=(6400, 63)), -1, "pixel stride"), (dict(x_stride=(-1, 64)), -1, "stride"), (dict(y_stride=(6400, 0)), -1, "pixel stride"),
])
def test_group_norm_refuses(kw, code, frag):
    lib, p, n = O._library(), _group(**kw), C.c_size_t(0)
    queries = lib.paraanya_group_norm_workspace, lib.paraanya_group_norm_backward_workspace
    for i in range(2):
        _refused(_group_calls(p)[0] if i == 0 else lib.paraanya_group_norm_backward(C.byref(p), *[PTR] * 9, PTR, BIG, None), code, frag)
        _refused(queries[i](C.byref(p), C.byref(n)), code, frag)


def test_group_norm_refuses_pointers_strides_and_workspaces():
    lib, p, n = O._library(), _group(pixels=100000, x_stride=(BIG >> 12, 64), y_stride=(BIG >> 12, 64), dx_stride=(BIG >> 12, 64)), C.c_size_t(0)
    fwd, bwd = lib.paraanya_group_norm, lib.paraanya_group_norm_backward
    _refused(fwd(None, PTR, None, None, PTR, None, None, PTR, BIG, None), I, "NULL")
    _refused(fwd(C.byref(p), None, None, None, PTR, None, None, PTR, BIG, None), I, "NULL")
    _refused(fwd(C.byref(p), C.c_void_p(4097), None, None, PTR, None, None, PTR, BIG, None), I, "aligned")
    _refused(fwd(C.byref(p), PTR, None, None, PTR, C.c_void_p(4098), None, PTR, BIG, None), I, "aligned")
    _refused(fwd(C.byref(p), PTR, None, None, PTR, None, None, None, 0, None), I, "workspace")
    _refused(bwd(C.byref(p), PTR, PTR, None, None, None, PTR, PTR, PTR, PTR, PTR, BIG, None), I, "NULL")
    assert lib.paraanya_group_norm_workspace(C.byref(p), C.byref(n)) == B.PA_OK and n.value > 0
    _refused(fwd(C.byref(p), PTR, None, None, PTR, None, None, PTR, n.value - 1, None), I, "too small")
    assert lib.paraanya_group_norm_backward_workspace(C.byref(p), C.byref(n)) == B.PA_OK and n.value > 0
    _refused(bwd(C.byref(p), *[PTR] * 9, PTR, n.value - 1, None), I, "too small")
    _refused(bwd(C.byref(p), *[PTR] * 9, C.c_void_p(4100), BIG, None), I, "256-byte")
    _refused(lib.paraanya_group_norm_workspace(C.byref(p), None), I, "NULL")
    q = _group(y_stride=(0, 64))                # an input may repeat a sample, an output may not overlap itself
    _refused(fwd(C.byref(q), PTR, None, None, PTR, None, None, PTR, BIG, None), I, "y overlaps")
    assert lib.paraanya_group_norm_backward_workspace(C.byref(q), C.byref(n)) == B.PA_OK
    _refused(bwd(C.byref(_group(dx_stride=(64, 64))), *[PTR] * 9, PTR, BIG, None), I, "dx overlaps")
    assert lib.paraanya_group_norm_workspace(C.byref(_group(x_stride=(0, 64), y_stride=(64, 128))), C.byref(n)) == B.PA_OK
    for kw in (dict(batch=0), dict(pixels=0)):
        z = _group(**kw)
        assert fwd(C.byref(z), None, None, None, None, None, None, None, 0, None) == B.PA_OK
    assert bwd(C.byref(p), *[PTR] * 6, None, None, None, None, 0, None) == B.PA_OK


# ------------------------------------------------------------------ feed-forward block
FEED = dict(rows=200, in_features=64, hidden_features=96, out_features=32, dtype=O.PA_BF16, activation=O.PA_ACT_GELU, alignment=16,
            x_stride=64, gate_stride=64, up_stride=64, down_stride=96, y_stride=32)


@pytest.mark.parametrize("kw,code,frag", [
    (dict(rows=-1), -1, "rows"), (dict(rows=(1 << 30) + 1), -1, "rows"), (dict(in_features=0), -1, "in_features"),
    (dict(hidden_features=(1 << 20) + 1), -1, "hidden_features"), (dict(out_features=0), -1, "out_features"), (dict(dtype=O.PA_F32), -6, "fp32"),
    (dict(dtype=9), -1, "dtype"), (dict(activation=-1), -1, "activation"), (dict(alignment=3), -1, "alignment"), (dict(alignment=32), -1, "alignment"),
    (dict(x_stride=63), -1, "strides"), (dict(gate_stride=1), -1, "strides"), (dict(up_stride=0), -1, "strides"),
    (dict(down_stride=95), -1, "strides"), (dict(y_stride=31), -1, "strides"),
    (dict(rows=1 << 30, in_features=64), -6, "elements"),
    (dict(rows=1 << 30, in_features=16, hidden_features=8, out_features=8), -6, "tiles"), (dict(hidden_features=1 << 20, down_stride=1 << 20, in_features=1 << 20, x_stride=1 << 20,
                                                                gate_stride=1 << 20, up_stride=1 << 20), -6, "elements"),
])
def test_feed_forward_refuses(kw, code, frag):
    lib, p, n, g = O._library(), O.Feed(**{**FEED, **kw}), C.c_size_t(0), O.FeedGrad(*[4096] * 7)
    _refused(lib.paraanya_feed_forward(C.byref(p), *[PTR] * 9, BIG, PTR, BIG, None), code, frag)
    _refused(lib.paraanya_feed_forward_backward(C.byref(p), C.byref(g), *[PTR] * 6, BIG, PTR, BIG, None), code, frag)
    _refused(lib.paraanya_feed_forward_saved(C.byref(p), C.byref(n)), code, frag)
    _refused(lib.paraanya_feed_forward_workspace(C.byref(p), 0, C.byref(n)), code, frag)
    _refused(lib.paraanya_feed_forward_backward_workspace(C.byref(p), C.byref(n)), code, frag)


def test_feed_forward_refuses_pointers_and_workspaces():
    lib, p, n = O._library(), O.Feed(**FEED), C.c_size_t(0)
    fwd, bwd = lib.paraanya_feed_forward, lib.paraanya_feed_forward_backward

    def forward(p, *, x=PTR, gate=PTR, gate_bias=PTR, y=PTR, saved=PTR, saved_bytes=BIG, ws=PTR, ws_bytes=BIG):
        return fwd(p, x, gate, gate_bias, PTR, PTR, PTR, PTR, y, saved, saved_bytes, ws, ws_bytes, None)

    _refused(forward(None), I, "NULL")
    _refused(forward(C.byref(p), x=None), I, "NULL")
    _refused(forward(C.byref(p), y=None), I, "NULL")
    _refused(forward(C.byref(p), gate=C.c_void_p(4104)), I, "16 bytes")
    _refused(forward(C.byref(p), gate_bias=C.c_void_p(4097)), I, "element")
    _refused(forward(C.byref(p), saved=None, ws=None), I, "workspace")
    _refused(forward(C.byref(p), saved=C.c_void_p(4112)), I, "saved must be 256-byte")
    assert lib.paraanya_feed_forward_saved(C.byref(p), C.byref(n)) == B.PA_OK and n.value >= 3 * 200 * 96 * 2
    _refused(forward(C.byref(p), saved_bytes=n.value - 1), I, "too small")
    # Without saved the gated product is in the workspace.
    assert lib.paraanya_feed_forward_workspace(C.byref(p), 0, C.byref(n)) == B.PA_OK and n.value >= 200 * 96 * 2
    _refused(forward(C.byref(p), saved=None, ws_bytes=n.value - 1), I, "too small")
    # Copies only where rows are not in whole pieces.
    assert lib.paraanya_feed_forward_workspace(C.byref(p), 1, C.byref(n)) == B.PA_OK and n.value == 0
    for kw in (dict(alignment=2), dict(x_stride=65), dict(in_features=63), dict(up_stride=72), dict(down_stride=1 << 23)):
        q = O.Feed(**{**FEED, **kw})
        assert lib.paraanya_feed_forward_workspace(C.byref(q), 1, C.byref(n)) == B.PA_OK and n.value > 0, kw
        _refused(forward(C.byref(q), ws=None), I, "workspace")
    g = O.FeedGrad(*[4096] * 7)
    args = [C.byref(g), PTR, PTR, PTR, PTR, PTR]
    _refused(bwd(C.byref(p), None, *args[1:], PTR, BIG, PTR, BIG, None), I, "NULL")
    _refused(bwd(C.byref(p), args[0], None, *args[2:], PTR, BIG, PTR, BIG, None), I, "NULL")
    _refused(bwd(C.byref(p), *args, None, BIG, PTR, BIG, None), I, "saved")
    _refused(bwd(C.byref(p), *args, PTR, 256, PTR, BIG, None), I, "too small")
    assert lib.paraanya_feed_forward_backward_workspace(C.byref(p), C.byref(n)) == B.PA_OK and n.value > 0
    _refused(bwd(C.byref(p), *args, PTR, BIG, PTR, n.value - 1, None), I, "too small")
    lone = O.FeedGrad(None, None, None, None, 4096, None, None)
    _refused(bwd(C.byref(p), C.byref(lone), *args[1:], PTR, BIG, PTR, BIG, None), I, "weight's")
    odd = O.FeedGrad(4097)
    _refused(bwd(C.byref(p), C.byref(odd), *args[1:], PTR, BIG, PTR, BIG, None), I, "element")
    none = O.FeedGrad()
    assert bwd(C.byref(p), C.byref(none), *args[1:], None, 0, None, 0, None) == B.PA_OK
    z = O.Feed(**{**FEED, "rows": 0})
    assert fwd(C.byref(z), *[None] * 9, 0, None, 0, None) == B.PA_OK
    assert bwd(C.byref(z), C.byref(O.FeedGrad(4096)), *[None] * 6, 0, None, 0, None) == B.PA_OK    # dx without rows: nothing


# ------------------------------------------------------------------ 8-bit integers
QUANT = dict(rows=8, cols=100, dtype=O.PA_F32, x_stride=100, q_stride=112)
INT8 = dict(rows=8, in_features=100, out_features=32, dtype=O.PA_F16, x_stride=112, w_stride=112, y_stride=32)


@pytest.mark.parametrize("kw,code,frag", [
    (dict(rows=-1), -1, "rows"), (dict(cols=0), -1, "cols"), (dict(cols=(1 << 20) + 1), -1, "cols"), (dict(dtype=3), -1, "dtype"),
    (dict(x_stride=99), -1, "strides"), (dict(q_stride=96), -1, "strides"), (dict(q_stride=120), -1, "multiple of 16")])
def test_quantize_rows_refuses(kw, code, frag):
    p = O.Quantize(**{**QUANT, **kw})
    _refused(O._library().paraanya_quantize_rows(C.byref(p), PTR, PTR, PTR, None), code, frag)


@pytest.mark.parametrize("kw,code,frag", [
    (dict(rows=-1), -1, "rows"), (dict(in_features=0), -1, "in_features"), (dict(in_features=1 << 17, x_stride=1 << 17, w_stride=1 << 17), -6, "in_features"),
    (dict(out_features=0), -1, "out_features"), (dict(dtype=O.PA_F32), -6, "fp32"), (dict(dtype=-1), -1, "dtype"), (dict(x_stride=96), -1, "strides"),
    (dict(w_stride=104), -1, "multiples of 16"), (dict(y_stride=31), -1, "strides"), (dict(w_stride=(1 << 22) + 16), -6, "2^22"),
    (dict(rows=1 << 30, out_features=1 << 20, y_stride=1 << 20), -6, "outputs")])
def test_int8_linear_refuses(kw, code, frag):
    p = O.Int8Linear(**{**INT8, **kw})
    _refused(O._library().paraanya_int8_linear(C.byref(p), *[PTR] * 6, None), code, frag)


def test_8_bit_calls_refuse_pointers():
    lib, q, p = O._library(), O.Quantize(**QUANT), O.Int8Linear(**INT8)
    odd = C.c_void_p(4098)
    _refused(lib.paraanya_quantize_rows(None, PTR, PTR, PTR, None), I, "NULL")
    _refused(lib.paraanya_quantize_rows(C.byref(q), PTR, None, PTR, None), I, "NULL")
    _refused(lib.paraanya_quantize_rows(C.byref(q), odd, PTR, PTR, None), I, "aligned")
    _refused(lib.paraanya_quantize_rows(C.byref(q), PTR, C.c_void_p(4104), PTR, None), I, "16-byte")
    f = lib.paraanya_int8_linear
    _refused(f(None, *[PTR] * 6, None), I, "NULL")
    _refused(f(C.byref(p), PTR, PTR, PTR, None, PTR, PTR, None), I, "NULL")
    _refused(f(C.byref(p), C.c_void_p(4104), PTR, PTR, PTR, PTR, PTR, None), I, "16-byte")
    _refused(f(C.byref(p), PTR, odd, PTR, PTR, PTR, PTR, None), I, "aligned")
    assert f(C.byref(O.Int8Linear(**{**INT8, "rows": 0})), *[None] * 6, None) == B.PA_OK
    assert lib.paraanya_quantize_rows(C.byref(O.Quantize(**{**QUANT, "rows": 0})), None, None, None, None) == B.PA_OK


# ------------------------------------------------------------------ the Python functions' own checks
def _z(*s, dt=torch.bfloat16):
    return torch.zeros(s, dtype=dt)


@pytest.mark.parametrize("call,frag", [
    (lambda: O.group_norm(_z(2, 4, 6, dt=torch.float64), 2), "not built"), (lambda: O.group_norm(_z(6), 2), "shape"),
    (lambda: O.group_norm(_z(2, 4, 6), 4), "multiple"), (lambda: O.group_norm(_z(2, 4, 6), 0), "multiple"),
    (lambda: O.group_norm(_z(2, 4, 6), 2, _z(5)), "weight"), (lambda: O.group_norm(_z(2, 4, 6), 2, activation="relu"), "activation"),
    (lambda: O.group_norm_backward(_z(2, 4, 6), _z(2, 4, 6), _z(2, 2), _z(2, 2)), "mean and rstd"),
    (lambda: O.group_norm_backward(_z(2, 3, 6), _z(2, 4, 6), _z(2, 2, dt=torch.float32), _z(2, 2, dt=torch.float32)), "dy"),
    (lambda: O.feed_forward(_z(2, 4, dt=torch.float32), _z(8, 4), _z(8, 4), _z(4, 8)), "not built"),
    (lambda: O.feed_forward(_z(2, 4), _z(8, 4), _z(8, 5), _z(4, 8)), "fit together"),
    (lambda: O.feed_forward(_z(2, 4), _z(8, 4), _z(8, 4), _z(4, 8), _z(7)), "bias"),
    (lambda: O.feed_forward(_z(2, 4), _z(8, 4), _z(8, 4, dt=torch.float16), _z(4, 8)), "one type"),
    (lambda: O.feed_forward(_z(2, 4), _z(8, 4), _z(8, 4), _z(4, 8), activation="tanh"), "activation"),
    (lambda: O.feed_forward_backward(_z(2, 5), _z(2, 4), _z(8, 4), _z(8, 4), _z(4, 8), _z(1)), "dy"),
    (lambda: O.quantize_rows(_z(2, 4, dt=torch.int8)), "not built"), (lambda: O.quantize_rows(_z(2, 0)), "column"),
    (lambda: O.quantize_rows(_z(2, 4).requires_grad_()), "no gradients"),
    (lambda: O.int8_linear(_z(2, 4), _z(2, dt=torch.float32), _z(3, 4), _z(3, dt=torch.float32)), "int8"),
    (lambda: O.int8_linear(_z(2, 4, dt=torch.int8), _z(3, dt=torch.float32), _z(3, 4, dt=torch.int8), _z(3, dt=torch.float32)), "scale"),
    (lambda: O.int8_linear(_z(2, 4, dt=torch.int8), _z(2, dt=torch.float32), _z(3, 5, dt=torch.int8), _z(3, dt=torch.float32)), "expected q"),
    (lambda: O.int8_linear(_z(2, 4, dt=torch.int8), _z(2, dt=torch.float32), _z(3, 4, dt=torch.int8), _z(3, dt=torch.float32), _z(3, dt=torch.float16)), "bias"),
    (lambda: O.int8_linear(_z(2, 4, dt=torch.int8), _z(2, dt=torch.float32), _z(3, 4, dt=torch.int8), _z(3, dt=torch.float32), dtype=torch.float32), "not built"),
    (lambda: O.int8_linear(_z(2, 4, dt=torch.int8), _z(2, dt=torch.float32).requires_grad_(), _z(3, 4, dt=torch.int8), _z(3, dt=torch.float32)), "no gradients"),
])
def test_python_checks(call, frag):
    with pytest.raises(ValueError, match=frag):
        call()


# ------------------------------------------------------------------ the formulas against differences
@pytest.fixture
def exact(monkeypatch):
    for t in (R.U, R.TINY):
        monkeypatch.setitem(t, torch.float64, 0.0)
    assert R.U is ops_reference.U


def _slope(f, args, which, direction, h=1e-5):
    up, dn = list(args), list(args)
    up[which], dn[which] = args[which] + h * direction, args[which] - h * direction
    return float((f(*up) - f(*dn)) / (2 * h))


def _draw(seed, *shapes):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g, dtype=torch.float64) for s in shapes]


@pytest.mark.parametrize("act", [None, "silu", "gelu"])
def test_group_norm_formula_against_differences(exact, act):
    x, w, b, dy = _draw(0, (2, 5, 6), (6,), (6,), (2, 5, 6))
    ref = R.group_norm(x, 3, w, b, 1e-3, act, dy)
    assert torch.allclose(R.group_norm(x, 3, w, b, 1e-3)["y"][0], torch.nn.functional.group_norm(x.transpose(1, 2), 3, w, b, 1e-3).transpose(1, 2))
    for which, name in enumerate(("dx", "dw", "db")):
        e, = _draw(7 + which, (x, w, b)[which].shape)
        got = _slope(lambda *a: (R.group_norm(a[0], 3, a[1], a[2], 1e-3, act)["y"][0] * dy).sum(), (x, w, b), which, e)
        assert abs(got - float((ref[name][0] * e).sum())) < 1e-7, name


@pytest.mark.parametrize("act", [None, "silu", "gelu"])
def test_feed_forward_formula_against_differences(exact, act):
    x, gate, up, down, bg, bu, bd, dy = _draw(1, (4, 5), (7, 5), (7, 5), (3, 7), (7,), (7,), (3,), (4, 3))
    args = (x, gate, up, down, bg, bu, bd)
    ref = R.feed_forward(x, gate, up, down, (bg, bu, bd), act, dy)
    for which, name in enumerate(O.FeedGradients._fields):
        e, = _draw(9 + which, args[which].shape)
        got = _slope(lambda *a: (R.feed_forward(*a[:4], a[4:], act)["y"][0] * dy).sum(), args, which, e)
        assert abs(got - float((ref[name][0] * e).sum())) < 1e-6, name


def test_autograd_returns_a_gradient_for_each_argument(exact, monkeypatch):
    """The autograd functions on formulas in the kernels' place: every argument gets its own gradient, in order."""
    x, gate, up, down, bg, bu, bd, dy = _draw(2, (4, 5), (7, 5), (7, 5), (3, 7), (7,), (7,), (3,), (4, 3))
    monkeypatch.setattr(O, "feed_forward_forward", lambda x, g, u, d, *b, activation, save: (R.feed_forward(x, g, u, d, b, activation)["y"][0], torch.zeros(1)))

    def backward(dy, x, g, u, d, saved, *, activation, need):
        ref = R.feed_forward(x, g, u, d, (bg, bu, bd), activation, dy)
        return O.FeedGradients(*(ref[n][0] for n in O.FeedGradients._fields))

    monkeypatch.setattr(O, "feed_forward_backward", backward)
    leaves = [t.requires_grad_() for t in (x, gate, up, down, bg, bu, bd)]
    O.feed_forward(*leaves, activation="gelu").backward(dy)
    ref = R.feed_forward(x.detach(), gate.detach(), up.detach(), down.detach(), (bg.detach(), bu.detach(), bd.detach()), "gelu", dy)
    for t, name in zip(leaves, O.FeedGradients._fields):
        assert torch.equal(t.grad, ref[name][0]), name
    grad, = torch.autograd.grad(O.feed_forward(*leaves).square().sum() + x.pow(3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.square().sum().backward()

    monkeypatch.setattr(O, "group_norm_forward", lambda x, n, w, b, eps, activation: (R.group_norm(x, n, w, b, eps, activation)["y"][0], torch.zeros(2, n), None))

    def group_backward(dy, x, mean, rstd, w, b, *, activation):
        ref = R.group_norm(x, mean.shape[1], w, b, 1e-5, activation, dy)
        return tuple(ref[n][0] for n in ("dx", "dw", "db"))

    monkeypatch.setattr(O, "group_norm_backward", group_backward)
    x, w, b, dy = _draw(3, (2, 5, 6), (6,), (6,), (2, 5, 6))
    leaves = [t.requires_grad_() for t in (x, w, b)]
    O.group_norm(x, 3, w, b, activation="silu").backward(dy)
    ref = R.group_norm(x.detach(), 3, w.detach(), b.detach(), 1e-5, "silu", dy)
    assert all(torch.equal(t.grad, ref[n][0]) for t, n in zip(leaves, ("dx", "dw", "db")))
    grad, = torch.autograd.grad(O.group_norm(x, 3, w, b).square().sum() + x.pow(3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.square().sum().backward()
