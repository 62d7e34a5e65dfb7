"""Group norm, the gated feed-forward block and the 8-bit projection on the device against their definitions
in 64 bits (tests/block_ops_reference.py), at the sizes, strides and types where they can go wrong."""
import math

import pytest
import torch

import block_ops_reference as R
from ops_reference import TINY, U, check
from paper_2609_36522_amd import binding as B
from paper_2609_36522_amd import ops

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = dict(argvalues=[BF16, F16], ids=["bf16", "f16"])


@pytest.fixture(autouse=True)
def _lib(gpu_lib):
    return gpu_lib


def _gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *s, dtype=F32, f=1.0):
    return (f * torch.randn(s, generator=g, device="cuda")).to(dtype)


# ------------------------------------------------------------------ group norm
def _group_case(Bn, P, C, dt, pt=None, seed=0, affine="wb"):
    g = _gen(seed)
    x = (_randn(g, Bn, P, C) * (0.5 + torch.rand(C, generator=g, device="cuda")) + 0.5 * _randn(g, C) + 0.3 * _randn(g, Bn, 1, C)).to(dt)
    w = (1 + _randn(g, C, f=0.3)).to(pt or dt) if "w" in affine else None
    b = _randn(g, C, dtype=pt or dt, f=0.3) if "b" in affine else None
    return x, w, b, _randn(g, Bn, P, C, dtype=dt)


def _check_group(x, groups, w, b, dy, act=None, eps=1e-5):
    y, mean, rstd = ops.group_norm_forward(x, groups, w, b, eps, activation=act)
    dx, dw, db = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation=act)
    Bn, C = x.shape[0], x.shape[-1]
    ref = R.group_norm(x.reshape(Bn, -1, C), groups, w, b, eps, act, dy.reshape(Bn, -1, C))
    for name, got in (("y", y.reshape(Bn, -1, C)), ("dx", dx.reshape(Bn, -1, C)), ("dw", dw), ("db", db)):
        check(got, *ref[name], f"{name} of {tuple(x.shape)} {x.dtype} {act}")


# Pixels and channels about the block's 512 threads of 8 channels and its registers: one launch, several chunks,
# several slabs, groups that are no whole pieces.
@pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("Bn,P,C,G", [
    (1, 1, 8, 1), (2, 3, 5, 1), (1, 17, 7, 7), (3, 64, 320, 32), (2, 65, 320, 32), (1, 1024, 320, 32), (2, 1961, 330, 11),
    (1, 4096, 40, 8), (1, 5000, 12, 4), (2, 333, 1280, 32), (1, 97, 4096, 1), (1, 50, 6144, 2), (1, 33, 8200, 8200),
    (2, 129, 1001 * 3, 3), (1, 70001, 6, 2), (40, 9, 640, 32), (1, 16384, 96, 3), (3, 257, 4104, 27), (1, 600, 24, 24)])
def test_group_norm(Bn, P, C, G, dt):
    _check_group(*_group_args(Bn, P, C, G, dt))


def _group_args(Bn, P, C, G, dt, **kw):
    x, w, b, dy = _group_case(Bn, P, C, dt, **kw)
    return x, G, w, b, dy


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("Bn,P,C,G", [(2, 64, 320, 32), (2, 2000, 330, 11), (1, 4096, 40, 5)])
def test_group_norm_with_an_activation(Bn, P, C, G, dt, act):
    _check_group(*_group_args(Bn, P, C, G, dt), act)


@pytest.mark.parametrize("affine", ["", "w", "b", "wb"])
@pytest.mark.parametrize("P", [30, 3000])
@pytest.mark.parametrize("dt", **TYPES)
def test_group_norm_parameters_in_32_bits(P, dt, affine):
    _check_group(*_group_args(2, P, 48, 6, dt, pt=F32, affine=affine), "silu")


@pytest.mark.parametrize("P", [20, 2500])
def test_group_norm_strides_and_alignment(P):
    """Pixels apart, channels that start at any element, samples side by side, several pixel dimensions, a
    channels-last image tensor, a repeated sample."""
    x, w, b, dy = _group_case(3, P, 67, BF16)
    w, b = w[:60].contiguous(), b[:60].contiguous()
    _check_group(x[..., 1:61], 5, w, b, dy[..., 3:63], "silu")
    _check_group(x[..., :60].transpose(0, 1).contiguous().transpose(0, 1), 5, w, b, dy[..., :60], "silu")
    _check_group(x[..., :60].reshape(3, P // 5, 5, 60), 5, w, b, dy[..., :60].reshape(3, P // 5, 5, 60))
    image = x[..., :60].reshape(3, P // 5, 5, 60).permute(0, 3, 1, 2).contiguous(memory_format=torch.channels_last)
    _check_group(image.permute(0, 2, 3, 1), 5, w, b, dy[..., :60].reshape(3, P // 5, 5, 60))
    _check_group(x[:1, :, :60].expand(3, P, 60), 5, w, b, dy[..., :60])
    _check_group(x[:, :1, :60].expand(3, P, 60), 5, w, b, dy[..., :60])


@pytest.mark.parametrize("P", [100, 5000])
def test_group_norm_offset_far_beyond_its_spread(P):
    """A mean of 1000 times the deviation: squares are taken of differences."""
    x, w, b, dy = _group_case(2, P, 64, F32)
    _check_group(x * 1e-2 + 10.0, 4, w, b, dy)


@pytest.mark.parametrize("P", [50, 4000])
def test_group_norm_not_a_number_stays_in_its_group(P):
    x, w, b, dy = _group_case(2, P, 64, BF16)
    x[1, P // 2, 20] = math.nan
    y, mean, rstd = ops.group_norm_forward(x, 4, w, b, activation="silu")
    dx, dw, _ = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu")
    want = torch.zeros(2, P, 64, dtype=torch.bool, device="cuda")
    want[1, :, 16:32] = True
    assert torch.equal(torch.isnan(y), want) and torch.equal(torch.isnan(dx), want)
    assert torch.equal(torch.isnan(dw), want[1, 0])


# Slabs enough for a block on most CUs, pixels about what a block's registers hold (8, 14, 21 in fp32 and 42 for each of 128
# threads, 102 of them for 80 channels in slabs of 40), and about two blocks a CU.
@pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("Bn,P,C,G", [
    (3, 1024, 96, 3), (3, 1025, 96, 3), (2, 1792, 64, 4), (180, 1793, 32, 4), (180, 2100, 32, 1), (180, 2689, 32, 8), (172, 5376, 32, 4),
    (172, 5377, 32, 4), (90, 4000, 80, 8), (170, 4284, 40, 4), (350, 2500, 32, 2)])
def test_group_norm_of_many_slabs(Bn, P, C, G, dt):
    x, w, b, dy = _group_case(Bn, P, C, dt)
    _check_group(x, G, w, b, dy, "silu")
    y, mean, rstd = ops.group_norm_forward(x, G, w, b, activation="silu")
    bad = x.clone()
    bad[1, P - 1, C // 2] = math.inf
    z, _, r = ops.group_norm_forward(bad, G, w, b, activation="silu")
    width = C // G
    at = C // 2 // width
    z[1, :, at * width:(at + 1) * width] = y[1, :, at * width:(at + 1) * width]      # the group that has no mean
    r[1, at] = rstd[1, at]
    assert torch.equal(z, y) and torch.equal(r, rstd)
    assert torch.equal(ops.group_norm_forward(x.transpose(0, 1).contiguous().transpose(0, 1), G, w, b, activation="silu")[0], y)


def test_group_norm_constant_groups_and_nothing():
    x = torch.full((2, 30, 24), 2.5, device="cuda")
    y, mean, rstd = ops.group_norm_forward(x, 3)
    assert not y.any() and torch.equal(mean, torch.full((2, 3), 2.5, device="cuda"))
    for shape in ((0, 30, 24), (2, 0, 24)):
        e = torch.empty(shape, device="cuda")
        y, mean, rstd = ops.group_norm_forward(e, 3)
        assert y.shape == shape and mean.shape == (shape[0], 3)
        dx, dw, db = ops.group_norm_backward(e, e, mean, rstd)
        assert dx.shape == shape and dw.shape == (24,) and not dw.any() and not db.any()


@pytest.mark.parametrize("Bn,P", [(2, 60), (2, 1500), (2, 3000), (64, 3000)])
def test_group_norm_in_place(Bn, P):
    """y may be x and dx may be dy (C ABI); gradients one at a time give the same."""
    import ctypes as C
    x, w, b, dy = _group_case(Bn, P, 96, BF16)
    y, mean, rstd = ops.group_norm_forward(x, 4, w, b, activation="gelu")
    want = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="gelu")
    lib, st = ops._library(), torch.cuda.current_stream().cuda_stream
    s = (P * 96, 96)
    p = ops.GroupNorm(Bn, P, 96, 4, ops.PA_BF16, ops.PA_BF16, ops.PA_ACT_GELU, 0, 1e-5, s, s, s)
    n = C.c_size_t(0)
    B._check(lib.paraanya_group_norm_backward_workspace(C.byref(p), C.byref(n)))
    ws = torch.empty(n.value + (1 << 22), dtype=torch.uint8, device="cuda")
    x2, d2 = x.clone(), dy.clone()
    B._check(lib.paraanya_group_norm(C.byref(p), x2.data_ptr(), w.data_ptr(), b.data_ptr(), x2.data_ptr(), None, None, ws.data_ptr(),
                                     ws.numel(), st))
    assert torch.equal(x2, y)
    only = torch.empty_like(w)
    args = (x.data_ptr(), w.data_ptr(), b.data_ptr(), mean.data_ptr(), rstd.data_ptr())
    B._check(lib.paraanya_group_norm_backward(C.byref(p), d2.data_ptr(), *args, None, only.data_ptr(), None, ws.data_ptr(), ws.numel(), st))
    assert torch.equal(only, want[1])
    B._check(lib.paraanya_group_norm_backward(C.byref(p), d2.data_ptr(), *args, None, None, only.data_ptr(), ws.data_ptr(), ws.numel(), st))
    assert torch.equal(only, want[2])
    B._check(lib.paraanya_group_norm_backward(C.byref(p), d2.data_ptr(), *args, d2.data_ptr(), None, None, ws.data_ptr(), ws.numel(), st))
    assert torch.equal(d2, want[0])


def _slopes(f, args, grads, h, dirs):
    """Central differences of the scalar f along a random direction of each argument against its gradient."""
    for i, (name, grad) in enumerate(grads):
        e = dirs[i]
        up, dn = list(args), list(args)
        up[i], dn[i] = args[i] + h * e, args[i] - h * e
        yield name, float((f(up) - f(dn)) / (2 * h)), float((grad.double() * e.double()).sum())


@pytest.mark.parametrize("act", [None, "silu", "gelu"])
def test_group_norm_gradient_against_differences(act):
    """In fp32, step 1e-2: the difference's error is h^2 times a third derivative, and the outputs' rounding
    over h; sums of 4000 products of size 1 take 3e-3 of their size with room."""
    x, w, b, dy = _group_case(2, 100, 20, F32, seed=5)
    xs = x.clone().requires_grad_(), w.clone().requires_grad_(), b.clone().requires_grad_()
    ops.group_norm(xs[0], 4, xs[1], xs[2], activation=act).backward(dy)

    def f(a):
        return (ops.group_norm_forward(a[0], 4, a[1], a[2], activation=act)[0].double() * dy.double()).sum()

    g = _gen(9)
    for name, got, want in _slopes(f, [x, w, b], [(n, t.grad) for n, t in zip(("x", "w", "b"), xs)], 1e-2, [_randn(g, *t.shape) for t in xs]):
        assert abs(got - want) <= 3e-3 * (abs(want) + math.sqrt(dy.numel())), (name, got, want)


# ------------------------------------------------------------------ feed-forward block
def _feed_case(M, K, H, N, dt, bias=True, seed=0, f=1.0):
    g = _gen(seed)
    x = _randn(g, M, K, dtype=dt)
    gate, up = (_randn(g, H, K, dtype=dt, f=1 / math.sqrt(K)) for _ in range(2))
    down = _randn(g, N, H, dtype=dt, f=1 / math.sqrt(H))
    biases = tuple(_randn(g, n, dtype=dt, f=0.2) if bias else None for n in (H, H, N))
    return x, gate, up, down, biases, _randn(g, M, N, dtype=dt, f=f)


def _check_feed(x, gate, up, down, biases, dy, act="silu"):
    y, saved = ops.feed_forward_forward(x, gate, up, down, *biases, activation=act)
    plain, none = ops.feed_forward_forward(x, gate, up, down, *biases, activation=act, save=False)
    assert none is None and torch.equal(plain, y)
    grads = ops.feed_forward_backward(dy, x, gate, up, down, saved, activation=act)
    K, N = x.shape[-1], down.shape[0]
    ref = R.feed_forward(x.reshape(-1, K), gate, up, down, biases, act, dy.reshape(-1, N))
    for name, got in (("y", y.reshape(-1, N)), *grads._asdict().items()):
        what = f"{name} of {tuple(x.shape)} H {gate.shape[0]} N {N} {x.dtype} {act}"
        check(got.reshape(ref[name][0].shape), *ref[name], what)
        # At most four roundings on the way to a result, each of an independent sign: their share is at most as
        # many units of it, also where a row's bound is loose. A result below the type's normal numbers is off by up to
        # half of their least spacing: n of them by sqrt(n) times that in the norm.
        want = ref[name][0]
        if want.numel() > 1000:
            off = float((got.reshape(want.shape).double() - want).norm())
            assert off < 4 * U[x.dtype] * float(want.norm()) + TINY[x.dtype] * math.sqrt(want.numel()), what


# Rows about the few-row kernels' 16, 32 and 64 and the tiles' sizes; widths about a part of the reduction (64), pieces of
# 8, and shorter than a piece.
@pytest.mark.parametrize("dt", **TYPES)
@pytest.mark.parametrize("M,K,H,N", [
    (1, 64, 128, 64), (1, 1, 1, 1), (2, 3, 5, 7), (5, 8, 8, 8), (16, 72, 100, 33), (17, 129, 65, 40), (33, 1024, 256, 96), (64, 200, 264, 136),
    (65, 64, 64, 64), (65, 7, 3, 2), (100, 72, 136, 200), (129, 131, 67, 77), (257, 320, 264, 129), (300, 1100, 683, 514),
    (1000, 264, 1000, 264), (70, 2056, 72, 8), (66, 8, 2056, 16)])
def test_feed_forward(M, K, H, N, dt):
    _check_feed(*_feed_case(M, K, H, N, dt))


# Enough tiles of each size that the larger ones are taken.
@pytest.mark.parametrize("M,K,H,N", [(2048, 136, 2048, 2048), (4096, 72, 4104, 520), (4100, 64, 2060, 4100)])
def test_feed_forward_of_many_tiles(M, K, H, N):
    _check_feed(*_feed_case(M, K, H, N, BF16))


@pytest.mark.parametrize("act", [None, "gelu"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("dt", **TYPES)
def test_feed_forward_activations_and_biases(M, dt, bias, act):
    _check_feed(*_feed_case(M, 96, 200, 72, dt, bias), act)


@pytest.mark.parametrize("M", [9, 300])
def test_feed_forward_strides_and_alignment(M):
    """Rows apart, at any element, several leading dimensions, weights of different strides, transposed weights."""
    x, gate, up, down, biases, dy = _feed_case(M, 80, 120, 64, BF16)

    def apart(t, at, extra):
        wide = torch.full((t.shape[0], t.shape[1] + extra), math.nan, dtype=t.dtype, device="cuda")
        wide[:, at:at + t.shape[1]] = t
        return wide[:, at:at + t.shape[1]]

    _check_feed(apart(x, 1, 3), gate, up, down, biases, dy)
    _check_feed(x, apart(gate, 8, 16), apart(up, 8, 16), down, biases, apart(dy, 8, 8))
    _check_feed(x, apart(gate, 0, 8), up, apart(down, 3, 5), biases, apart(dy, 5, 6))
    _check_feed(x, gate.t().contiguous().t(), up, down.t().contiguous().t(), biases, dy)
    _check_feed(x.reshape(3, M // 3, 80), gate, up, down, biases, dy.reshape(3, M // 3, 64))
    _check_feed(x[:1].expand(M, 80), gate, up, down, biases, dy[:1].expand(M, 64))


@pytest.mark.parametrize("f", [1e-6, 1e-3, 1e3])
@pytest.mark.parametrize("M", [40, 200])
def test_feed_forward_in_fp16_keeps_small_and_large_gradients(M, f):
    """dy near fp16's least and largest numbers: intermediate gradients are scaled by its largest value."""
    _check_feed(*_feed_case(M, 64, 96, 64, F16, f=f))


@pytest.mark.parametrize("M", [20, 300])
def test_feed_forward_in_fp16_with_a_large_gain(M):
    """dz up to 2^17 times the largest dy: finite in fp16, and to be kept so by the scale."""
    x, gate, up, down, biases, dy = _feed_case(M, 64, 96, 1024, F16, f=2.0**-12)
    gate, up, down = (gate.float() / 64).half(), (up.float() * 1024).half(), (down.float() * 2 * math.sqrt(96)).half()
    ref = R.feed_forward(x, gate, up, down, biases, None, dy)
    assert float(ref["x"][0].abs().max()) < 65504
    _, saved = ops.feed_forward_forward(x, gate, up, down, *biases, activation=None)
    grads = ops.feed_forward_backward(dy, x, gate, up, down, saved, activation=None)
    for name in ("x", "gate", "up", "gate_bias", "up_bias"):
        got = getattr(grads, name)
        assert bool(torch.isfinite(got).all()) or not bool((ref[name][0].abs() < 65504).all()), name
        check(got, *ref[name], name)


def test_feed_forward_not_a_number_stays_in_its_row():
    for M in (20, 150):
        x, gate, up, down, biases, dy = _feed_case(M, 60, 90, 50, BF16)
        x[4, 13], x[7, 2] = math.nan, math.inf
        y, saved = ops.feed_forward_forward(x, gate, up, down, *biases)
        clean = torch.ones(M, dtype=torch.bool, device="cuda")
        clean[[4, 7]] = False
        assert bool(torch.isfinite(y[clean]).all()) and bool(torch.isnan(y[4]).all())
        g = ops.feed_forward_backward(dy, x, gate, up, down, saved)
        assert bool(torch.isfinite(g.x[clean]).all()) and not bool(torch.isfinite(g.x[4]).any())


def test_feed_forward_without_rows():
    x, gate, up, down, biases, dy = _feed_case(0, 64, 96, 40, BF16)
    y, saved = ops.feed_forward_forward(x, gate, up, down, *biases)
    assert y.shape == (0, 40)
    g = ops.feed_forward_backward(dy, x, gate, up, down, saved)
    assert g.x.shape == (0, 64) and all(not bool(t.any()) for t in g[1:])


def test_feed_forward_gradients_one_at_a_time():
    x, gate, up, down, biases, dy = _feed_case(150, 64, 96, 40, F16)
    y, saved = ops.feed_forward_forward(x, gate, up, down, *biases)
    every = ops.feed_forward_backward(dy, x, gate, up, down, saved)
    for i in range(7):
        got = ops.feed_forward_backward(dy, x, gate, up, down, saved, need=[k == i for k in range(7)])
        assert torch.equal(got[i], every[i]), ops.FeedGradients._fields[i]
        assert [k for k in range(7) if got[k] is not None] == sorted({i, i if i < 4 else i - 3})
    leaves = [t.clone().requires_grad_(i in (1, 6)) for i, t in enumerate((x, gate, up, down, *biases))]
    ops.feed_forward(*leaves).backward(dy)
    assert torch.equal(leaves[1].grad, every.gate) and torch.equal(leaves[6].grad, every.down_bias)
    assert all(t.grad is None for i, t in enumerate(leaves) if i not in (1, 6))
    with torch.no_grad():
        assert torch.equal(ops.feed_forward(x, gate, up, down, *biases), y)


def test_feed_forward_gradient_against_differences():
    """bf16 cannot be stepped finely: the 64-bit formulas' gradients, which the kernels are held to above, against
    differences of the 64-bit forward formula, relative to the step's third derivative (1e-4 squared)."""
    x, gate, up, down, biases, dy = (t if isinstance(t, tuple) else t.double() for t in _feed_case(6, 16, 24, 10, BF16))
    args = [x, gate, up, down, *(t.double() for t in biases)]
    ref = R_feed64(args, dy)

    def f(a):
        p, q = a[0] @ a[1].T + a[4], a[0] @ a[2].T + a[5]
        return ((torch.nn.functional.silu(p) * q @ a[3].T + a[6]) * dy).sum()

    g = _gen(11)
    for name, got, want in _slopes(f, args, ref, 1e-4, [_randn(g, *t.shape, dtype=torch.float64) for t in args]):
        assert abs(got - want) <= 1e-6 * (1 + abs(want)), (name, got, want)


def R_feed64(args, dy):
    low = [t.to(BF16) for t in args]           # drawn in bf16: exact
    ref = R.feed_forward(*low[:4], tuple(low[4:]), "silu", dy.to(BF16))
    return [(n, ref[n][0]) for n in ops.FeedGradients._fields]


# ------------------------------------------------------------------ 8-bit integers
@pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (5, 16), (4, 17), (9, 511), (3, 512), (2, 513), (7, 1024), (2, 1025), (5, 2048), (3, 2050),
                                 (2, 4097), (3, 8192), (2, 8200), (2, 20001), (600, 40)])
def test_quantize_rows(M, K, dt):
    g = _gen(K)
    x = (_randn(g, M, K) * torch.exp(_randn(g, K))).to(dt)
    q, scale = ops.quantize_rows(x)
    want, s = R.quantize_rows(x)
    assert torch.equal(scale, s) and torch.equal(q, want)
    assert q.stride(0) % 16 == 0
    wide = torch.as_strided(q, (M, q.stride(0)), (q.stride(0), 1))
    assert not bool(wide[:, K:].any())


def test_quantize_rows_special_rows():
    """Zeros, infinities, NaN, the type's least and largest numbers, ties; strides."""
    x = torch.zeros(8, 100, device="cuda")
    x[1, 3], x[2, 5], x[3, 7] = math.inf, math.nan, -math.inf
    x[4] = torch.finfo(F32).max
    x[5, 0], x[5, 1] = 1e-44, -1e-45
    x[6] = torch.arange(100, device="cuda") * 0.5
    x[6, 99] = 127.0
    x[7, 50] = torch.finfo(F32).tiny
    q, scale = ops.quantize_rows(x)
    want, s = R.quantize_rows(x)
    assert torch.equal(q, want) and torch.equal(torch.nan_to_num(scale, nan=-1.0), torch.nan_to_num(s, nan=-1.0))
    assert scale[0] == 0 and bool(torch.isnan(scale[1:4]).all()) and not bool(q[:4].any())
    w = torch.randint(-128, 128, (20, 100), dtype=torch.int8, device="cuda")
    y = ops.int8_linear(q, scale, w, torch.ones(20, device="cuda"))
    assert not bool(y[0].any()) and bool(torch.isnan(y[1:4]).all())
    g = _gen(4)
    wide = _randn(g, 6, 130, dtype=BF16)
    for t in (wide[:, 1:100], wide[:, ::2], wide.reshape(2, 3, 130), wide[:1].expand(6, 130)):
        q, scale = ops.quantize_rows(t)
        want, s = R.quantize_rows(t)
        assert q.shape == t.shape and scale.shape == t.shape[:-1] and torch.equal(q, want) and torch.equal(scale, s)
    assert ops.quantize_rows(wide[:0])[0].shape == (0, 130)


def _int8_case(M, K, N, dt, bias=True, seed=0):
    g = _gen(seed)
    q = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
    s, ws = (torch.rand(n, device="cuda", generator=g) / math.sqrt(K) / 50 for n in (M, N))
    return q, s, w, ws, _randn(g, N, dtype=dt) if bias else None


@pytest.mark.parametrize("dt", **TYPES)
@pytest.mark.parametrize("M,K,N", [
    (1, 1, 1), (1, 1024, 96), (3, 15, 17), (16, 64, 33), (17, 100, 64), (33, 2049, 16), (64, 130, 130), (65, 128, 64), (66, 5, 3), (100, 129, 200),
    (129, 127, 65), (300, 1100, 683), (1000, 264, 2056), (2048, 272, 4104), (2100, 144, 8200)])
def test_int8_linear(M, K, N, dt):
    q, s, w, ws, bias = _int8_case(M, K, N, dt)
    for b in (bias, None):
        check(ops.int8_linear(q, s, w, ws, b, dtype=dt), *R.int8_linear(q, s, w, ws, b, dt), f"y of {M}x{K}x{N} {dt}")


def test_int8_linear_largest_sums():
    """The longest reduction of the largest products stays within 32 bits."""
    K = ops.PA_INT8_MAX_IN
    q = torch.full((3, K), -128, dtype=torch.int8, device="cuda")
    q[1] = 127
    w = torch.full((2, K), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(3, device="cuda")
    for M in (3, 70):
        big = q[torch.arange(M, device="cuda") % 3]
        y = ops.int8_linear(big, torch.ones(M, device="cuda"), w, one[:2], dtype=BF16)
        check(y, *R.int8_linear(big, torch.ones(M, device="cuda"), w, one[:2], None, BF16), "y")


@pytest.mark.parametrize("M", [20, 200])
def test_int8_linear_strides_and_what_lies_past_a_row(M):
    """Views of wider matrices: what follows a row has no effect; rows at odd addresses are copied."""
    q, s, w, ws, bias = _int8_case(M, 200, 70, F16)
    for at, K in ((0, 200), (16, 100), (32, 161), (1, 150), (0, 7), (0, 16)):
        a, b = q[:, at:at + K], w[:, at:at + K]
        check(ops.int8_linear(a, s, b, ws, bias, dtype=F16), *R.int8_linear(a, s, b, ws, bias, F16), f"y at {at} of {K}")
    y = ops.int8_linear(q.reshape(4, M // 4, 200), s.reshape(4, M // 4), w, ws, bias, dtype=F16)
    assert torch.equal(y.reshape(M, 70), ops.int8_linear(q, s, w, ws, bias, dtype=F16))
    assert ops.int8_linear(q[:0], s[:0], w, ws, bias, dtype=F16).shape == (0, 70)


# ------------------------------------------------------------------ streams, graphs, repetition
def _calls():
    """Every entry point at a few-row or one-launch size and at a larger one: (name, inputs, call)."""
    out = []
    for P in (64, 3000):
        x, w, b, dy = _group_case(2, P, 96, BF16, seed=P)

        def group(x, dy, w=w, b=b):
            y, mean, rstd = ops.group_norm_forward(x, 4, w, b, activation="silu")
            return (y, *ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu"))

        out.append((f"group norm {P}", (x, dy), group))
    for M, dt in ((8, BF16), (200, F16), (3000, BF16)):
        x, gate, up, down, biases, dy = _feed_case(M, 200, 520, 136, dt, seed=M)

        def feed(x, dy, gate=gate, up=up, down=down, biases=biases):
            y, saved = ops.feed_forward_forward(x, gate, up, down, *biases)
            return (y, *ops.feed_forward_backward(dy, x, gate, up, down, saved))

        out.append((f"feed forward {M}", (x, dy), feed))
        wq, ws = ops.quantize_rows(gate)

        def int8(x, dy, wq=wq, ws=ws, dt=dt):
            q, s = ops.quantize_rows(x)
            return ops.int8_linear(q, s, wq, ws, dtype=dt), q, s

        out.append((f"int8 {M}", (x, dy), int8))
    return out


def test_repeated_calls_and_other_streams_give_the_same_bits():
    for name, args, call in _calls():
        want = call(*args)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = [call(*args) for _ in range(2)]
        torch.cuda.current_stream().wait_stream(side)
        for r in (*got, call(*args)):
            assert all(torch.equal(a, b) for a, b in zip(r, want)), name


def test_captured_calls_replay_on_new_inputs():
    for name, args, call in _calls():
        held = [t.clone() for t in args]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(*held)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call(*held)
        for k in range(3):
            for h, t in zip(held, args):
                h.copy_(t.roll(k, 0))
            graph.replay()
            want = call(*held)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, k)


def test_captured_training_steps_replay_on_new_inputs():
    """Forward and backward through autograd in one graph (of leaves that no eager graph holds), replayed among eager steps."""
    x, w, b, dy = _group_case(2, 700, 96, BF16)
    _, gate, up, down, biases, _ = _feed_case(1, 96, 200, 96, BF16)

    def step(x, dy):
        leaves = [t.detach().requires_grad_() for t in (x, w, b, gate, up, down, *biases)]
        y = ops.feed_forward(ops.group_norm(leaves[0], 4, *leaves[1:3], activation="silu"), *leaves[3:])
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, dy)
    for k in range(3):
        x.copy_(x.roll(1, 1)), dy.copy_(dy.roll(k, 1))
        graph.replay()
        want = step(x, dy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


# ------------------------------------------------------------------ more than 2^31 elements or bytes
def test_group_norm_offsets_beyond_31_bits():
    g = _gen(1)
    w, b = _randn(g, 320, dtype=BF16), _randn(g, 320, dtype=BF16)
    x = torch.zeros(2250, 3000, 320, dtype=BF16, device="cuda")          # long samples: 2.2e9 elements
    dy = torch.zeros_like(x)
    x[-1], dy[-1] = _randn(g, 3000, 320, dtype=BF16), _randn(g, 3000, 320, dtype=BF16)
    y, mean, rstd = ops.group_norm_forward(x, 32, w, b, activation="silu")
    got = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu")
    ref = R.group_norm(x[-1:], 32, w, b, 1e-5, "silu", dy[-1:])
    for name, t in (("y", y[-1:]), ("dx", got[0][-1:]), ("dw", got[1]), ("db", got[2])):
        check(t, *ref[name], name)
    flat = x.view(-1)
    far = flat.as_strided((1, 64, 320), (0, 34_200_000, 1))
    far.copy_(_randn(g, 1, 64, 320))
    check(ops.group_norm_forward(far, 32, w, b)[0], *R.group_norm(far, 32, w, b, 1e-5, None)["y"], "pixels far apart")


def test_feed_forward_offsets_beyond_31_bits():
    """2.3e9 elements in each intermediate; only the last rows have gradients, so that the weights' are theirs."""
    x, gate, up, down, biases, _ = _feed_case(140_000, 32, 16384, 24, BF16)
    dy = torch.zeros(140_000, 24, dtype=BF16, device="cuda")
    dy[-50:] = _randn(_gen(3), 50, 24, dtype=BF16)
    y, saved = ops.feed_forward_forward(x, gate, up, down, *biases)
    grads = ops.feed_forward_backward(dy, x, gate, up, down, saved)
    ref = R.feed_forward(x[-50:], gate, up, down, biases, "silu", dy[-50:])
    check(y[-50:], *ref["y"], "y")
    check(grads.x[-50:], *ref["x"], "x")
    assert not bool(grads.x[:-50].any())
    for name in ops.FeedGradients._fields[1:]:
        check(getattr(grads, name), *ref[name], name)


def test_8_bit_offsets_beyond_31_bits():
    g = _gen(5)
    x = torch.zeros(70_000, 32768, dtype=BF16, device="cuda")
    x[-40:] = _randn(g, 40, 32768)
    q, scale = ops.quantize_rows(x)
    want, s = R.quantize_rows(x[-40:])
    assert torch.equal(q[-40:], want) and torch.equal(scale[-40:], s)
    del x
    wq, ws = ops.quantize_rows(_randn(g, 24, 32768))
    check(ops.int8_linear(q, scale, wq, ws)[-40:], *R.int8_linear(q[-40:], scale[-40:], wq, ws, None, BF16), "reading far rows")
    q, s, w, ws, bias = _int8_case(70_000, 24, 32768, BF16)
    check(ops.int8_linear(q, s, w, ws, bias)[-40:], *R.int8_linear(q[-40:], s[-40:], w, ws, bias, BF16), "writing far rows")


def test_a_gradients_gradient_is_refused():
    x, w, b, _ = _group_case(1, 20, 16, F32)
    x.requires_grad_()
    g, = torch.autograd.grad(ops.group_norm(x, 2, w, b).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()
    x, gate, up, down, biases, _ = _feed_case(4, 16, 24, 8, BF16)
    x.requires_grad_()
    g, = torch.autograd.grad(ops.feed_forward(x, gate, up, down, *biases).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()
