"""Group norm, the feed-forward block and the 8-bit projection on the device where a call is at the edge of what it takes:
the largest grids, values near the largest numbers, every tile."""
import pytest
import torch

import block_ops_reference as R
import feed_reference as F
from ops_reference import TINY, U, check
from paper_2609_36522_amd import ops
from tile_shapes import FEED_TILES, INT8_TILES

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(autouse=True)
def _lib(gpu_lib):
    return gpu_lib


def _randn(g, *s, dtype=F32):
    return torch.randn(s, generator=g, device="cuda", dtype=dtype)


# ------------------------------------------------------------------ group norm
def test_group_norm_in_ranges_of_samples():
    """8200 samples of 65536 groups: more than 2^20 blocks over the samples in every pass, 2^23 slabs and more, so that each
    pass takes several launches. Both ends of both ranges' samples, and the parameters' gradients over all of them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    Bn, P, C = 8200, 2, 65536
    x, dy = _randn(g, Bn, P, C, dtype=BF16), _randn(g, Bn, P, C, dtype=BF16)
    w, b = _randn(g, C, dtype=BF16), _randn(g, C, dtype=BF16)
    y, mean, rstd = ops.group_norm_forward(x, C, w, b, activation="silu")
    dx, dw, db = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu")
    cols = torch.tensor([0, 1, 511, 512, 32767, 65024, 65535], device="cuda")
    at = {n: t[:, :, cols].contiguous() for n, t in (("x", x), ("y", y), ("dy", dy), ("dx", dx))}
    ref = R.group_norm(at["x"], len(cols), w[cols], b[cols], 1e-5, "silu", at["dy"])
    for name, got in (("y", at["y"]), ("dx", at["dx"]), ("dw", dw[cols]), ("db", db[cols])):
        check(got, *ref[name], name)
    some = [0, 1, 8190, 8191, 8192, 8199]
    ref = R.group_norm(x[some], C, w, b, 1e-5, "silu", dy[some])
    check(y[some], *ref["y"], "y of whole samples")
    check(dx[some], *ref["dx"], "dx of whole samples")


# Fewer pixels than lanes, as many as a block's registers hold (8 and 42 a thread), several chunks.
@pytest.mark.parametrize("Bn,P,C,G", [(2, 3, 64, 8), (1, 1, 24, 3), (2, 500, 64, 8), (180, 2689, 32, 8), (2, 4000, 64, 8), (3, 3000, 330, 33)])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_group_norm_of_values_whose_squares_overflow(Bn, P, C, G, dt):
    """A mean of 2^64 and more, whose square is no number in fp32: with no spread, and with one whose squares are."""
    g = torch.Generator(device="cuda").manual_seed(P)
    w, b = _randn(g, C, dtype=dt), _randn(g, C, dtype=dt)
    x = torch.full((Bn, P, C), 2.0**66, dtype=dt, device="cuda")
    y, mean, rstd = ops.group_norm_forward(x, G, w, b, activation="silu")
    assert bool((mean == 2.0**66).all())
    check(y, *R.group_norm(x, G, w, b, 1e-5, "silu")["y"], "y of a constant")
    if dt == BF16:
        # Two neighbours: 2^57 apart, at most 24000 squares of 2^112.
        x = 2.0**64 * (1 + torch.randint(0, 2, (Bn, P, C), generator=g, device="cuda") / 128)
    else:
        x = 2.0**66 * (1 + 1e-4 * _randn(g, Bn, P, C))
    x, dy = x.to(dt), _randn(g, Bn, P, C, dtype=dt)
    y, mean, rstd = ops.group_norm_forward(x, G, w, b, activation="silu")
    dx, dw, db = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu")
    ref = R.group_norm(x, G, w, b, 1e-5, "silu", dy)
    for name, got in (("y", y), ("dx", dx), ("dw", dw), ("db", db)):
        check(got, *ref[name], name)


def _activation_bounds(act, z, exact):
    """(value, derivative, bound of each before it is rounded to its type) for an activation of fp32 numbers z. The shares, in
    units u = 2^-24: an exponential unit's result is off by 2 u of itself, a reciprocal by 2 u, each product or sum by one."""
    u, a, z = 2.0**-24, z.double().abs(), z.double()
    if act == "silu":
        # 2^(-z log2 e): the constant and the product are rounded, |z| u each in the exponential; of p that is its share 1 - p.
        p, r = torch.sigmoid(z), torch.sigmoid(-z)
        ep = p * u * (2 * a * r + 2 * r + 4)
        v, d = z * p, p + z * p * r
        # v (1 - p) + p: 1 - p is off by ep and a rounding.
        return v, d, a * ep + u * v.abs() + 2.0**-120, ep + a * r * (ep + u * p) + a * p * (ep + u * r) + u * (p + d.abs()) + 2.0**-120
    # (torch.special.ndtr loses its digits in the tail.)
    upper, lower = (torch.special.erfc(t / 2**0.5) / 2 for t in (a, -z))
    phi = torch.exp(-z * z / 2) / (2 * torch.pi)**0.5
    v, d = z * lower, lower + z * phi
    # The density: 0.72 z^2 from two products and a rounded constant, 0.72 ln2 z^2 = z^2 / 2 u each, and 3 more products.
    ephi = phi * u * (3 + 1.5 * a * a)
    if not exact:
        return v, d, 1.5e-7 * a.clamp(min=1) + u * v.abs(), 4e-6 + a * ephi + 2 * u
    # 2 Q = 2^-P: steps of P's evaluation are rounded (sums of up to 8 times P) and its fit is within 20 u beyond 3; beyond 8 the
    # result is at most what it is there.
    eq = upper * u * (4 + 8 * -torch.log2(2 * upper) + 20 * (a > 3)) + 7e-16 * (a > 8)
    return v, d, a * eq + u * v.abs(), eq + a * ephi + u * (lower + d.abs())


@pytest.mark.parametrize("P", [1, 5000])
@pytest.mark.parametrize("dt", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_group_norm_activation_and_its_derivative(act, dt, P):
    """A weight of 0: y is the activation of the bias, and dbias, where dy is 1 in one pixel, its derivative. Parameters
    in fp32, so that the derivative is not rounded to x's type."""
    C = 65536 if P == 1 else 2048
    z = torch.linspace(-14, 14, C, device="cuda")
    z[: C // 4] = torch.linspace(-1, 1, C // 4, device="cuda") ** 5
    x = _randn(torch.Generator(device="cuda").manual_seed(1), 1, P, C, dtype=dt)
    dy = torch.zeros_like(x)
    dy[0, P // 2] = 1
    w = torch.zeros_like(z)
    y, mean, rstd = ops.group_norm_forward(x, 32, w, z, activation=act)
    _, _, db = ops.group_norm_backward(dy, x, mean, rstd, w, z, activation=act)
    v, d, ev, ed = _activation_bounds(act, z, dt == F32)
    for row in (0, P - 1):
        check(y[0, row], v, ev + (0 if dt == F32 else U[dt]) * v.abs() + TINY[dt], f"{act} in {dt}")
    check(db, d, ed, f"the derivative of {act} in {dt}")


@pytest.mark.parametrize("P", [60, 3000])
def test_group_norm_gradients_one_at_a_time(P):
    g = torch.Generator(device="cuda").manual_seed(P)
    x, dy, w, b = (_randn(g, *s, dtype=BF16) for s in ((2, P, 96), (2, P, 96), (96,), (96,)))
    _, mean, rstd = ops.group_norm_forward(x, 4, w, b, activation="silu")
    every = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu")
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, False, True), (False,) * 3):
        got = ops.group_norm_backward(dy, x, mean, rstd, w, b, activation="silu", need=need)
        assert all(a is None if not k else torch.equal(a, e) for a, e, k in zip(got, every, need)), need
    for i in range(3):
        leaves = [t.clone().requires_grad_(k == i) for k, t in enumerate((x, w, b))]
        ops.group_norm(leaves[0], 4, *leaves[1:], activation="silu").backward(dy)
        assert torch.equal(leaves[i].grad, every[i]) and sum(t.grad is not None for t in leaves) == 1
    x.requires_grad_()
    y = ops.group_norm(x, 4, activation="silu")          # no parameters
    y.backward(dy)
    _, mean, rstd = ops.group_norm_forward(x.detach(), 4, activation="silu")
    assert torch.equal(x.grad, ops.group_norm_backward(dy, x.detach(), mean, rstd, activation="silu")[0])


# ------------------------------------------------------------------ feed-forward block
def _feed(M, K, H, N, dt, act, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, gate, up, down = (f * _randn(g, *s) for s, f in (((M, K), 1), ((H, K), K**-0.5), ((H, K), K**-0.5), ((N, H), H**-0.5)))
    biases = tuple((0.2 * _randn(g, n)).to(dt) for n in (H, H, N))
    args = tuple(t.to(dt) for t in (x, gate, up, down))
    dy = _randn(g, M, N).to(dt)
    y, saved = ops.feed_forward_forward(*args, *biases, activation=act)
    grads = ops.feed_forward_backward(dy, *args, saved, activation=act)
    ref = F.feed_forward(*args, biases, act, dy)
    for name, got in (("y", y), *grads._asdict().items()):
        what = f"{name} of {M}x{K}x{H}x{N} {dt} {act}"
        want, bound = ref.pop(name)
        check(got, want, bound, what)
        if want.numel() >= 1000:
            off, limit = float((got.double() - want).norm()), F.norm_limit(name, want, dt, M * H)
            assert off < limit, f"{what}: off by {off / float(want.norm()) / U[dt]:.3f} roundings' size, of {limit / float(want.norm()) / U[dt]:.3f}"


@pytest.mark.parametrize("M,K,H,N", FEED_TILES)
@pytest.mark.parametrize("dt", [BF16, F16], ids=["bf16", "f16"])
def test_feed_forward_of_every_tile(M, K, H, N, dt):
    _feed(M, K, H, N, dt, "silu" if M % 2 else "gelu", seed=M)


# The few-row kernels; sizes in whole pieces, which are read in place.
@pytest.mark.parametrize("M,K,H,N", [(1, 1000, 3000, 1500), (17, 264, 2048, 1032), (32, 77, 999, 333), (40, 1024, 2048, 512), (2048, 1024, 2048, 1024),
                                     (1500, 264, 1000, 520)])
@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("dt", [BF16, F16], ids=["bf16", "f16"])
def test_feed_forward_roundings(M, K, H, N, dt, act):
    _feed(M, K, H, N, dt, act, seed=M + K)


@pytest.mark.parametrize("M", [20, 300])
def test_feed_forward_in_fp16_with_projections_beyond_its_range(M):
    """u about 2^17, g about 2^-8: h is a number in fp16, u is not, and dz 2^17 times dy is by its scale. Rows without a
    gradient stay so."""
    g = torch.Generator(device="cuda").manual_seed(M)
    K, H, N = 64, 96, 48
    x, gate, up, down = (_randn(g, *s) * f for s, f in (((M, K), 4), ((H, K), 2.0**-13), ((H, K), 4096), ((N, H), 0.07)))
    args = tuple(t.half() for t in (x, gate, up, down))
    dy = (_randn(g, M, N) * 2.0**-10).half()
    dy[3] = 0
    assert float((args[0].double() @ args[2].double().T).abs().median()) > 65504
    y, saved = ops.feed_forward_forward(*args, activation=None)
    grads = ops.feed_forward_backward(dy, *args, saved, activation=None)
    ref = F.feed_forward(*args, (None,) * 3, None, dy)
    assert all(bool((ref[n][0].abs() < 65504).all()) for n in ("y", "x", "gate", "up", "down"))
    for name, got in (("y", y), *grads._asdict().items()):
        check(got, *ref[name], name)
    assert not bool(grads.x[3].any())


# ------------------------------------------------------------------ 8-bit integers
@pytest.mark.parametrize("M,K,N", INT8_TILES + [(16, 500, 4111), (17, 500, 4111), (50, 1100, 5000), (64, 129, 4096)])
@pytest.mark.parametrize("dt", [BF16, F16], ids=["bf16", "f16"])
def test_int8_linear_of_every_tile(M, K, N, dt):
    g = torch.Generator(device="cuda").manual_seed(M)
    q, w = (torch.randint(-128, 128, s, dtype=torch.int8, device="cuda", generator=g) for s in ((M, K), (N, K)))
    s, ws = (torch.rand(n, device="cuda", generator=g) / K**0.5 / 50 for n in (M, N))
    bias = _randn(g, N).to(dt)
    check(ops.int8_linear(q, s, w, ws, bias, dtype=dt), *R.int8_linear(q, s, w, ws, bias, dt), f"y of {M}x{K}x{N} {dt}")
