"""What the operators launch, recorded without a GPU (launch_record.py): grids within the limits of a launch at the largest
sizes that are accepted, and the tiles that the listed sizes of tile_shapes.py take."""
import math
import os

import pytest

import launch_record as L
from paper_2609_36522_amd import build as B
from paper_2609_36522_amd import ops as O
from tile_shapes import FEED_TILES, INT8_TILES


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    if not os.path.exists(B.LIB):             # built by __graft_entry__.build(); here only where nothing is
        B.build()
    return L.build(str(tmp_path_factory.mktemp("launches")))


# Samples x pixels x channels in groups of one, of a few and of many channels: more than 2^23 blocks over all samples
# in either pass, many chunks, one chunk.
SIZES = [(65535, 1, 65536, 65536), (32768, 2, 131072, 131072), (65535, 1, 1 << 20, 1 << 20), (65535, 1, 1 << 20, 1 << 18),
         (65535, 1, 4096, 32), (9, 1025, 1 << 20, 1 << 20), (65535, 16384, 320, 32), (1, 1 << 30, 8, 1), (3, 1 << 20, 4096, 1),
         (600, 5000, 1 << 20, 256), (8, 4096, 640, 32)]


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dtype", [O.PA_F32, O.PA_BF16])
def test_group_norm_grids(recorder, backward, dtype):
    calls = [f"group {backward} {' '.join(map(str, s))} {dtype} {O.PA_ACT_SILU}" for s in SIZES]
    for call, (status, launches) in zip(calls, L.record(recorder, calls)):
        assert status == 0 and launches, call
        blocks = {}
        for k in launches:
            # Fewer than 2^32 threads, along an axis and in all.
            assert math.prod(k.grid) * math.prod(k.block) < 1 << 32 and max(k.grid[1:]) < 1 << 16, (call, k)
            blocks[k.name] = blocks.get(k.name, 0) + math.prod(k.grid)
        batch, _, channels, groups = map(int, call.split()[2:6])
        # The launches of a kernel cover every sample alike (and those of the parameters' sums 512 of 2 x channels values a block).
        params = -(-2 * channels // 512)
        if backward and "k_group_params" not in blocks:
            blocks["k_group_dx"] -= params
        for name, n in blocks.items():
            assert n == params if name == "k_group_params" else n % batch == 0 and n > 0, (call, name, n)
        assert blocks.get("k_group_join", batch * groups) == batch * groups, call


def test_group_norm_backward_in_one_pass(recorder):
    """Up to 4 pixels a thread, or up to 8 where half of the CUs have a block (320 channels: 8 slabs of 102 lanes a sample)."""
    calls = [(1, 408, True), (1, 409, False), (15, 816, False), (16, 816, True), (16, 817, False), (400, 817, False), (400, 816, True)]
    for (batch, pixels, one), (status, launches) in zip(
            calls, L.record(recorder, [f"group 1 {b} {p} 320 32 {O.PA_BF16} {O.PA_ACT_SILU}" for b, p, _ in calls])):
        names = [k.name for k in launches]
        assert status == 0 and names == (["k_group_bwd_whole", "k_group_params"] if one else ["k_group_sums", "k_group_join", "k_group_dx"]), (batch, pixels)


# Matrices at the limits of elements (2^34), of tiles (2^23 of 64 x 64) and of a width (2^20).
FEED_SIZES = [(1 << 29, 1, 1, 1), (1 << 29, 32, 8, 32), (1 << 14, 1 << 20, 1 << 14, 1 << 14), (33, 1 << 14, 1 << 20, 1 << 14), (33, 1 << 20, 1 << 14, 1 << 20),
              (1 << 14, 8, 1 << 20, 3), ((1 << 14) + 1, 1 << 14, 1 << 20, 1 << 14), (1, 1 << 14, 1 << 20, 1 << 14), (1 << 19, 1 << 15, 1, 1 << 15)]


@pytest.mark.parametrize("dtype,alignment", [(O.PA_BF16, 16), (O.PA_F16, 2)])
def test_feed_forward_grids(recorder, dtype, alignment):
    calls = [f"feed {b} {' '.join(map(str, s))} {dtype} {O.PA_ACT_SILU} {alignment}" for s in FEED_SIZES for b in (0, 1)]
    for call, (status, launches) in zip(calls, L.record(recorder, calls)):
        rows, *widths = map(int, call.split()[2:6])
        assert status == 0 if rows * max(widths) <= 1 << 34 else (status == -6 and not launches), (call, status)
        for k in launches:
            assert math.prod(k.grid) * math.prod(k.block) < 1 << 32 and max(k.grid[1:]) < 1 << 16, (call, k)


def test_int8_linear_grids(recorder):
    sizes = [(1 << 29, 16, 64), (1 << 15, 131071, 1 << 20), (1 << 30, 1, 1), (65, 64, 1 << 20), (1, 64, 1 << 20)]
    calls = [f"int8 {' '.join(map(str, s))} {O.PA_F16}" for s in sizes]
    for call, (status, launches) in zip(calls, L.record(recorder, calls)):
        rows, _, out = map(int, call.split()[1:4])
        assert status == 0 if -(-rows // 64) * -(-out // 64) <= 1 << 23 else (status == -6 and not launches), (call, status)
        for k in launches:
            assert math.prod(k.grid) * math.prod(k.block) < 1 << 32 and max(k.grid[1:]) < 1 << 16, (call, k)


# ------------------------------------------------------------------ the tiles that tile_shapes.py is to take
# Waves over features and over rows, 32-wide tiles a wave of each, stages.
BIG, TALL, WIDE, MID, DEEP, SMALL = (2, 4, 4, 2, 2), (4, 2, 2, 2, 3), (2, 2, 2, 3, 2), (2, 2, 2, 2, 2), (2, 2, 2, 2, 3), (2, 2, 1, 1, 4)
GATED_SMALL = (1, 4, 2, 1, 3)


def _up(n, d):
    return -(-n // d)


def _taken(launches, joined, product, sizes, parts):
    """{(product, tile, split)} of a call's launch, if a range of its reduction has 2 x stages + 1 parts or more."""
    out = set()
    for k in launches:
        if k.name != product:
            continue
        features, rows = k.tile[0] * k.tile[2] * 32, k.tile[1] * k.tile[3] * 32
        if k.name == "k_feed_gate":
            features //= 2
        ranges, rest = divmod(k.grid[0], sum(_up(f, features) * _up(r, rows) for f, r in sizes))
        assert rest == 0 and (ranges > 1) == any(j.name == joined for j in launches), k
        if parts // ranges >= 2 * k.tile[4] + 1:
            out.add((product, k.tile, ranges > 1))
    return out


def test_listed_sizes_take_every_tile_of_the_feed_forward_block(recorder):
    for dtype in (O.PA_BF16, O.PA_F16):
        of_type = set()
        for M, K, H, N in FEED_TILES:
            (fs, forward), (bs, backward) = L.record(recorder, [f"feed {b} {M} {K} {H} {N} {dtype} {O.PA_ACT_SILU} 16" for b in (0, 1)])
            assert fs == 0 and bs == 0
            of_type |= _taken(forward, None, "k_feed_gate", [(H, M)], _up(K, 64))
            of_type |= {("y", *t[1:]) for t in _taken(forward, "k_feed_join", "k_feed_plain", [(N, M)], _up(H, 64))}
            of_type |= _taken(backward, None, "k_feed_grad", [(H, M)], _up(N, 64))
            of_type |= {("dx", *t[1:]) for t in _taken(backward, "k_feed_join", "k_feed_plain", [(K, M)], 2 * _up(H, 64))}
            of_type |= _taken(backward, "k_feed_weights_join", "k_feed_weights", [(K, H), (K, H), (H, N)], _up(M, 64))
        want = {("k_feed_gate", t, False) for t in (BIG, WIDE, MID, DEEP, GATED_SMALL)}
        want |= {("k_feed_grad", t, False) for t in (BIG, TALL, WIDE, MID, DEEP, SMALL)}
        want |= {(p, t, s) for p in ("y", "dx", "k_feed_weights") for t in (BIG, TALL, WIDE, MID, DEEP, SMALL) for s in (False, True)}
        assert of_type == want, (dtype, want - of_type, of_type - want)


def test_listed_sizes_take_every_tile_of_the_8_bit_projection(recorder):
    got = set()
    for M, K, N in INT8_TILES:
        (status, launches), = L.record(recorder, [f"int8 {M} {K} {N} {O.PA_BF16}"])
        assert status == 0
        got |= _taken(launches, None, "k_int8_tile", [(N, M)], _up(K, 128))
    assert got == {("k_int8_tile", t, False) for t in (BIG, TALL, WIDE, MID, DEEP, SMALL)}


def test_few_rows_of_the_8_bit_projection(recorder):
    """Straight from memory where a CU has one block of 16 features, up to 64 rows, and with 16 rows at any width."""
    calls = [(64, 4096, True), (65, 4096, False), (16, 4097, True), (17, 4097, False), (1, 1 << 20, True), (64, 1, True)]
    for (rows, out, few), (status, (k,)) in zip(calls, L.record(recorder, [f"int8 {m} 200 {n} {O.PA_F16}" for m, n, _ in calls])):
        assert status == 0 and k.name == ("k_int8_few" if few else "k_int8_tile"), (rows, out)
