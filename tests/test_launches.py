"""What the operators launch, recorded without a GPU (launch_record.py): grids within the limits of a launch at the largest
sizes that are accepted."""
import math
import os

import pytest

import launch_record as L
from paper_2609_36522_amd import build as B
from paper_2609_36522_amd import ops as O


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
