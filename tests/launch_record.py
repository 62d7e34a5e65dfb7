"""The kernels that a call of an operator launches, recorded without a GPU (tests/launches/launches.cpp)."""
import os
import re
import subprocess
from typing import NamedTuple

from paper_2609_36522_amd import build as B

SRC = os.path.join(os.path.dirname(__file__), "launches", "launches.cpp")


class Launch(NamedTuple):
    name: str              # of the kernel, without its namespace and arguments
    tile: tuple            # waves over features and over rows, 32-wide tiles of each and stages of its Tile, if it has one
    mangled: str
    grid: tuple
    block: tuple


def build(folder):
    exe = os.path.join(folder, "launches")
    subprocess.run([B.hipcc(), "-O1", "-std=c++17", "-x", "c++", SRC, "-I", B.INCLUDE, "-rdynamic",
                    "-L", os.path.dirname(B.LIB), "-l:" + os.path.basename(B.LIB), f"-Wl,-rpath,{os.path.dirname(B.LIB)}", "-o", exe],
                   check=True, timeout=300)
    return exe


def _launch(line):
    mangled, *n = line.split()
    n = tuple(map(int, n))
    length, name = re.search(r"GLOBAL__N_1(\d+)(k_\w+)", mangled).groups()
    tile = re.search(r"4TileI[^L]*((?:Li\d+E){5})", mangled)
    return Launch(name[:int(length)], tuple(map(int, re.findall(r"\d+", tile.group(1)))) if tile else (), mangled, n[:3], n[3:])


def record(exe, calls):
    """(status, [Launch]) of each call, a line of the driver's input."""
    r = subprocess.run([exe], input="".join(c + "\n" for c in calls), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    out, launches = [], []
    for line in r.stdout.splitlines():
        if line.startswith("call "):
            out.append((int(line[5:]), launches))
            launches = []
        else:
            launches.append(_launch(line))
    assert len(out) == len(calls)
    return out
