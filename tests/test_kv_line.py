"""The line of key tiles that the attention kernels cut into pieces, compiled for the host (kv_line_host.cpp): the arrival
counters of cut units come back to zero whichever CTAs give up on the way, so a call behind one that timed out joins nothing early."""
import os
import random
import shutil
import subprocess

import pytest

from paper_2605_18817_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def line(tmp_path_factory):
    nvcc = shutil.which(build._nvcc()) or "/usr/local/cuda/bin/nvcc"
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    exe = str(tmp_path_factory.mktemp("line") / "line")
    subprocess.run(["g++", "-w", "-std=c++17", "-O1", "-I", cuda, "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "kv_line_host.cpp"),
                    "-o", exe], check=True)
    return exe


# rows and keys of a tile, lead: the few-row kernel, the 128-row ones, the one on warp-level products
@pytest.mark.parametrize("rows,tile,lead", [(16, 128, 2), (128, 128, 3), (256, 128, 4), (16, 64, 0)])
def test_counters_are_zero_behind_a_call_that_gave_up(line, rows, tile, lead):
    rng = random.Random(rows + tile)
    text = []
    for i in range(200):
        n = rng.choice([1, 1, 2, 5, 30])
        heads, g = rng.choice([(1, 1), (2, 4), (8, 4), (5, 3), (1, 20)])
        window = rng.choice([0, 0, 1, 100, 1500])
        lens = " ".join("%d %d" % (rng.choice([0, 3, 127, 128, rng.randrange(5000)]), rng.choice([0, 1, 4, rng.randrange(400)])) for _ in range(n))
        text.append("%d %d %d %d %d %d %d %d %d %d %d %s" % (rows, tile, heads, g, rng.randrange(3), window, rng.choice([0, 4, 300]), lead,
                                                               rng.choice([148, 148, 132, 296]), i, n, lens))
    out = subprocess.run([line], input="\n".join(text), capture_output=True, text=True, check=True, timeout=300).stdout.splitlines()
    assert len(out) == len(text)
    cut = 0
    for case, got in zip(text, out):
        w = got.split()
        assert w[3] == "0" and w[5] == "0", (case, got)
        cut += int(w[1])
    assert cut > 1000
