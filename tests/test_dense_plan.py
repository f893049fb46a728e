"""The launches that the dense operators' products are given, on the host (CPU only): the sizes of
tests/dense_tiles.py take the tiles that they are listed for, so that a change of the estimates
behind the choice cannot leave a kernel without its tests unseen."""
import os
import shutil
import subprocess

import pytest

from paper_2609_13846_amd import dtp
from tests.dense_tiles import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PER_CU = {256: 1, 128: 2, 64: 3}  # bf16 blocks of a compute unit


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ is not available")
    exe = tmp_path_factory.mktemp("plan") / "plan"
    build = subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                            "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2609_13846_amd", "csrc"),
                            os.path.join(ROOT, "tests", "host_plan", "driver.cpp"), "-o", str(exe)],
                           capture_output=True, text=True, timeout=300)
    assert build.returncode == 0, build.stderr[-4000:]

    def ask(lines, cus=256):
        """For each (kind, tokens, in, out, dtype, act): {product: {"m", "n", "splits", ..}}."""
        text = "\n".join(" ".join(map(str, line)) for line in lines) + "\n"
        run = subprocess.run([str(exe), str(cus)], input=text, capture_output=True, text=True, timeout=300)
        assert run.returncode == 0, run.stderr[-4000:]
        out = []
        for line in run.stdout.splitlines():
            f = line.split()
            out.append({f[i]: dict(zip(("m", "n", "splits", "stages", "per", "tiles", "threads"), map(int, f[i + 1:i + 8])))
                        for i in range(0, len(f), 8)})
        assert len(out) == len(lines)
        return out

    return ask


def test_sizes_take_the_tiles_that_they_are_listed_for(plans):
    got = plans([(kind, T, K, N, dtype, dtp.DTP_ACT_SILU if kind == "gated" else dtp.DTP_ACT_NONE)
                 for kind, dtype, T, K, N, _ in CASES])
    for (kind, dtype, T, K, N, want), g in zip(CASES, got):
        for name, (cols, parts, many) in want.items():
            p = g[name]
            case = (kind, dtype, T, K, N, name, p)
            assert p["n"] == cols and p["m"] == max(cols, 128), case
            assert (p["splits"] > 1) == (parts == "split"), case
            assert p["stages"] >= 3, case
            if many:
                assert p["tiles"] * p["splits"] > 256 * PER_CU[cols], case


def test_every_kernel_of_large_tiles_is_listed():
    """Kind, dtype, product, tile and splitting; for bf16 forward rows, whether they end inside a piece of eight."""
    def reached(kind, dtype, name, cols, parts, odd=None, many=""):
        return any(c[0] == kind and c[1] == dtype and c[5].get(name, (0, ""))[:2] == (cols, parts) and
                   many in c[5][name][2] and (odd is None or (c[4] % 8 != 0) == odd) for c in CASES)
    for kind in ("linear", "gated"):
        for dtype, cols in (("bf16", 256), ("f32", 128)):
            for name in ("forward", "dx", "dw"):
                for parts in ("whole", "split"):
                    assert reached(kind, dtype, name, cols, parts), (kind, dtype, name, parts)
        for cols in (64, 128, 256):
            for odd in (False, True):
                assert reached(kind, "bf16", "forward", cols, "whole", odd, "many"), (kind, cols, odd)
            for name in ("dx", "dw"):
                assert cols == 256 or reached(kind, "bf16", name, cols, "whole", many="many"), (kind, cols, name)


def test_splits_cover_the_contraction(plans):
    """Every split has stages, together they are all of them, and bf16 items have an even number."""
    lines = [(kind, T, K, N, dtype, 1) for kind in ("linear", "gated") for dtype in ("bf16", "f32")
             for T in (1, 8, 9, 16, 17, 100, 777, 4096, 30000) for K, N in ((1, 1), (40, 24), (1040, 2810), (14336, 4096), (7, 20000))]
    for line, got in zip(lines, plans(lines)):
        for name, p in got.items():
            assert (p["splits"] - 1) * p["per"] < p["stages"] <= p["splits"] * p["per"], (line, name, p)
            if p["m"] and line[4] == "bf16":
                assert p["per"] % 2 == 0 and p["stages"] % 2 == 0, (line, name, p)


def test_launches_have_fewer_than_2_to_the_32_threads(plans):
    """Of the longest and narrowest tensors that are taken, whose results still fit the GPU."""
    lines = [(kind, T, K, N, dtype, 1) for kind in ("linear", "gated") for dtype in ("bf16", "f32")
             for T in (1 << 28, (1 << 29) + 70, (1 << 30) - 1, 1 << 30) for K, N in ((1, 1), (1, 64), (1, 65), (65, 1), (1, 129))]
    for line, got in zip(lines, plans(lines)):
        for name, p in got.items():
            assert 0 < p["threads"] < 2 ** 32, (line, name, p)


def test_plans_follow_the_compute_units(plans):
    """A part of the GPU gets no more blocks than it holds at a time, and splits the contraction for no
    more than it has; what fills the whole GPU is split on neither."""
    few, some, many = ("linear", 16, 14336, 4096, "bf16", 0), ("linear", 400, 4096, 1024, "f32", 0), ("gated", 8192, 4096, 14336, "bf16", 1)
    whole, part = plans([few, some, many]), plans([few, some, many], 32)
    for w, p in zip(whole[:2], part):
        assert w["forward"]["splits"] > p["forward"]["splits"]
    for cus, g in ((256, whole[2]), (32, part[2])):
        assert g["forward"]["splits"] == 1 and g["forward"]["m"] == 256 and g["forward"]["threads"] == 512 * cus
