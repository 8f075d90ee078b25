"""The 4-bit layer's rules (csrc/w4_plan.h), compiled for the host alone: the arg-max's workspace against what its kernels leave there."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2011_09208_amd import buildlib

SHIM = """#include "%s"
using namespace ws;
extern "C" {
int parts_(int B, int D, int C) { return w4_parts(w4_plan(B, D, C, true), B); }
int way_(int B, int D, int C) { return w4_plan(B, D, C, true).way; }
int groups_(int B, int D, int C) { return w4_plan(B, D, C, true).groups; }
}
"""
MAX_ROWS, MAX_CLASSES = 1 << 20, (1 << 30) - 65536


@pytest.fixture(scope="module")
def ws():
    if buildlib.is_stale():
        buildlib.build()
    from paper_2011_09208_amd import binding
    return binding


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    folder = str(tmp_path_factory.mktemp("w4_plan"))
    src, lib = os.path.join(folder, "rules.cpp"), os.path.join(folder, "rules.so")
    with open(src, "w") as f:
        f.write(SHIM % os.path.join(buildlib.PKG, "csrc", "w4_plan.h"))
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", src, "-o", lib], check=True)
    return ctypes.CDLL(lib)


def _drawn(n, seed):
    rng = random.Random(seed)
    for _ in range(n):
        B = int(MAX_ROWS ** rng.random()) if rng.random() < 0.5 else rng.randint(1, 300)
        C = int(MAX_CLASSES ** rng.random()) if rng.random() < 0.7 else 16 * rng.randint(1, 2100) + rng.choice((-1, 0, 1))
        yield B, 64 * int((1 << 21) ** rng.random()) if rng.random() < 0.3 else 64 * rng.randint(1, 260), C


def test_the_workspace_holds_every_candidate(rules, ws):
    ways = set()
    edges = [(B, D, C) for B in (1, 16, 17, 32, 33, 64, 65, 1 << 15, MAX_ROWS) for D in (64, 1024, 1088, 2048, 4096, 8192, 8256, 1 << 27)
             for C in (1, 16, 17, 16 * 256 + 1, 16 * 1024, 16 * 1024 + 1, 16 * 2048, 16 * 2048 + 1, 2 ** 20, MAX_CLASSES)]
    for B, D, C in [*edges, *_drawn(60000, 1)]:
        parts = rules.parts_(B, D, C)
        assert 1 <= parts <= rules.groups_(B, D, C)
        assert 8 * B * parts <= ws.w4_top1_workspace_bytes(B, C), (B, D, C)
        ways.add(rules.way_(B, D, C))
    assert ways == {0, 1, 2}


def test_the_workspace_is_no_more_than_some_call_of_this_size_writes(rules, ws):
    """Beyond the border where waves share a contraction, exactly what the largest number of candidates takes."""
    for B, _, C in _drawn(3000, 2):
        if ((C + 15) // 16) * ((B + 31) // 32) > 2048:
            most = max(rules.parts_(B, D, C) for D in (64, 128, 1024, 2048, 4096, 16384, 1 << 20))
            assert ws.w4_top1_workspace_bytes(B, C) == 8 * B * most, (B, C)


def test_many_rows_ask_for_little(ws):
    assert ws.w4_top1_workspace_bytes(8192, 100000) <= 26 << 20
    assert ws.w4_top1_workspace_bytes(MAX_ROWS, 100000) <= 1 << 28
    assert ws.w4_top1_workspace_bytes(1, 100000) <= 1 << 15
