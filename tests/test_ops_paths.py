"""CPU test: the batches of ops_paths.py take the ways that they are there for."""
import os
import subprocess

import numpy as np
import pytest

from ops_paths import PATHS, tables

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan_paths(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "plan_paths")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(HERE, "native", "plan_paths.cpp"), "-o", exe])
    return exe


@pytest.mark.parametrize("name", list(PATHS))
def test_batches_take_their_ways(plan_paths, name):
    (H, D, B, dtype, scales), G, lens, q_lens, shared, want = PATHS[name]
    N = sum(-(-n // B) for n in lens) + 3
    rows = tables(np.random.default_rng(0), N, lens, B, shared)
    off = np.concatenate([[0], np.cumsum([len(r) for r in rows])])
    text = " ".join(str(int(x)) for x in [H, G, B, D, N, dtype == "fp8_e4m3", len(lens), *lens, *q_lens, *off, *np.concatenate(rows)])
    r = subprocess.run([plan_paths], input=text, capture_output=True, text=True, timeout=60)
    assert r.returncode == 0
    assert want <= set(r.stdout.split()), r.stdout
