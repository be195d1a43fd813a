"""CPU tests of the host side of the operators on the pool's contents: kvops.hip, unchanged, on the stand-in HIP runtime, with launches that
are recorded (tests/native/ops_on_mock_hip.cpp says what each check looks at)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CLANGXX = os.environ.get("HOST_CLANGXX", "/opt/rocm/llvm/bin/clang++")
CSRC = os.path.join(ROOT, "paper_2510_02758_amd", "csrc")
MOCK = os.path.join(HERE, "native", "mockhip")


@pytest.fixture(scope="module")
def ops(tmp_path_factory):
    if not os.path.exists(CLANGXX):
        pytest.skip("no host clang++ for the kernel source")
    exe = str(tmp_path_factory.mktemp("ops") / "ops_on_mock_hip")
    subprocess.check_call([CLANGXX, "-std=c++17", "-O1", "-g", "-pthread", "-Wno-unused-function", "-Wno-keyword-macro", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", MOCK, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", os.path.join(HERE, "native"),
                           "-o", exe, os.path.join(HERE, "native", "ops_on_mock_hip.cpp"), os.path.join(MOCK, "mockhip.cpp")])
    return exe


@pytest.mark.parametrize("name", ["replay_then_set", "captures_draw_no_tickets", "an_earlier_error", "launches_of_a_large_eviction", "room_is_grown_by_set", "far_positions", "set_that_fails",
                                  "captured_evictions_have_no_requests"])
def test_host_side(ops, name):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:detect_stack_use_after_return=0")
    r = subprocess.run([ops, name], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_which_evictions_reach_shared_blocks(tmp_path):
    exe = str(tmp_path / "rewrites_shared")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "native", "rewrites_shared.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "checks ok" in r.stdout, r.stdout + r.stderr
