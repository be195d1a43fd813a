"""CPU tests of batches with drafted trees at their edges: padding to a fixed size, sizes near what 32 bits count."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CLANGXX = os.environ.get("HOST_CLANGXX", "/opt/rocm/llvm/bin/clang++")


def _plain(tmp_path, name):
    """A program that needs the plan only."""
    exe = str(tmp_path / name)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "native", name + ".cpp"), "-o", exe])
    return exe


def test_padded_requests_leave_the_others_their_workgroups(tmp_path):
    r = subprocess.run([_plain(tmp_path, "padded_drafts")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "plans ok" in r.stdout, r.stdout + r.stderr


def _on_mock_hip(where, name):
    """A program that is built with the kernels' or the host side's source."""
    if not os.path.exists(CLANGXX):
        pytest.skip("no host clang++ for the kernel source")
    exe, mock = str(where / name), os.path.join(HERE, "native", "mockhip")
    subprocess.check_call([CLANGXX, "-std=c++17", "-O1", "-g", "-pthread", "-Wno-unused-function", "-Wno-keyword-macro", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", mock, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2510_02758_amd", "csrc"),
                           "-I", os.path.join(HERE, "native"), "-o", exe, os.path.join(HERE, "native", name + ".cpp"), os.path.join(mock, "mockhip.cpp")])
    return exe


@pytest.fixture(scope="module")
def edges(tmp_path_factory):
    return _on_mock_hip(tmp_path_factory.mktemp("edges"), "tree_edges_on_cpu")


@pytest.mark.parametrize("name", ["weights_of_rows_that_see_nothing", "paths_of_padded_trees"])
def test_kernels_at_their_edges(edges, name):
    r = subprocess.run([edges, name], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_stack_use_after_return=0"))
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_sizes_that_no_launch_could_have(tmp_path):
    r = subprocess.run([_on_mock_hip(tmp_path, "tree_sizes_on_mock_hip")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_lengths_near_what_32_bits_count(tmp_path):
    r = subprocess.run([_plain(tmp_path, "lengths_near_2g")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "lengths ok" in r.stdout, r.stdout + r.stderr


def test_prompts_beside_drafts_are_as_precise(tmp_path):
    r = subprocess.run([_plain(tmp_path, "prompts_beside_drafts")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "plans ok" in r.stdout, r.stdout + r.stderr
