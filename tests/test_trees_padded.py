"""CPU tests of batches with drafted trees at their edges: padding to a fixed size, sizes near what 32 bits count."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def _plain(tmp_path, name):
    """A program that needs the plan only."""
    exe = str(tmp_path / name)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "native", name + ".cpp"), "-o", exe])
    return exe


def test_padded_requests_leave_the_others_their_workgroups(tmp_path):
    r = subprocess.run([_plain(tmp_path, "padded_drafts")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "plans ok" in r.stdout, r.stdout + r.stderr
