"""CPU tests of drafted trees over the paged pool and of positions with several axes: the plan and the tree's kernels against plain loops, refusals, and what
accepted drafts do to the bookkeeping of host copies (plan-only handles make no HIP call)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import trees_ref as TR
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CLANGXX = os.environ.get("HOST_CLANGXX", "/opt/rocm/llvm/bin/clang++")
ONE = 16  # stands for a device pointer: a plan-only handle never follows it


def test_plan_and_kernels_against_plain_loops(tmp_path):
    if not os.path.exists(CLANGXX):
        pytest.skip("no host clang++ for the kernel source")
    exe = str(tmp_path / "trees_on_cpu")
    mock = os.path.join(HERE, "native", "mockhip")
    subprocess.check_call([CLANGXX, "-std=c++17", "-O1", "-g", "-pthread", "-Wno-unused-function", "-Wno-keyword-macro", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", mock, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2510_02758_amd", "csrc"),
                           "-I", os.path.join(HERE, "native"), "-o", exe, os.path.join(HERE, "native", "trees_on_cpu.cpp"), os.path.join(mock, "mockhip.cpp")])
    r = subprocess.run([exe, "300"], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_stack_use_after_return=0"))
    assert r.returncode == 0 and "trees ok" in r.stdout, r.stdout + r.stderr


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not os.path.exists(CLANGXX):
        pytest.skip("no host clang++ for the kernel source")
    exe, mock = str(tmp_path_factory.mktemp("trees") / "trees_host"), os.path.join(HERE, "native", "mockhip")
    subprocess.check_call([CLANGXX, "-std=c++17", "-O1", "-g", "-pthread", "-Wno-unused-function", "-Wno-keyword-macro", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", mock, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2510_02758_amd", "csrc"),
                           "-I", os.path.join(HERE, "native"), "-o", exe, os.path.join(HERE, "native", "trees_host_on_mock_hip.cpp"), os.path.join(mock, "mockhip.cpp")])
    return exe


@pytest.mark.parametrize("name", ["trees_of_a_batch", "captures_and_replays", "launches_of_an_acceptance", "launches_of_large_trees"])
def test_host_side(host, name):
    r = subprocess.run([host, name], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:detect_stack_use_after_return=0"))
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_the_oracle_notices_mistakes():
    """What the plain implementation says of a small tree, by hand; a planted mistake would differ."""
    #        0 - 1 - 3          2 hangs on 0, 4 on 2; 5 is in no tree, nor is 6, which hangs on it; 7 is a root of its own
    parents = [-1, 0, 0, 1, 2, -2, 5, -1]
    inside, family = TR.ancestry(parents)
    assert inside.tolist() == [True] * 5 + [False, False, True]
    assert [np.nonzero(f)[0].tolist() for f in family] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4], [], [], [7]]
    assert TR.depth(parents).tolist() == [0, 1, 1, 2, 2, 0, 0, 0]
    seen = TR.sight(10, 8, parents)
    assert np.nonzero(seen[4])[0].tolist() == [0, 1, 2, 4, 6] and not seen[6].any() and np.nonzero(seen[7])[0].tolist() == [0, 1, 9]
    tokens = [9, 5, 6, 7, 7, 1, 1, 9]
    assert TR.accepted(parents, tokens, [6, 0, 7, 0, 3, 0, 0, 0]) == ([0, 2, 4], 3)
    assert TR.accepted(parents, tokens, [4, 0, 7, 0, 3, 0, 0, 0]) == ([0], 4)
    assert TR.accepted([-1, 0, 0], [0, 8, 8], [8, 1, 2]) == ([0, 1], 1)
    assert TR.accepted([-2, -1], [0, 8], [8, 1]) == ([], -1)


def _pool(**kw):
    g = W.Geometry(**dict(dict(L=2, H=2, D=64, B=4, dtype="bf16", N=64, scales=False), **kw))
    return g, kv.KVPool(g, flags=kv.KV_PLAN_ONLY, staging_bytes=32 * g.S)


def test_trees_that_are_refused():
    g, p = _pool(N=1024)
    b = kv.KVBatch(p)
    i32 = lambda x: np.ascontiguousarray(x, np.int32)  # noqa: E731

    def set_(off, ids, lens, q, trees=None, parents=ONE, heads=4):
        return kv.kv_batch_set_trees(b.h, i32(off), i32(ids), i32(lens), i32(q), heads, parents, trees)

    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [3, 1]) == kv.KV_OK
    kv_rc, info = kv.kv_batch_query(b.h)
    assert kv_rc == kv.KV_OK and info["rows"] == 4
    assert set_([0, 2, 3], [5, 6, 7], [9, 1], [1, 1]) == kv.KV_EINVAL        # as kv_batch_set
    assert set_([0, 2, 3], [5, 6, 1024], [8, 1], [1, 1]) == kv.KV_ERANGE
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [9, 1]) == kv.KV_EINVAL
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [-1, 1]) == kv.KV_EINVAL
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [1, 1], heads=3) == kv.KV_EINVAL
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [3, 1], parents=None) == kv.KV_EINVAL
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [3, 1], trees=[False, False], parents=None) == kv.KV_OK   # nothing is read
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [3, 0], trees=[False, True], parents=None) == kv.KV_OK
    assert set_([0, 2, 3], [5, 6, 7], [8, 1], [3, 1], trees=[False, True], parents=None) == kv.KV_EINVAL
    assert set_([0], [], [], [], parents=None) == kv.KV_OK and kv.kv_batch_query(b.h)[1]["rows"] == 0
    blocks = np.arange(300)
    assert set_([0, 300], blocks, [1200], [kv.KV_TREE_MAX]) == kv.KV_OK
    assert set_([0, 300], blocks, [1200], [kv.KV_TREE_MAX + 1]) == kv.KV_EINVAL
    assert set_([0, 300], blocks, [1200], [kv.KV_TREE_MAX + 1], trees=[False]) == kv.KV_OK
    assert kv._lib.kv_batch_set_trees(None, 0, None, None, None, None, 4, None, None, None) == kv.KV_EINVAL
    assert kv._lib.kv_batch_set_trees(b.h, -1, None, None, None, None, 4, None, ONE, None) == kv.KV_EINVAL
    assert kv._lib.kv_batch_set_trees(b.h, 1, None, None, None, None, 4, None, ONE, None) == kv.KV_EINVAL


def _accept_args(**kw):
    a = kv.kv_accept_args()
    for k, v in dict(dict(layer=0, num_layers=2, tokens=ONE, chosen=ONE, count=ONE, path=ONE, next=ONE, path_cap=3, path_stride=3, weights_cap=8), **kw).items():
        setattr(a, k, v)
    return a


def test_acceptances_that_are_refused():
    g, p = _pool()
    b = kv.KVBatch(p)
    i32 = lambda *x: np.array(x, np.int32)  # noqa: E731
    accept = lambda **kw: kv.kv_accept(b.h, _accept_args(**kw))  # noqa: E731
    assert accept() == kv.KV_OK                                        # no requests: nothing is looked at
    kv.kv_check(kv.kv_batch_set_trees(b.h, i32(0, 2, 3), i32(5, 6, 7), i32(8, 1), i32(3, 1), 4, ONE))
    assert accept() == kv.KV_OK and accept(num_layers=0) == kv.KV_OK and accept(weights=ONE) == kv.KV_OK and accept(layer=1, num_layers=1) == kv.KV_OK
    for bad in (dict(layer=1), dict(layer=-1), dict(num_layers=-1), dict(num_layers=3), dict(tokens=None), dict(chosen=None), dict(count=None),
                dict(path=None), dict(next=None), dict(path_cap=2), dict(weights=ONE, weights_cap=7)):
        assert accept(**bad) == kv.KV_EINVAL, bad
    a = _accept_args()
    a.struct_size = ctypes.sizeof(a) - 8
    assert kv._lib.kv_accept(b.h, ctypes.byref(a), None) == kv.KV_EINVAL
    assert kv._lib.kv_accept(None, ctypes.byref(a), None) == kv.KV_EINVAL and kv._lib.kv_accept(b.h, None, None) == kv.KV_EINVAL
    # a block with drafted tokens in it that another request has, too
    kv.kv_check(kv.kv_batch_set_trees(b.h, i32(0, 2, 4), i32(5, 6, 5, 6), i32(8, 7), i32(3, 1), 4, ONE))
    assert accept() == kv.KV_EDUP and accept(num_layers=0) == kv.KV_OK
    kv.kv_check(kv.kv_batch_set_trees(b.h, i32(0, 2, 4), i32(5, 6, 5, 7), i32(8, 7), i32(3, 1), 4, ONE))
    assert accept() == kv.KV_OK                                        # the first block is in front of all of them: 5 .. 7 are in the second
    kv.kv_check(kv.kv_batch_set_trees(b.h, i32(0, 2, 4), i32(5, 6, 5, 6), i32(8, 7), i32(1, 1), 4, ONE))
    assert accept() == kv.KV_OK                                        # single tokens never move
    # without trees tokens and path are not needed
    kv.kv_check(b.set([0, 2, 3], [5, 6, 7], [8, 1], [3, 1], 4))
    assert accept(tokens=None, path=None, path_cap=0) == kv.KV_OK


def test_axes_that_are_refused():
    g, p = _pool()
    b = kv.KVBatch(p)
    kv.kv_check(b.set([0, 2], [5, 6], [8], [1], 4))

    def append(axes, pair_axes, **kw):
        a = kv.kv_append_args()
        for k, v in dict(dict(layer=1, io_dtype=kv.KV_BF16, rot=64, q=ONE, k=ONE, v=ONE, q_out=ONE, turns=ONE, positions=ONE), **kw).items():
            setattr(a, k, v)
        a.struct_size = ctypes.sizeof(a)
        w = None if pair_axes is None else np.ascontiguousarray(pair_axes, np.int32)
        return kv._lib.kv_append_axes(b.h, ctypes.byref(a), axes, None if w is None else w.ctypes.data, 1, None)

    good = np.arange(32) % 3
    assert append(3, good) == kv.KV_OK and append(4, good) == kv.KV_OK and append(1, np.zeros(32)) == kv.KV_OK
    assert append(2, good) == kv.KV_EINVAL and append(3, good - 1) == kv.KV_EINVAL and append(3, None) == kv.KV_EINVAL
    assert append(0, good) == kv.KV_EINVAL and append(5, good) == kv.KV_EINVAL and append(-1, good) == kv.KV_EINVAL
    assert append(3, good, positions=None) == kv.KV_EINVAL
    assert append(3, None, rot=0, positions=None, turns=None) == kv.KV_OK
    for bad in (dict(layer=2), dict(io_dtype=kv.KV_F16), dict(rot=63), dict(rot=66), dict(k=None), dict(v=None), dict(q=None), dict(turns=None), dict(k_scale=ONE)):
        assert append(3, good, **bad) == kv.KV_EINVAL, bad
    a = kv.kv_append_args()
    assert kv._lib.kv_append_axes(None, ctypes.byref(a), 3, good.ctypes.data, 1, None) == kv.KV_EINVAL
    assert kv._lib.kv_append_axes(b.h, None, 3, good.ctypes.data, 1, None) == kv.KV_EINVAL
    assert kv._lib.kv_append_axes(b.h, ctypes.byref(a), 3, good.ctypes.data, 1, None) == kv.KV_EINVAL  # struct_size


def test_tensors_that_do_not_fit_are_refused():
    """The binding sees shapes, types and devices that the C side cannot."""
    import torch
    g, p = _pool()
    b = kv.KVBatch(p)
    b.device = torch.device("cpu")
    b._stream = lambda s: None
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    set_ = lambda parents, trees=None: b.set_trees([0, 2, 3], [5, 6, 7], [8, 1], [3, 1], 4, parents, trees)  # noqa: E731
    assert set_(i32(4)) == kv.KV_OK and (b.n, b.T, b.max_tree) == (2, 4, 3)
    for bad in (i32(3), i32(5), i32(4, 1), torch.zeros(4, dtype=torch.int64), i32(8)[::2]):
        assert set_(bad) == kv.KV_EINVAL
    assert set_(i32(4), [True]) == kv.KV_EINVAL and set_(i32(4), [False, True]) == kv.KV_OK and b.max_tree == 1
    kv.kv_check(set_(i32(4)))
    args = dict(tokens=i32(4), chosen=i32(4), count=i32(2), path=i32(2, 3), next_token=i32(2))
    accept = lambda **kw: b.accept(0, 2, **dict(args, **kw))  # noqa: E731
    assert accept() == kv.KV_OK and accept(path=i32(2, 9)[:, :3]) == kv.KV_OK and accept(weights=torch.zeros(2, 2, 2, 8)) == kv.KV_OK
    for bad in (dict(tokens=i32(3)), dict(tokens=torch.zeros(4)), dict(chosen=i32(5)), dict(count=i32(1)), dict(count=torch.zeros(2, dtype=torch.int64)), dict(path=i32(2, 2)),
                dict(path=i32(3, 3)), dict(path=i32(3, 2).t()), dict(next_token=i32(3)), dict(weights=torch.zeros(1, 2, 2, 8)), dict(weights=torch.zeros(2, 2, 2, 7)),
                dict(weights=torch.zeros(2, 2, 2, 8).half()), dict(tokens=None), dict(path=None), dict(req_ids=[1])):
        assert accept(**bad) == kv.KV_EINVAL, bad
    k, turns = torch.zeros(4, 2, 64).bfloat16(), torch.zeros(32, dtype=torch.int64)
    append = lambda positions, pair_axes: b.append(0, None, k, k, turns=turns, positions=positions, pair_axes=pair_axes)  # noqa: E731
    good = np.arange(32) % 3
    assert append(i32(3, 4), good) == kv.KV_OK and append(i32(3, 9)[:, :4], good) == kv.KV_OK
    for bad in ((None, good), (i32(4), good), (i32(2, 4), good), (i32(3, 5), good), (i32(4, 3).t(), good), (i32(3, 4), good[:31]), (torch.zeros(3, 4), good),
                (i32(5, 4), good), (i32(3, 4), good + 1)):
        assert append(*bad) == kv.KV_EINVAL
    b.close()
    assert set_(i32(4)) == kv.KV_EINVAL and accept() == kv.KV_EINVAL


def test_accepted_drafts_make_host_copies_stale():
    """What a tree's tokens may move in is no longer as it was written through; requests that do not draft keep their copies."""
    g, p = _pool()
    b = kv.KVBatch(p)
    rows = [np.arange(0, 5), np.arange(10, 15), np.arange(20, 25)]
    off, ids = np.array([0, 5, 10, 15], np.int32), np.concatenate(rows).astype(np.int32)
    rc, *_ = p.swap_out_delta(np.array([1, 2, 3], np.uint64), off, ids, np.array([20, 20, 20], np.int32))
    assert rc == kv.KV_OK
    assert [p.query(i)[1]["wm"] for i in (1, 2, 3)] == [5, 5, 5]
    a = _accept_args(path_cap=8)
    req = np.array([1, 2, 3], np.uint64)
    a.req_ids = req.ctypes.data
    # 11 cached before the drafts of the first: tokens 12 .. 17 may move to 12 .. 16, in blocks from the fourth on
    kv.kv_check(kv.kv_batch_set_trees(b.h, off, ids, np.array([18, 18, 18], np.int32), np.array([7, 7, 1], np.int32), 4, ONE, [True, False, True]))
    assert kv.kv_accept(b.h, a) == kv.KV_OK
    assert [p.query(i)[1]["wm"] for i in (1, 2, 3)] == [3, 5, 5]
    # not of a request that is swapped out
    assert p.swap_out(np.array([3], np.uint64), np.array([0, 5], np.int32), ids[10:], np.array([20], np.int32)) == kv.KV_OK
    assert kv.kv_accept(b.h, a) == kv.KV_EEXIST
