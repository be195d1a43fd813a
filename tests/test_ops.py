"""CPU tests of the operators on the pool's contents: the attention's plan, the rotary frequencies, refusals, and what an eviction does to
the bookkeeping of host copies (plan-only handles make no HIP call)."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W

HERE = os.path.dirname(os.path.abspath(__file__))


def test_plan_covers_every_pair_once(tmp_path):
    exe = str(tmp_path / "batch_plan")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "native", "batch_plan.cpp"), "-o", exe])
    r = subprocess.run([exe, "600"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "plans ok" in r.stdout, r.stdout + r.stderr


def _pool(**kw):
    g = W.Geometry(**dict(dict(L=2, H=2, D=64, B=4, dtype="bf16", N=64, scales=False), **kw))
    return g, kv.KVPool(g, flags=kv.KV_PLAN_ONLY, staging_bytes=32 * g.S)


def test_batches_that_are_refused():
    g, p = _pool()
    b = kv.KVBatch(p)
    ok = lambda off, ids, lens, q, heads=4: b.set(np.array(off), np.array(ids), lens, q, heads)  # noqa: E731
    assert ok([0, 2, 3], [5, 6, 7], [8, 1], [1, 1]) == kv.KV_OK
    assert b.query()["rows"] == 2 and b.query()["cached_tokens"] == 9
    assert ok([0, 2, 3], [5, 6, 7], [9, 1], [1, 1]) == kv.KV_EINVAL        # two blocks do not hold nine tokens
    assert ok([0, 2, 3], [5, 6, 64], [8, 1], [1, 1]) == kv.KV_ERANGE
    assert ok([0, 2, 3], [5, -1, 6], [8, 1], [1, 1]) == kv.KV_ERANGE
    assert ok([0, 2, 3], [5, 6, 64], [8, 0], [1, 1]) == kv.KV_OK           # behind what the tokens need nothing is looked at
    assert ok([0, 2, 1], [5, 6, 7], [8, 1], [1, 1]) == kv.KV_EINVAL
    assert ok([0, 2], [5, 6, 7], [8, 1], [1, 1]) == kv.KV_EINVAL
    assert ok([0, 2, 5], [5, 6, 7], [8, 1], [1, 1]) == kv.KV_EINVAL
    assert ok([0, 2, 3], [5, 6, 7], [8, 1], [9, 1]) == kv.KV_EINVAL        # more new tokens than tokens
    assert ok([0, 2, 3], [5, 6, 7], [8, 0], [1, 2]) == kv.KV_EINVAL
    assert ok([0, 2, 3], [5, 6, 7], [8, -1], [1, 1]) == kv.KV_EINVAL
    assert ok([0, 2, 3], [5, 6, 7], [8, 1], [1, -1]) == kv.KV_EINVAL
    assert ok([0, 2, 3], [5, 6, 7], [8, 1], [1, 1], 3) == kv.KV_EINVAL     # three query heads on two KV heads
    assert ok([0, 2, 3], [5, 6, 7], [8, 1], [1, 1], 0) == kv.KV_EINVAL
    assert ok([0], [], [], []) == kv.KV_OK and b.query()["rows"] == 0
    b.close()
    assert ok([0], [], [], []) == kv.KV_EINVAL
    for D in (4, 12, 136, 264, 512):
        g, p = _pool(D=D, H=4)
        with pytest.raises(kv.KVSwapError):
            kv.KVBatch(p)


def test_calls_that_are_refused():
    g, p = _pool()
    b = kv.KVBatch(p)
    kv.kv_check(b.set([0, 2], [5, 6], [8], [1], 4))
    one = 16  # stands for a device pointer: a plan-only handle never follows it

    def append(**kw):
        a = kv.kv_append_args()
        for k, v in dict(dict(layer=1, io_dtype=kv.KV_BF16, rot=64, q=one, k=one, v=one, q_out=one, turns=one), **kw).items():
            setattr(a, k, v)
        return kv.kv_append(b.h, a)

    assert append() == kv.KV_OK
    for bad in (dict(layer=2), dict(layer=-1), dict(io_dtype=kv.KV_F16), dict(io_dtype=kv.KV_FP8_E4M3), dict(rot=63), dict(rot=-2), dict(rot=66),
                dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(turns=None), dict(k_scale=one), dict(k_scale=one, v_scale=one)):
        assert append(**bad) == kv.KV_EINVAL, bad
    assert append(q=None, q_out=None) == kv.KV_OK and append(rot=0, turns=None) == kv.KV_OK

    def attn(**kw):
        a = kv.kv_attn_args()
        for k, v in dict(dict(layer=1, io_dtype=kv.KV_BF16, scale=0.1, q=one, out=one, weights_cap=8), **kw).items():
            setattr(a, k, v)
        return kv.kv_attn(b.h, a)

    assert attn() == kv.KV_OK and attn(weights=one) == kv.KV_OK
    for bad in (dict(layer=2), dict(layer=-1), dict(io_dtype=kv.KV_F16), dict(q=None), dict(out=None), dict(weights=one, weights_cap=7),
                dict(scale=math.nan), dict(scale=math.inf)):
        assert attn(**bad) == kv.KV_EINVAL, bad

    def evict(**kw):
        a = kv.kv_evict_args()
        for k, v in dict(dict(layer=0, num_layers=2, keep=4, keep_first=1, keep_last=1, weights=one, kept=one, weights_cap=8), **kw).items():
            setattr(a, k, v)
        return kv.kv_evict(b.h, a)

    assert evict() == kv.KV_OK
    for bad in (dict(layer=1), dict(layer=-1), dict(num_layers=-1), dict(num_layers=3), dict(keep=1), dict(keep_first=-1), dict(keep_last=-1),
                dict(keep=-1, keep_first=0, keep_last=0), dict(weights=None), dict(kept=None), dict(weights_cap=7)):
        assert evict(**bad) == kv.KV_EINVAL, bad
    assert evict(num_layers=0) == kv.KV_OK

    for name in ("kv_append", "kv_attn", "kv_evict"):
        f = getattr(kv._lib, name)
        args = getattr(kv, name + "_args")()
        args.struct_size = ctypes.sizeof(args) - 8
        assert f(b.h, ctypes.byref(args), None) == kv.KV_EINVAL
        assert f(None, ctypes.byref(args), None) == kv.KV_EINVAL and f(b.h, None, None) == kv.KV_EINVAL
    assert kv._lib.kv_batch_create(None, None) == kv.KV_EINVAL and kv._lib.kv_batch_destroy(None) == kv.KV_EINVAL
    assert kv._lib.kv_batch_set(None, 0, None, None, None, None, 4, None) == kv.KV_EINVAL
    assert kv._lib.kv_batch_query(b.h, None) == kv.KV_EINVAL

    # the two 16-bit types on an fp8 pool, and its scales
    g, p8 = _pool(dtype="fp8_e4m3")
    b = kv.KVBatch(p8)
    kv.kv_check(b.set([0, 2], [5, 6], [8], [1], 4))
    assert append() == kv.KV_OK and append(io_dtype=kv.KV_F16) == kv.KV_OK and append(io_dtype=kv.KV_FP8_E4M3) == kv.KV_EINVAL
    assert append(k_scale=one, v_scale=one) == kv.KV_EINVAL


def test_tensors_that_do_not_fit_are_refused():
    """The binding sees shapes, types and devices that the C side cannot."""
    import torch
    g, p = _pool()
    b = kv.KVBatch(p)
    b.device = torch.device("cpu")
    b._stream = lambda s: None
    kv.kv_check(b.set([0, 2], [5, 6], [8], [2], 4))
    T, bf = 2, torch.bfloat16
    q, k = torch.zeros(T, 4, 64, dtype=bf), torch.zeros(T, 2, 64, dtype=bf)
    lse, w = torch.zeros(T, 4), torch.zeros(1, 2, 8)
    assert b.attn(0, q, q, 1.0, lse=lse, weights=w) == kv.KV_OK
    wide = torch.zeros(T, 4, 128, dtype=bf)
    for bad in (q[:1], q[:, :3], q[..., :32], q.float(), wide[..., ::2], q[0], q.half()):
        assert b.attn(0, bad, q, 1.0) == kv.KV_EINVAL and b.attn(0, q, bad, 1.0) == kv.KV_EINVAL
    assert b.attn(0, wide[..., :64], wide[..., 64:], 1.0) == kv.KV_OK
    for bad in (lse[:1], lse.double(), lse.t()):
        assert b.attn(0, q, q, 1.0, lse=bad) == kv.KV_EINVAL
    for bad in (w[..., :7], w[:, :1], w[0], w.double()):
        assert b.attn(0, q, q, 1.0, weights=bad) == kv.KV_EINVAL
    turns = torch.zeros(32, dtype=torch.int64)
    assert b.append(0, q, k, k, turns=turns, positions=torch.zeros(T, dtype=torch.int32)) == kv.KV_OK
    assert b.append(0, None, k, k) == kv.KV_OK
    assert b.append(0, q, k[:1], k) == kv.KV_EINVAL and b.append(0, q, k, k.half()) == kv.KV_EINVAL and b.append(0, k, k, k) == kv.KV_EINVAL
    assert b.append(0, q, k, k, turns=turns.int()) == kv.KV_EINVAL
    assert b.append(0, q, k, k, turns=torch.zeros(33, dtype=torch.int64)) == kv.KV_EINVAL
    assert b.append(0, q, k, k, positions=torch.zeros(T)) == kv.KV_EINVAL
    assert b.append(0, q, k, k, positions=torch.zeros(T + 1, dtype=torch.int32)) == kv.KV_EINVAL
    w, kept = torch.zeros(2, 1, 2, 8), torch.zeros(2, 1, 2, 4, dtype=torch.int32)
    assert b.evict(0, 2, w, kept, 4) == kv.KV_OK
    assert b.evict(0, 2, w, kept, 5) == kv.KV_EINVAL and b.evict(0, 1, w, kept, 4) == kv.KV_EINVAL
    assert b.evict(0, 2, w, kept.long(), 4) == kv.KV_EINVAL and b.evict(0, 2, w, kept, 4, weights_out=torch.zeros(2, 1, 2, 9)[..., :8]) == kv.KV_EINVAL
    assert b.evict(0, 2, w, kept, 4, req_ids=[1, 2]) == kv.KV_EINVAL


def test_an_eviction_makes_host_copies_stale():
    g, p = _pool()  # blocks of 4 tokens
    kv.kv_check(p.swap_out_delta([7], [0, 4], [1, 2, 3, 4], [16])[0])
    kv.kv_check(p.wq_post([7], [0, 4], [1, 2, 3, 4], [16]))
    kv.kv_check(p.swap_out([8], [0, 1], [20], [4]))
    b = kv.KVBatch(p)
    kv.kv_check(b.set([0, 4, 5], [1, 2, 3, 4, 9], [16, 3], [1, 1], 4))
    a = kv.kv_evict_args()
    a.num_layers, a.keep, a.keep_first, a.weights, a.kept, a.weights_cap = 2, 10, 6, 16, 16, 16

    def evict(ids):
        ids = np.array(ids, np.uint64)
        a.req_ids = ids.ctypes.data
        return kv.kv_evict(b.h, a)

    assert p.query(7)[1]["wm"] == 4 and p.wq_pending()[2] == 0
    assert evict([7, 8]) == kv.KV_EEXIST       # 8 is swapped out: it has no blocks to evict from
    assert p.query(7)[1]["wm"] == 4
    kv.kv_check(evict([7, 99]))                # 99 is not known, and has little enough
    q = p.query(7)[1]
    assert (q["wm"], q["staged"], q["cap"], q["swapped"]) == (1, 1, 4, 0)  # the block in front of the first that is written
    assert p.wq_remove(7) == kv.KV_ENOENT
    # what is written through next begins there, with the tokens that are left
    rc, moved = p.swap_out_delta([7], [0, 3], [1, 2, 3], [10])
    assert rc == kv.KV_OK and list(moved) == [1]
    # the same block twice: not where it would be written
    kv.kv_check(b.set([0, 4, 8], [1, 2, 3, 4, 1, 6, 7, 8], [16, 16], [1, 1], 4))
    a.req_ids = None
    assert kv.kv_evict(b.h, a) == kv.KV_OK
    a.keep_first = 3
    assert kv.kv_evict(b.h, a) == kv.KV_EDUP
    a.keep = 16
    assert kv.kv_evict(b.h, a) == kv.KV_OK     # nobody has more


def test_rotary_frequencies():
    """Against the formulas, in the words' own resolution: 2^-52 of the frequency and half a word."""
    two_pi = 2 * math.pi

    def check(words, want):
        got = [int(w) for w in words]
        for g, w in zip(got, want):
            assert abs(g - w * 2.0 ** 64) <= w * 2.0 ** 64 * 2.0 ** -48 + 1

    rot, base = 128, 10000.0
    plain = [base ** (-2 * j / rot) / two_pi for j in range(rot // 2)]
    rc, t, m = kv.kv_rope_freqs(rot, base)
    assert rc == kv.KV_OK and m == 1.0 and t.dtype == np.int64 and len(t) == 64
    check(t, plain)
    rc, t, m = kv.kv_rope_freqs(rot, base, kv.KV_ROPE_LINEAR, factor=4.0)
    check(t, [x / 4 for x in plain])
    rc, t, m = kv.kv_rope_freqs(rot, base, kv.KV_ROPE_BASE, factor=4.0)
    check(t, [(base * 4.0 ** (rot / (rot - 2))) ** (-2 * j / rot) / two_pi for j in range(rot // 2)])
    assert abs(int(t[-1]) / (plain[-1] * 2.0 ** 64 / 4.0) - 1) < 1e-9   # the slowest pair is stretched by just the factor
    rc, t, m = kv.kv_rope_freqs(rot, base, kv.KV_ROPE_PARTS, factor=8.0, trained=8192, low=1.0, high=4.0)
    want = []
    for x in plain:
        turns = 8192 * x
        k = 0.0 if turns <= 1 else 1.0 if turns >= 4 else (turns - 1) / 3
        want.append(x / 8 * (1 - k) + x * k)
    check(t, want)
    assert m == 1.0 and int(t[0]) == round(plain[0] * 2.0 ** 64) and abs(int(t[-1]) * 8 / (plain[-1] * 2.0 ** 64) - 1) < 1e-9
    rc, t, m = kv.kv_rope_freqs(rot, base, kv.KV_ROPE_YARN, factor=8.0, trained=4096, low=1.0, high=32.0)
    at = lambda n: rot * math.log(4096 / (n * two_pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = math.floor(at(32.0)), math.ceil(at(1.0))
    check(t, [x / 8 * r + x * (1 - r) for x, r in ((x, min(1.0, max(0.0, (j - lo) / (hi - lo)))) for j, x in enumerate(plain))])
    assert abs(m - (0.1 * math.log(8.0) + 1)) < 1e-6
    for bad in ((0,), (3,), (258,), (-2,), (64, 1.0), (64, math.nan), (64, 1e4, 9), (64, 1e4, kv.KV_ROPE_LINEAR, 0.5),
                (64, 1e4, kv.KV_ROPE_YARN, 2.0, 0.0), (64, 1e4, kv.KV_ROPE_PARTS, 2.0, 8192, 4.0, 4.0)):
        assert kv.kv_rope_freqs(*bad)[0] == kv.KV_EINVAL, bad
