"""Calls of a serving loop one after the other, on a real MI355X."""
import numpy as np
import pytest

import ops_ref as R
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W
from test_gpu_ops import Pool, _tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep", [64, 96])
def test_appending_after_an_eviction_with_scales(gpu, keep):
    """A pool whose blocks differ in their scales: an eviction that keeps whole blocks, then appends with scales of their own.  What was kept
    stands for what it did after the eviction, the new tokens for what was appended, and attention sees both."""
    import torch
    L, H, D, B, G, lens = 1, 2, 64, 16, 4, [150, 133]
    N = 30
    p = Pool(gpu, W.Geometry(L, H, D, B, "fp8_e4m3", N, scales=True), seed=21)
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    torch.manual_seed(keep)
    o, ids = R.csr(rows)
    weights = torch.rand(L, 2, H, max(lens), device=gpu)
    kept = torch.zeros(L, 2, H, keep, dtype=torch.int32, device=gpu)
    kv.kv_check(p.batch.set(o, ids, lens, [0, 0], G * H))
    kv.kv_check(p.batch.evict(0, L, weights, kept, keep, 4, 8))
    torch.cuda.synchronize()
    stood = [R.request_rows(p.values()[0], rows[i], keep, B) for i in range(2)]
    new = []
    for step in range(3):
        lens_now = [keep + step + 1] * 2
        kv.kv_check(p.batch.set(o, ids, lens_now, [1, 1], G * H))
        k, v = (torch.randn(2, H, D, device=gpu).bfloat16() for _ in range(2))
        scale = [torch.tensor([0.011, 0.014], device=gpu), torch.tensor([0.009, 0.02], device=gpu)]
        kv.kv_check(p.batch.append(0, None, k, v, k_scale=scale[0], v_scale=scale[1]))
        q, out = torch.randn(2, G * H, D, device=gpu).bfloat16(), torch.empty(2, G * H, D, dtype=torch.bfloat16, device=gpu)
        kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
        torch.cuda.synchronize()
        new.append((k.double().cpu().numpy(), v.double().cpu().numpy()))
        values = p.values()[0]
        for i in range(2):
            there = R.request_rows(values, rows[i], lens_now[i], B)
            assert np.array_equal(there[:, :keep], stood[i])
            for s, both in enumerate(new):
                for c in range(2):  # beyond +-448 scales as these, and rounded to fp8 once: half of 2^-3 of itself, or of the smallest step
                    sc = scale[c].double().cpu().numpy()[:, None]
                    x = np.clip(both[c][i], -448 * sc, 448 * sc)
                    assert (np.abs(there[c, keep + s] - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * sc).all()
        ref, tol, _, _, _, _ = R.attention(values, rows, lens_now, [1, 1], q.double().cpu().numpy(), D ** -0.5, "bf16", B)
        assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
