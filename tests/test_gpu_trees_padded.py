"""Drafted trees on a real MI355X where a batch is padded or a cache holds what is not finite, against plain implementations in 64 bits (trees_ref.py)."""
import numpy as np
import pytest

import ops_ref as R
import trees_ref as TR
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W
from test_gpu_ops import Pool, _tables, _torch_type

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(2, 128, 16, 4), (2, 72, 5, 3), (1, 256, 32, 4)])
@pytest.mark.parametrize("new", [5, 30])     # row tiles, whose products are kept, and big ones, whose products are computed again
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_row_of_no_tree_gives_no_weight_to_an_infinite_key(gpu, dtype, new, shape):
    """A cached key with an infinity that every row in the tree has a product of -inf with has weight 0; rows of no tree, whatever their queries are, change
    nothing about that."""
    import torch
    H, D, B, G = shape
    n, far, d = 170, 3, 9
    N = -(-n // B) + 2
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, N), seed=new + D)
    rows = _tables(p.rng, N, [n], B)
    p.fill(rows, [n])
    parents = [TR.ROOT] + [TR.NONE if j % 3 == 1 else 0 for j in range(1, new)]
    inside, _ = TR.ancestry(parents)
    q = torch.from_numpy(p.rng.standard_normal((new, G * H, D))).to(_torch_type(dtype)).to(gpu)
    q[:, :, d] = -q[:, :, d].abs() - 0.1
    # the reference: the same without that key, which is behind everything that is seen of it
    x = np.delete(np.arange(n), far)
    table = np.asarray(rows[0], np.int64)
    without = p.values()[0][:, table[x // B], x % B][:, :, None]
    ref, tol, rlse, ltol, rw, wtol = TR.attention(without, [np.arange(n - 1)], [n - 1], [new], [parents], q.double().cpu().numpy(), D ** -0.5, dtype, 1)
    p.bits()[0, 0, int(table[far // B]), far % B, :, d] = {"bf16": 0x7F80, "f16": 0x7C00}[dtype]
    for j in np.nonzero(~inside)[0]:
        q[int(j)] = float("nan") if j % 2 else 0.0
    o, ids = R.csr(rows)
    out, lse = torch.empty_like(q), torch.empty(new, G * H, device=gpu)
    start = torch.rand(1, H, n, device=gpu)
    weights = start.clone()
    kv.kv_check(p.batch.set_trees(o, ids, [n], [new], G * H, torch.tensor(parents, dtype=torch.int32, device=gpu)))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5, lse=lse, weights=weights))
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    gl = lse.double().cpu().numpy()
    assert (gl[~inside] == -np.inf).all() and (np.abs(gl[inside] - rlse[inside]) <= ltol[inside]).all()
    added = (weights.double() - start.double())[0].cpu().numpy()
    assert (added[:, far] == 0).all()
    slack = (2.0 ** -22 * (1 + np.abs(rw[0])) + wtol[0]) * (1 + new)     # (as in test_gpu_trees.py)
    assert (np.abs(added[:, x] - rw[0]) <= slack).all()


def test_paths_of_padded_requests(gpu):
    """Every row of a tree has an entry of `path`, that of a padded request, too; a request whose new tokens are no tree has none."""
    import torch
    lens, q_lens, trees = [40, 0, 9, 30, 0], [4, 1, 0, 3, 1], [True, True, True, False, False]
    p = Pool(gpu, W.Geometry(2, 2, 64, 16, "bf16", 12), seed=8)
    rows = _tables(p.rng, 12, lens, 16)
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=gpu)  # noqa: E731
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, 4, dev([-1, 0, 1, -2, -1, 3, 3, 3, 3]), trees))
    count, nxt, path = dev([-9] * 5), dev([-9] * 5), torch.full((5, 6), -9, dtype=torch.int32, device=gpu)
    kv.kv_check(p.batch.accept(0, 2, dev([7] * 9), dev([7] * 9), count, path, nxt))
    assert count.tolist() == [3, 0, 0, 3, 0] and nxt.tolist() == [7, -1, -1, 7, -1]
    none = [-9] * 6
    assert path.tolist() == [[0, 1, 2, -1, -9, -9], [-1] + none[1:], none, none, none]


@pytest.mark.parametrize("shape", [(2, 128, 8), (3, 72, 6)])
def test_accepted_rows_between_scales_far_apart(gpu, shape):
    """A row that comes with a scale beyond 2^128 times that of its new block: what is not 0 becomes +-448, and a 0 stays one."""
    import torch
    H, D, B = shape
    base, new = B, 3 * B
    p = Pool(gpu, W.Geometry(2, H, D, B, "fp8_e4m3", 8, scales=True), seed=D)
    rows = _tables(p.rng, 8, [base + new], B)
    p.fill(rows, [base + new])
    first, last = int(rows[0][1]), int(rows[0][3])
    row = 2 * B + 1                                # in the last block; it goes to place 1 of the first with new tokens
    bits = p.bits()
    bits[:, :, last, 1, :, ::3] = 0
    bits[:, :, last, 1, :, 1] = 0x80
    p.scale[:, :, first] = 1e-30
    p.scale[:, :, last] = 1e30
    before = bits.clone()
    o, ids = R.csr(rows)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=gpu)  # noqa: E731
    kv.kv_check(p.batch.set_trees(o, ids, [base + new], [new], H, dev([TR.ROOT] + [0] * (new - 1))))
    tokens, chosen = dev([0] * new), dev([5] * new)
    tokens[row] = 5
    count, nxt, path = dev([0]), dev([0]), torch.zeros(1, new, dtype=torch.int32, device=gpu)
    kv.kv_check(p.batch.accept(0, 2, tokens, chosen, count, path, nxt))
    assert count.tolist() == [2] and path[0, :3].tolist() == [0, row, -1]
    want = before.clone()
    was = before[:, :, last, 1]
    want[:, :, first, 1] = torch.where(was & 0x7F == 0, was, was & 0x80 | 0x7E)
    assert torch.equal(p.bits(), want)
