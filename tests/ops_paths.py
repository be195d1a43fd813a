"""Batches that take the attention's ways through its kernels which small ones do not: several heads a workgroup, workgroups with several items, rows
of very many pieces, big tiles that are cut along their keys, heads with more query heads than a big tile has rows.  test_ops_paths.py checks on
the plan that they do (a set of words of native/plan_paths.cpp), test_gpu_ops_paths.py what the kernels make of them."""
import numpy as np


def spread(n, lo, hi, step=7):
    """n numbers over lo..hi in a mixed order."""
    return [lo + (hi - lo) * ((i * step) % n) // max(1, n - 1) for i in range(n)]


def behind(groups, blocks):
    """(request, of which request, blocks): consecutive groups of requests, each behind its first one's blocks."""
    out, at = [], 0
    for n in groups:
        out += [(at + i, at, blocks) for i in range(1, n)]
        at += n
    return tuple(out)


# name: geometry (H, D, B, dtype, scales), query heads a KV head, lengths, new tokens, shared beginnings, ways
PATHS = {
    "four heads a workgroup": ((4, 64, 16, "bf16", False), 2, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many", "stream", "join1"}),
    "four heads a workgroup, f16": ((8, 64, 32, "f16", False), 1, spread(200, 30, 1000), [1] * 200, (), {"hw4", "rows_many", "stream"}),
    "four heads a workgroup, d 128": ((4, 128, 16, "bf16", False), 3, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many", "stream"}),
    "four heads a workgroup, d 256": ((4, 256, 16, "bf16", False), 1, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many", "stream"}),
    "four heads a workgroup, fp8": ((4, 64, 16, "fp8_e4m3", True), 2, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many", "stream"}),
    "four heads a workgroup, fp8, d 128": ((4, 128, 32, "fp8_e4m3", True), 1, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many", "stream"}),
    "four heads a workgroup, odd blocks": ((4, 72, 5, "bf16", False), 3, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many"}),
    "four heads a workgroup, odd blocks, fp8": ((4, 96, 6, "fp8_e4m3", True), 3, spread(400, 30, 1000), [1] * 400, (), {"hw4", "rows_many"}),
    "four heads a workgroup, some with two new tokens": ((4, 64, 16, "bf16", False), 2, spread(400, 30, 1000), [1, 2, 1, 1] * 100, (), {"hw4", "rows_many", "rows_mixed"}),
    "four heads a workgroup, two new tokens, fp8": ((4, 64, 16, "fp8_e4m3", True), 2, spread(400, 30, 1000), [2, 2, 1, 1] * 100, (), {"hw4", "rows_many", "rows_mixed"}),
    "two heads a workgroup": ((6, 64, 16, "bf16", False), 2, spread(160, 30, 1200), [1] * 160, (), {"hw2", "rows_many", "stream"}),
    "two heads a workgroup, fp8": ((6, 64, 16, "fp8_e4m3", True), 1, spread(160, 30, 1200), [1] * 160, (), {"hw2", "rows_many", "stream"}),
    "two heads a workgroup, odd blocks": ((2, 64, 5, "f16", False), 2, spread(420, 30, 1300), [1, 1, 2, 1, 1] * 84, (), {"hw2", "rows_many", "rows_mixed"}),
    "many short requests": ((1, 128, 16, "bf16", False), 4, spread(700, 0, 61), [1] * 700, (), {"hw1", "rows_many", "rows_whole", "stream"}),
    "many short requests, fp8": ((2, 64, 16, "fp8_e4m3", True), 3, spread(400, 1, 61), [1] * 400, (), {"hw1", "rows_many", "stream"}),
    "many short requests, odd blocks": ((4, 80, 3, "f16", False), 3, spread(200, 2, 61), [1, 1, 1, 2] * 50, (), {"hw1", "rows_many", "rows_mixed"}),
    "very many pieces": ((1, 64, 16, "bf16", False), 4, [60011, 333], [1, 1], (), {"hw1", "join16", "stream"}),
    "very many pieces, d 256, odd blocks": ((1, 256, 7, "f16", False), 3, [52003, 40], [1, 1], (), {"join16"}),
    "very many pieces, fp8, two new tokens": ((1, 96, 4, "fp8_e4m3", False), 3, [52003, 40], [2, 1], (), {"join16", "rows_mixed"}),
    "a long prefix": ((2, 128, 16, "bf16", False), 8, [4112 + 4 + 11 * (i % 24) for i in range(60)], [1] * 60, behind([60], 257), {"both", "big_cut", "fine"}),
    "a long prefix, f16": ((2, 64, 16, "f16", False), 8, [7632 + 4 + 11 * (i % 24) for i in range(60)], [1] * 60, behind([60], 477), {"both", "big_cut", "fine"}),
    "a long prefix, fp8": ((2, 128, 16, "fp8_e4m3", True), 8, [7632 + 4 + 11 * (i % 24) for i in range(60)], [1] * 60, behind([60], 477), {"both", "big_cut", "fine"}),
    "a long prefix, d 256": ((1, 256, 16, "bf16", False), 8, [4112 + 4 + 11 * (i % 24) for i in range(60)], [1] * 60, behind([60], 257), {"both", "big_cut", "fine"}),
    "a long prefix, odd blocks": ((2, 72, 5, "bf16", False), 8, [6775 + 4 + 11 * (i % 24) for i in range(60)], [1] * 60, behind([60], 1355), {"big_cut", "fine"}),
    "a long prefix, odd blocks, fp8": ((2, 72, 6, "fp8_e4m3", True), 8, [13542 + 4 + 11 * (i % 24) for i in range(60)], [1] * 60, behind([60], 2257), {"big_cut", "fine"}),
    "a long prefix, one with a prompt": ((2, 128, 16, "bf16", False), 8, [4112 + 4 + 11 * (i % 24) for i in range(60 - 1)] + [4112 + 320], [1] * (60 - 1) + [300], behind([60], 257),
                                         {"both", "big_cut", "big_mixed", "fine"}),
    "a long prompt": ((2, 128, 16, "bf16", False), 4, [2600, 1500], [300, 70], (), {"big_cut", "big_cut_mixed", "big_blind"}),
    "a long prompt, f16": ((1, 64, 16, "f16", False), 4, [3001, 1500], [700, 70], (), {"big_cut", "big_cut_mixed", "big_blind"}),
    "a long prompt, fp8": ((2, 128, 16, "fp8_e4m3", True), 4, [2600, 1500], [300, 70], (), {"big_cut", "big_cut_mixed", "big_blind"}),
    "a long prompt, d 256": ((1, 256, 16, "bf16", False), 4, [2600, 1500], [300, 70], (), {"big_cut", "big_cut_mixed", "big_blind"}),
    "a long prompt, odd blocks": ((2, 72, 5, "bf16", False), 4, [2600, 1500], [300, 70], (), {"big_cut", "big_cut_mixed", "big_blind"}),
    "a long prompt, odd blocks, fp8": ((2, 192, 6, "fp8_e4m3", True), 4, [2600, 1500], [300, 70], (), {"big_cut", "big_cut_mixed", "big_blind"}),
    "many tiles of prompts": ((8, 64, 16, "bf16", False), 8, [1100, 1300], [500, 700], (), {"big_many", "big_mixed", "big_cut"}),
    "many tiles of prompts, fp8": ((8, 128, 16, "fp8_e4m3", True), 8, [1100, 1300], [500, 700], (), {"big_many", "big_mixed", "big_cut"}),
    "many tiles of prompts, d 256": ((8, 256, 16, "f16", False), 8, [900, 700], [230, 170], (), {"big_many", "big_mixed"}),
    "many tiles of prompts, odd blocks": ((16, 72, 5, "bf16", False), 8, [700, 600], [300, 290], (), {"big_many", "big_mixed"}),
    "few behind a prefix": ((2, 128, 16, "bf16", False), 4, [700, 710, 720, 900], [1, 1, 1, 1], behind([4], 43), {"rows_shared", "stream", "join1"}),
    "few behind a prefix, new tokens": ((2, 64, 16, "f16", False), 2, [700, 710, 720, 900], [1, 3, 1, 2], behind([4], 43), {"rows_shared", "rows_mixed"}),
    "few behind a prefix, fp8": ((2, 128, 16, "fp8_e4m3", True), 4, [700, 710, 720, 900], [1, 1, 1, 1], behind([4], 43), {"rows_shared", "stream"}),
    "few behind a prefix, odd blocks, fp8": ((2, 72, 6, "fp8_e4m3", True), 4, [700, 710, 720, 900], [1, 2, 1, 0], behind([4], 116), {"rows_shared", "rows_mixed"}),
    "a prefix and nothing else": ((1, 128, 16, "bf16", False), 2, [640, 640, 640], [1, 1, 1], behind([3], 40), {"rows_shared", "stream"}),
    "a tree of prefixes": ((1, 64, 16, "f16", False), 2, [2400, 2400, 2410, 2500, 1090, 533, 2390], [1, 2, 1, 3, 1, 1, 1],
                           ((1, 0, 140), (2, 0, 140), (3, 1, 80), (4, 0, 65), (5, 4, 32), (6, 3, 100)), {"rows_shared", "rows_mixed"}),
    "many prefixes": ((8, 64, 16, "bf16", False), 16, [1637 + i % 9 for i in range(140)], [1] * 140, behind([2] * 70, 102), {"big_many", "fine", "both", "rows_many"}),
    "many prefixes, fp8": ((8, 64, 16, "fp8_e4m3", True), 16, [3237 + i % 9 for i in range(140)], [1] * 140, behind([2] * 70, 202), {"big_many", "fine", "both", "rows_many"}),
    "many prefixes, odd blocks": ((8, 80, 5, "f16", False), 16, [1295 + i % 9 for i in range(140)], [1] * 140, behind([2] * 70, 258), {"big_many", "fine", "rows_many"}),
    "more query heads than rows": ((2, 64, 16, "bf16", False), 150, [300, 45, 0], [1, 3, 1], (), {"huge", "big_mixed", "big_whole"}),
    "more query heads than rows, a prefix": ((1, 128, 16, "f16", False), 150, [8020 + i % 7 for i in range(60)], [3] + [1] * 59, behind([60], 500), {"huge", "fine"}),
    "more query heads than rows, fp8": ((2, 64, 16, "fp8_e4m3", True), 150, [300, 45], [1, 3], (), {"huge", "big_mixed"}),
    "more query heads than rows, d 256": ((1, 256, 16, "bf16", False), 70, [300, 45], [1, 3], (), {"huge", "big_mixed"}),
    "more query heads than rows, cut": ((1, 64, 1, "bf16", False), 150, [4000, 45], [3, 1], (), {"huge", "huge_cut", "huge_cut_mixed"}),
    "more query heads than rows, cut, blind": ((1, 72, 1, "f16", False), 130, [1925, 45], [30, 1], (), {"huge", "huge_cut", "huge_blind"}),
}


def tables(rng, N, lens, B, shared):
    """Tables of distinct blocks; shared: (request, of which request, blocks) begins with the other's first blocks."""
    perm, at, rows = rng.permutation(N).astype(np.int32), 0, []
    for n in lens:
        need = -(-n // B)
        rows.append(perm[at:at + need].copy())
        at += need
    for i, of, k in shared:
        assert k <= len(rows[i]) and k <= len(rows[of])
        rows[i][:k] = rows[of][:k]
    return rows
