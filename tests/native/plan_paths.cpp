// Which ways through the attention's kernels a batch takes: its plan (batch.hpp) for a GPU of 256 CUs, in words.
// stdin: H G B D N fp8 n, then n lengths, n query lengths, n + 1 offsets, and the table's blocks.
#include <cstdio>
#include <map>
#include <set>
#include <string>
#include <tuple>

#include "../../paper_2510_02758_amd/csrc/batch.hpp"

int main() {
  int H, G, B, D, N, fp8, n;
  if (std::scanf("%d%d%d%d%d%d%d", &H, &G, &B, &D, &N, &fp8, &n) != 7) return 2;
  auto read = [](size_t k) {
    std::vector<int32_t> v(k);
    for (int32_t& x : v)
      if (std::scanf("%d", &x) != 1) std::exit(2);
    return v;
  };
  const auto len = read(n), q = read(n), off = read(n + 1), ids = read(off[n]);
  kvswap::BatchPlan p;
  const kvswap::BatchShape shape = kvswap::batch_shape(H, D, B, N, 256, fp8 != 0);
  if (p.set(n, off.data(), ids.data(), len.data(), q.data(), G * H, shape) != KV_OK) return 3;
  std::set<std::string> paths;
  paths.insert("hw" + std::to_string(p.heads));
  for (size_t k = 0; k + 1 < p.wg_items.size(); k++)
    if (p.wg_items[k + 1] - p.wg_items[k] > 1) paths.insert("rows_many");   // a workgroup of row tiles with several items
  for (size_t k = 0; k + 1 < p.wg_big.size(); k++)
    if (p.wg_big[k + 1] - p.wg_big[k] > 1) paths.insert("big_many");
  std::map<std::pair<int, int>, std::set<int>> runs;   // (tokens, row0) of a big tile -> where its runs of keys begin
  std::map<int, std::set<int>> tiles;                  // token -> tiles of its own
  for (size_t k = 0; k < p.items.size(); k++) {
    const kvswap::AttnItem& it = p.items[k];
    const bool big = (int)k >= p.big_first;
    const bool mixed = it.clear < it.k1;
    paths.insert(big ? "big" : "rows");
    if (mixed) paths.insert(big ? "big_mixed" : "rows_mixed");
    if (!big && it.fine) paths.insert("rows_shared");
    if (it.part < 0) paths.insert(big ? "big_whole" : "rows_whole");
    if (!big) continue;
    if (it.fine) paths.insert("fine");
    auto& r = runs[{it.tokens, it.row0}];
    r.insert(it.k0);
    const char* kind = G > shape.big_tile ? "huge" : "big";
    if (G > shape.big_tile) paths.insert("huge");
    if (r.size() > 1) paths.insert(std::string(kind) + "_cut");
    if (it.k0 > 0 && mixed) paths.insert(std::string(kind) + "_cut_mixed");
    for (int row = it.row0; row < it.row0 + it.rows; row++)
      if (it.k1 > it.k0 && p.tok_limit[p.lists[it.tokens + row / G]] <= it.k0) paths.insert(std::string(kind) + "_blind");   // a row that sees none of the item's keys
  }
  if (p.most_parts > 96) paths.insert("join16");
  else if (p.most_parts > 32) paths.insert("join4");
  else if (p.most_parts > 0) paths.insert("join1");
  const bool fast = (D == 64 || D == 128 || D == 256) && B % 16 == 0;
  if (fast && !p.mixed && paths.count("rows") && paths.count("big")) paths.insert("both");
  if (fast && !p.mixed && paths.count("rows")) paths.insert("stream");
  for (const std::string& s : paths) std::printf("%s ", s.c_str());
  std::printf("\n");
  return 0;
}
