// Drafted trees on the CPU, under the sanitizers: the plan of batches that have some (batch.hpp), and the two kernels that find out what rows see and
// which path is accepted (tree.hip.inc, unchanged, lane by lane), against plain loops, over random batches.  Device memory is as large as it has to be and
// no larger.
//
// usage: trees_on_cpu SEEDS   (prints "trees ok")
#include "mock_device.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#undef __shared__
#define __shared__ static  // one workgroup at a time, its lanes share it

#include "pool_view.hpp"
#include "attn.hpp"
#include "append.hip.inc"
#include "tree.hip.inc"

#define CHECK(cond, ...)                                                              \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      fprintf(stderr, "seed %d: %s:%d: %s failed ", seed, __FILE__, __LINE__, #cond); \
      fprintf(stderr, __VA_ARGS__);                                                   \
      fprintf(stderr, "\n");                                                          \
      return 1;                                                                       \
    }                                                                                 \
  } while (0)

int main(int argc, char** argv) {
  const int seeds = argc > 1 ? atoi(argv[1]) : 200;
  long masked_pairs = 0, moved = 0, shared_seen = 0, refused = 0;
  for (int seed = 0; seed < seeds; seed++) {
    std::mt19937 rng(seed);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    kvswap::BatchShape s;
    const int Bs[] = {1, 3, 4, 16, 20, 32};
    s.B = Bs[pick(0, 5)];
    s.H = pick(1, 3);
    const int G = pick(0, 9) ? pick(1, 12) : pick(60, 150);
    s.N = 1 << 14;
    s.wgs = pick(0, 1) ? 1024 : pick(1, 64);
    s.big_tile = pick(0, 1) ? 128 : 64;
    s.big_wgs = pick(0, 1) ? 512 : pick(1, 64);
    s.least = pick(0, 1) ? 512 : 128;
    s.big_least = pick(0, 1) ? 512 : 128;
    s.row_tile = pick(0, 1) ? 32 : 16;
    s.row_step = pick(0, 1) ? 32 : 0;
    s.big_step = pick(0, 1) ? 64 : 0;
    const int n = pick(1, 8);
    std::vector<int32_t> off{0}, ids, len, ql;
    std::vector<uint8_t> trees;
    int fresh = 0;
    for (int i = 0; i < n; i++) {
      std::vector<int32_t> row;
      if (i && pick(0, 2)) {  // begins as an earlier one does
        const int o = pick(0, i - 1), have = off[o + 1] - off[o];
        const int take = pick(0, have);
        row.assign(ids.begin() + off[o], ids.begin() + off[o] + take);
      }
      const int l = pick(0, 9) ? (int)row.size() * s.B + pick(0, 250) : 0;
      row.resize(std::min(row.size(), (size_t)((l + s.B - 1) / s.B)));
      while ((int)row.size() * s.B < l) row.push_back(fresh++);
      len.push_back(l);
      trees.push_back(pick(0, 3) != 0);
      ql.push_back(l == 0 ? pick(0, 1) : pick(0, 9) ? pick(1, std::min(l, 70)) : pick(0, std::min(l, 300)));
      ids.insert(ids.end(), row.begin(), row.end());
      off.push_back((int32_t)ids.size());
    }
    if (fresh > s.N) continue;
    kvswap::BatchPlan p;
    CHECK(p.set(n, off.data(), ids.data(), len.data(), ql.data(), G * s.H, s, trees.data()) == KV_OK, " ");
    if (p.T == 0) continue;
    // parents, mostly good ones
    std::vector<int32_t> parents((size_t)p.T);
    for (int i = 0; i < n; i++)
      for (int j = 0; j < ql[i]; j++) {
        const int kind = pick(0, 30);
        parents[p.q_first[i] + j] = kind == 0 ? -2 : kind == 1 ? j : kind == 2 ? INT32_MIN + pick(0, 3) : kind == 3 ? INT32_MAX - pick(0, 3)
                                    : kind < 6 || j == 0 ? -1 : pick(std::max(0, j - (kind < 20 ? 5 : 300)), j - 1);
      }
    // what every row sees, and its depth
    std::vector<std::vector<uint8_t>> sees((size_t)p.T);
    std::vector<int> depth((size_t)p.T, 0), inside((size_t)p.T, 1);
    for (int i = 0; i < n; i++)
      for (int j = 0; j < ql[i]; j++) {
        const int t = p.q_first[i] + j, base = len[i] - ql[i];
        sees[t].assign((size_t)len[i], 0);
        if (len[i] == 0) continue;
        if (!trees[i]) {
          for (int x = 0; x <= base + j; x++) sees[t][x] = 1;
          depth[t] = j;
          continue;
        }
        const int32_t up = parents[t];
        if (up == -1)
          for (int x = 0; x < base; x++) sees[t][x] = 1;
        else if (up >= 0 && up < j && inside[p.q_first[i] + up]) {
          sees[t] = sees[p.q_first[i] + up];
          depth[t] = depth[p.q_first[i] + up] + 1;
        } else
          inside[t] = 0;
        if (inside[t]) sees[t][base + j] = 1;
      }
    // the kernel that finds out
    std::vector<int32_t> parent((size_t)p.T, -99), position((size_t)p.T, -99), limit = p.tok_limit;
    std::vector<uint32_t> bits((size_t)p.tree_words, 0xDEADBEEF);
    {
      TreeArgs a{p.tree_reqs.data(), parents.data(), (p.tree_units + 255) / 256, parent.data(), position.data(), limit.data(), bits.data()};
      if (a.chunks) mockhip::run_grid(dim3((unsigned)(n * a.chunks)), dim3(256), 16, [&] { kv_tree_kernel(a); });
    }
    // the tiles: every pair of a row and a key that it sees once; what it does not see is masked, by a limit or by a bit, where a tile masks at all
    std::vector<std::map<int, int>> seen((size_t)p.T * G);
    for (const auto& it : p.items) {
      const bool big = &it - p.items.data() >= p.big_first;
      CHECK(it.clear >= it.k1 || (big ? p.big_mixed : p.mixed), "mixed");
      for (int r = it.row0; r < it.row0 + it.rows; r++) {
        const int tok = p.lists[it.tokens + r / G], row = tok * G + r % G, req = p.tok_req[tok];
        const kvswap::TreeSight sight = it.tree < 0 ? kvswap::TreeSight{-1, 0} : kvswap::TreeSight{it.tree + (tok - it.tree_first) * it.tree_words, it.tree_origin};
        CHECK(it.tree < 0 || (sight.word == p.tree_sight[tok].word && sight.origin == p.tree_sight[tok].origin), "where the bits of row %d are", tok);
        for (int x = it.k0; x < it.k1; x++) {
          CHECK(p.ids[it.table + x / s.B] == ids[off[req] + x / s.B], "block of key %d", x);
          const bool may = x < limit[tok];
          bool bit = true;
          if (sight.word >= 0 && x >= sight.origin) {
            const int step = big ? 64 : 32;
            CHECK((x - (x - it.k0) % step - sight.origin) % step == 0, "a step does not begin with a word");
            const size_t at = (size_t)sight.word + (x - sight.origin) / 32;
            CHECK(at < bits.size(), "word %zu of %zu", at, bits.size());
            bit = bits[at] >> ((x - sight.origin) % 32) & 1;
          }
          const bool shown = x < it.clear || (may && bit), does = sees[tok][x];
          if (inside[tok]) CHECK(shown == does, "row %d, key %d: %d instead of %d", tok, x, shown, does);
          masked_pairs += !does;
          if (does) seen[row][x]++;
        }
      }
    }
    for (int t = 0; t < p.T; t++) {
      const int req = p.tok_req[t];
      CHECK(position[t] == len[req] - ql[req] + depth[t] || len[req] == 0, "position of row %d", t);
      CHECK(limit[t] == (!len[req] || !inside[t] ? 0 : trees[req] ? len[req] : p.tok_limit[t]), "limit of row %d", t);
      int count = 0;
      for (uint8_t x : sees[t]) count += x;
      for (int g = 0; g < G; g++) {
        CHECK((int)seen[(size_t)t * G + g].size() == count, "row %d sees %zu of %d", t, seen[(size_t)t * G + g].size(), count);
        for (auto& k : seen[(size_t)t * G + g]) CHECK(k.second == 1, "key %d %d times", k.first, k.second);
      }
    }
    shared_seen += p.read < p.cached;
    // is a tail in two tables?
    std::map<int, int> times;
    for (int32_t x : p.ids) times[x]++;
    bool twice = false;
    for (int i = 0; i < n; i++)
      if (trees[i] && ql[i] > 1)
        for (int k = (len[i] - ql[i]) / s.B; k < (len[i] + s.B - 1) / s.B; k++) twice = twice || times[ids[off[i] + k]] > 1;
    CHECK(twice == p.tree_tails_shared, "shared tails");
    refused += twice;
    if (twice) continue;
    // the accepted path, and the move: rows of `row` bytes in blocks of their own
    const int vec = pick(0, 1) ? 16 : 8, row = vec * (pick(0, 4) ? pick(1, 40) : pick(250, 700)), layers = pick(1, 2);
    const int64_t block = (int64_t)row * s.B, plane = block * std::max(fresh, 1);
    std::vector<char> pool((size_t)(plane * 2 * layers));
    for (char& c : pool) c = (char)rng();
    std::vector<int32_t> tokens((size_t)p.T), chosen((size_t)p.T), count((size_t)n, -9), next((size_t)n, -9);
    for (int32_t& x : tokens) x = pick(0, 3);
    for (int32_t& x : chosen) x = pick(0, 3);
    int most = 1;
    for (int i = 0; i < n; i++)
      if (trees[i]) most = std::max(most, ql[i]);
    std::vector<int32_t> path((size_t)n * most, -9);
    std::vector<float> weights((size_t)layers * n * s.H * std::max(1, *std::max_element(len.begin(), len.end())));
    const int64_t cap = (int64_t)weights.size() / layers / n / s.H;
    for (float& x : weights) x = (float)pick(1, 1000);
    std::vector<char> want = pool;
    std::vector<float> wwant = weights;
    std::vector<int> wcount, wnext;
    for (int i = 0; i < n; i++) {
      const int f = p.q_first[i], base = len[i] - ql[i];
      std::vector<int> way;
      if (!trees[i] || len[i] == 0) {
        wcount.push_back(len[i] ? ql[i] : 0);
        wnext.push_back(len[i] && ql[i] ? chosen[f + ql[i] - 1] : -1);
        continue;
      }
      for (int u = ql[i] && inside[f] ? 0 : -1; u >= 0;) {
        way.push_back(u);
        int to = -1;
        for (int j = u + 1; j < ql[i] && to < 0; j++)
          if (inside[f + j] && parents[f + j] == u && tokens[f + j] == chosen[f + u]) to = j;
        u = to;
      }
      wcount.push_back((int)way.size());
      wnext.push_back(way.empty() ? -1 : chosen[f + way.back()]);
      for (size_t k = 0; k < way.size(); k++) {
        const int x = base + way[k], y = base + (int)k;
        moved += way[k] != (int)k;
        for (int l = 0; l < layers * 2; l++)
          std::memcpy(want.data() + l * plane + ids[off[i] + y / s.B] * block + (int64_t)(y % s.B) * row,
                      pool.data() + l * plane + ids[off[i] + x / s.B] * block + (int64_t)(x % s.B) * row, (size_t)row);
      }
      for (int l = 0; l < layers; l++)
        for (int h = 0; h < s.H; h++)
          for (int k = 0; k < ql[i]; k++) {
            const int64_t at = ((int64_t)(l * n + i) * s.H + h) * cap + base;
            wwant[at + k] = k < (int)way.size() ? weights[at + way[k]] : 0.f;
          }
    }
    AcceptArgs a{};
    a.reqs = p.tree_reqs.data();
    a.parent = parent.data();
    a.tokens = tokens.data();
    a.chosen = chosen.data();
    a.q_first = p.q_first.data();
    a.len = p.len.data();
    a.off = p.off.data();
    a.table = p.ids.data();
    a.count = count.data();
    a.path = path.data();
    a.next = next.data();
    a.path_stride = most;
    a.n = n;
    a.layers = layers;
    a.H = s.H;
    a.B = s.B;
    a.pool = pool.data();
    a.ls = 2 * plane;
    a.vk = plane;
    a.bs = block;
    a.row = row;
    a.groups = pick(1, 2 * layers);
    a.cols = (row / vec + 255) / 256;
    a.vecs = (row / vec + a.cols - 1) / a.cols;
    a.weights = weights.data();
    a.ws[0] = cap * s.H * n;
    a.ws[1] = cap * s.H;
    a.ws[2] = cap;
    auto run = [&](auto kern) { mockhip::run_grid(dim3((unsigned)(a.groups * n * a.cols)), dim3(256), 16, [&] { kern(a); }); };
    if (pick(0, 1))
      vec == 16 ? run(kv_accept_kernel<u32x4, false, 1>) : run(kv_accept_kernel<u32x2, false, 1>);
    else
      vec == 16 ? run(kv_accept_kernel<u32x4, false, 2>) : run(kv_accept_kernel<u32x2, false, 2>);
    for (int i = 0; i < n; i++) CHECK(count[i] == wcount[i] && next[i] == wnext[i], "request %d: %d rows, then %d, instead of %d, %d", i, count[i], next[i], wcount[i], wnext[i]);
    CHECK(pool == want, "the pool");
    CHECK(weights == wwant, "the weights");
  }
  // the join's launch: a row of its own lanes for every head of every token, and never more lanes than 32 bits count
  for (int64_t T : {1ll, 1000ll, 16777215ll, 16777216ll, 20000000ll, 500000000ll})
    for (int heads : {1, 3, 8, 64, 128})
      for (int D : {8, 64, 72, 128, 136, 256}) {
        const int seed = -1;  // (none)
        const int64_t wgs = join_few_wgs(T, heads, D);
        CHECK(wgs * 256 <= UINT32_MAX, "%ld tokens of %d heads of %d: %ld workgroups", (long)T, heads, D, (long)wgs);
        if (T <= 1000) CHECK(wgs == T * join_few_chunks(heads, D) && wgs * 256 >= T * heads * join_few_stride(D) && join_few_stride(D) * 4 >= D, "%ld workgroups", (long)wgs);
      }
  if (!masked_pairs || !moved || !shared_seen || !refused) return fprintf(stderr, "nothing was looked at: %ld %ld %ld %ld\n", masked_pairs, moved, shared_seen, refused), 1;
  printf("trees ok\n");
  return 0;
}
