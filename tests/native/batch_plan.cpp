// The attention's plan (batch.hpp) against what it has to cover: over random batches with shared prefixes, every (row, key it sees)
// pair is in exactly one item, by the right block; no key outside a row's sight is left unmasked; every partial row belongs to one (item,
// row), and each row's list for the join names exactly its own.  Exits 0 when all of it holds.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>

#include "../../paper_2510_02758_amd/csrc/batch.hpp"

#define CHECK(cond, ...)                                                       \
  do {                                                                         \
    if (!(cond)) {                                                             \
      fprintf(stderr, "seed %d: %s:%d: %s failed ", seed, __FILE__, __LINE__, #cond); \
      fprintf(stderr, __VA_ARGS__);                                            \
      fprintf(stderr, "\n");                                                   \
      return 1;                                                                \
    }                                                                          \
  } while (0)

int main(int argc, char** argv) {
  const int seeds = argc > 1 ? atoi(argv[1]) : 400;
  long shared_nodes = 0, joined = 0, direct = 0, dealt = 0, big_dealt = 0;
  for (int seed = 0; seed < seeds; seed++) {
    std::mt19937 rng(seed);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    kvswap::BatchShape s;
    const int Bs[] = {1, 3, 4, 16, 20, 32};
    s.B = Bs[pick(0, 5)];
    s.H = pick(1, 4);
    const int G = pick(0, 9) ? pick(1, 20) : pick(60, 150);
    s.N = 1 << 20;
    s.wgs = pick(0, 1) ? 1024 : pick(1, 64);
    s.big_tile = pick(0, 1) ? 128 : 64;
    s.big_wgs = pick(0, 1) ? 512 : pick(1, 64);
    s.least = pick(0, 1) ? 512 : 128;
    s.big_least = pick(0, 1) ? 512 : 128;
    const int n = pick(0, 12);
    std::vector<int32_t> off{pick(0, 3)}, ids((size_t)off[0], -7), len, ql;
    int fresh = 0;
    for (int i = 0; i < n; i++) {
      std::vector<int32_t> row;
      if (i && pick(0, 2)) {  // begins as an earlier one does
        const int o = pick(0, i - 1);
        const int have = off[o + 1] - off[o], take = pick(0, have);
        row.assign(ids.begin() + off[o], ids.begin() + off[o] + take);
      }
      for (int k = pick(0, 200 / s.B + 2); k > 0; k--) row.push_back(fresh++);
      const int most = (int)row.size() * s.B;
      const int l = most ? std::max(0, most - pick(0, std::min(most, 2 * s.B))) : 0;
      len.push_back(l);
      ql.push_back(l == 0 ? pick(0, 1) : pick(0, 3) ? 1 : pick(0, std::min(l, 40)));
      ids.insert(ids.end(), row.begin(), row.end());
      off.push_back((int32_t)ids.size());
    }
    kvswap::BatchPlan p;
    const int rc = p.set(n, off.data(), ids.data(), len.data(), ql.data(), G * s.H, s);
    CHECK(rc == KV_OK, "%d", rc);
    std::vector<std::map<int, int>> seen((size_t)p.T * G);  // row -> key -> times
    std::map<int, int> part_row;                          // partial row -> row
    std::vector<int> finished((size_t)p.T * G, 0);
    for (const auto& it : p.items) {
      const bool big = &it - p.items.data() >= p.big_first;
      CHECK(it.rows >= 1 && it.rows <= (big ? s.big_tile : p.kRowTile), "rows %d", it.rows);
      CHECK(it.clear >= it.k1 || (big ? p.big_mixed : p.mixed), "mixed");
      CHECK(it.k0 >= 0 && it.k1 >= it.k0, "keys %d %d", it.k0, it.k1);
      if (it.k1 > it.k0) {
        const int b0 = it.k0 / s.B, b1 = (it.k1 - 1) / s.B;
        CHECK(b1 - b0 + 1 <= kvswap::BatchPlan::kMaxEntries, "%d entries", b1 - b0 + 1);
        CHECK(it.table + b1 < (int)p.ids.size(), "table");
      }
      for (int r = it.row0; r < it.row0 + it.rows; r++) {
        CHECK(it.tokens + r / G < (int)p.lists.size(), "list");
        const int tok = p.lists[it.tokens + r / G], row = tok * G + r % G, req = p.tok_req[tok];
        for (int x = it.k0; x < it.k1; x++) {
          const bool masked = x >= p.tok_limit[tok];
          CHECK(!masked || x >= it.clear, "key %d is not masked", x);
          if (masked) continue;
          CHECK(p.ids[it.table + x / s.B] == ids[off[req] + x / s.B], "block of key %d", x);
          seen[row][x]++;
        }
        if (it.part >= 0) {
          const int pr = it.part + r - it.row0;
          CHECK(pr < p.partial_rows && !part_row.count(pr), "partial row %d", pr);
          part_row[pr] = row;
        } else {
          finished[row]++;
        }
      }
    }
    for (int t = 0; t < p.T; t++) {
      const int req = p.tok_req[t], limit = len[req] ? len[req] - ql[req] + (t - p.q_first[req]) + 1 : 0;
      CHECK(limit == p.tok_limit[t], "limit");
      const auto& at = p.places[t];
      CHECK(at.index == limit - 1 && at.block == (limit ? ids[off[req] + (limit - 1) / s.B] : -1) && at.place == (limit ? (limit - 1) % s.B : 0), "place");
      const int nj = p.join_off[t + 1] - p.join_off[t];
      for (int g = 0; g < G; g++) {
        const int row = t * G + g;
        CHECK((int)seen[row].size() == limit, "row %d sees %zu of %d", row, seen[row].size(), limit);
        for (auto& k : seen[row]) CHECK(k.second == 1 && k.first < limit, "key %d %d times", k.first, k.second);
        CHECK(finished[row] == (nj ? 0 : 1), "row %d finished %d times, %d partial", row, finished[row], nj);
        std::set<int> mine, listed;
        for (auto& x : part_row)
          if (x.second == row) mine.insert(x.first);
        for (int k = p.join_off[t]; k < p.join_off[t + 1]; k++) listed.insert(p.join[k] + g);
        CHECK(mine == listed && (int)listed.size() == nj, "join of row %d", row);
        nj ? joined++ : direct++;
      }
    }
    CHECK((p.heads == 1 || p.heads == 2 || p.heads == 4) && s.H % p.heads == 0, "%d heads of %d", p.heads, s.H);
    // every row tile's item has its workgroup
    CHECK(p.wg_items.size() >= 1 && p.wg_items.back() == p.big_first, "workgroups");
    for (size_t k = 0; k + 1 < p.wg_items.size(); k++) CHECK(p.wg_items[k] < p.wg_items[k + 1] && (k || p.wg_items[0] == 0), "workgroup %zu", k);
    CHECK(p.wg_big.size() >= 1 && p.wg_big[0] == p.big_first && p.wg_big.back() == (int)p.items.size(), "workgroups of big tiles");
    for (size_t k = 0; k + 1 < p.wg_big.size(); k++) {
      CHECK(p.wg_big[k] < p.wg_big[k + 1], "workgroup %zu of big tiles", k);
      big_dealt += p.wg_big[k + 1] - p.wg_big[k] > 1;
    }
    for (size_t k = 0; k + 1 < p.wg_items.size(); k++) dealt += p.wg_items[k + 1] - p.wg_items[k] > 1;
    int64_t cached = 0;
    for (int i = 0; i < n; i++)
      if (ql[i]) cached += len[i];
    CHECK(p.read <= cached, "reads %lld of %lld", (long long)p.read, (long long)cached);
    shared_nodes += p.read < cached;
    // kept products: every (row, key) of a row tile has a place of its own, and each request's keys are summed once, from
    // kept products by the places that its rows wrote, or computed again
    std::map<int64_t, std::pair<int, int>> place;  // -> (row, key)
    for (int n2 = 0; n2 < p.big_first; n2++) {
      const auto& it = p.items[n2];
      for (int r = 0; r < it.rows; r++)
        for (int x = it.k0; x < it.k1; x++) {
          const int64_t at = (int64_t)it.score * 16 + (int64_t)r * it.score_row + x - it.score_from;
          CHECK(at >= 0 && at < p.scores && !place.count(at) && it.score_row % 16 == 0 && x - it.score_from < it.score_row, "place of a product");
          place[at] = {p.lists[it.tokens + (it.row0 + r) / G] * G + (it.row0 + r) % G, x};
        }
    }
    std::vector<std::map<int, int>> summed((size_t)n);
    for (const auto& it : p.sitems) {
      CHECK(it.k1 - it.k0 <= p.kScoreKeys && (it.k0 - it.score_from) % 4 == 0 && it.rows == ql[it.req] * G, "score item");
      for (int x = it.k0; x < it.k1; x++) {
        summed[it.req][x]++;
        for (int r = 0; r < it.rows; r++) {
          const auto f = place.find((int64_t)it.score * 16 + (int64_t)(it.row0 + r) * it.score_row + x - it.score_from);
          CHECK(f != place.end() && f->second == std::make_pair(p.q_first[it.req] * G + r, x), "product of row %d, key %d", r, x);
        }
      }
    }
    for (const auto& it : p.wrest)
      for (int k = it.first; k < it.first + it.count; k++)
        for (int x = it.k0; x < it.k1; x++) summed[p.wreqs[k]][x]++;
    for (int i = 0; i < n; i++) {
      CHECK((int)summed[i].size() == (ql[i] ? len[i] : 0), "keys of %d summed", i);
      for (auto& k : summed[i]) CHECK(k.second == 1 && k.first < len[i], "key %d of %d summed %d times", k.first, i, k.second);
    }
    // weight items: every key of a request with rows once
    std::vector<std::map<int, int>> w((size_t)n);
    for (const auto& it : p.witems) {
      CHECK(it.k1 > it.k0 && it.k1 - it.k0 <= p.kWeightKeys && it.count >= 1 && it.first + it.count <= (int)p.wreqs.size(), "weight item");
      for (int k = it.first; k < it.first + it.count; k++)
        for (int x = it.k0; x < it.k1; x++) {
          CHECK(p.ids[it.table + x / s.B] == ids[off[p.wreqs[k]] + x / s.B], "block of key %d of %d", x, p.wreqs[k]);
          w[p.wreqs[k]][x]++;
        }
    }
    for (int i = 0; i < n; i++) {
      CHECK((int)w[i].size() == (ql[i] ? len[i] : 0), "weights of %d", i);
      for (auto& k : w[i]) CHECK(k.second == 1 && k.first < len[i], "weight of key %d", k.first);
    }
  }
  if (!shared_nodes || !joined || !direct || !dealt || !big_dealt) {
    fprintf(stderr, "the batches do not reach every kind: %ld shared, %ld joined, %ld direct, %ld and %ld dealt\n", shared_nodes, joined, direct, dealt, big_dealt);
    return 1;
  }
  printf("plans ok: %ld batches with shared keys, %ld rows joined, %ld finished at once\n", shared_nodes, joined, direct);
  return 0;
}
