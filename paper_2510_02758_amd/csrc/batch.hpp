// Host side of a batch (kv_batch_set): checks the tables and lays out the attention's work.  Pure C++ (no HIP), as planner.hpp.
//
// Requests whose tables begin with the same blocks share a prefix.  The tables form a tree: every node is a run of blocks that a set
// of requests has in common behind its parent's, a leaf what a request has for itself.  Attention over a node's keys is one
// product with the queries of all its requests; what a row got at the nodes on its way down is joined by its softmax
// statistics.  Only blocks that lie in front of every new token of all their requests go to shared nodes, so no row of one needs a mask.
#pragma once

#include <algorithm>
#include <cstdint>
#include <unordered_map>
#include <utility>
#include <vector>

#include "../../include/kvswap.h"

namespace kvswap {

// One piece of attention work for one KV head: a tile of rows against a run of keys.
// Row r of a node is new token tokens[first + r / G] with query head r % G of the group.
struct AttnItem {
  int32_t table;    // where the row of the table begins that names the blocks of the keys
  int32_t k0, k1;   // keys [k0, k1), as indices of that row's request
  int32_t clear;    // keys below are seen by every row of the tile
  int32_t tokens;   // the node's list of tokens
  int32_t row0, rows;
  int32_t part;     // partial row of row0; -1: the rows are finished here
};
// One piece of weight accumulation: keys [k0, k1) of a request.
struct WeightItem {
  int32_t req, k0, k1, pad;
};

struct BatchShape {
  int32_t H = 1, G = 1, B = 1;
  int64_t N = 0;
  int wgs = 1024;       // workgroups that fill the device
};

class BatchPlan {
 public:
  int32_t n = 0, T = 0, G = 1;
  int64_t cached = 0, read = 0;
  std::vector<int32_t> off, ids, len, q_len, q_first;        // per request (off, q_first: n + 1)
  std::vector<int32_t> tok_req, tok_limit;                   // per row of the tensors: request, keys it sees
  std::vector<int32_t> lists;                                // the nodes' tokens
  std::vector<AttnItem> items;
  std::vector<int32_t> join_off, join;                       // per token: partial rows of its first query head
  std::vector<WeightItem> witems;
  int32_t partial_rows = 0;
  bool mixed = false;  // some item has keys that some of its rows see and others do not

  // Entries of the table that an item may need: its part of the table is held on chip.
  static constexpr int32_t kMaxEntries = 2048;
  static constexpr int32_t kTile = 16;  // rows of an item
  static constexpr int32_t kWeightKeys = 512;

  int set(int32_t n_, const int32_t* offsets, const int32_t* blocks, const int32_t* tokens, const int32_t* q_lens, int32_t num_q_heads,
          const BatchShape& s) {
    if (n_ < 0 || num_q_heads <= 0 || num_q_heads % s.H) return KV_EINVAL;
    if (n_ && (!offsets || !tokens || !q_lens || offsets[0] < 0)) return KV_EINVAL;
    int64_t rows = 0, keys = 0, table = 0;
    for (int32_t i = 0; i < n_; i++) {
      if (offsets[i + 1] < offsets[i] || tokens[i] < 0 || q_lens[i] < 0) return KV_EINVAL;
      if (q_lens[i] > tokens[i] && !(tokens[i] == 0 && q_lens[i] == 1)) return KV_EINVAL;
      const int64_t need = ((int64_t)tokens[i] + s.B - 1) / s.B;
      if ((int64_t)offsets[i + 1] - offsets[i] < need) return KV_EINVAL;
      rows += q_lens[i];
      keys += tokens[i];
      table += need;
    }
    const int32_t g = num_q_heads / s.H;
    if (rows * g > INT32_MAX / 4 || table > INT32_MAX) return KV_EINVAL;
    if (table && !blocks) return KV_EINVAL;
    for (int32_t i = 0; i < n_; i++) {
      const int64_t need = ((int64_t)tokens[i] + s.B - 1) / s.B;
      for (int64_t k = offsets[i]; k < offsets[i] + need; k++)
        if (blocks[k] < 0 || blocks[k] >= s.N) return KV_ERANGE;
    }
    // nothing fails from here on but allocation: a batch that could not be set describes nothing
    n = T = 0;
    try {
      lay_out(n_, offsets, blocks, tokens, q_lens, g, (int32_t)rows, keys, (size_t)table, s);
    } catch (...) {
      n = T = 0;
      throw;
    }
    return KV_OK;
  }

  // Would rewriting blocks [first_block, keep_blocks) of the requests with more than `keep` tokens reach a block that the batch has twice?
  bool rewrites_shared(int32_t keep, int32_t first_block, int32_t keep_blocks) const {
    std::vector<int32_t> sorted(ids);
    std::sort(sorted.begin(), sorted.end());
    for (int32_t i = 0; i < n; i++) {
      if (len[i] <= keep) continue;
      for (int32_t k = off[i] + first_block; k < off[i] + keep_blocks; k++) {
        const auto r = std::equal_range(sorted.begin(), sorted.end(), ids[k]);
        if (r.second - r.first > 1) return true;
      }
    }
    return false;
  }

 private:
  struct Node {
    std::vector<int32_t> reqs;
    int32_t from, to;  // keys
  };

  void lay_out(int32_t n_, const int32_t* offsets, const int32_t* blocks, const int32_t* tokens, const int32_t* q_lens, int32_t g, int32_t rows,
               int64_t keys, size_t table, const BatchShape& s) {
    G = g;
    cached = keys;
    len.assign(tokens, tokens + n_);
    q_len.assign(q_lens, q_lens + n_);
    off.assign(1, 0);
    q_first.assign(1, 0);
    ids.clear();
    ids.reserve(table);
    tok_req.clear();
    tok_limit.clear();
    tok_req.reserve(rows);
    tok_limit.reserve(rows);
    for (int32_t i = 0; i < n_; i++) {
      const int32_t need = (int32_t)(((int64_t)tokens[i] + s.B - 1) / s.B);
      ids.insert(ids.end(), blocks + offsets[i], blocks + offsets[i] + need);
      off.push_back((int32_t)ids.size());
      q_first.push_back(q_first.back() + q_lens[i]);
      for (int32_t j = 0; j < q_lens[i]; j++) {
        tok_req.push_back(i);
        tok_limit.push_back(tokens[i] ? tokens[i] - q_lens[i] + j + 1 : 0);
      }
    }
    n = n_;
    T = rows;
    find_nodes(s.B);
    cut(s);
    cut_weights();
  }

  // Blocks of request i that every one of its rows sees whole.
  int32_t open_blocks(int32_t i, int32_t B) const { return len[i] ? (len[i] - q_len[i] + 1) / B : 0; }

  std::vector<Node> nodes_;

  void find_nodes(int32_t B) {
    nodes_.clear();
    struct Work {
      std::vector<int32_t> reqs;
      int32_t from, at;  // blocks in front of `from` are done with, those in front of `at` are known to be the same
    };
    std::vector<Work> todo(1);
    todo[0].from = todo[0].at = 0;
    for (int32_t i = 0; i < n; i++)
      if (q_len[i]) todo[0].reqs.push_back(i);
    std::vector<std::pair<int32_t, int32_t>> next;  // (block at the fork, request)
    while (!todo.empty()) {
      Work w = std::move(todo.back());
      todo.pop_back();
      int32_t at = w.at;
      if (w.reqs.size() > 1) {
        int32_t most = INT32_MAX;
        for (int32_t i : w.reqs) most = std::min(most, open_blocks(i, B));
        const int32_t* a = ids.data() + off[w.reqs[0]];
        if (w.at > 0)
          for (size_t k = 1; k < w.reqs.size() && most > at; k++) {
            const int32_t* b = ids.data() + off[w.reqs[k]];
            int32_t x = at;
            while (x < most && a[x] == b[x]) x++;
            most = x;
          }
        else
          most = 0;  // the root has no block yet
        at = std::max(at, most);
        // A node costs its rows a partial result each; it is worth it from kShared tokens on that it spares.
        if ((int64_t)(at - w.from) * B * (int64_t)(w.reqs.size() - 1) >= kShared) {
          nodes_.push_back({w.reqs, w.from * B, at * B});
          w.from = at;
        }
      }
      next.clear();
      for (int32_t i : w.reqs) {
        if (w.reqs.size() > 1 && at < open_blocks(i, B))
          next.push_back({ids[off[i] + at], i});
        else
          nodes_.push_back({{i}, w.from * B, len[i]});
      }
      std::stable_sort(next.begin(), next.end(), [](const auto& x, const auto& y) { return x.first < y.first; });
      for (size_t k = 0; k < next.size();) {
        size_t e = k;
        while (e < next.size() && next[e].first == next[k].first) e++;
        Work child;
        child.from = w.from;
        child.at = at + 1;
        for (size_t j = k; j < e; j++) child.reqs.push_back(next[j].second);
        if (child.reqs.size() == 1)
          nodes_.push_back({child.reqs, w.from * B, len[child.reqs[0]]});
        else
          todo.push_back(std::move(child));
        k = e;
      }
    }
  }
  static constexpr int64_t kShared = 128;

  void cut(const BatchShape& s) {
    lists.clear();
    items.clear();
    mixed = false;
    struct Tile {
      int32_t node, list, row0, rows, limit, clear;
    };
    std::vector<Tile> tiles;
    std::vector<int32_t> seen((size_t)T, 0);  // nodes with keys, per token
    read = 0;
    int64_t work = 0;
    for (size_t d = 0; d < nodes_.size(); d++) {
      const Node& node = nodes_[d];
      const int32_t list = (int32_t)lists.size();
      for (int32_t i : node.reqs)
        for (int32_t t = q_first[i]; t < q_first[i + 1]; t++) lists.push_back(t);
      read += node.to - node.from;
      const int64_t rows = (int64_t)((int32_t)lists.size() - list) * G;
      for (int64_t r = 0; r < rows; r += kTile) {
        Tile t{(int32_t)d, list, (int32_t)r, (int32_t)std::min<int64_t>(kTile, rows - r), 0, INT32_MAX};
        for (int64_t j = r / G; j <= (r + t.rows - 1) / G; j++) {
          const int32_t limit = std::min(node.to, tok_limit[lists[list + j]]);
          t.limit = std::max(t.limit, limit);
          t.clear = std::min(t.clear, limit);
        }
        work += std::max(t.limit - node.from, 0);
        tiles.push_back(t);
      }
      for (size_t j = list; j < lists.size(); j++)
        if (node.to > node.from) seen[lists[j]]++;
    }
    // Equal runs of keys, so many that the device is full.
    int64_t chunk = (work * s.H + s.wgs - 1) / s.wgs;
    const int64_t most = std::min<int64_t>((int64_t)(kMaxEntries - 1) * s.B, INT32_MAX / 2) / kStep * kStep;
    chunk = std::min<int64_t>(most, std::max<int64_t>(kLeast, (chunk + kStep - 1) / kStep * kStep));
    // Rows that end up in a single piece need no partial results: that holds for a whole node or not at all.
    std::vector<std::vector<std::pair<int32_t, int32_t>>> parts;  // per node: (partial row of its first row, pieces)
    partial_rows = 0;
    std::vector<int32_t> count((size_t)T, 0);
    struct Use {
      int32_t list, tokens, part;
    };
    std::vector<Use> uses;
    for (size_t k = 0; k < tiles.size();) {
      size_t e = k;
      while (e < tiles.size() && tiles[e].node == tiles[k].node) e++;
      const Node& node = nodes_[tiles[k].node];
      int32_t pieces = 1;
      bool alone = true;
      for (size_t j = k; j < e; j++)
        pieces = std::max<int32_t>(pieces, (int32_t)((std::max(tiles[j].limit - node.from, 0) + chunk - 1) / chunk));
      const int32_t ntok = (tiles[e - 1].row0 + tiles[e - 1].rows) / G;
      for (int32_t j = 0; j < ntok; j++) alone = alone && seen[lists[tiles[k].list + j]] <= 1;
      const bool empty = node.to <= node.from;
      if (empty && !alone_empty(seen, tiles[k].list, ntok)) {  // its rows have all they see at other nodes
        k = e;
        continue;
      }
      const bool direct = pieces == 1 && alone;
      // every tile is cut at the same keys, so that partial rows of a piece are a run
      const int32_t span = node.to - node.from;
      const int32_t step = pieces > 1 ? (int32_t)(((span + pieces - 1) / pieces + kStep - 1) / kStep * kStep) : span;
      for (int32_t c = 0; c < pieces; c++) {
        const int32_t k0 = node.from + (int32_t)std::min<int64_t>(span, (int64_t)c * step);
        const int32_t k1 = c + 1 < pieces ? node.from + (int32_t)std::min<int64_t>(span, (int64_t)(c + 1) * step) : node.to;
        if (c && k0 >= k1) break;
        const int32_t part = direct ? -1 : partial_rows;
        if (!direct) {
          partial_rows += ntok * G;
          uses.push_back({tiles[k].list, ntok, part});
        }
        for (size_t j = k; j < e; j++) {
          const Tile& t = tiles[j];
          items.push_back({off[node.reqs[0]], k0, std::max(k0, std::min(k1, t.limit)), std::min(k1, t.clear), t.list, t.row0, t.rows,
                           direct ? -1 : part + t.row0});
          mixed = mixed || items.back().clear < items.back().k1;
        }
      }
      k = e;
    }
    join_off.assign((size_t)T + 1, 0);
    for (const Use& u : uses)
      for (int32_t j = 0; j < u.tokens; j++) join_off[lists[u.list + j] + 1]++;
    for (int32_t t = 0; t < T; t++) join_off[t + 1] += join_off[t];
    join.assign((size_t)join_off[T], 0);
    std::vector<int32_t> at(join_off.begin(), join_off.end() - 1);
    for (const Use& u : uses)
      for (int32_t j = 0; j < u.tokens; j++) join[at[lists[u.list + j]]++] = u.part + j * G;
  }
  static constexpr int32_t kLeast = 128, kStep = 128;

  bool alone_empty(const std::vector<int32_t>& seen, int32_t list, int32_t ntok) const {
    for (int32_t j = 0; j < ntok; j++)
      if (seen[lists[list + j]] == 0) return true;
    return false;
  }

  void cut_weights() {
    witems.clear();
    for (int32_t i = 0; i < n; i++)
      for (int32_t k = 0; q_len[i] && k < len[i]; k += kWeightKeys) witems.push_back({i, k, std::min(len[i], k + kWeightKeys), 0});
  }
};

}  // namespace kvswap
