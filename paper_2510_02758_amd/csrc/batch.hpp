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

// One piece of attention work for one KV head: a tile of rows against a run of keys.  Nodes of few rows are tiles of their own (at
// most kRowTile rows), nodes of more rows are cut into big tiles; either kind is dealt out to workgroups in even shares of keys.
// Row r of a node is new token tokens[first + r / G] with query head r % G of the group.
struct AttnItem {
  int32_t table;    // where the row of the table begins that names the blocks of the keys
  int32_t k0, k1;   // keys [k0, k1), as indices of that row's request
  int32_t clear;    // keys below are seen by every row of the tile
  int32_t tokens;   // the node's list of tokens
  int32_t row0, rows;
  int32_t part;     // partial row of row0; -1: the rows are finished here
  // Row tiles: where the products of the tile's rows and keys go if they are wanted: row r (of 16), key x at 16 score + r score_row + x - score_from.
  int32_t score, score_row, score_from;
  int32_t fine;  // keys that several requests share.  In big tiles their weights are as precise as in row tiles, whatever these requests' number
};
// One piece of weight accumulation whose products are computed again: keys [k0, k1) that `count` requests have in common, for the
// rows of these, requests wreqs[first ..].
struct WeightItem {
  int32_t table, k0, k1, first, count, pad[3];
};
// The same from products that were kept: the request's rows are row0 .. row0+rows-1 of their tile.
struct ScoreItem {
  int32_t req, k0, k1, score, score_row, score_from, row0, rows;
};

// Where a new token goes: place `place` of block `block` (-1: nowhere), cache index `index`.
struct TokenPlace {
  int32_t block, place, index, pad;
};

struct BatchShape {
  int32_t H = 1, G = 1, B = 1;
  int64_t N = 0;
  int wgs = 512;        // workgroups of row tiles that are to run at a time
  int least = 512;      // keys below which a run is not cut for their sake
  int big_wgs = 512;    // the same two for big tiles
  int big_least = 512;
  int big_tile = 128;   // rows of a big tile
  int big_cu = 2;       // workgroups of big tiles that share a CU
  int key_rows = 50;    // rows of partial results, of all heads, that cost as much as a workgroup's time for one key
  // A prefix is shared from so many tokens on, by rows of one row tile and by more rows; the latter if all of them together spare `spared` tokens.
  int few_prefix = 64, big_prefix = 64;
  int64_t spared = 0;
};

// Rows of a big tile: what a wavefront's registers hold of their outputs.
constexpr int big_tile(int D) { return D <= 128 ? 128 : 64; }

// What a pool's batches are laid out for on a GPU of `cus` compute units.  Two workgroups of row tiles a CU: with three, more places of the pool are
// read at a time, and each more slowly (64 requests of 512 to 4096 tokens on 8 heads of 128 in bf16: 103 us with two, 122 with three, 140 with
// one; 32 of 256 to 8192 on 32 heads in fp8: 181, 185, 242).
inline BatchShape batch_shape(int32_t H, int32_t D, int32_t B, int64_t N, int cus, bool fp8) {
  BatchShape s;
  s.H = H;
  s.B = B;
  s.N = N;
  s.wgs = cus * 2;
  s.big_cu = D <= 128 ? 2 : 1;
  s.big_wgs = cus * s.big_cu;
  s.key_rows = fp8 ? 100 : 50;
  // Sharing a prefix costs a join of partial results (3 to 5 us), and for more than 16 rows big tiles, which take 25 us (fp8: 30) however little there is
  // to do; and repeated reads of a short prefix come from the caches.  Decode steps, 8 heads of 128 with 4 query heads each, prefix shared / read by each
  // request, bf16 us, then fp8.  Up to 16 rows: 2 requests behind 256 tokens 11.5 / 9.7, 11.0 / 8.6, behind 1024 13.2 / 12.4, 13.2 / 12.3; 32 pairs
  // behind 256 59.3 / 60.7, 36.8 / 37.4, 32 fours behind 512 68 / 73, 47 / 42, behind 1024 63 / 104, 39 / 58.  More rows: 8 requests behind 1024 25 / 16,
  // 30 / 14, behind 8192 27 / 46, 31 / 32; 32 behind 1024 30 / 23, 34 / 19, behind 2048 31 / 37, 35 / 31, behind 4096 32 / 70, 37 / 46; 128 behind 512
  // 60 / 47, 46 / 38, behind 1024 62 / 61, 51 / 48, behind 2048 67 / 89, 53 / 72; 8 eights behind 1024 36 / 44, 36 / 33.  So: from 512 tokens, and from
  // 1024 where what is spared would take 35 us to read at 6.6 TB/s (57000 tokens of these in bf16).
  s.few_prefix = 512;
  s.big_prefix = 1024;
  s.spared = (int64_t)230000000 / (2 * (int64_t)H * D * (fp8 ? 1 : 2));
  s.big_tile = big_tile(D);
  return s;
}

class BatchPlan {
 public:
  int32_t n = 0, T = 0, G = 1;
  int64_t cached = 0, read = 0;
  std::vector<int32_t> off, ids, len, q_len, q_first;        // per request (off, q_first: n + 1)
  std::vector<int32_t> tok_req, tok_limit;                   // per row of the tensors: request, keys it sees
  std::vector<TokenPlace> places;                            // per row
  std::vector<int32_t> lists;                                // the nodes' tokens
  std::vector<AttnItem> items;                               // first those of row tiles, workgroup by workgroup, then those of big tiles
  std::vector<int32_t> wg_items, wg_big;                     // where each workgroup's items begin, and their end
  int32_t heads = 1;                                         // heads of a workgroup of row tiles: 1, 2 or 4
  int32_t big_first = 0;                                     // first item of a big tile
  std::vector<int32_t> join_off, join;                       // per token: partial rows of its first query head
  // Weights: of all keys from products computed again; or of row tiles' keys from kept ones, and of the others computed again.
  std::vector<WeightItem> witems, wrest;
  std::vector<int32_t> wreqs;
  std::vector<ScoreItem> sitems;
  int64_t scores = 0;                                        // kept products of one KV head
  int32_t partial_rows = 0, most_parts = 0;
  bool mixed = false, big_mixed = false;  // some row tile (big tile) has keys that some of its rows see and others do not

  // Entries of the table that an item may need: its part of the table is held on chip.
  static constexpr int32_t kMaxEntries = 2048;
  static constexpr int32_t kRowTile = 16;
  static constexpr int32_t kWeightKeys = 256, kWeightReqs = 16, kScoreKeys = 1024;

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
    if (rows * g > INT32_MAX / 4 || table > INT32_MAX || (keys + 16 * (int64_t)n_) * kRowTile / 16 > INT32_MAX) return KV_EINVAL;
    if (table && !blocks) return KV_EINVAL;
    for (int32_t i = 0; i < n_; i++) {
      const int64_t need = ((int64_t)tokens[i] + s.B - 1) / s.B;
      for (int64_t k = offsets[i]; k < offsets[i] + need; k++)
        if (blocks[k] < 0 || blocks[k] >= s.N) return KV_ERANGE;
    }
    // nothing fails from here on but allocation: a batch that could not be set describes nothing
    n = T = 0;
    blocks_ = s.N;
    try {
      lay_out(n_, offsets, blocks, tokens, q_lens, g, (int32_t)rows, keys, (size_t)table, s);
    } catch (...) {
      n = T = 0;
      throw;
    }
    return KV_OK;
  }

  // Would rewriting blocks [first_block, keep_blocks) of the requests with more than `keep` tokens reach a block that the batch has twice?
  // These blocks are marked, then all others looked up: 128 requests behind 8192 tokens, 69260 blocks, 31 us on the host.
  bool rewrites_shared(int32_t keep, int32_t first_block, int32_t keep_blocks) {
    marked_.resize((size_t)blocks_, 0);
    auto each = [&](auto what) {  // blocks [from, to) of the table that are rewritten
      for (int32_t i = 0; i < n; i++)
        if (len[i] > keep) what(off[i] + first_block, off[i] + keep_blocks);
    };
    bool twice = false;
    each([&](int32_t from, int32_t to) {
      for (int32_t k = from; k < to; k++) {
        twice |= marked_[ids[k]];
        marked_[ids[k]] = 1;
      }
    });
    uint8_t hit = 0;
    int32_t at = 0;
    auto look_up = [&](int32_t to) {
      for (; at < to; at++) hit |= marked_[ids[at]];
    };
    each([&](int32_t from, int32_t to) {
      look_up(from);
      at = std::max(at, to);
    });
    look_up((int32_t)ids.size());
    each([&](int32_t from, int32_t to) {
      for (int32_t k = from; k < to; k++) marked_[ids[k]] = 0;
    });
    return twice || hit;
  }

 private:
  std::vector<uint8_t> marked_;  // by block, all 0 between calls
  int64_t blocks_ = 0;

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
    places.clear();
    places.reserve(rows);
    tok_req.reserve(rows);
    tok_limit.reserve(rows);
    for (int32_t i = 0; i < n_; i++) {
      const int32_t need = (int32_t)(((int64_t)tokens[i] + s.B - 1) / s.B);
      ids.insert(ids.end(), blocks + offsets[i], blocks + offsets[i] + need);
      off.push_back((int32_t)ids.size());
      q_first.push_back(q_first.back() + q_lens[i]);
      for (int32_t j = 0; j < q_lens[i]; j++) {
        tok_req.push_back(i);
        const int32_t x = tokens[i] ? tokens[i] - q_lens[i] + j : -1;
        tok_limit.push_back(x + 1);
        places.push_back({x < 0 ? -1 : ids[off[i] + x / s.B], x < 0 ? 0 : x % s.B, x, 0});
      }
    }
    n = n_;
    T = rows;
    const int64_t spared = find_nodes(s, true);
    if (spared > 0 && spared < s.spared) find_nodes(s, false);
    cut(s);
  }

  // Blocks of request i that every one of its rows sees whole.
  int32_t open_blocks(int32_t i, int32_t B) const { return len[i] ? (len[i] - q_len[i] + 1) / B : 0; }

  std::vector<Node> nodes_;

  // -> tokens that big tiles do not read again.
  int64_t find_nodes(const BatchShape& s, bool share_big) {
    const int32_t B = s.B;
    int64_t spared = 0;
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
        const int64_t keys = (int64_t)(at - w.from) * B;
        int64_t rows = 0;
        for (int32_t i : w.reqs) rows += (int64_t)q_len[i] * G;
        if (rows <= kRowTile ? keys >= s.few_prefix : share_big && keys >= s.big_prefix) {
          nodes_.push_back({w.reqs, w.from * B, at * B});
          w.from = at;
          if (rows > kRowTile) spared += keys * (int64_t)(w.reqs.size() - 1);
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
    return spared;
  }

  struct Tile {
    int32_t node, list, tokens, row0, rows, limit, clear;
    int32_t score = 0, score_row = 0;
  };
  struct Use {
    int32_t list, tokens, part;  // every row of these tokens has a partial row from here on
  };
  std::vector<Tile> few_, big_, huge_;
  int big_cu_ = 1;
  double row_cost_ = 0;  // keys that the partial rows of a big tile's piece cost
  std::vector<int32_t> seen_;  // nodes with keys, per token
  std::vector<Use> uses_;

  void cut(const BatchShape& s) {
    lists.clear();
    items.clear();
    few_.clear();
    big_.clear();
    huge_.clear();
    uses_.clear();
    wrest.clear();
    witems.clear();
    wreqs.clear();
    sitems.clear();
    scores = 0;
    seen_.assign((size_t)T, 0);
    mixed = big_mixed = false;
    partial_rows = 0;
    read = 0;
    // Tiles have whole tokens, so that a token's rows are together wherever a tile's keys are cut; where one token has more rows than a
    // big tile, its tiles are cut alike instead.
    const int32_t big_tokens = s.big_tile / G;
    big_cu_ = s.big_cu;
    row_cost_ = (double)s.big_tile * s.H / s.key_rows;
    for (size_t d = 0; d < nodes_.size(); d++) {
      const Node& node = nodes_[d];
      const int32_t list = (int32_t)lists.size();
      for (int32_t i : node.reqs)
        for (int32_t t = q_first[i]; t < q_first[i + 1]; t++) lists.push_back(t);
      read += node.to - node.from;
      const int32_t tokens = (int32_t)lists.size() - list;
      const int64_t rows = (int64_t)tokens * G;
      auto tile = [&](int32_t at, int32_t n, int32_t row0, int32_t tile_rows) {
        Tile t{(int32_t)d, list + at, n, row0, tile_rows, 0, INT32_MAX};
        for (int32_t j = row0 / G; j <= (row0 + tile_rows - 1) / G; j++) {
          const int32_t limit = std::min(node.to, tok_limit[lists[list + at + j]]);
          t.limit = std::max(t.limit, limit);
          t.clear = std::min(t.clear, limit);
        }
        return t;
      };
      if (rows <= kRowTile) {
        Tile t = tile(0, tokens, 0, (int32_t)rows);
        t.score_row = (std::max(t.limit - node.from, 0) + 15) / 16 * 16;
        t.score = (int32_t)(scores / 16);
        scores += (int64_t)rows * t.score_row;
        int32_t row0 = 0;
        for (int32_t i : node.reqs) {
          for (int32_t k = node.from; k < t.limit; k += kScoreKeys)
            sitems.push_back({i, k, std::min(t.limit, k + kScoreKeys), t.score, t.score_row, node.from, row0, q_len[i] * G});
          row0 += q_len[i] * G;
        }
        few_.push_back(t);
      } else if (big_tokens > 0) {
        for (int32_t at = 0; at < tokens; at += big_tokens) {
          const int32_t n = std::min(big_tokens, tokens - at);
          big_.push_back(tile(at, n, 0, n * G));
        }
      } else {
        for (int64_t r = 0; r < rows; r += s.big_tile)
          huge_.push_back(tile(0, tokens, (int32_t)r, (int32_t)std::min<int64_t>(s.big_tile, rows - r)));
      }
      const int32_t reqs = (int32_t)node.reqs.size(), first = (int32_t)wreqs.size();
      wreqs.insert(wreqs.end(), node.reqs.begin(), node.reqs.end());
      for (int32_t k = node.from; k < node.to; k += kWeightKeys)
        for (int32_t r = 0; r < reqs; r += kWeightReqs) {
          witems.push_back({off[node.reqs[0]], k, std::min(node.to, k + kWeightKeys), first + r, std::min(kWeightReqs, reqs - r), {}});
          if (rows > kRowTile) wrest.push_back(witems.back());
        }
      for (size_t j = list; j < lists.size(); j++)
        if (node.to > node.from) seen_[lists[j]]++;
    }
    heads = 1;
    int64_t work = 0;
    for (const Tile& t : few_) work += std::max(t.limit - nodes_[t.node].from, 0);
    // Where there is enough for every workgroup, its four wavefronts take four heads (two, if the head count is no multiple of four) rather
    // than four runs of one head's keys: they then read neighbouring bytes at the same time.  64 requests of 512 to 4096 tokens with 8
    // heads of 128 in bf16: 103 us instead of 135, 32 requests of 256 to 8192 with 32 heads in fp8: 175 to 181 instead of 207.
    heads = work * s.H / std::max(1, s.wgs) < kMany ? 1 : s.H % 4 == 0 ? 4 : s.H % 2 == 0 ? 2 : 1;
    wg_items.clear();
    deal_out(few_, s.wgs * heads / s.H, s.least / heads, s.B, &wg_items, &mixed);
    big_first = (int32_t)items.size();
    wg_big.clear();
    deal_out(big_, s.big_wgs / s.H, s.big_least, s.B, &wg_big, &big_mixed);
    cut_alike(s.B);

    join_off.assign((size_t)T + 1, 0);
    for (const Use& u : uses_)
      for (int32_t j = 0; j < u.tokens; j++) join_off[lists[u.list + j] + 1]++;
    for (int32_t t = 0; t < T; t++) join_off[t + 1] += join_off[t];
    join.assign((size_t)join_off[T], 0);
    most_parts = 0;
    for (int32_t t = 0; t < T; t++) most_parts = std::max(most_parts, join_off[t + 1] - join_off[t]);
    std::vector<int32_t> at(join_off.begin(), join_off.end() - 1);
    for (const Use& u : uses_)
      for (int32_t j = 0; j < u.tokens; j++) join[at[lists[u.list + j]]++] = u.part + j * G;
  }
  static constexpr int32_t kStep = 128;  // keys that a workgroup takes at a time
  static constexpr int64_t kMany = 1024;  // keys of one head a workgroup

  // Does a tile without keys have something to do?  Only where its rows have no keys at any node.
  bool idle(const Tile& t) const {
    if (nodes_[t.node].to > nodes_[t.node].from) return false;
    for (int32_t j = 0; j < t.tokens; j++)
      if (seen_[lists[t.list + j]] == 0) return false;
    return true;
  }
  bool alone(const Tile& t) const {
    for (int32_t j = 0; j < t.tokens; j++)
      if (seen_[lists[t.list + j]] > 1) return false;
    return true;
  }
  int64_t most_keys(int32_t B) const { return std::min<int64_t>((int64_t)(kMaxEntries - 1) * B, INT32_MAX / 2) / kStep * kStep; }

  void add(const Tile& t, int32_t k0, int32_t k1, int32_t part, bool* any_mixed) {
    const int32_t end = std::max(k0, std::min(k1, t.limit));
    items.push_back({off[nodes_[t.node].reqs[0]], k0, end, std::min(end, t.clear), t.list, t.row0, t.rows, part,
                     t.score, t.score_row, nodes_[t.node].from, nodes_[t.node].reqs.size() > 1});
    if (items.back().clear < end) *any_mixed = true;
  }
  int32_t take_rows(const Tile& t, int32_t rows) {
    const int32_t part = partial_rows;
    partial_rows += rows;
    uses_.push_back({t.list, t.tokens, part});
    return part;
  }

  int64_t keys_of(const Tile& t) const { return std::max(t.limit - nodes_[t.node].from, 0); }

  // Tiles that all have a workgroup of their own: is it better to leave them whole, though some are longer than a share, than to cut them and have
  // partial results?
  // Row tiles: up to one and a half shares.  Whole against cut, 8 heads of 128 in bf16, lengths from .. to: longest 1.3 to 1.46 shares, 250 requests of 500
  // to 1000 129 / 162 us, 250 of 1500 to 3000 372 / 368, 200 of 2500 to 3000 354 / 426, 30 of 500 to 700 20 / 25; 1.56 shares, 250 of 100 to 1000
  // 109 / 104, 200 of 500 to 1000 113 / 112; 1.8 shares and more, 200 of 1000 to 3000 301 / 265, 150 of 500 to 700 77 / 71, 200 of 100 to 3000 274 / 208.
  // Big tiles: what they take whole, by the longest pair of workgroups that share a CU (three quarters of the time a key for one that is left alone: 23
  // ns for 31), against a share and the way of the partial rows through memory: in bf16 50 rows of all heads a key (45 to 110 us for 13500 rows of 8
  // heads), in fp8, where a key takes longer, 100.  New tokens of all cached, whole / cut in bf16, then in fp8: 2000 of 2000 64 / 94 us, 94 / 124; 1500
  // of 9000 in three requests 101 / 114, 151 / 148; 1024 of 8001 and 517 of 5000 206 / 213, 324 / 283; 1280 of 6000 181 / 151, 277 / 203; 1024 of 8192
  // 190 / 164, 302 / 222; 1408 of 12000 355 / 303, 548 / 404.  Over 48 such prompts the rule is 1 % from the better of the two on average.
  bool stay_whole(const std::vector<Tile>& tiles, int64_t held, int64_t share, int64_t longest, int64_t pieces) const {
    if (&tiles == &few_) return 2 * longest <= 3 * share;
    int64_t whole = 0;  // in quarters of a key
    if (big_cu_ == 1) whole = 4 * longest;
    for (size_t j = 0; big_cu_ > 1 && j < tiles.size(); j++) {
      const size_t other = j + (size_t)held / 2;
      const int64_t a = keys_of(tiles[j]), b = other < tiles.size() ? keys_of(tiles[other]) : 0;
      whole = std::max(whole, 4 * std::min(a, b) + 3 * std::abs(a - b));
    }
    const int64_t parts = pieces > held ? (int64_t)tiles.size() + held : pieces;
    return whole - 4 * share <= 4 * row_cost_ * parts;
  }

  // Tiles of whole tokens.  If one piece of at most `share` keys for each of the workgroups that are to run at a time (`held`) is enough,
  // every tile is cut by itself, and each piece has its workgroup.  Otherwise the tiles' keys are one line that is cut into equal shares:
  // a workgroup may take the end of one tile, whole ones and the beginning of another.
  void deal_out(const std::vector<Tile>& tiles, int64_t held, int64_t least, int32_t B, std::vector<int32_t>* wgs, bool* any_mixed) {
    int64_t work = 0;
    for (const Tile& t : tiles) work += keys_of(t);
    held = std::max<int64_t>(1, held);
    const int64_t most = most_keys(B);
    int64_t share = std::max<int64_t>(least, (work + held - 1) / held);
    share = std::min(most, (share + kStep - 1) / kStep * kStep);
    int64_t longest = 0, pieces = 0;
    auto count = [&] {
      pieces = 0;
      for (const Tile& t : tiles) pieces += std::max<int64_t>(1, (keys_of(t) + share - 1) / share);
    };
    for (const Tile& t : tiles) longest = std::max(longest, keys_of(t));
    count();
    if ((int64_t)tiles.size() <= held && longest > share && longest <= most && stay_whole(tiles, held, share, longest, pieces)) {
      share = longest;
      count();
    }
    const bool line = pieces > held;
    int64_t room = 0;  // keys that the current workgroup still takes
    for (const Tile& t : tiles) {
      if (idle(t)) continue;
      const int32_t from = nodes_[t.node].from, keys = std::max(t.limit - from, 0);
      const bool whole_alone = alone(t);
      if (!line || keys == 0 || room < kStep) {
        wgs->push_back((int32_t)items.size());
        room = share;
      }
      if (!line) {  // equal pieces
        const int32_t n = (int32_t)std::max<int64_t>(1, (keys + share - 1) / share);
        const int32_t step = (int32_t)(((int64_t)(keys + n - 1) / n + kStep - 1) / kStep * kStep);
        for (int32_t c = 0; c < n && (c == 0 || (int64_t)c * step < keys); c++) {
          if (c) wgs->push_back((int32_t)items.size());
          const int32_t part = n == 1 && whole_alone ? -1 : take_rows(t, t.rows);
          add(t, from + c * step, from + (int32_t)std::min<int64_t>(keys, (int64_t)(c + 1) * step), part, any_mixed);
        }
        continue;
      }
      // a rest below half a step is taken along rather than left to another workgroup
      for (int32_t k = 0; k < keys || keys == 0;) {
        int32_t n = (int32_t)std::min<int64_t>(keys - k, room);
        if (keys - k - n < kStep / 2 && keys - k <= most) n = keys - k;
        const int32_t part = n == keys && whole_alone ? -1 : take_rows(t, t.rows);
        add(t, from + k, from + k + n, part, any_mixed);
        k += n;
        room -= (n + kStep - 1) / kStep * kStep;
        if (keys == 0) break;
        if (k < keys) {
          wgs->push_back((int32_t)items.size());
          room = share;
        }
      }
    }
    wgs->push_back((int32_t)items.size());
  }

  // Tiles that share tokens: all of a node's are cut at the same keys, as seldom as may be.  They follow the big tiles.
  void cut_alike(int32_t B) {
    const int64_t most = most_keys(B);
    for (size_t k = 0; k < huge_.size();) {
      size_t e = k;
      while (e < huge_.size() && huge_[e].node == huge_[k].node) e++;
      const Node& node = nodes_[huge_[k].node];
      const int64_t keys = node.to - node.from;
      if (!idle(huge_[k]))
        for (int64_t c = 0; c == 0 || c < keys; c += most) {
          const int32_t part = keys <= most && alone(huge_[k]) ? -1 : take_rows(huge_[k], huge_[k].tokens * G);
          for (size_t j = k; j < e; j++) {
            add(huge_[j], node.from + (int32_t)c, node.from + (int32_t)std::min(keys, c + most), part < 0 ? -1 : part + huge_[j].row0, &big_mixed);
            wg_big.push_back((int32_t)items.size());
          }
        }
      k = e;
    }
  }
};

}  // namespace kvswap
