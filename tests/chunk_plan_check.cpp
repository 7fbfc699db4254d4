// The chunk attention's plan (the first part of csrc/chunk.hpp) on the CPU: the plan's rounds over a batch and the
// kernels' walks over the queues, one at a time where the device scans lanes.  Returns 0, or the line that failed.
#include "chunk.hpp"

#include <algorithm>
#include <map>
#include <set>
#include <tuple>
#include <vector>

using namespace sdb;

#define NEED(x) \
  if (!(x)) return __LINE__

extern "C" int check_chunk(int S, int Hkv, int G, int causal, const int *ctx, const int *B, int slots, int *items_out,
                           int *pieces_out, double *largest) {
  const int P = kChunkRows / G;
  std::vector<ChunkSeq> seq;
  std::vector<int> order(S);
  double total = 0;
  for (int s = 0; s < S; ++s) {
    seq.push_back(ChunkSeq{ctx[s], B[s], P, G, causal});
    order[s] = s;
    total += seq[s].all_units() * Hkv;
    double sum = 0;
    for (int j = 0; j < seq[s].tiles(); ++j) {
      NEED(seq[s].rows(j) >= 1 && seq[s].rows(j) <= kChunkRows && seq[s].before(j) == sum);
      sum += seq[s].units(j);
    }
    NEED(sum == seq[s].all_units());
  }
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return (float)seq[x].longest() > (float)seq[y].longest(); });
  std::vector<ChunkEntry> entry(S);
  double after = 0, slot = 0;
  int merges = 0;
  for (int r = S - 1; r >= 0; --r) {
    const ChunkSeq &q = seq[order[r]];
    ChunkSplit sp = q.tiles() ? chunk_split(q, Hkv, after, total) : ChunkSplit{0, 1};
    NEED(sp.js >= 0 && sp.js <= q.tiles() && sp.np >= 1 && sp.np <= 64 && (sp.np > 1) == (sp.js > 0));
    const double want = sp.np > 1 ? (double)sp.js * sp.np * Hkv : 0;
    const double slot0 = slot;
    slot += want;
    if (slot > slots) sp = ChunkSplit{0, 1};
    entry[r] = ChunkEntry{order[r], q.ctx, q.B, 0, q.tiles(), sp.js, sp.np, (int)(sp.js ? slot0 : 0), q.tiles() - sp.js + sp.js * sp.np, merges, {0, 0}};
    merges += sp.js * Hkv;
    after += q.all_units() * Hkv;
  }
  NEED(merges <= slots / 2 && after == total);
  std::map<std::tuple<int, int, int>, std::vector<std::pair<int, int>>> keys;  // tile -> pieces
  std::set<int> used;
  int items = 0, pieces = 0;
  *largest = 0;
  for (int x = 0; x < kChunkQueues; ++x) {
    const int n = chunk_groups((long long)S * Hkv, x);
    NEED(n <= (S * Hkv + kChunkQueues - 1) / kChunkQueues);
    for (int k = 0; k < n; ++k) {
      const int group = x + kChunkQueues * k, r = group / Hkv, g = group - r * Hkv;
      NEED(group < S * Hkv);
      const ChunkEntry &e = entry[r];
      const ChunkSeq &q = seq[e.s];
      for (int i = 0; i < e.items; ++i, ++items) {
        const int j = e.tile(i), p = e.piece(i), nk = q.keys(j);
        NEED(j >= 0 && j < e.nt && p < e.np);
        const int k0 = p < 0 ? 0 : chunk_piece(nk, e.np, p), k1 = p < 0 ? nk : chunk_piece(nk, e.np, p + 1);
        NEED(k0 >= 0 && k0 <= k1 && k1 <= nk && k0 % kChunkKT == 0 && (k1 % kChunkKT == 0 || k1 == nk));
        const double w = (double)chunk_weight(q.rows(j)) * (k1 - k0 + kChunkPieceCost);
        if (w > *largest) *largest = w;
        if (p >= 0) {
          const int sl = e.slot(g, j, p);
          NEED(sl >= 0 && sl < slots && used.insert(sl).second);
          ++pieces;
        }
        if (k0 < k1) keys[{e.s, g, j}].push_back({k0, k1});
      }
    }
  }
  size_t tiles = 0;
  for (int s = 0; s < S; ++s)
    for (int g = 0; g < Hkv; ++g)
      for (int j = 0; j < seq[s].tiles(); ++j, ++tiles) {
        auto v = keys[{s, g, j}];
        std::sort(v.begin(), v.end());
        int at = 0;
        for (auto &k : v) {
          NEED(k.first == at);
          at = k.second;
        }
        NEED(at == seq[s].keys(j));
      }
  NEED(keys.size() == tiles);
  *items_out = items;
  *pieces_out = pieces;
  *largest /= total > 0 ? total / kChunkGrid : 1;
  return 0;
}
