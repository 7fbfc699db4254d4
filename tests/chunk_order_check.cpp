// The chunk attention's plan on the CPU in the order in which the device makes it (csrc/chunk.hpp): the order of the
// sequences, the split of each against what lies behind it, the queues' items, the slots and the merge's list.  Returns
// 0, or the line that failed.
#include "chunk.hpp"

#include <math.h>
#include <set>
#include <vector>

using namespace sdb;

#define NEED(x) \
  if (!(x)) return __LINE__

// order_out [S]; longest_out: units of the longest item, share_out: of a workgroup's even share.
extern "C" int check_order(int S, int Hkv, int G, int causal, const int *ctx, const int *B, int slots, int *order_out,
                           double *longest_out, double *share_out, int *dropped_out) {
  const int P = kChunkRows / G;
  std::vector<ChunkSeq> seq;
  std::vector<float> key(S), work(S), place(S);
  double total = 0;
  for (int s = 0; s < S; ++s) {
    seq.push_back(ChunkSeq{ctx[s], B[s], P, G, causal});
    key[s] = chunk_key(seq[s]);
    work[s] = (float)seq[s].all_units();
    total += seq[s].all_units() * Hkv;
  }
  // the order
  std::vector<int> order(S, -1);
  if (S <= kChunkSortSeqs) {
    for (int s = 0; s < S; ++s) place[s] = chunk_place(key.data(), work.data(), S, s);
    for (int s = 0; s < S; ++s) {
      const int r = chunk_rank(place.data(), S, s);
      NEED(r >= 0 && r < S && order[r] == -1);  // each rank once
      order[r] = s;
    }
    // Places are sums of at most S works in fp32 over their total: each within (S + 2) 2^-24 of its value.  Neighbours of a
    // kind are half of both their works apart, so only works below this share of the total may change places.
    const double edge = (S + 2) * ldexp(1, -22);
    float last[2] = {INFINITY, INFINITY};
    double done[2] = {0, 0}, all[2] = {0, 0};
    for (int s = 0; s < S; ++s) all[key[s] < 0] += seq[s].all_units();
    bool rows = true;
    for (int r = 0; r < S; ++r) {
      const int s = order[r], kind = key[s] < 0;
      if (B[s] <= 0) {
        rows = false;
        continue;
      }
      const double units = seq[s].all_units();
      NEED(rows || units <= edge * all[kind]);  // sequences without rows come last
      NEED(fabsf(key[s]) <= last[kind] || units <= edge * all[kind]);  // a kind's longest first
      if (units > edge * all[kind]) last[kind] = fabsf(key[s]);
      // The kinds' shares keep step: a sequence that is half done is at most where the other kind's next one is then (1e-3:
      // the places' error above, and what changed places).
      const double half = units / 2, at = (done[kind] + half) / all[kind];
      if (all[!kind] > 0) {
        double next = 0;  // the first of the other kind that is still to come
        for (int q = r + 1; q < S; ++q)
          if (B[order[q]] > 0 && (key[order[q]] < 0) != kind) {
            next = seq[order[q]].all_units() / 2;
            NEED((done[!kind] + next) / all[!kind] >= at - 1e-3);
            break;
          }
      }
      done[kind] += 2 * half;
    }
  } else {
    for (int s = 0; s < S; ++s) order[s] = s;
  }
  // the entries, from the last, 64 at a time: what lies behind is the sum of the later rounds and of the later lanes
  std::vector<ChunkEntry> entry(S);
  double after = 0, filed = 0;
  int merges = 0, dropped = 0;
  for (int c0 = (S - 1) / 64 * 64; c0 >= 0; c0 -= 64) {
    double behind = after, slot0 = filed;
    int merge0 = merges;
    for (int r = (c0 + 63 < S - 1 ? c0 + 63 : S - 1); r >= c0; --r) {
      const ChunkSeq &q = seq[order[r]];
      ChunkSplit sp = q.tiles() ? chunk_split(q, Hkv, behind, total) : ChunkSplit{0, 1};
      NEED(sp.js >= 0 && sp.js <= q.tiles() && sp.np >= 1 && sp.np <= 64 && (sp.np > 1) == (sp.js > 0));
      const double want = sp.np > 1 ? (double)sp.js * sp.np * Hkv : 0;
      if (slot0 + want > slots) sp = ChunkSplit{0, 1}, ++dropped;
      entry[r] = ChunkEntry{order[r], q.ctx, q.B, 0, q.tiles(), sp.js, sp.np, (int)(sp.js ? slot0 : 0),
                            q.tiles() - sp.js + sp.js * sp.np, merge0, {0, 0}};
      slot0 += want;
      merge0 += sp.js * Hkv;
      behind += q.all_units() * Hkv;
    }
    after = behind;
    filed = slot0;
    merges = merge0;
  }
  NEED(after == total && merges <= slots / 2);
  // the queues: every key of every tile once, slots once each, tiles of one merge entry each
  std::set<int> used, merged;
  double keys = 0, want_keys = 0;
  *longest_out = 0;
  for (int x = 0; x < kChunkQueues; ++x) {
    const int n = chunk_groups((long long)S * Hkv, x);
    for (int k = 0; k < n; ++k) {
      const int group = x + kChunkQueues * k, r = group / Hkv, g = group - r * Hkv;
      const ChunkEntry &e = entry[r];
      const ChunkSeq &q = seq[e.s];
      std::vector<int> at(e.nt, 0);
      for (int i = 0; i < e.items; ++i) {
        const int j = e.tile(i), p = e.piece(i);
        NEED(j >= 0 && j < e.nt && p < e.np);
        const int k0 = p < 0 ? 0 : chunk_piece(q.keys(j), e.np, p), k1 = p < 0 ? q.keys(j) : chunk_piece(q.keys(j), e.np, p + 1);
        NEED(k0 == at[j] && k1 >= k0);  // a tile's pieces follow one another in the queue
        at[j] = k1;
        keys += k1 - k0;
        const double w = (double)chunk_weight(q.rows(j)) * (k1 - k0 + kChunkPieceCost);
        if (w > *longest_out) *longest_out = w;
        if (p >= 0) {
          const int sl = e.slot(g, j, p);
          NEED(sl >= 0 && sl < slots && used.insert(sl).second);
        }
        if (p == 0) {
          const int m = e.merge0 + g * e.js + j;
          NEED(m >= 0 && m < merges && merged.insert(m).second);
        }
      }
      for (int j = 0; j < e.nt; ++j) {
        NEED(at[j] == q.keys(j));
        want_keys += q.keys(j);
      }
    }
  }
  NEED(keys == want_keys && (int)merged.size() == merges);
  *share_out = total / kChunkGrid;
  *dropped_out = dropped;
  for (int r = 0; r < S; ++r) order_out[r] = order[r];
  return 0;
}
