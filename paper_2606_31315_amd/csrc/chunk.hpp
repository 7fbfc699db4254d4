// chunk.hpp -- attention of chunks of new tokens over page pools: the B_s rows of sequence s, any
// number of them, attend to their committed context and to the chunk itself.
//
// A query tile is P = 256 / G positions of one (sequence, kv head) with the G query heads of each, up
// to 256 rows, so a key row that a workgroup fetches serves all of them.  A workgroup of eight
// wavefronts takes a tile, 32 rows a wavefront, and walks its keys 64 at a time:
//   S^T = K Q^T    (32x32x16 bf16 matrix products, fp32 sums)
//   P = exp2(S^T c - m), reference m near the running row maximum, row sum l in fp32
//   O^T = O^T 2^(m_old - m) + V^T P^T   (P rounded to bf16 for the product; O^T fp32 in registers)
// Scores come transposed, so a lane holds the scores of one query row (32 of a step's 64 keys, its
// partner lane the others) and the softmax needs no exchange but, now and then, one between two
// lanes.  The weights then are the right operand of the second product as they stand: the products'
// inner index runs over keys in the order in which the first product left them, and V^T is read in
// that order.  P is rounded because the matrix cores take bf16: 2^-8 of each weight, independent from key
// to key; sums and O stay fp32.
//
// Bound, for long chunks, by the matrix cores and the power they draw: 2048 rows at 65536 keys (32 heads on 4) take
// 1.83 to 1.94 ms from card to card, 1.15 to 1.22 PFLOP/s, where a matrix product of 16384^3 reaches 1.37.  The matrix
// units are busy 62% of the cycles at a clock of 2.0 GHz (a step is 2048 cycles of products and took 3400 before its
// first operands were read ahead; then, in copies that skip them, they were busy 65% without the tile loads, 77% at
// 1.81 GHz without LDS reads, 80% without LDS reads and softmax).  LDS reads (256 KB a step) are the next bound, without
// bank conflicts; the L2 serves 96% of the tile loads.  At head_dim 64, half the products to a softmax: 1.13 to 1.26 ms,
// 0.89 to 0.99 PFLOP/s.
// Tried and slower: four wavefronts of 64 rows (half the LDS reads, but 512 registers, half of which only the
// matrix units address: 3.2 ms); eight without turns at the matrix unit (2.1 ms); row sums by bf16 dot
// products of two (1.95 against 1.87); asking for the next item before the last steps (2.01 against 1.97); the
// tile loads with the softmax instead of the products (1.89 against 1.87); equal wave priorities (1.94 against 1.87).
#pragma once

#include "attn.hpp"

namespace sdb {

constexpr int kChunkRows = 256;  // query rows of a tile
constexpr int kChunkKT = 64;     // keys of a step

// ---- plan --------------------------------------------------------------------------
// Query tiles have from one key step to thousands, and their number seldom fits the device.  A small
// launch orders the sequences, longest tiles first, deals their kv heads to eight
// queues, one per XCD, and decides which tiles are cut into pieces of keys: those near the end of the
// order, whose length the work behind them could not even out.  Workgroups take the next item of
// their XCD's queue, and of another when that is empty.  The tiles of one kv head are neighbours in a queue, so
// the workgroups of an XCD walk the same keys at about the same time and fetch them once into its L2 (a chunk of
// 2048 rows at 65536 keys, 8 query heads to a kv head: 2.21 ms with an equal share of a line of all tiles for
// every workgroup, whose walks are spread over the keys, 1.94 ms in step).  Pieces file their
// unnormalised sums, and a third launch joins them.
constexpr int kChunkQueues = 8;
constexpr int kChunkGrid = 256;       // workgroups at most: one fills a CU
constexpr int kChunkSlots = 1024;     // pieces at most
constexpr int kChunkSortSeqs = 1024;  // batches past this keep their order
constexpr int kChunkPieceCost = 128;  // keys' worth of starting and ending an item
constexpr int kChunkMinPiece = 512;   // keys of a piece at least
constexpr int kChunkFew = 128;        // batches of less than this many tiles are cut throughout
constexpr int kChunkSpread = 64;      // else a tile is cut where less than this many of its kind are left
constexpr int kChunkEndPieces = 3;    // into this many pieces
constexpr int kChunkPieceExtra = 512; // keys' worth of cutting: sums filed and joined

// Relative time of a key by the tile's rows.  A step of few rows still goes through both phases and their barriers: 1024
// tiles over the same 4096 keys take 509 us with 256 rows, 438 with 192, 357 with 128, 335 with 64 and 320 with 4, that is
// 8 : 6.9 : 5.6 : 5.3 : 5.0 (head_dim 64: 326, 295, 268, 252, 239); with keys of their own 604, 533, 445, 414, 397.  With 6 for
// the least, batches take the same (400 rows at 4000 keys 50.8 and 50.9 us, prompt chunks of 200 to 900 rows beside single
// tokens of 64 sequences 1134 and 1137); with 3 for sequences of few rows, too (1138 and 1134; at head_dim 64, 16
// sequences, 192 and 200).
SDB_HD int chunk_weight(int rows) { return plan_max((rows + 31) / 32, 5); }

struct ChunkSeq {
  int ctx, B, P, G, causal;
  SDB_HD int tiles() const { return B > 0 ? (B + P - 1) / P : 0; }
  SDB_HD int rows(int j) const { return plan_min(P, B - P * j) * G; }           // of tile j
  SDB_HD int keys(int j) const { return ctx + (causal ? plan_min(P * (j + 1), B) : B); }
  // Work of tile j, and of the tiles before it (which are all full): whole numbers, below 2^53 (the host checks).
  SDB_HD double units(int j) const { return (double)chunk_weight(rows(j)) * ((double)keys(j) + kChunkPieceCost); }
  SDB_HD double before(int j) const {
    const double n = j, each = (double)(causal ? ctx : ctx + B) + kChunkPieceCost;
    return chunk_weight(P * G) * (n * each + (causal ? n * (n + 1) / 2 * P : 0));
  }
  SDB_HD double all_units() const { const int n = tiles(); return n ? before(n - 1) + units(n - 1) : 0; }
  SDB_HD bool few() const { return B > 0 && B <= 64 / G; }  // rows: bound by its keys' way from memory
  SDB_HD double longest() const {  // the last tile may have few rows
    const int n = tiles();
    const double u = n ? units(n - 1) : 0, v = n > 1 ? units(n - 2) : 0;
    return u > v ? u : v;
  }
};

// Tiles 0 .. js - 1 of each of a sequence's heads are cut into np pieces, the others are whole.  after: work of the
// sequences behind it, total: of the batch.
struct ChunkSplit {
  int js, np;
};
SDB_HD ChunkSplit chunk_split(const ChunkSeq &q, int Hkv, double after, double total) {
  const int nt = q.tiles();
  int lo = 0, hi = nt;
  for (int j = nt - 1; lo < hi; j = lo + (hi - lo) / 2) {  // the first tile that is not cut (a search, as if there were one)
    if (total < kChunkFew * q.units(j) || after + Hkv * (q.before(j) + q.units(j)) < kChunkSpread * q.units(j)) lo = j + 1;
    else hi = j;
  }
  if (lo == 0) return ChunkSplit{0, 1};
  double longest = q.units(lo - 1);
  if (lo > 1 && q.units(lo - 2) > longest) longest = q.units(lo - 2);
  const double tiles = total / longest;  // tiles like this one
  int np = 1;
  if (tiles >= kChunkFew) {  // the end of a long batch
    np = kChunkEndPieces;
  } else {  // all of it: the number of rounds over the device, of as many pieces as fit it, that ends first
    const double extra = (double)chunk_weight(kChunkRows) * kChunkPieceExtra;
    double best = longest;
    for (int k = 1; k <= 4; ++k) {
      const int n = plan_min((int)(kChunkGrid * k / tiles), 64);
      const double t = k * (longest / plan_max(n, 1) + extra);
      if (n > 1 && t < best) {
        best = t;
        np = n;
      }
    }
  }
  const int most = (int)(longest / ((double)chunk_weight(kChunkRows) * kChunkMinPiece));
  if (np > most) np = most;
  return np > 1 ? ChunkSplit{lo, np} : ChunkSplit{0, 1};
}
// First key of piece i of np of n keys (i = np: n): whole steps, evenly; a piece may be empty.
SDB_HD int chunk_piece(int n, int np, int i) {
  const long long steps = (n + kChunkKT - 1) / kChunkKT;
  return i == np ? n : (int)(steps * i / np) * kChunkKT;
}

#if defined(__HIPCC__)
#define SDB_UNROLL4 _Pragma("unroll 4")
#else
#define SDB_UNROLL4
#endif
// The order of the sequences: those of few rows, which memory bounds, and the others, which the products bound, each kind
// longest first, the two interleaved by the share of their work that is done by then.
// A sequence's length, its kind marked by the sign.
SDB_HD float chunk_key(const ChunkSeq &q) { return (float)q.longest() * (q.few() ? -1.f : 1.f); }
// Share of its kind's work done when sequence t is half done, from all keys and units of work.
SDB_HD float chunk_place(const float *key, const float *work, int S, int t) {
  const float k = key[t];
  float before = 0.f, all = 0.f;
  SDB_UNROLL4
  for (int i = 0; i < S; ++i) {
    const float u = key[i], au = u < 0.f ? -u : u, ak = k < 0.f ? -k : k, w = (u < 0.f) == (k < 0.f) ? work[i] : 0.f;
    all += w;
    before += au > ak || (u == k && i < t) ? w : 0.f;
  }
  return all > 0.f ? (before + 0.5f * work[t]) / all : 2.f;  // sequences without rows come last
}
// Its rank by these.
SDB_HD int chunk_rank(const float *place, int S, int t) {
  const float at = place[t];
  int rank = 0;
  SDB_UNROLL4
  for (int i = 0; i < S; ++i) rank += place[i] < at || (place[i] == at && i < t);
  return rank;
}

// What the plan says of a sequence, in the order of the queues.
struct ChunkEntry {
  int s, ctx, B, qoff;
  int nt, js, np, slot0;  // slot0: partial slot of piece 0 of tile 0 of head 0
  int items;              // of each of its heads
  int merge0;             // first of its cut tiles in the list of the merge
  int pad[2];
  // Item i of a head: the whole tiles from the last on, then the first pieces of the others, the second ones, ...
  SDB_HD int whole() const { return nt - js; }
  SDB_HD int tile(int i) const { return i < whole() ? nt - 1 - i : js - 1 - (i - whole()) % js; }
  SDB_HD int piece(int i) const { return i < whole() ? -1 : (i - whole()) / js; }  // -1: a whole tile
  SDB_HD int slot(int g, int j, int p) const { return slot0 + (g * js + j) * np + p; }
};
// Kv head g of the r-th sequence is group r * Hkv + g; queue x holds groups x, x + 8, ...
SDB_HD int chunk_groups(long long groups, int x) { return groups > x ? (int)((groups - x + kChunkQueues - 1) / kChunkQueues) : 0; }

// A cut tile, for the merge.
struct ChunkMerge {
  int row0, g, rows, keys, np, slot, pad[2];  // row0: its first position in q and out
};

struct ChunkHead {
  struct {
    int v, pad[63];
  } next[kChunkQueues];     // items taken: a line each, atomics on one line wait for each other
  int count[kChunkQueues];  // items
  int merges;
};

#if defined(__HIPCC__)

}  // namespace sdb
#include <type_traits>
namespace sdb {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4c __attribute__((ext_vector_type(4)));
typedef short s16x8c __attribute__((ext_vector_type(8)));

struct ChunkArgs {
  const void *q;             // [total_q, Hq, D]
  const void *k, *v;         // [num_pages, Hkv, page_size, D]
  void *out;                 // [total_q, Hq, D]
  const int *ctx_lens, *chunk_lens, *q_offsets, *block_table;
  int S, Hq, Hkv, G;
  int P;                     // positions of a tile
  int page_log2, max_pages, num_pages;
  int causal;
  float scale_log2;          // softmax scale * log2(e)
  int slots, grid;           // partial slots, workgroups
  // workspace
  ChunkHead *head;
  ChunkEntry *entries;       // [S]
  int *prefix;               // [8, ceil(S Hkv / 8)] first item of each group of a queue
  ChunkMerge *merges;        // [slots / 2]
  float *part_o;             // [slots, 256, D] unnormalised sums
  float2 *part_ml;           // [slots, 256] (reference of the weights in log2 units, row sum)
};

template <int D>
struct ChunkTile {
  static constexpr int ROWB = D * 2;                   // bytes of a key row
  static constexpr int CPR = ROWB / 16;                // 16-byte vectors of a row
  static constexpr int TILEB = kChunkKT * ROWB;        // bytes of a K (or V) tile
  static constexpr int STAGEB = 2 * TILEB;             // K, then V
  static constexpr int NV = 16 * CPR / 64;             // vectors a lane fetches: 16 rows of K or of V a wavefront
  // A row's vectors are stored at their index XOR these, so that the 16 lanes an operand read serves at a
  // time touch distinct banks: 16 rows at one vector index of K, 4 rows at 4 indices of V.
  __device__ static int swz_k(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  __device__ static int swz_v(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }
};

// A context below 0, which no caller may give, counts as 0: no read lies before the sequence's row of the block table.
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs &a, int s) {
  return ChunkSeq{max(a.ctx_lens[s], 0), a.chunk_lens[s], a.P, a.G, a.causal};
}

// The plan, by one workgroup.  Sums of work are whole numbers in doubles and every order is fixed: the same lengths
// give the same plan.
// Its order costs two walks over the batch for every sequence, its entries one wavefront's 64 at a time: 5.5 us for one
// sequence, 9 to 12 for 32, 23 for 128, 43 for 256, 87 for 512, 207 for 1024 (an eighth of such a call: single tokens of
// nine sequences in ten, contexts of 500 to 2000 keys, 354 us for 256 and 1436 for 1024), 36 for 1025, which are not ordered.
constexpr int kChunkPlanThreads = 1024;
static_assert(kChunkSortSeqs <= kChunkPlanThreads, "a thread per sequence");
__global__ __launch_bounds__(kChunkPlanThreads) void chunk_plan_kernel(ChunkArgs a) {
  __shared__ float key[kChunkSortSeqs], place[kChunkSortSeqs];
  __shared__ int order[kChunkSortSeqs], items[kChunkSortSeqs];
  __shared__ double sums[kChunkPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, S = a.S;
  const bool sorted = S <= kChunkSortSeqs;
  // the batch's work, and the order
  double mine = 0;
  float k = 0.f, work = 0.f;
  for (int s = tid; s < S; s += kChunkPlanThreads) {
    const ChunkSeq q = chunk_seq(a, s);
    const double u = q.all_units();
    mine += u * a.Hkv;
    k = chunk_key(q);
    work = (float)u;
  }
  if (tid < kChunkSortSeqs) key[tid] = k, place[tid] = work;
  mine = wave_sum_d(mine);
  if (lane == 0) sums[wave] = mine;
  __syncthreads();
  double total = 0;
  for (int w = 0; w < kChunkPlanThreads / 64; ++w) total += sums[w];
  if (sorted) {
    const float at = tid < S ? chunk_place(key, place, S, tid) : 0.f;
    __syncthreads();
    if (tid < S) place[tid] = at;
    __syncthreads();
    if (tid < S) order[chunk_rank(place, S, tid)] = tid;
  }
  __syncthreads();
  // entries from the last to the first, 64 a round: what lies behind each is known then
  if (wave == 0) {
    double after = 0, slots = 0;
    int merges = 0;
    for (int c0 = (S - 1) / 64 * 64; c0 >= 0; c0 -= 64) {
      const int r = min(c0 + lane, S - 1);
      const bool live = c0 + lane < S;
      ChunkEntry e{};
      e.s = sorted ? order[r] : r;
      const ChunkSeq q = chunk_seq(a, e.s);
      e.ctx = q.ctx;
      e.B = q.B;
      e.qoff = a.q_offsets[e.s];
      e.nt = live ? q.tiles() : 0;
      double excl;
      const double units = live ? q.all_units() * a.Hkv : 0.0, incl = wave_scan_d(units, &excl), all = readlane_d(incl, 63);
      ChunkSplit sp = e.nt ? chunk_split(q, a.Hkv, after + (all - incl), total) : ChunkSplit{0, 1};
      const double want = sp.np > 1 ? (double)sp.js * sp.np * a.Hkv : 0.0, wi = wave_scan_d(want, &excl), wall = readlane_d(wi, 63);
      const double slot0 = slots + (wall - wi);  // of the sequences behind
      if (slot0 + want > a.slots) sp = ChunkSplit{0, 1};
      e.js = sp.js;
      e.np = sp.np;
      e.slot0 = sp.js ? (int)slot0 : 0;
      e.items = e.nt - sp.js + sp.js * sp.np;
      const int mi = wave_scan_i(sp.js * a.Hkv), mall = __builtin_amdgcn_readlane(mi, 63);
      e.merge0 = merges + mall - mi;
      if (live) {
        a.entries[r] = e;
        if (sorted) items[r] = e.items;
      }
      after += all;
      slots += wall;
      merges += mall;
    }
    if (lane == 0) a.head->merges = merges;
  }
  __threadfence_block();
  __syncthreads();
  if (wave < kChunkQueues) {  // a queue each
    const int x = wave, n = chunk_groups((long long)S * a.Hkv, x), stride = (S * a.Hkv + kChunkQueues - 1) / kChunkQueues;
    int base = 0;
    for (int k0 = 0; k0 < n; k0 += 64) {
      const int k = min(k0 + lane, n - 1);
      const int r = (x + kChunkQueues * k) / a.Hkv, m = k0 + lane < n ? (sorted ? items[r] : a.entries[r].items) : 0;
      const int incl = wave_scan_i(m);
      if (k0 + lane < n) a.prefix[x * stride + k] = base + incl - m;
      base += __builtin_amdgcn_readlane(incl, 63);
    }
    if (lane == 0) {
      a.head->next[x].v = ((int)a.grid - x + kChunkQueues - 1) / kChunkQueues;  // each workgroup's first item is its own
      a.head->count[x] = base;
    }
  } else {  // the list of cut tiles: the sequences that have some go round the other wavefronts
    int turn = wave;
    constexpr int kTurns = kChunkPlanThreads / 64 - kChunkQueues;
    for (int c0 = 0; c0 < S; c0 += 64) {
      const ChunkEntry e = a.entries[min(c0 + lane, S - 1)];
      unsigned long long cut = __ballot(c0 + lane < S && e.js > 0);
      while (cut) {
        const int l = __ffsll((long long)cut) - 1;
        cut &= cut - 1;
        if (turn++ % kTurns) continue;
        ChunkEntry u{};
        u.ctx = __builtin_amdgcn_readlane(e.ctx, l);
        u.B = __builtin_amdgcn_readlane(e.B, l);
        u.qoff = __builtin_amdgcn_readlane(e.qoff, l);
        u.js = __builtin_amdgcn_readlane(e.js, l);
        u.np = __builtin_amdgcn_readlane(e.np, l);
        u.slot0 = __builtin_amdgcn_readlane(e.slot0, l);
        u.merge0 = __builtin_amdgcn_readlane(e.merge0, l);
        const ChunkSeq q{u.ctx, u.B, a.P, a.G, a.causal};
        for (int t = lane; t < u.js * a.Hkv; t += 64) {
          const int g = t / u.js, j = t - g * u.js;
          a.merges[u.merge0 + t] = ChunkMerge{u.qoff + j * a.P, g, q.rows(j), q.keys(j), u.np, u.slot(g, j, 0), {0, 0}};
        }
      }
    }
  }
}

// Another queue that has items left, or -1.  (One that was empty once stays so.)
__device__ __forceinline__ int chunk_other(const ChunkArgs &a, int x) {
  int next[kChunkQueues], found = -1;
#pragma unroll
  for (int o = 1; o < kChunkQueues; ++o)
    next[o] = __hip_atomic_load(&a.head->next[x ^ o].v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
  for (int o = 1; o < kChunkQueues; ++o)
    if (next[o] < a.head->count[x ^ o]) found = x ^ o;
  return found;
}
__device__ __forceinline__ int chunk_take(const ChunkArgs &a, int x) {
  return __hip_atomic_fetch_add(&a.head->next[x].v, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The group of queue x that holds item i: the last whose first item is at most i.  k: where to look from, and its place.
__device__ __forceinline__ int chunk_group(const ChunkArgs &a, int x, int i, int &k, int *first) {
  const int lane = threadIdx.x & 63;
  const int n = chunk_groups((long long)a.S * a.Hkv, x), stride = (a.S * a.Hkv + kChunkQueues - 1) / kChunkQueues;
  for (int k0 = k & ~63; k0 < n; k0 += 64) {
    const int p = a.prefix[x * stride + min(k0 + lane, n - 1)];
    const unsigned long long le = __ballot(k0 + lane < n && p <= i);
    if (!le) break;
    const int l = 63 - __clzll((long long)le);
    k = k0 + l;
    *first = __builtin_amdgcn_readlane(p, l);
    if (l < 63) break;
  }
  return x + kChunkQueues * k;
}

// Tile b of the batch, sequences in order, within one the heads, within one the tiles: its sequence, head and number.
__device__ __forceinline__ bool chunk_tile(const ChunkArgs &a, int b, ChunkEntry &e, int &g, int &j) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int c0 = 0; c0 < a.S; c0 += 64) {
    const int k = min(c0 + lane, a.S - 1);  // clamped: no per-load branch
    const ChunkSeq q = chunk_seq(a, k);
    const int off = a.q_offsets[k], nt = c0 + lane < a.S ? q.tiles() : 0;
    const int items = nt * a.Hkv, incl = before + wave_scan_i(items);
    const unsigned long long hit = __ballot(incl > b && incl - items <= b);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;  // wave-uniform
      e.s = c0 + l;
      e.ctx = __builtin_amdgcn_readlane(q.ctx, l);
      e.B = __builtin_amdgcn_readlane(q.B, l);
      e.qoff = __builtin_amdgcn_readlane(off, l);
      const int n = __builtin_amdgcn_readlane(nt, l), r = b - __builtin_amdgcn_readlane(incl - items, l);
      g = r / n;
      j = r - g * n;
      return true;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// Weights are taken against the row's maximum when it was last looked for.  It is looked for again only
// where a lane's 32 weights of a step sum to more than this: bf16 and fp32 hold such weights no less exactly,
// and nearly every step does without the maximum, its exchange between lanes and the rescaling of O.
constexpr float kChunkSum = 4096.f;

// Fetches 16 bytes a lane from base + off to LDS bytes dst + 16 * lane.  As assembly without outputs: the
// compiler knows of no transfer in flight and so makes no LDS read wait for all of them, as it does
// after the builtin; the waits are chunk_phase_end's.  (Its own waits for vector loads count the transfers
// as well, so they only grow stricter.)  The five wait states are those between a lane read that may
// have written the base and a vector load from it, which the compiler sees to only for its own.
__device__ __forceinline__ void chunk_load_lds(const char *base, unsigned off, unsigned dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(off), "s"(base)
               : "m0", "memory");
}

// Ends a phase: this wavefront's LDS reads are done, and all but its N youngest transfers (N < 0: no
// matter which), before the barrier.  (__syncthreads would wait for every transfer in flight.)
template <int N>
__device__ __forceinline__ void chunk_phase_end() {
  if constexpr (N < 0) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int V>
using Int = std::integral_constant<int, V>;

// How the workgroups find their work: items of the plan; whole tiles by their index; the same with tiles of 128
// rows, whose steps the two halves of the workgroup take in turn and join at the end: twice the workgroups, each
// with half the steps of half the rows, where a batch leaves CUs idle (100 rows at 500 keys, 32 heads on 8: 17.2 us, of
// which ten steps of 256 rows would take 21.8; a step of 128 keys takes the 3400 cycles of one of 64 with 256 rows).
enum ChunkMode { kPlanned, kDirect, kHalves };

template <int D, ChunkMode MODE>
__global__ __launch_bounds__(512) void chunk_attn_kernel(ChunkArgs a) {
  constexpr bool PLANNED = MODE == kPlanned, HALVES = MODE == kHalves;
  using T = ChunkTile<D>;
  constexpr int NST = D / 16, NDT = D / 32, EB = 2;
  __shared__ __attribute__((aligned(1024))) char stages[4 * T::STAGEB];  // a K and a V tile each
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups take the items of their XCD's queue, then those of the others.  Any may take any item: no result
  // depends on which.  The next item is asked for at the end of one.
  __shared__ int ticket[2];
  int queue = blockIdx.x % kChunkQueues, ahead = blockIdx.x / kChunkQueues;
  [[maybe_unused]] int looked = -1, place = 0;
  for (;;) {  // one pass per item
    ChunkEntry e{};
    int g, j, piece, n, k0, k1;  // keys [0, n) are visible to some row; the item takes [k0, k1)
    if constexpr (PLANNED) {
      if (tid == 0) {
        while (ahead >= a.head->count[queue]) {
          queue = chunk_other(a, queue);
          if (queue < 0) break;
          ahead = chunk_take(a, queue);
        }
        ticket[0] = queue;
        ticket[1] = ahead;
      }
      __syncthreads();
      const int x = __builtin_amdgcn_readfirstlane(ticket[0]), item = __builtin_amdgcn_readfirstlane(ticket[1]);
      __syncthreads();  // read by all before the next
      if (x < 0) break;
      if (x != looked) place = 0;  // a queue's items come in order
      looked = x;
      int first = 0;
      const int group = chunk_group(a, x, item, place, &first), er = group / a.Hkv;
      g = group - er * a.Hkv;
      typedef const __attribute__((address_space(4))) ChunkEntry CE;  // scalar loads
      CE *ep = (CE *)(a.entries + er);
      e.s = ep->s, e.ctx = ep->ctx, e.B = ep->B, e.qoff = ep->qoff;
      e.nt = ep->nt, e.js = ep->js, e.np = ep->np, e.slot0 = ep->slot0;
      j = e.tile(item - first);
      piece = e.piece(item - first);
      n = ChunkSeq{e.ctx, e.B, a.P, a.G, a.causal}.keys(j);
      k0 = piece < 0 ? 0 : chunk_piece(n, e.np, piece);
      k1 = piece < 0 ? n : chunk_piece(n, e.np, piece + 1);
      if (k0 >= k1) {  // uniform per workgroup
        if (tid == 0) ahead = chunk_take(a, queue);
        continue;
      }
    } else {  // workgroup b takes whole tile b, if there is one
      if (!chunk_tile(a, blockIdx.x, e, g, j)) break;
      piece = -1;
      n = ChunkSeq{e.ctx, e.B, a.P, a.G, a.causal}.keys(j);
      k0 = 0;
      k1 = n;
    }
    const ChunkSeq seq{e.ctx, e.B, a.P, a.G, a.causal};
    const int p0 = j * a.P, M = seq.rows(j);  // the tile's first position and its rows

    // ---- query operands: element e of step st is dim st*16 + h*8 + e of row m ----
    bf16x8 qop[NST];
    const int rwave = HALVES ? wave & 3 : wave;  // which 32 rows
    const int m = rwave * 32 + l32, mc = min(m, M - 1), mp = mc / a.G;  // rows past the tile: its last
    const int lim = a.causal ? e.ctx + p0 + mp + 1 : n;            // keys the row sees
    {
      const char *qrow = (const char *)a.q + ((size_t)(e.qoff + p0 + mp) * a.Hq + g * a.G + (mc - mp * a.G)) * D * EB;
#pragma unroll
      for (int st = 0; st < NST; ++st) qop[st] = *(const bf16x8 *)(qrow + (st * 16 + h * 8) * EB);
    }
    const int vis_all = min(k1, a.causal ? e.ctx + p0 + min(rwave * 32, M - 1) / a.G + 1 : n);  // keys that all its rows see
    const bool act = rwave * 32 < M;  // the wavefront has rows

    f32x16 oacc[NDT];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;

    // ---- key and value tiles: wavefronts 0-3 fetch rows 16w .. 16w + 15 of K, 4-7 those of V; they lie in one page ----
    const int *table = a.block_table + (size_t)e.s * a.max_pages;
    const bool isv = wave >= 4;
    const int frow = (wave & 3) * 16;
    const char *pool = (const char *)(isv ? a.v : a.k);
    const int pmask = (1 << a.page_log2) - 1;
    constexpr int RPI = 64 / T::CPR;  // rows of one load of a wavefront
    const int lane_row = lane / T::CPR;
    // The lane's vector of load i: row i * RPI + lane_row, whose swizzle differs from load 0's by 4i (K) or
    // not at all (V).
    const unsigned off0 = ((lane % T::CPR) ^ (isv ? T::swz_v(lane_row) : T::swz_k(lane_row))) * 16 + lane_row * T::ROWB;
    const unsigned flip = isv ? 0 : 64;
    auto page_of = [&](int t) __attribute__((always_inline)) {
      const int kw = __builtin_amdgcn_readfirstlane(min(k0 + t * kChunkKT + frow, k1 - 1));
      return ld_uniform(table, min(kw >> a.page_log2, a.max_pages - 1));
    };
    const unsigned lds0 = (unsigned)(uintptr_t)(char SDB_LDS *)(SDB_LDS void *)stages;
    const char *src;  // of tile t: the wavefront's first row, in its page; rows past the last key re-read it (what
    unsigned dst;     // lies behind it may hold anything), and a tile behind the last one is that key throughout
    int most;         // the wavefront's last row that holds a key
    auto start = [&](int t, int page_id) __attribute__((always_inline)) {
      const int pg = min(max(page_id, 0), a.num_pages - 1), kw = k0 + t * kChunkKT + frow, last = k1 - 1;
      most = max(last - kw, 0);
      src = pool + ((((size_t)pg * a.Hkv + g) << a.page_log2) + (min(kw, last) & pmask)) * T::ROWB;
      dst = lds0 + (t & 3) * T::STAGEB + (isv ? T::TILEB : 0) + frow * T::ROWB;
    };
    auto load = [&](int i) __attribute__((always_inline)) {
      const int back = max(i * RPI + lane_row - most, 0);
      chunk_load_lds(src, (off0 ^ (i * flip)) + i * 1024 - back * T::ROWB, dst + i * 1024);
    };
    // LDS addresses of the lane's operands in stage 0.  K: row l32, its 16-byte vectors 2 st + h.  V^T: lane l of
    // a 16-lane group reads 4 dims of key row (l % 16) / 4 of four and receives, of dim 16 ((l / 16) % 2) +
    // l % 16 of 32, those four keys.  Step st and dims dt only flip bits of the address.
    const unsigned kaddr = lds0 + l32 * T::ROWB + ((h ^ T::swz_k(l32)) << 4);
    const int vrow = 4 * h + ((lane & 15) >> 2);
    const unsigned vaddr = lds0 + T::TILEB + vrow * T::ROWB + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ T::swz_v(vrow)) << 4) +
                           ((lane & 1) << 3);

    // Step t of a wavefront takes tile t; of a half's, tile 2t or 2t + 1, which may lie behind the last key.
    const int nsteps = (k1 - k0 + kChunkKT * (HALVES ? 2 : 1) - 1) / (kChunkKT * (HALVES ? 2 : 1));
    auto tile_of = [&](int t) __attribute__((always_inline)) { return HALVES ? 2 * t + (wave >= 4) : t; };
    // ---- the products and the softmax of a step ----
    f32x16 sacc[2];  // [kb]: register i is key kb*32 + 8*(i/4) + 4h + i%4 of row l32
    bf16x8 pop[4];   // the weights of 16 keys each
    // Products FROM .. TO - 1 of a step: NP of O^T += V^T P^T (tile t - 1), then those of S^T = K Q^T (tile t).
    // Each product's left operand is read kAhead products before it; the order stays as written.
    constexpr int NP = 4 * NDT, NPQ = NP + 2 * NST, kAhead = D == 128 ? 8 : 6;
    auto operand = [&](int i, unsigned va, unsigned ka) __attribute__((always_inline)) {
      if (i < NP) {
        const int ks = i / NDT, dt = i % NDT;
        s16x4c vv[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          vv[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (s16x4c SDB_LDS *)(uintptr_t)((va ^ (dt << 6)) + (ks * 16 + u * 8) * T::ROWB));
        const s16x8c v8 = {vv[0][0], vv[0][1], vv[0][2], vv[0][3], vv[1][0], vv[1][1], vv[1][2], vv[1][3]};
        return __builtin_bit_cast(bf16x8, v8);
      }
      const int st = (i - NP) / 2, kb = (i - NP) % 2;
      return *(const bf16x8 SDB_LDS *)(uintptr_t)((ka ^ (st << 5)) + kb * 32 * T::ROWB);
    };
    // The first operands of P V of step t are read at the end of its softmax, before the phase that multiplies, so
    // that its products need not wait for them (2048 rows at 65536 keys 1.91 -> 1.85 ms, 8192 rows 501 -> 489 us).  V of step
    // t is there by then, but not in a workgroup of halves.  At head_dim 64 the softmax is the longer phase, and what is
    // added to it costs more (1.25 ms without, 1.33 with).
    constexpr bool EARLY = D == 128 && !HALVES;
    bf16x8 first[kAhead];
    auto read_first = [&](int t) __attribute__((always_inline)) {
      unsigned va = vaddr + (tile_of(t) & 3) * T::STAGEB;
      asm("" : "+v"(va));
#pragma unroll
      for (int i = 0; i < kAhead; ++i) first[i] = operand(i, va, 0);
    };
    auto products = [&](auto from_c, auto to_c, int t, auto loads_c) __attribute__((always_inline)) {
      constexpr int FROM = decltype(from_c)::value, TO = decltype(to_c)::value;
      unsigned va = vaddr + (tile_of(t - 1) & 3) * T::STAGEB, ka = kaddr + (tile_of(t) & 3) * T::STAGEB;
      asm("" : "+v"(va), "+v"(ka));  // the operands' addresses are made here, in the products' shadow, not kept in registers
      bf16x8 op[NPQ];
      auto read = [&](int i) __attribute__((always_inline)) { op[i] = operand(i, va, ka); };
#pragma unroll
      for (int i = FROM; i < FROM + kAhead; ++i) {
        if (FROM == 0 && EARLY) {
          op[i] = first[i];
        } else {
          read(i);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = FROM; i < TO; ++i) {
        if (i < NP) {
          oacc[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], pop[i / NDT], oacc[i % NDT], 0, 0, 0);
        } else {
          const int st = (i - NP) / 2, kb = (i - NP) % 2;
          if (st == 0) {
            f32x16 zero;
#pragma unroll
            for (int e = 0; e < 16; ++e) zero[e] = 0.f;
            sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], qop[0], zero, 0, 0, 0);
          } else {
            sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], qop[st], sacc[kb], 0, 0, 0);
          }
        }
        if (i + kAhead < TO) read(i + kAhead);
        if (decltype(loads_c)::value && i % 2 == 1 && i / 2 < T::NV) load(i / 2);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto softmax = [&](int kt) __attribute__((always_inline)) {
      if (kt + kChunkKT > vis_all) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (kt + kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3) >= min(lim, k1)) sacc[kb][i] = -INFINITY;
      }
      // The weights against a reference (log2 units), to the second product's operands; their sum.
      auto weights = [&](float ref) __attribute__((always_inline)) {
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x16 &sc = sacc[ks >> 1];
            const int i = 8 * (ks & 1) + 2 * e;
            const float x = fast_exp2(fmaf(sc[i], a.scale_log2, -ref)), y = fast_exp2(fmaf(sc[i + 1], a.scale_log2, -ref));
            w[e] = cvt_pk_bf16(x, y);
            sum[0] += x;
            sum[1] += y;
          }
          pop[ks] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
        }
        return sum[0] + sum[1];
      };
      float sum = weights(m_run);
      if (__any(!(sum <= kChunkSum))) {  // also before the first key (the reference is -inf) and where a sum is no number
        float tmax = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, sacc[kb][i]);
        const float2 pm = pair_x32(tmax);
        const float mnew = fmaxf(m_run, fmaxf(pm.x, pm.y) * a.scale_log2);
        const float alpha = mnew == -INFINITY ? 1.f : fast_exp2(m_run - mnew);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) oacc[dt] *= alpha;
        m_run = mnew;
        sum = weights(mnew == -INFINITY ? 0.f : mnew);
      }
      l_run += sum;
    };

    // ---- the steps ----
    // The two wavefronts of a SIMD (w and w + 4) take turns at its matrix unit: in phase 2t the first four
    // multiply P V of step t - 1 and Q K of step t while the others take the softmax of step t - 1, in
    // phase 2t + 1 the first take the softmax of step t while the others multiply.  A barrier ends each
    // phase.  A wavefront fetches its part of tile t + 2 while it multiplies, in phase 2t or 2t + 1, into the
    // stage that was last read in phase 2t - 1; it has to be there for phase 2t + 4.
    const bool second = wave >= 4;
    auto load_all = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < T::NV; ++i) load(i);
    };
    if constexpr (HALVES) {
      // Both tiles of a step are fetched together, and the ring holds two steps: the first half fetches K of step t + 1
      // in phase 2t, as its stages were last read in phase 2t - 1, to be there for phase 2t + 2; the second half V of
      // step t + 1 in phase 2t + 2, as its stages were last read in phase 2t + 1, for phase 2t + 4.  (Each half its own
      // tiles, three phases ahead, was no faster.)
      auto fetch = [&](int t, int i0, int i1) __attribute__((always_inline)) {
        start(2 * t, i0);
        load_all();
        start(2 * t + 1, i1);
        load_all();
      };
      {
        const int i0 = page_of(0), i1 = page_of(1), i2 = page_of(2), i3 = page_of(3);
        fetch(0, i0, i1);
        fetch(1, i2, i3);
      }
      int i0 = page_of(4), i1 = page_of(5);
#pragma unroll
      for (int st = 0; st < NST; ++st) asm volatile("" : "+v"(qop[st]));
      chunk_phase_end<2 * T::NV>();       // the first step's tiles are here
      if (second) chunk_phase_end<-1>();  // phase 0
      if (act) products(Int<NP>{}, Int<NPQ>{}, 0, Int<0>{});
      if (second) chunk_phase_end<0>();
      else chunk_phase_end<-1>();
      if (act) softmax(k0 + tile_of(0) * kChunkKT);
      if (second) chunk_phase_end<-1>();
      else chunk_phase_end<0>();
      for (int t = 1; t < nsteps; ++t) {
        if (!second) fetch(t + 1, i0, i1);
        if (act) {
          __builtin_amdgcn_s_setprio(1);
          products(Int<0>{}, Int<NPQ>{}, t, Int<0>{});
          __builtin_amdgcn_s_setprio(0);
        }
        if (second) {
          chunk_phase_end<0>();
          fetch(t + 1, i0, i1);
        } else {
          chunk_phase_end<-1>();
        }
        i0 = page_of(2 * t + 4);
        i1 = page_of(2 * t + 5);
        if (act) softmax(k0 + tile_of(t) * kChunkKT);
        if (second) chunk_phase_end<-1>();
        else chunk_phase_end<0>();
      }
    } else {
      {
        const int id0 = page_of(0), id1 = page_of(1);
        start(0, id0);
        load_all();
        start(1, id1);
        load_all();
      }
      int id = page_of(2);
#pragma unroll
      for (int st = 0; st < NST; ++st) asm volatile("" : "+v"(qop[st]));  // waited for here, not in the loop
      chunk_phase_end<T::NV>();                // tile 0 is here
      if (second) chunk_phase_end<-1>();  // phase 0
      start(2, id);
      id = page_of(3);
      load_all();
      if (act) products(Int<NP>{}, Int<NPQ>{}, 0, Int<0>{});
      auto between = [&]() __attribute__((always_inline)) {  // the products of a step and its softmax
        if (second) chunk_phase_end<T::NV>();  // the next tile is here
        else chunk_phase_end<-1>();
      };
      auto behind = [&](int t) __attribute__((always_inline)) {  // the softmax of step t
        if (EARLY && act) read_first(t);
        if (second) chunk_phase_end<-1>();
        else chunk_phase_end<T::NV>();
      };
      between();
      if (act) softmax(k0);
      behind(0);
      for (int t = 1; t < nsteps; ++t) {
        start(t + 2, id);
        id = page_of(t + 3);
        if (act) {
          __builtin_amdgcn_s_setprio(1);
          products(Int<0>{}, Int<NPQ>{}, t, Int<1>{});
          __builtin_amdgcn_s_setprio(0);
        } else {
          load_all();
        }
        between();
        if (act) softmax(k0 + t * kChunkKT);
        behind(t);
      }
    }
    if constexpr (PLANNED) {
      if (tid == 0) ahead = chunk_take(a, queue);
    }
    if (act) products(Int<0>{}, Int<NP>{}, nsteps, Int<0>{});
    chunk_phase_end<0>();  // no transfer is on its way, and (second) every wavefront is done with the tiles
    if (!second) chunk_phase_end<-1>();

    // ---- output: register i of oacc[dt] is dim dt*32 + 8*(i/4) + 4h + i%4 of row l32 ----
    const float2 pl = pair_x32(l_run);
    const float lsum = pl.x + pl.y;
    if constexpr (HALVES) {
      // Each half takes the dims of half of O and gives its partner's to it.
      float4 *const give = (float4 *)stages + wave * (NDT * 2) * 64 + lane, *const take = (float4 *)stages + (wave ^ 4) * (NDT * 2) * 64 + lane;
      float2 *const ml = (float2 *)(stages + 8 * (NDT * 2) * 64 * 16);
      auto give_half = [&](auto own_c) __attribute__((always_inline)) {
        constexpr int OTHER = decltype(own_c)::value ? 0 : NDT / 2;
#pragma unroll
        for (int d = 0; d < NDT / 2; ++d)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const f32x16 &o = oacc[OTHER + d];
            give[(d * 4 + c) * 64] = float4{o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]};
          }
      };
      if (second) give_half(Int<1>{});
      else give_half(Int<0>{});
      if (h == 0) ml[wave * 32 + l32] = float2{m_run, lsum};
      __syncthreads();
      const float2 x = ml[(wave ^ 4) * 32 + l32];
      const float mx = fmaxf(m_run, x.x);
      const float wo = m_run == -INFINITY ? 0.f : fast_exp2(m_run - mx), wx = x.x == -INFINITY ? 0.f : fast_exp2(x.x - mx);
      const float inv = 1.f / (lsum * wo + x.y * wx);
      auto join = [&](auto own_c) __attribute__((always_inline)) {
        constexpr int OWN = decltype(own_c)::value ? NDT / 2 : 0;
        char *orow = (char *)a.out + ((size_t)(e.qoff + p0 + mp) * a.Hq + g * a.G + (m - mp * a.G)) * D * EB;
#pragma unroll
        for (int d = 0; d < NDT / 2; ++d)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const f32x16 &o = oacc[OWN + d];
            const float4 y = take[(d * 4 + c) * 64];
            const float z0 = (o[4 * c] * wo + y.x * wx) * inv, z1 = (o[4 * c + 1] * wo + y.y * wx) * inv;
            const float z2 = (o[4 * c + 2] * wo + y.z * wx) * inv, z3 = (o[4 * c + 3] * wo + y.w * wx) * inv;
            *(uint2 *)(orow + ((OWN + d) * 32 + c * 8 + h * 4) * EB) = uint2{cvt_pk_bf16(z0, z1), cvt_pk_bf16(z2, z3)};
          }
      };
      if (m < M) {
        if (second) join(Int<1>{});
        else join(Int<0>{});
      }
    } else if (m < M && piece < 0) {
      const float inv = 1.f / lsum;
      char *orow = (char *)a.out + ((size_t)(e.qoff + p0 + mp) * a.Hq + g * a.G + (m - mp * a.G)) * D * EB;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x16 &o = oacc[dt];
          *(uint2 *)(orow + (dt * 32 + c * 8 + h * 4) * EB) =
              uint2{cvt_pk_bf16(o[4 * c] * inv, o[4 * c + 1] * inv), cvt_pk_bf16(o[4 * c + 2] * inv, o[4 * c + 3] * inv)};
        }
    } else if (m < M) {
      // as the registers stand, so that a store is 1 KB in one place: vector (wave, dt, c, lane) of the slot
      const size_t slot = e.slot(g, j, piece);
      f32x4 *po = (f32x4 *)(a.part_o + slot * kChunkRows * D) + (wave * NDT * 4) * 64 + lane;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x16 &o = oacc[dt];
          __builtin_nontemporal_store(f32x4{o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]}, po + (dt * 4 + c) * 64);
        }
      if (h == 0) a.part_ml[slot * kChunkRows + m] = float2{m_run, lsum};
    }
    if constexpr (!PLANNED) break;
  }
}

// Joins the pieces of the cut tiles:
//   O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i,  M = max_i m_i
// A workgroup takes the 32 rows that were one wavefront's, its four wavefronts a quarter of their vectors each.
constexpr int kChunkMergeUnits = 8;  // of a tile
template <int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a) {
  constexpr int NVEC = D / 8 / 4;  // vectors a lane joins
  const int lane = threadIdx.x & 63, quarter = threadIdx.x >> 6, h = lane >> 5;
  const int units = ld_uniform(&a.head->merges, 0) * kChunkMergeUnits;
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const ChunkMerge t = a.merges[u / kChunkMergeUnits];
    const int wave = u % kChunkMergeUnits, m = wave * 32 + (lane & 31);
    if (m >= t.rows) continue;
    const float2 *ml = a.part_ml + (size_t)t.slot * kChunkRows + m;
    const f32x4 *po = (const f32x4 *)(a.part_o + (size_t)t.slot * kChunkRows * D) + (wave * (D / 8) + quarter * NVEC) * 64 + lane;
    float mx = -INFINITY, lsum = 0.f;
    f32x4 acc[NVEC];
#pragma unroll
    for (int v = 0; v < NVEC; ++v) acc[v] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
    for (int k = 0; k < t.np; ++k) {
      if (chunk_piece(t.keys, t.np, k) >= chunk_piece(t.keys, t.np, k + 1)) continue;  // an empty piece
      const float2 x = ml[(size_t)k * kChunkRows];
      f32x4 o[NVEC];
#pragma unroll
      for (int v = 0; v < NVEC; ++v) o[v] = po[(size_t)k * (kChunkRows * D / 4) + v * 64];
      // a piece with no visible key (one whose scores are no numbers has no reference either, but a sum that is none)
      if (x.x == -INFINITY && x.y == 0.f) continue;
      const float mn = fmaxf(mx, x.x), wo = mx == -INFINITY ? 0.f : fast_exp2(mx - mn), wn = fast_exp2(x.x - mn);
      lsum = lsum * wo + x.y * wn;
#pragma unroll
      for (int v = 0; v < NVEC; ++v) acc[v] = acc[v] * wo + o[v] * wn;
      mx = mn;
    }
    const float inv = 1.f / lsum;
    const int mp = m / a.G;
    char *orow = (char *)a.out + ((size_t)(t.row0 + mp) * a.Hq + t.g * a.G + (m - mp * a.G)) * D * 2;
#pragma unroll
    for (int v = 0; v < NVEC; ++v) {
      const int i = quarter * NVEC + v;  // dt * 4 + c
      *(uint2 *)(orow + ((i >> 2) * 32 + (i & 3) * 8 + h * 4) * 2) =
          uint2{cvt_pk_bf16(acc[v][0] * inv, acc[v][1] * inv), cvt_pk_bf16(acc[v][2] * inv, acc[v][3] * inv)};
    }
  }
}

#endif  // __HIPCC__

}  // namespace sdb
