// chunk.hpp -- attention of chunks of new tokens over page pools: the B_s rows of sequence s, any
// number of them, attend to their committed context and to the chunk itself.
//
// A query tile is P = 256 / G positions of one (sequence, kv head) with the G query heads of each, up
// to 256 rows, so a key row that a workgroup fetches serves all of them.  A workgroup of eight
// wavefronts takes a tile, 32 rows a wavefront, and walks its keys 64 at a time:
//   S^T = K Q^T    (32x32x16 bf16 matrix products, fp32 sums)
//   P = exp2(S^T c - m), running row maximum m and row sum l in fp32
//   O^T = O^T 2^(m_old - m) + V^T P^T   (P rounded to bf16 for the product; O^T fp32 in registers)
// Scores come transposed, so a lane holds the scores of one query row (32 of a tile's 64 keys, its
// partner lane the others) and the softmax needs one exchange between two lanes.  The weights then
// are the right operand of the second product as they stand: the products' inner index runs over
// keys in the order in which the first product left them, and V^T is read in that order.
#pragma once

#include "attn.hpp"

namespace sdb {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4c __attribute__((ext_vector_type(4)));
typedef short s16x8c __attribute__((ext_vector_type(8)));

constexpr int kChunkRows = 256;  // query rows of a tile
constexpr int kChunkKT = 64;     // keys of a step

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
};

template <int D>
struct ChunkTile {
  static constexpr int ROWB = D * 2;                   // bytes of a key row
  static constexpr int CPR = ROWB / 16;                // 16-byte vectors of a row
  static constexpr int TILEB = kChunkKT * ROWB;        // bytes of a K (or V) tile
  static constexpr int NV = 16 * CPR / 64;             // vectors a lane fetches: 16 rows of K or of V a wavefront
  // A row's vectors are stored at their index XOR these, so that the 16 lanes an operand read serves at a
  // time touch distinct banks: 16 rows at one vector index of K, 4 rows at 4 indices of V.
  __device__ static int swz_k(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  __device__ static int swz_v(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }
};

struct ChunkItem {
  int s, g, ctx, B, qoff, p0;  // p0: the tile's first position in the chunk
};

// Tile b of the batch: sequences in order, within one the kv heads in order, within one the tiles from
// the last to the first (under the causal mask the last has the most keys).
__device__ __forceinline__ bool chunk_item(const ChunkArgs &a, int b, ChunkItem &it) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int c0 = 0; c0 < a.S; c0 += 64) {
    const int k = min(c0 + lane, a.S - 1);  // clamped: no per-load branch
    const int ctx = a.ctx_lens[k], B = a.chunk_lens[k], off = a.q_offsets[k];
    const int nt = c0 + lane < a.S && B > 0 ? (B + a.P - 1) / a.P : 0;
    const int items = nt * a.Hkv, incl = before + wave_scan_i(items);
    const unsigned long long hit = __ballot(incl > b && incl - items <= b);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;  // wave-uniform
      it.s = c0 + l;
      it.ctx = __builtin_amdgcn_readlane(ctx, l);
      it.B = __builtin_amdgcn_readlane(B, l);
      it.qoff = __builtin_amdgcn_readlane(off, l);
      const int n = __builtin_amdgcn_readlane(nt, l), r = b - __builtin_amdgcn_readlane(incl - items, l);
      it.g = r / n;
      it.p0 = (n - 1 - (r - it.g * n)) * a.P;
      return true;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// The running maximum may lag behind a row's scores by this much (log2 units) before the sums are
// rescaled: weights then are at most 2^8 instead of 1, which changes no relative rounding, and the
// rescaling of O, half as much work as the rest of the softmax, is left out of nearly every step.
constexpr float kChunkLag = 8.f;

template <int D>
__global__ __launch_bounds__(512) void chunk_attn_kernel(ChunkArgs a) {
  using T = ChunkTile<D>;
  constexpr int NST = D / 16, NDT = D / 32, EB = 2;
  __shared__ __attribute__((aligned(1024))) char lds_raw[2][2 * T::TILEB];
  ChunkItem it;
  if (!chunk_item(a, blockIdx.x, it)) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int np = min(a.P, it.B - it.p0), M = np * a.G;  // the tile's positions and rows
  const int k1 = it.ctx + (a.causal ? it.p0 + np : it.B);  // keys [0, k1) are visible to some row

  // ---- query operands: element e of step st is dim st*16 + h*8 + e of row m ----
  bf16x8 qop[NST];
  const int m = wave * 32 + l32, mc = min(m, M - 1), mp = mc / a.G;  // rows past the tile: its last
  const int lim = a.causal ? it.ctx + it.p0 + mp + 1 : k1;           // keys the row sees
  {
    const char *qrow = (const char *)a.q + ((size_t)(it.qoff + it.p0 + mp) * a.Hq + it.g * a.G + (mc - mp * a.G)) * D * EB;
#pragma unroll
    for (int st = 0; st < NST; ++st) qop[st] = *(const bf16x8 *)(qrow + (st * 16 + h * 8) * EB);
  }
  // keys that all / some of the wavefront's rows see
  const int pw0 = min(wave * 32, M - 1) / a.G, pw1 = min(wave * 32 + 31, M - 1) / a.G;
  const int vis_all = a.causal ? it.ctx + it.p0 + pw0 + 1 : k1;
  const int vis_any = wave * 32 >= M ? 0 : a.causal ? it.ctx + it.p0 + pw1 + 1 : k1;

  f32x16 oacc[NDT];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;

  // ---- key and value tiles: wavefronts 0-3 fetch rows 16w .. 16w + 15 of K, 4-7 those of V; they lie in one page ----
  const int *table = a.block_table + (size_t)it.s * a.max_pages;
  const bool isv = wave >= 4;
  const int frow = (wave & 3) * 16;
  const char *pool = (const char *)(isv ? a.v : a.k);
  v4u32 reg[T::NV];  // a vector type: an array of the u32x4 struct is copied through private memory
  const int pmask = (1 << a.page_log2) - 1;
  auto fetch = [&](int key0) {  // rows past the last key re-read it (rows behind it may hold anything)
    const int kw = __builtin_amdgcn_readfirstlane(min(key0 + frow, k1 - 1));
    const int pg = min(max(ld_uniform(table, min(kw >> a.page_log2, a.max_pages - 1)), 0), a.num_pages - 1);
    const char *page = pool + ((((size_t)pg * a.Hkv + it.g) << a.page_log2)) * T::ROWB;
#pragma unroll
    for (int i = 0; i < T::NV; ++i) {
      const int v = i * 64 + lane, r = v / T::CPR, c = v % T::CPR;
      const int key = min(key0 + frow + r, k1 - 1);
      reg[i] = *(const v4u32 *)(page + (unsigned)((key & pmask) * T::ROWB + c * 16));
    }
  };
  auto stash = [&](char *stage) {
#pragma unroll
    for (int i = 0; i < T::NV; ++i) {
      const int v = i * 64 + lane, r = frow + v / T::CPR, c = v % T::CPR;
      *(v4u32 *)(stage + (isv ? T::TILEB : 0) + r * T::ROWB + ((c ^ (isv ? T::swz_v(r) : T::swz_k(r))) << 4)) = reg[i];
    }
  };
  // V^T operand: lane l of a 16-lane group reads 4 dims of key row (l % 16) / 4 of four and receives, of
  // dim 16 * ((l / 16) % 2) + l % 16 of the 32, those four keys.
  const int vrow = 4 * h + ((lane & 15) >> 2);
  const int vcol = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);  // 16-byte vector of the 32 dims

  const int ntiles = (k1 + kChunkKT - 1) / kChunkKT;
  fetch(0);
  for (int t = 0; t < ntiles; ++t) {
    char *stage = lds_raw[t & 1];
    stash(stage);
    __syncthreads();  // the tile is there for every wavefront
    const int kt = t * kChunkKT;
    if (t + 1 < ntiles) fetch(kt + kChunkKT);
    if (kt >= vis_any) continue;  // uniform per wavefront

    f32x16 sacc[2];  // [kb]: register i is key kb*32 + 8*(i/4) + 4h + i%4 of row l32
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sacc[kb][i] = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int st = 0; st < NST; ++st) {
        const int r = kb * 32 + l32;
        const bf16x8 kf = *(const bf16x8 *)(stage + r * T::ROWB + (((2 * st + h) ^ T::swz_k(r)) << 4));
        sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qop[st], sacc[kb], 0, 0, 0);
      }
    if (kt + kChunkKT > vis_all) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (kt + kb * 32 + 8 * (i >> 2) + 4 * h + (i & 3) >= lim) sacc[kb][i] = -INFINITY;
    }
    float tmax = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, sacc[kb][i]);
    const float2 pm = pair_x32(tmax);
    const float mt = fmaxf(pm.x, pm.y) * a.scale_log2;
    if (__any(mt > m_run + kChunkLag)) {
      const float mnew = fmaxf(m_run, mt);
      const float alpha = mnew == -INFINITY ? 1.f : fast_exp2(m_run - mnew);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) oacc[dt] *= alpha;
      m_run = mnew;
    }
    const float muse = m_run == -INFINITY ? 0.f : m_run;
    float psum[2] = {0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sacc[kb][i] = fast_exp2(fmaf(sacc[kb][i], a.scale_log2, -muse));
        psum[kb] += sacc[kb][i];
      }
    l_run += psum[0] + psum[1];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const f32x16 &p = sacc[ks >> 1];
      const int i0 = 8 * (ks & 1);
      const u32x4 raw{cvt_pk_bf16(p[i0], p[i0 + 1]), cvt_pk_bf16(p[i0 + 2], p[i0 + 3]),
                      cvt_pk_bf16(p[i0 + 4], p[i0 + 5]), cvt_pk_bf16(p[i0 + 6], p[i0 + 7])};
      const bf16x8 pop = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        s16x4c vv[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = ks * 16 + u * 8 + vrow;
          const char *p8 = stage + T::TILEB + r * T::ROWB + (((4 * dt + vcol) ^ T::swz_v(r)) << 4) + ((lane & 1) << 3);
          vv[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4c SDB_LDS *)p8);
        }
        const s16x8c v8 = {vv[0][0], vv[0][1], vv[0][2], vv[0][3], vv[1][0], vv[1][1], vv[1][2], vv[1][3]};
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v8), pop, oacc[dt], 0, 0, 0);
      }
    }
  }

  // ---- output: register i of oacc[dt] is dim dt*32 + 8*(i/4) + 4h + i%4 of row l32 ----
  const float2 pl = pair_x32(l_run);
  const float inv = 1.f / (pl.x + pl.y);
  if (m >= M) return;
  char *orow = (char *)a.out + ((size_t)(it.qoff + it.p0 + mp) * a.Hq + it.g * a.G + (m - mp * a.G)) * D * EB;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const f32x16 &o = oacc[dt];
      *(uint2 *)(orow + (dt * 32 + c * 8 + h * 4) * EB) =
          uint2{cvt_pk_bf16(o[4 * c] * inv, o[4 * c + 1] * inv), cvt_pk_bf16(o[4 * c + 2] * inv, o[4 * c + 3] * inv)};
    }
}

}  // namespace sdb
