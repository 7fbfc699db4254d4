// rope.hpp -- norm of queries and keys per head and their rotation by position, in one pass, with
// or without the append of keys and values to page pools on the way.
//
// For a head's D dims x of a token at position t:
//   x^ = x / sqrt(mean(x^2) + eps) * w                                        (with a weight w [D])
//   pair i < R/2 turns by the angle t w_i:  (a, b) -> (a c - b s, b c + a s),  c, s = f cos, f sin
// Pair i is dims (i, R/2 + i), or neighbours (2i, 2i + 1); dims from R on pass.
//
// Bound by memory: every element is read once and written once, with about 10 operations between.
// 8192 bf16 tokens of 32 + 8 heads of 128 (168 MB) take 32.8 us, 5.1 TB/s, the rate of a large copy; prompt
// chunks of 5.9 thousand tokens appended to pages of 16 (145 MB) 30.9 us, 4.7 TB/s.  One token: 3.2 us, all latency.
// A lane takes the 8 pairs 8j .. 8j + 7 of one head (two 16-byte vectors in bf16, so both dims of a
// pair are in one lane and nothing is exchanged), D/16 lanes a head, so a wavefront takes 8 (D = 128) or
// 16 (D = 64) heads of one token; queries, keys and values of a token are one list of heads.  Each
// lane computes one angle, and the wavefront hands the cosines and sines round through LDS.  Four tokens of
// the same heads to a workgroup, in place of four parts of one token, were slower (appended chunks 36.2
// against 34.4 us).
// Everything between the load and the store is fp32, with one rounding to the element type at the
// end.  The angle is reduced in 64 bits, in turns (t * w_i / 2 pi less its nearest integer): in
// 32 bits position 2^20 alone would lose 0.06 rad.
#pragma once

#include "common.hpp"
#include "kvstep.hpp"

namespace sdb {

struct RopeArgs {
  const void *q, *k, *v;     // rows of q_stride / k_stride / v_stride elements
  void *q_out, *k_out;       // k_out, k_stride: contiguous callers only
  const float *inv_freq;     // [rot / 2]
  const void *qw, *kw;       // [D] or null: no norm
  const int *positions;      // [total_q]; the paged call goes by ctx_lens and q_offsets
  long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  int total_q, Hq, Hkv, rot, interleaved;
  float eps, rot_scale;
  int groups;                // wavefronts a token's heads take
  int once;                  // rows are loaded past the caches
  // paged call
  void *k_pages, *v_pages;   // [num_pages, Hkv, page_size, D]
  const int *ctx_lens, *q_offsets, *block_table;
  int S, page_log2, max_pages, num_pages;
};

// 16-byte vectors of 8 elements and their fp32 values.
template <bool BF16>
struct Vec8 {
  static constexpr int NV = BF16 ? 1 : 2;
  u32x4 raw[NV];
  __device__ __forceinline__ void load(const char *p) {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = reinterpret_cast<const u32x4 *>(p)[i];
  }
  __device__ __forceinline__ void load_once(const char *p) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const v4u32 v = __builtin_nontemporal_load(reinterpret_cast<const v4u32 *>(p) + i);
      raw[i] = u32x4{v[0], v[1], v[2], v[3]};
    }
  }
  __device__ __forceinline__ void store(char *p) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) reinterpret_cast<u32x4 *>(p)[i] = raw[i];
  }
  __device__ __forceinline__ void get(float *x) const {
    const uint32_t *w = &raw[0].x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (BF16) x[i] = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
      else x[i] = __uint_as_float(w[i]);
    }
  }
  __device__ __forceinline__ void set(const float *x) {
    uint32_t *w = &raw[0].x;
#pragma unroll
    for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
      if constexpr (BF16) w[i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
      else w[i] = __float_as_uint(x[i]);
    }
  }
};

// Sum over the D/16 lanes of a head (aligned groups of 4 or 8), the same in each.
template <int D>
__device__ __forceinline__ float head_sum(float x) {
  x += dpp_f<0xb1>(x);   // quad_perm 1,0,3,2
  x += dpp_f<0x4e>(x);   // quad_perm 2,3,0,1
  if constexpr (D == 128) x += dpp_f<0x141>(x);  // row_half_mirror: the other quad of the eight
  return x;
}

template <bool BF16, int D, bool PAGED>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int EB = BF16 ? 2 : 4;
  constexpr int LPH = D / 16;     // lanes per head
  constexpr int HPW = 64 / LPH;   // heads per wavefront
  __shared__ __attribute__((aligned(16))) float turn[4][2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LPH;
  const bool turned = 16 * j < a.rot;
  // the lane's two vectors: the halves of its pairs, or 16 dims in a row
  const int R2 = a.rot >> 1;
  const bool apart = turned && !a.interleaved;
  const int d0 = apart ? 8 * j : 16 * j, d1 = apart ? R2 + 8 * j : 16 * j + 8;
  const float freq = lane < R2 ? a.inv_freq[lane] : 0.f;
  const double per_turn = (double)freq * 0.15915494309189533577;  // turns per position
  float(&cs)[64] = turn[wave][0], (&sn)[64] = turn[wave][1];

  const long long n = (long long)a.total_q * a.groups;
  for (long long t = (long long)blockIdx.x * 4 + wave; t < n; t += (long long)gridDim.x * 4) {
    const int r = __builtin_amdgcn_readfirstlane((int)(t / a.groups));
    const int hh = (int)(t - (long long)r * a.groups) * HPW + lane / LPH;
    const int kv = hh < a.Hq ? 0 : hh < a.Hq + a.Hkv ? 1 : 2;  // query, key, value
    const bool live = hh < a.Hq + (PAGED ? 2 : 1) * a.Hkv;
    const int h = hh - (kv == 0 ? 0 : kv == 1 ? a.Hq : a.Hq + a.Hkv);
    const char *src = kv == 0 ? (const char *)a.q + ((long long)r * a.q_stride + h * D) * EB
                      : kv == 1 ? (const char *)a.k + ((long long)r * a.k_stride + h * D) * EB
                                : (const char *)a.v + ((long long)r * a.v_stride + h * D) * EB;
    Vec8<BF16> v0, v1;
    if (live && a.once) {
      v0.load_once(src + d0 * EB);
      v1.load_once(src + d1 * EB);
    } else if (live) {
      v0.load(src + d0 * EB);
      v1.load(src + d1 * EB);
    }
    // the token's position, and where its keys and values go
    int pos, seq = 0, pg = -1;
    if constexpr (PAGED) {
      row_owner_pos(a.q_offsets, a.ctx_lens, a.S, r, seq, pos);
      if (r >= ld_uniform(a.q_offsets, a.S)) continue;  // behind the last sequence: left as it was
      seq = __builtin_amdgcn_readfirstlane(seq);
      pos = __builtin_amdgcn_readfirstlane(pos);
      if (pos >= 0 && (pos >> a.page_log2) < a.max_pages)
        pg = ld_uniform(a.block_table, (long long)seq * a.max_pages + (pos >> a.page_log2));
    } else {
      pos = ld_uniform(a.positions, r);
    }
    {
      const double ang = (double)pos * per_turn;
      float s, c;
      sincospif((float)(2.0 * (ang - rint(ang))), &s, &c);
      cs[lane] = c * a.rot_scale;
      sn[lane] = s * a.rot_scale;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    if (!live) continue;
    char *dst;
    if (kv == 0) {
      dst = (char *)a.q_out + ((long long)r * a.q_out_stride + h * D) * EB;
    } else if constexpr (PAGED) {
      if (pg < 0 || pg >= a.num_pages) continue;  // past the table or outside the pool: not written
      const size_t row = (((size_t)pg * a.Hkv + h) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
      dst = (char *)(kv == 1 ? a.k_pages : a.v_pages) + row * D * EB;
    } else {
      dst = (char *)a.k_out + ((long long)r * a.k_out_stride + h * D) * EB;
    }
    if (kv != 2) {
      float x[16];
      v0.get(x);
      v1.get(x + 8);
      const char *w = (const char *)(kv == 0 ? a.qw : a.kw);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
      ss = head_sum<D>(ss);
      if (w) {
        const float inv = rsqrtf(ss * (1.f / D) + a.eps);
        Vec8<BF16> w0, w1;
        float wf[16];
        w0.load(w + d0 * EB);
        w1.load(w + d1 * EB);
        w0.get(wf);
        w1.get(wf + 8);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= inv * wf[i];
      }
      if (turned) {
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          c[i] = cs[8 * j + i];
          s[i] = sn[8 * j + i];
        }
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float xa = x[2 * i], xb = x[2 * i + 1];
            x[2 * i] = xa * c[i] - xb * s[i];
            x[2 * i + 1] = xb * c[i] + xa * s[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float xa = x[i], xb = x[8 + i];
            x[i] = xa * c[i] - xb * s[i];
            x[8 + i] = xb * c[i] + xa * s[i];
          }
        }
      }
      v0.set(x);
      v1.set(x + 8);
    }
    v0.store(dst + d0 * EB);
    v1.store(dst + d1 * EB);
  }
}

}  // namespace sdb
