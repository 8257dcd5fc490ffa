// Masked attention of 32 own tokens by one wavefront, with every operand straight from memory: for the rows whose result in the fast kernels
// is not finite.  There a weight of 0 meets whatever a token that is not seen holds, and 0 times an infinity or a NaN is a NaN.  Here the
// products take the streamed values that are finite, and the others are added one by one to the rows that see them; sums in a fixed order.
// The forward takes the weights' sum first, so that sums of weights above 1 that overflowed are finite here too.
// Bound: the latency of the loads, one block of 32 streamed tokens after the other.  A call all of whose rows come here takes up to 13 times as
// long as otherwise: 16 heads of 128 sharing 2, 8192 tokens, causal, capped, one infinite value of v that all but five rows see: forward 4.1
// ms instead of 0.34; 92 tokens of NaN as padding 3.7 ms, both ways 8.2 instead of 0.76; backward of all tokens 12 ms instead of 1.4.  Where
// every value of a row has become NaN the rest is left out (everything NaN: backward 1.6 ms; the forward's sums of weights tell, 0.32).  One row
// at a time the same calls took 30 to 340 times as long as otherwise.
#ifndef SBP_LM_ATTENTION_ROWS_H_
#define SBP_LM_ATTENTION_ROWS_H_

#include "sbp_attention_tiles.h"
#include "sbp_lm_internal.h"

namespace sbp {

static constexpr int kLmTile = 64;                         // streamed tokens per tile

static constexpr int kLmChunk = 128;                       // own tokens per workgroup of the backward

// What the first kernel of the backward writes (workspace): npad = rows rounded up to whole tiles.
struct LmTables {
  float *l2, *nd;                // [B*h][npad]
  float* pos;                    // [B][npad], NaN past the last token: no comparison with it is true
  int32_t* doc;                  // [B][npad]
  int4* range;                   // [B][npad / 64]: positions, documents (0, 0 without documents) of the tile's tokens
  float* part;                   // [parts][B*rows][hk][2][D]: dK, dV of the parts of a key / value head
  int npad, parts, nchunks;
};

__device__ __forceinline__ uint32_t lm_bits(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t lm_bits(const uint16_t* p) { return *p; }

__device__ __forceinline__ float lm_dot(const float* a, const float* b, int d) {
  float s = 0.f;
  for (int c = 0; c < d; c += 4) {
    const float4 x = *reinterpret_cast<const float4*>(a + c), y = *reinterpret_cast<const float4*>(b + c);
    s = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s))));
  }
  return s;
}
__device__ __forceinline__ float lm_dot(const uint16_t* a, const uint16_t* b, int d) {
  float s = 0.f;
  for (int c = 0; c < d; c += 8) {
    const uint4 x = *reinterpret_cast<const uint4*>(a + c), y = *reinterpret_cast<const uint4*>(b + c);
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fmaf(bf16_lo(xw[e]), bf16_lo(yw[e]), fmaf(bf16_hi(xw[e]), bf16_hi(yw[e]), s));
  }
  return s;
}
// where token t of sample b stands, and the document it belongs to
__device__ __forceinline__ int lm_pos(const MaskedAttention& a, int b, int t) { return a.idx ? a.idx[(long long)b * a.rows + t] - b * a.n : t; }
__device__ __forceinline__ int lm_doc(const MaskedAttention& a, int b, int pos) { return a.doc ? a.doc[(long long)b * a.n + pos] : 0; }
// (no position is below 0: differences of prefix and a position stay within 32 bits)
__device__ __forceinline__ int lm_prefix(const MaskedAttention& a, int b) { return a.prefix ? max(a.prefix[b], 0) : 0; }
__device__ __forceinline__ bool lm_visible(const MaskedAttention& a, int prefix, int pi, int di, int pj, int dj) {
  return (!a.causal || pj <= pi || pj < prefix) && di == dj && di >= 0;
}
// tanh to about a step of fp32, without branches: up to 0.55, about (ln 3) / 2, an odd polynomial (fitted for the least largest error, 2^-29 of the
// value), beyond it 1 - 2 / (exp(2 |x|) + 1); the split and the upper branch as in Cody and Waite, Software Manual for the Elementary
// Functions.  (tanhf() takes both of its ways where the lanes differ.)
__device__ __forceinline__ float lm_tanh(float x) {
  const float u = x * x, y = fabsf(x);
  const float near = fmaf(x * u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -0.0062824725f, 0.021077758f), -0.05385386f), 0.13332602f), -0.3333332f), x);
  const float far = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * (2.f * kLog2e)) + 1.f), 1.f);
  return y > 0.55f ? copysignf(far, x) : near;
}
// score of z = q.k at this distance; tanh of the cap's argument in t
__device__ __forceinline__ float lm_score(const MaskedAttention& a, float slope, float z, float distance, float* t) {
  float s = a.scale * z;
  *t = 0.f;
  if (a.cap > 0.f) { *t = lm_tanh(z * a.per_cap); s = a.cap * *t; }
  return slope == 0.f ? s : s - slope * distance;
}
__device__ __forceinline__ bool lm_finite(float v) { return fabsf(v) < INFINITY; }
// four elements of a row, at a multiple of four
__device__ __forceinline__ void lm_load4(const float* p, float (&v)[4]) {
  const float4 x = *reinterpret_cast<const float4*>(p);
  v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
}
__device__ __forceinline__ void lm_load4(const uint16_t* p, float (&v)[4]) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  v[0] = bf16_lo(x.x); v[1] = bf16_hi(x.x); v[2] = bf16_lo(x.y); v[3] = bf16_hi(x.y);
}
__device__ __forceinline__ void lm_store4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void lm_store4(uint16_t* p, const float (&v)[4]) { *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3])); }

// Products of 32 own tokens (columns: lane & 31) with 32 streamed ones, whose register e is row 8 (e >> 2) + 4 u + (e & 3), u = lane >> 5.
template <typename T, int D>
struct LmBlock {
  static constexpr int W = D < 32 ? D : 32, Q4 = W / 8;       // head dimensions of a product ...
  static constexpr int CB = D == 128 ? 4 : 1;                // ... and products at a time (the kernels of d = 128 have the registers)
  static __device__ __forceinline__ int row(int e, int u) { return 8 * (e >> 2) + 4 * u + (e & 3); }
  // streamed x own^T; the lane's streamed row and own row
  static __device__ __forceinline__ f32x16_t scores(const T* streamed, const T* own, int u) {
    f32x16_t s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_t*>(streamed + 16 * ks + 8 * u),
                                                    *reinterpret_cast<const bf16x8_t*>(own + 16 * ks + 8 * u), s, 0, 0, 0);
    } else {
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        float x[4], y[4];
        lm_load4(streamed + 8 * c + 4 * u, x);
        lm_load4(own + 8 * c + 4 * u, y);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], s, 0, 0, 0);
      }
    }
    return s;
  }
  // acc += rows^T w: W columns of 32 rows from `base` on (at most `last` rows on).  see: bit e, the own token sees row e (elsewhere w is 0).
  // WEIGHT: w are weights exp(..), above 0 even where they are too small for fp32.
  template <bool WEIGHT>
  static __device__ __forceinline__ void add(f32x16_t& acc, const T* base, uint32_t ld, int last, const f32x16_t& w, uint32_t see, int lane) {
    const int u = lane >> 5;
    constexpr uint32_t TOP = sizeof(T) == 2 ? 0x7f80u : 0x7f800000u;       // the exponent of infinities and NaN
    uint32_t holes = 0;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      __builtin_amdgcn_sched_barrier(0);
      uint32_t x[8];                                         // (as they lie in memory)
      bool fine = true;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = lm_bits(base + ((uint32_t)min(row(8 * ks + i, u), last) * ld + (uint32_t)(lane & (W - 1))));
#pragma unroll
      for (int i = 0; i < 8; ++i) fine = fine && (x[i] & TOP) != TOP;
      if (__ballot(!fine)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const unsigned long long m = __ballot((x[i] & TOP) == TOP);
          holes |= ((uint32_t)m ? 1u << row(8 * ks + i, 0) : 0u) | ((uint32_t)(m >> 32) ? 1u << row(8 * ks + i, 1) : 0u);
          x[i] = (x[i] & TOP) == TOP ? 0u : x[i];
        }
      }
      if constexpr (sizeof(T) == 2) {
        const uint4 p = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, p), pack8(w, ks), acc, 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[i]), w[8 * ks + i], acc, 0, 0, 0);
      }
    }
    // the values that are not finite, for the own tokens that see them, unless nothing can change any more
    __builtin_amdgcn_sched_barrier(0);
    if (last < 31) holes &= (2u << last) - 1u;
#pragma unroll 1
    for (; holes; holes &= holes - 1) {
      const int r = __ffs((int)holes) - 1, e0 = (r >> 3) * 4 + (r & 3), from = (lane & 31) + 32 * ((r >> 2) & 1);
      bool open = false;
#pragma unroll
      for (int e = 0; e < 4 * Q4; ++e) open = open || acc[e] == acc[e];
      const bool on = __shfl((int)see, from) >> e0 & 1;
      if (!__ballot(on && open)) continue;
      float f = 1.f;
      if constexpr (!WEIGHT) {
        f = w[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) f = e == e0 ? w[e] : f;
        f = __shfl(f, from);
      }
      const T* p = base + ((uint32_t)r * ld + 4 * u);
#pragma unroll
      for (int q4 = 0; q4 < Q4; ++q4) {
        float x[4];
        lm_load4(p + 8 * q4, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[4 * q4 + e] = on && !lm_finite(x[e]) ? fmaf(f, x[e], acc[4 * q4 + e]) : acc[4 * q4 + e];
      }
    }
  }
  // W columns of the own token's row
  template <typename O>
  static __device__ __forceinline__ void store(O* out, const f32x16_t& acc, int u) {
#pragma unroll
    for (int q4 = 0; q4 < Q4; ++q4) {
      const float v[4] = {acc[4 * q4], acc[4 * q4 + 1], acc[4 * q4 + 2], acc[4 * q4 + 3]};
      lm_store4(out + 8 * q4 + 4 * u, v);
    }
  }
};
__device__ __forceinline__ void lm_clear(f32x16_t& v) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = 0.f;
}
// Something of it is a number: more terms change it.
template <int N>
__device__ __forceinline__ bool lm_open(const f32x16_t (&v)[N]) {
  bool open = false;
#pragma unroll
  for (int x = 0; x < N; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) open = open || v[x][e] == v[x][e];
  return open;
}

// A (lse has met scores alone) of the queries `again` (bit q: first + q) of (sample b, head), by one wavefront.
template <typename T, int D>
__device__ __forceinline__ void lm_forward_again(const MaskedAttention& a, int b, int head, int first, uint32_t again, int lane) {
  asm volatile("" : "+v"(lane));                             // (nothing of what follows is kept in registers through the caller's loop)
  using B = LmBlock<T, D>;
  const int n = a.n, u = lane >> 5, i = first + (lane & 31), own = min(i, n - 1), kv = head / (a.h / a.hk);
  const long long ld = (long long)(a.h + 2 * a.hk) * D, row0 = (long long)b * n;
  const T *q = (const T*)a.qkv + (row0 + own) * ld + head * D, *k = (const T*)a.qkv + row0 * ld + (long long)(a.h + kv) * D, *v = k + (long long)a.hk * D;
  const int32_t* doc = a.doc ? a.doc + row0 : nullptr;
  const int prefix = lm_prefix(a, b), di = lm_doc(a, b, own);
  const bool mine = again >> (lane & 31) & 1 && i < n;
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  const int reach = a.causal ? min(n, max(first + 32, prefix)) : n;
  // scores of the keys from j0 on, -inf where they are not seen; false: none of them is
  auto scores = [&](int j0, f32x16_t& s, uint32_t& see) {
    const int last = n - 1 - j0;
    see = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);     // (few of them under way: the registers are the main loop's)
      const int r = B::row(e, u);
      see |= mine && r <= last && lm_visible(a, prefix, own, di, j0 + r, doc ? doc[(uint32_t)(j0 + min(r, last))] : 0) ? 1u << e : 0u;
    }
    if (!__ballot(see != 0)) return false;
    s = B::scores(k + (j0 + min(lane & 31, last)) * ld, q, u);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
      float unused;
      s[e] = see >> e & 1 ? lm_score(a, slope, s[e], fabsf((float)(own - j0 - B::row(e, u))), &unused) : -INFINITY;
    }
    return true;
  };
  // the maximum and the sum of the weights first: weights that add up to 1 keep the sums below the largest value of v
  f32x16_t s;
  uint32_t see;
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int j0 = 0; j0 < reach; j0 += 32) {
    if (!scores(j0, s, see)) continue;
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
    const float mn = fmaxf(m, fmaxf(top, __shfl_xor(top, 32))), ms = mn == -INFINITY ? 0.f : mn;
    l *= mn > m ? expf(m - ms) : 1.f;
    m = mn;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
      l += see >> e & 1 ? expf(s[e] - ms) : 0.f;
    }
  }
  l += __shfl_xor(l, 32);
  const float inv = 1.f / l, ms = m == -INFINITY ? 0.f : m;
#pragma unroll 1
  for (int c = 0; c < D; c += B::CB * B::W) {
    f32x16_t o[B::CB];
#pragma unroll
    for (int x = 0; x < B::CB; ++x) lm_clear(o[x]);
#pragma unroll 1
    for (int j0 = 0; j0 < reach; j0 += 32) {
      if (!scores(j0, s, see)) continue;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
        s[e] = see >> e & 1 ? expf(s[e] - ms) * inv : 0.f;
      }
#pragma unroll
      for (int x = 0; x < B::CB; ++x) B::template add<true>(o[x], v + j0 * ld + c + x * B::W, (uint32_t)ld, n - 1 - j0, s, see, lane);
      if (!__ballot(mine && lm_open(o))) break;
    }
    if (mine) {
#pragma unroll
      for (int x = 0; x < B::CB; ++x) B::store((T*)a.out + (row0 + i) * ((long long)a.h * D) + head * D + c + x * B::W, o[x], u);
    }
  }
}

// dQ of the queries (KEY: dK and dV, from query heads h0 .. h0 + nh - 1, of the keys) `again` (bit t: token first + t) of sample b, by one
// wavefront.  part: fp32 rows of dK and dV, or NULL.
template <typename T, int D, bool KEY>
__device__ __forceinline__ void lm_backward_again(const MaskedAttention& a, const LmTables& w, int b, int kv, int h0, int nh, int first, uint32_t again, int lane,
                                                  float* part) {
  asm volatile("" : "+v"(lane));                             // (nothing of what follows is kept in registers through the caller's loop)
  using B = LmBlock<T, D>;
  const int rows = a.rows, u = lane >> 5, t = first + (lane & 31), own = min(t, rows - 1);
  const long long ld = (long long)(a.h + 2 * a.hk) * D, lda = (long long)a.h * D, row0 = (long long)b * rows, at0 = (long long)b * w.npad;
  const T *qkv = (const T*)a.qkv + row0 * ld, *dA = (const T*)a.dA + row0 * lda;
  const T* own1 = qkv + own * ld + (KEY ? a.h + kv : h0) * D;
  const T* own2 = KEY ? own1 + (long long)a.hk * D : dA + own * lda + h0 * D;
  const bool mine = again >> (lane & 31) & 1 && t < rows;
  const float* tpos = w.pos + at0;
  const int32_t* tdoc = w.doc + at0;
  const float own_pos = tpos[own], prefix = (float)lm_prefix(a, b);
  const int own_doc = tdoc[own];
  const float own_l = w.l2[((long long)b * a.h + h0) * w.npad + own], own_nd = w.nd[((long long)b * a.h + h0) * w.npad + own];      // (QUERY)
#pragma unroll 1
  for (int c = 0; c < D; c += B::CB * B::W) {
    f32x16_t acc[KEY ? 2 : 1][B::CB];
#pragma unroll
    for (int x = 0; x < B::CB; ++x) {
      lm_clear(acc[0][x]);
      if constexpr (KEY) lm_clear(acc[1][x]);
    }
    bool open = true;                                        // (for all lanes)
#pragma unroll 1
    for (int head = h0; open && head < h0 + nh; ++head) {
      const float slope = a.slopes ? a.slopes[head] : 0.f;
      const float *l2 = w.l2 + ((long long)b * a.h + head) * w.npad, *nd = w.nd + ((long long)b * a.h + head) * w.npad;
#pragma unroll 1
      for (int t0 = 0; open && t0 < rows; t0 += 32) {
        const int last = rows - 1 - t0, r0 = t0 + min(lane & 31, last);
        const uint32_t at = (uint32_t)(t0 + 4 * u);              // (the tables are whole tiles: rows past the end have no position)
        uint32_t see = 0;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const f32x4_t p = *reinterpret_cast<const f32x4_t*>(tpos + at + 8 * q4);
          const int4 d = *reinterpret_cast<const int4*>(tdoc + at + 8 * q4);
          const int dd[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float pi = KEY ? p[e] : own_pos, pj = KEY ? own_pos : p[e];
            see |= mine && p[e] == p[e] && dd[e] == own_doc && own_doc >= 0 && (!a.causal || pj <= pi || pj < prefix) ? 1u << (4 * q4 + e) : 0u;
          }
          __builtin_amdgcn_sched_barrier(0);                     // (few of them under way: the registers are the main loop's)
        }
        if (!__ballot(see != 0)) continue;
        const T* s1 = qkv + (KEY ? head : a.h + kv) * D;
        const T* s2 = KEY ? dA + head * D : qkv + (long long)(a.h + a.hk + kv) * D;
        const long long ld2 = KEY ? lda : ld;
        f32x16_t s = B::scores(s1 + r0 * ld, own1, u), dp = B::scores(s2 + r0 * ld2, own2, u);
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          __builtin_amdgcn_sched_barrier(0);
          f32x4_t l4, n4;
          const f32x4_t p4 = *reinterpret_cast<const f32x4_t*>(tpos + at + 8 * q4);
          if constexpr (KEY) {
            l4 = *reinterpret_cast<const f32x4_t*>(l2 + at + 8 * q4);
            n4 = *reinterpret_cast<const f32x4_t*>(nd + at + 8 * q4);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int e = 4 * q4 + k;
            float tanh;
            const float v = lm_score(a, slope, s[e], fabsf(p4[k] - own_pos), &tanh), l = KEY ? l4[k] : own_l;
            const float p = sizeof(T) == 2 ? exp2f(fmaf(v, kLog2e, -l)) : expf(v - l);
            const float d = p * (dp[e] + (KEY ? n4[k] : own_nd)) * (1.f - tanh * tanh) * a.scale;
            s[e] = see >> e & 1 ? p : 0.f;
            dp[e] = see >> e & 1 ? d : 0.f;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < B::CB; ++x) {
          B::template add<false>(acc[0][x], s1 + t0 * ld + c + x * B::W, (uint32_t)ld, last, dp, see, lane);
          if constexpr (KEY) B::template add<true>(acc[1][x], s2 + t0 * ld2 + c + x * B::W, (uint32_t)ld2, last, s, see, lane);
        }
        open = __ballot(mine && (lm_open(acc[0]) || (KEY && lm_open(acc[KEY ? 1 : 0])))) != 0;
      }
    }
    if (mine) {
      T* out = (T*)a.out + (row0 + t) * ld + c;
      float* p = part ? part + (long long)t * (a.hk * 2 * D) + c : nullptr;
#pragma unroll
      for (int x = 0; x < B::CB; ++x) {
        if constexpr (!KEY) {
          B::store(out + h0 * D + x * B::W, acc[0][x], u);
        } else if (p) {
          B::store(p + x * B::W, acc[0][x], u);
          B::store(p + D + x * B::W, acc[1][x], u);
        } else {
          B::store(out + (a.h + kv) * D + x * B::W, acc[0][x], u);
          B::store(out + (long long)(a.h + a.hk + kv) * D + x * B::W, acc[1][x], u);
        }
      }
    }
  }
}

}  // namespace sbp
#endif
