// Masked attention of fp32 tensors on the fp32 matrix cores (v_mfma_f32_32x32x2_f32: operands and sums in fp32; layouts at
// sbp_attention.hip).  A workgroup owns 32 tokens of one (sample, head); its 4 wavefronts share the blocks of 32 streamed tokens among
// them, in turn, and join their results through LDS, in order, at the end: a short sample then takes the time of a quarter of its blocks,
// and a long one loses nothing, since a product of 64 cycles hides the loads of its operands, which come from memory as they are (16
// bytes of a token's row for the scores, 4 bytes per lane of whole rows for the products with P and dM) without a stop in LDS.
// Bound: the fp32 matrix cores and, between their products, the latency of the rows' loads and the arithmetic of the weights (d = 64, 13 x 2
// heads, 1306 tokens: forward 195 us, 58 TFLOP/s of visible pairs; backward of 1273 kept ones 460 us, 59 TFLOP/s; d = 128 in documents of
// 300: 187 and 470 us).  Short samples: the chain of one block (2 x 3 heads of 64, 49 tokens forward: 8.5 us a call; 3 x 3 heads sharing 1, 99
// of 197 tokens backward: 19 us a call, 13 of them in the main kernel).
#include <algorithm>

#include "sbp_lm_attention_tiles.h"

namespace sbp {

template <int D> struct LmF32 {
  static constexpr int PITCH = D + 4;                      // of rows in LDS
  static constexpr int DB = D < 32 ? 1 : D / 32, W = D < 32 ? D : 32;      // blocks of head dimensions, dimensions of one
  // dimensions 8 c + 4 u .. + 3 of a row, in order
  static __device__ __forceinline__ void row(const float* p, int u, float (&v)[D / 2]) {
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      const float4 x = *reinterpret_cast<const float4*>(p + 8 * c + 4 * u);
      v[4 * c] = x.x; v[4 * c + 1] = x.y; v[4 * c + 2] = x.z; v[4 * c + 3] = x.w;
    }
  }
  // rows x own^T: rows are the streamed tokens (A), columns the own ones (B)
  static __device__ __forceinline__ f32x16_t scores(const float (&rows)[D / 2], const float (&own)[D / 2]) {
    f32x16_t s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(rows[i], own[i], s, 0, 0, 0);
    return s;
  }
  // ... with the own rows in LDS ([32][PITCH]: 16 bytes for four products)
  static __device__ __forceinline__ f32x16_t scores(const float (&rows)[D / 2], const float* own, int lane) {
    f32x16_t s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    const float* at = own + (lane & 31) * PITCH + 4 * (lane >> 5);
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(at + 8 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(rows[4 * c + e], x[e], s, 0, 0, 0);
    }
    return s;
  }
  // columns of a block: 32 rows from `base` on (ld elements apart, at most `last` rows on), register v of row 8 (v >> 2) + 4 u + (v & 3)
  static __device__ __forceinline__ void columns(float (&x)[16][DB], const float* base, long long ld, int last, int lane) {
    const int u = lane >> 5, col = lane & (W - 1);
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int b = 0; b < DB; ++b) x[v][b] = base[min(8 * (v >> 2) + 4 * u + (v & 3), last) * ld + col + 32 * b];
  }
  // acc += block^T w
  static __device__ __forceinline__ void add(f32x16_t (&acc)[DB], const float (&x)[16][DB], const f32x16_t& w) {
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int b = 0; b < DB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[v][b], w[v], acc[b], 0, 0, 0);
  }
  // the wavefront's accumulators to LDS: [32 own tokens][D + 4]
  static __device__ __forceinline__ void put(float* img, const f32x16_t (&acc)[DB], int lane) {
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int q4 = 0; q4 < (D < 32 ? D / 8 : 4); ++q4)
        *reinterpret_cast<float4*>(img + (lane & 31) * PITCH + 32 * b + 8 * q4 + 4 * (lane >> 5)) =
            make_float4(acc[b][4 * q4], acc[b][4 * q4 + 1], acc[b][4 * q4 + 2], acc[b][4 * q4 + 3]);
  }
};

// the score (natural units) of z = q.k and, capped, the square of its tanh
template <bool CAP>
__device__ __forceinline__ float lm_score_f32(const MaskedAttention& a, float slope, float z, float distance, float* t2) {
  float s = a.scale * z;
  if constexpr (CAP) {
    const float t = lm_tanh(z * a.per_cap);
    *t2 = t * t;
    s = a.cap * t;
  }
  return fmaf(-slope, distance, s);
}

template <int D, bool CAP>
__global__ void __launch_bounds__(256, D <= 32 ? 3 : D == 64 ? 2 : 1) masked_forward_f32_kernel(MaskedAttention a) {
  using F = LmF32<D>;
  __shared__ __attribute__((aligned(16))) float img[4 * 32 * F::PITCH];
  __shared__ float m_s[4][32], l_s[4][32];
  __shared__ uint32_t again_s;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), u = lane >> 5, n = a.n;
  const int nb = (n + 31) / 32, blk = a.causal ? nb - 1 - blockIdx.x / (a.B * a.h) : blockIdx.x / (a.B * a.h), bh = blockIdx.x % (a.B * a.h);
  const int b = bh / a.h, head = bh % a.h, kv = head / (a.h / a.hk), first = blk * 32, mine = first + (lane & 31), own = min(mine, n - 1);
  const long long ld = (long long)(a.h + 2 * a.hk) * D;
  const float* base = (const float*)a.qkv + (long long)b * n * ld;
  const float *k0 = base + (a.h + kv) * D, *v0 = k0 + a.hk * D;
  const bool docs = a.doc != nullptr;
  const int32_t* doc = docs ? a.doc + (long long)b * n : nullptr;
  const int prefix = lm_prefix(a, b), di = docs ? doc[own] : 0;
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  LmRange wq{first, min(first + 31, n - 1), 0, 0};
  if (docs) {
    LmDocs r;
    r.add(di);
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) r.join(m);
    r.close();
    wq.d0 = __builtin_amdgcn_readfirstlane(r.lo);
    wq.d1 = __builtin_amdgcn_readfirstlane(r.hi);
  }
  if (t == 0) again_s = 0;
  float q[D / 2];
  F::row(base + own * ld + head * D, u, q);
  f32x16_t o[F::DB];
#pragma unroll
  for (int x = 0; x < F::DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[x][e] = 0.f;
  float mx = -INFINITY, l = 0.f;
  const int reach = a.causal ? min(n, max(wq.p1 + 1, prefix)) : n;
  for (int j0 = 32 * wave; j0 < reach; j0 += 128) {
    LmRange r{j0, j0 + 31, 0, 0};
    int dj = 0;
    if (docs) {
      dj = doc[min(j0 + (lane & 31), n - 1)];
      LmDocs x;
      x.add(dj);
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) x.join(m);
      x.close();
      r.d0 = __builtin_amdgcn_readfirstlane(x.lo);
      r.d1 = __builtin_amdgcn_readfirstlane(x.hi);
    }
    const int cls = lm_class(wq, r, a.causal, prefix, docs);
    if (!cls) continue;
    float k[D / 2];
    F::row(k0 + min(j0 + (lane & 31), n - 1) * ld, u, k);
    f32x16_t s = F::scores(k, q);
    float v[16][F::DB];                                      // (under way while the weights are worked out)
    F::columns(v, v0 + j0 * ld, ld, n - 1 - j0, lane);
    __builtin_amdgcn_sched_barrier(0);
    const int rel = mine - j0 - 4 * u;
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float unused;
      s[e] = lm_score_f32<CAP>(a, slope, s[e], fabsf((float)(rel - (8 * (e >> 2) + (e & 3)))), &unused);
    }
    if (cls != 2 || j0 + 31 >= n) {
      int lim = n - j0 - 4 * u;
      if (a.causal) lim = min(lim, max(rel + 1, prefix - j0 - 4 * u));
      if (docs && di < 0) lim = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = 8 * (e >> 2) + (e & 3);
        const bool same = !docs || __shfl(dj, row + 4 * u) == di;
        s[e] = row < lim && same ? s[e] : -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__ballot(top > mx)) {
      const float mn = fmaxf(mx, top), f = mn > mx ? expf(mx - mn) : 1.f;
      mx = mn;
      l *= f;
#pragma unroll
      for (int x = 0; x < F::DB; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[x][e] *= f;
    }
    const float ms = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = expf(s[e] - ms);
      l += s[e];
    }
    F::add(o, v, s);
  }
  // join the wavefronts: their maxima, sums and outputs
  l += __shfl_xor(l, 32);
  F::put(img + wave * 32 * F::PITCH, o, lane);
  if (u == 0) { m_s[wave][lane] = mx; l_s[wave][lane] = l; }
  __syncthreads();
  float* out = (float*)a.out + (long long)b * n * (a.h * D) + head * D;
  for (int i = t; i < 32 * D / 4; i += 256) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    float m = m_s[0][row];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, m_s[w][row]);
    const float ms = m == -INFINITY ? 0.f : m;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = expf(m_s[w][row] - ms);
      const float4 v = *reinterpret_cast<const float4*>(img + (w * 32 + row) * F::PITCH + c);
      total = fmaf(f, l_s[w][row], total);
      s.x = fmaf(f, v.x, s.x); s.y = fmaf(f, v.y, s.y); s.z = fmaf(f, v.z, s.z); s.w = fmaf(f, v.w, s.w);
    }
    const bool empty = total == 0.f;
    const float f = empty ? 0.f : 1.f / total;
    if (lm_finite(total) && !(lm_finite(s.x) && lm_finite(s.y) && lm_finite(s.z) && lm_finite(s.w))) atomicOr(&again_s, 1u << row);
    if (first + row < n) {
      *reinterpret_cast<float4*>(out + (first + row) * ((long long)a.h * D) + c) = empty ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(s.x * f, s.y * f, s.z * f, s.w * f);
      if (a.lse_out && c == 0) a.lse_out[((long long)b * n + first + row) * a.h + head] = empty ? -INFINITY : ms + logf(total);
    }
  }
  __syncthreads();
  if (__builtin_expect(wave == 0 && again_s, 0)) lm_forward_again<float, D>(a, b, head, first, again_s, lane);      // (see sbp_lm_attention_fwd.h)
}

// ---- backward ------------------------------------------------------------------------------------------------------
template <int D, bool KEY, bool CAP>
__device__ __forceinline__ void masked_backward_f32_body(float* img, uint32_t* again_s, const MaskedAttention& a, const LmTables& w, int b, int group, int blk) {
  using F = LmF32<D>;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), u = lane >> 5;
  const int rows = a.rows, share = a.h / a.hk, nh = KEY ? share / w.parts : 1, kv = KEY ? group / w.parts : group / share;
  const int h0 = KEY ? kv * share + group % w.parts * nh : group;
  const long long ld = (long long)(a.h + 2 * a.hk) * D, lda = (long long)a.h * D, row0 = (long long)b * rows;
  const float *qkv = (const float*)a.qkv + row0 * ld, *dA = (const float*)a.dA + row0 * lda;
  const int first = blk * 32, mine = first + (lane & 31), own = min(mine, rows - 1), blocks = (rows + 31) / 32, tiles = w.npad / kLmTile;
  const bool docs = a.doc != nullptr;
  const int prefix = lm_prefix(a, b);
  const float own_pos = w.pos[(long long)b * w.npad + own];
  const int own_doc = w.doc[(long long)b * w.npad + own];
  float bound = KEY ? -3e38f : 3e38f;                       // streamed positions >= bound (KEY) or <= bound are visible
  if (a.causal) bound = KEY ? (own_pos < (float)prefix ? -3e38f : own_pos) : fmaxf(own_pos, (float)prefix - 1.f);
  if (docs && own_doc < 0) bound = KEY ? 3e38f : -3e38f;
  float own_l = 0.f, own_nd = 0.f;
  if constexpr (!KEY) {
    own_l = w.l2[((long long)b * a.h + h0) * w.npad + own];
    own_nd = w.nd[((long long)b * a.h + h0) * w.npad + own];
  }
  // k, v (KEY) or q, dA of the own tokens, in LDS: in registers they leave room for one wavefront per SIMD up to d = 64, and too little
  // for d = 128 (13 x 2 heads, 1273 tokens in documents of 300: d = 64 283 us, 209 so; d = 128 613 us, 466 so)
  const float* p1 = qkv + own * ld + (KEY ? a.h + kv : h0) * D;
  const float* p2 = KEY ? p1 + a.hk * D : dA + own * lda + h0 * D;
  for (int c = wave; c < D / 8; c += 4) {                    // 8 dimensions each
    float* at = img + (lane & 31) * F::PITCH + 8 * c + 4 * u;
    *reinterpret_cast<float4*>(at) = *reinterpret_cast<const float4*>(p1 + 8 * c + 4 * u);
    *reinterpret_cast<float4*>(at + 32 * F::PITCH) = *reinterpret_cast<const float4*>(p2 + 8 * c + 4 * u);
  }
  __syncthreads();
  f32x16_t acc[KEY ? 2 : 1][F::DB];
#pragma unroll
  for (int q = 0; q < (KEY ? 2 : 1); ++q)
#pragma unroll
    for (int x = 0; x < F::DB; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[q][x][e] = 0.f;
  if (t == 0) *again_s = 0;
  const int4* ranges = w.range + (long long)b * tiles;
  const int4 mr4 = ranges[blk >> 1];
  const LmRange mr{mr4.x, mr4.y, mr4.z, mr4.w};
  for (int i = wave; i < blocks * nh; i += 4) {
    const int head = h0 + i / blocks, t0 = i % blocks * 32, last = rows - 1 - t0;
    const int4 e4 = ranges[t0 >> 6];
    const LmRange r{e4.x, e4.y, e4.z, e4.w};
    const int cls = KEY ? lm_class(r, mr, a.causal, prefix, docs) : lm_class(mr, r, a.causal, prefix, docs);
    if (!cls) continue;
    const float slope = a.slopes ? a.slopes[head] : 0.f;
    const int row = t0 + min(lane & 31, last);
    const float* s1 = qkv + (KEY ? head : a.h + kv) * D;                     // q or k
    const float* s2 = KEY ? dA + head * D : qkv + (a.h + a.hk + kv) * D;     // dA or v
    const long long ld2 = KEY ? lda : ld;
    float x1[D / 2], x2[D / 2];
    F::row(s1 + row * ld, u, x1);
    F::row(s2 + row * ld2, u, x2);
    f32x4_t tl[4], tn[4], tp[4];
    int4 td[4];
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const long long at = (long long)b * w.npad + t0 + 8 * q4 + 4 * u, ah = ((long long)b * a.h + head) * w.npad + t0 + 8 * q4 + 4 * u;
      if constexpr (KEY) {
        tl[q4] = *reinterpret_cast<const f32x4_t*>(w.l2 + ah);
        tn[q4] = *reinterpret_cast<const f32x4_t*>(w.nd + ah);
      }
      tp[q4] = *reinterpret_cast<const f32x4_t*>(w.pos + at);
      td[q4] = *reinterpret_cast<const int4*>(w.doc + at);
    }
    f32x16_t s = F::scores(x1, img, lane), dp = F::scores(x2, img + 32 * F::PITCH, lane);
    float c[16][F::DB];                                      // (under way while the weights are worked out)
    F::columns(c, s1 + t0 * ld, ld, last, lane);
    __builtin_amdgcn_sched_barrier(0);
    const bool masked = cls != 2 || last < 31;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int q4 = e >> 2, k = e & 3;
      float t2 = 0.f;
      const float v = lm_score_f32<CAP>(a, slope, s[e], fabsf(tp[q4][k] - own_pos), &t2);
      float p = expf(v - (KEY ? tl[q4][k] : own_l)), m = p * (dp[e] + (KEY ? tn[q4][k] : own_nd)) * a.scale;
      if constexpr (CAP) m *= 1.f - t2;
      if (masked) {
        const int dd = k == 0 ? td[q4].x : k == 1 ? td[q4].y : k == 2 ? td[q4].z : td[q4].w;
        const bool see = (KEY ? tp[q4][k] >= bound : tp[q4][k] <= bound) && dd == own_doc;
        p = see ? p : 0.f;
        m = see ? m : 0.f;
      }
      s[e] = p;
      dp[e] = m;
    }
    if constexpr (KEY) {
      float c2[16][F::DB];                                   // (under way while the first products run)
      F::columns(c2, s2 + t0 * ld2, ld2, last, lane);
      __builtin_amdgcn_sched_barrier(0);
      F::add(acc[0], c, dp);
      F::add(acc[1], c2, s);
    } else {
      F::add(acc[0], c, dp);
    }
  }
  // join the wavefronts' sums in order
  float* out = (float*)a.out + row0 * ld;
  float* part = KEY && w.part ? w.part + (((long long)(group % w.parts) * a.B + b) * rows * a.hk + kv) * (2 * D) : nullptr;
#pragma unroll
  for (int q = 0; q < (KEY ? 2 : 1); ++q) {
    __syncthreads();
    F::put(img + wave * 32 * F::PITCH, acc[q], lane);
    __syncthreads();
    for (int i = t; i < 32 * D / 4; i += 256) {
      const int row = i / (D / 4), c = i % (D / 4) * 4;
      float4 s = *reinterpret_cast<const float4*>(img + row * F::PITCH + c);
#pragma unroll
      for (int x = 1; x < 4; ++x) {
        const float4 v = *reinterpret_cast<const float4*>(img + (x * 32 + row) * F::PITCH + c);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      if (!(lm_finite(s.x) && lm_finite(s.y) && lm_finite(s.z) && lm_finite(s.w))) atomicOr(again_s, 1u << row);
      if (first + row >= rows) continue;
      float* o = !KEY ? out + (first + row) * ld + h0 * D : part ? part + (long long)(first + row) * (a.hk * 2 * D) + q * D
                 : out + (first + row) * ld + (a.h + (q ? a.hk : 0) + kv) * D;
      *reinterpret_cast<float4*>(o + c) = s;
    }
  }
  __syncthreads();
  if (__builtin_expect(wave == 0 && *again_s, 0)) lm_backward_again<float, D, KEY>(a, w, b, kv, h0, nh, first, *again_s, lane, part);
}

template <int D, bool CAP>
__global__ void __launch_bounds__(256, D <= 64 ? 2 : 1) masked_backward_f32_kernel(MaskedAttention a, LmTables w) {
  __shared__ __attribute__((aligned(16))) float img[4 * 32 * LmF32<D>::PITCH];
  __shared__ uint32_t again_s;
  const int nk = a.B * a.hk * w.parts, nq = a.B * a.h, blocks = (a.rows + 31) / 32, rank = blockIdx.x / (nk + nq), k = blockIdx.x % (nk + nq);
  if (k < nk) masked_backward_f32_body<D, true, CAP>(img, &again_s, a, w, k / (a.hk * w.parts), k % (a.hk * w.parts), rank);
  else masked_backward_f32_body<D, false, CAP>(img, &again_s, a, w, (k - nk) / a.h, (k - nk) % a.h, a.causal ? blocks - 1 - rank : rank);
}

template <int D>
static void launch_f32(const MaskedAttention& a, const LmTables* w, hipStream_t s) {
  const bool cap = a.cap > 0.f;
  if (!w) {
    const dim3 grid((unsigned)((int64_t)a.B * a.h * ceil_div(a.n, 32)));
    if (cap) SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_forward_f32_kernel<D, true>), grid, dim3(256), 0, s, a);
    else SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_forward_f32_kernel<D, false>), grid, dim3(256), 0, s, a);
  } else {
    const dim3 grid((unsigned)((int64_t)a.B * (a.hk * w->parts + a.h) * ceil_div(a.rows, 32)));
    if (cap) SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_backward_f32_kernel<D, true>), grid, dim3(256), 0, s, a, *w);
    else SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_backward_f32_kernel<D, false>), grid, dim3(256), 0, s, a, *w);
  }
}
void launch_masked_f32(const MaskedAttention& a, const LmTables* w, hipStream_t s) {
  if (a.d == 16) launch_f32<16>(a, w, s);
  else if (a.d == 32) launch_f32<32>(a, w, s);
  else if (a.d == 64) launch_f32<64>(a, w, s);
  else launch_f32<128>(a, w, s);
}

}  // namespace sbp
