// Masked attention one row at a time: the definition, carried out by one wavefront with every sum in a fixed order.  Keys (or
// queries) that are not visible are skipped, never multiplied by zero, so nothing they hold reaches a result.
#ifndef SBP_LM_ATTENTION_ROWS_H_
#define SBP_LM_ATTENTION_ROWS_H_

#include "sbp_lm_internal.h"
#include "sbp_mfma_gemm.h"

namespace sbp {

__device__ __forceinline__ float lm_load(const float* p) { return *p; }
__device__ __forceinline__ float lm_load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void lm_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void lm_store(uint16_t* p, float v) { *p = (uint16_t)bf16_pack(v, v); }

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
__device__ __forceinline__ float lm_wave_sum(float v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ float lm_wave_max(float v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
  return v;
}

// where token t of sample b stands, and the document it belongs to
__device__ __forceinline__ int lm_pos(const MaskedAttention& a, int b, int t) { return a.idx ? a.idx[(long long)b * a.rows + t] - b * a.n : t; }
__device__ __forceinline__ int lm_doc(const MaskedAttention& a, int b, int pos) { return a.doc ? a.doc[(long long)b * a.n + pos] : 0; }
// (no position is below 0: differences of prefix and a position stay within 32 bits)
__device__ __forceinline__ int lm_prefix(const MaskedAttention& a, int b) { return a.prefix ? max(a.prefix[b], 0) : 0; }
__device__ __forceinline__ bool lm_visible(const MaskedAttention& a, int prefix, int pi, int di, int pj, int dj) {
  return (!a.causal || pj <= pi || pj < prefix) && di == dj && di >= 0;
}
// score of z = q.k; tanh of the cap's argument in t
__device__ __forceinline__ float lm_score(const MaskedAttention& a, float slope, float z, int pi, int pj, float* t) {
  float s = a.scale * z;
  *t = 0.f;
  if (a.cap > 0.f) { *t = tanhf(s / a.cap); s = a.cap * *t; }
  return slope == 0.f ? s : s - slope * fabsf((float)(pi - pj));
}

// A and lse of query t of (sample b, head)
template <typename T>
__device__ void lm_forward_row(const MaskedAttention& a, int b, int head, int t, int lane) {
  const int d = a.d, kv = head / (a.h / a.hk);
  const long long ld = (long long)(a.h + 2 * a.hk) * d, row0 = (long long)b * a.rows;
  const T* q = (const T*)a.qkv + (row0 + t) * ld + head * d;
  const T* k = (const T*)a.qkv + row0 * ld + (long long)(a.h + kv) * d;
  const T* v = k + (long long)a.hk * d;
  const int prefix = lm_prefix(a, b), pi = lm_pos(a, b, t), di = lm_doc(a, b, pi);
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  float m = -INFINITY, l = 0.f, acc0 = 0.f, acc1 = 0.f;
  for (int j0 = 0; j0 < a.rows; j0 += 64) {
    const int j = j0 + lane;
    float s = -INFINITY, unused;
    bool see = false;
    if (j < a.rows) {
      const int pj = lm_pos(a, b, j);
      see = lm_visible(a, prefix, pi, di, pj, lm_doc(a, b, pj));
      if (see) s = lm_score(a, slope, lm_dot(q, k + j * ld, d), pi, pj, &unused);
    }
    const unsigned long long any = __ballot(see);
    if (!any) continue;
    const float mn = fmaxf(m, lm_wave_max(s)), ms = mn == -INFINITY ? 0.f : mn;     // (a NaN among the scores reaches p, and the sums through it)
    const float f = m == -INFINITY ? 0.f : expf(m - ms), p = see ? expf(s - ms) : 0.f;
    l = l * f + lm_wave_sum(p);
    acc0 *= f; acc1 *= f;
    for (unsigned long long w = any; w; w &= w - 1) {
      const int jj = __ffsll((long long)w) - 1;
      const float pj = __shfl(p, jj);
      const T* vr = v + (j0 + jj) * ld;
      if (lane < d) acc0 = fmaf(pj, lm_load(vr + lane), acc0);
      if (lane + 64 < d) acc1 = fmaf(pj, lm_load(vr + lane + 64), acc1);
    }
    m = mn;
  }
  const bool empty = m == -INFINITY && l == 0.f;
  T* o = (T*)a.out + (row0 + t) * ((long long)a.h * d) + head * d;
  if (lane < d) lm_store(o + lane, empty ? 0.f : acc0 / l);
  if (lane + 64 < d) lm_store(o + lane + 64, empty ? 0.f : acc1 / l);
  if (a.lse_out && lane == 0) a.lse_out[(row0 + t) * a.h + head] = empty ? -INFINITY : m + logf(l);
}

// weight P and dM * scale of a visible pair
template <typename T>
__device__ __forceinline__ void lm_pair(const MaskedAttention& a, float slope, const T* q, const T* k, const T* g, const T* v, float delta,
                                        float lse, int pi, int pj, float* p, float* ds) {
  float t;
  const float s = lm_score(a, slope, lm_dot(q, k, a.d), pi, pj, &t);
  *p = lse == -INFINITY ? 0.f : expf(s - lse);               // (a row whose scores were all -inf)
  *ds = *p * (lm_dot(g, v, a.d) - delta) * (1.f - t * t) * a.scale;
}

// dQ of query t of (sample b, head)
template <typename T>
__device__ void lm_backward_query(const MaskedAttention& a, int b, int head, int t, int lane) {
  const int d = a.d, kv = head / (a.h / a.hk);
  const long long ld = (long long)(a.h + 2 * a.hk) * d, lda = (long long)a.h * d, row0 = (long long)b * a.rows;
  const T* q = (const T*)a.qkv + (row0 + t) * ld + head * d;
  const T* g = (const T*)a.dA + (row0 + t) * lda + head * d;
  const T* o = (const T*)a.A + (row0 + t) * lda + head * d;
  const T* k = (const T*)a.qkv + row0 * ld + (long long)(a.h + kv) * d;
  const T* v = k + (long long)a.hk * d;
  const int prefix = lm_prefix(a, b), pi = lm_pos(a, b, t), di = lm_doc(a, b, pi);
  const float slope = a.slopes ? a.slopes[head] : 0.f, delta = lm_dot(g, o, d), lse = a.lse[(row0 + t) * a.h + head];
  float acc0 = 0.f, acc1 = 0.f;
  for (int j0 = 0; j0 < a.rows; j0 += 64) {
    const int j = j0 + lane;
    float p = 0.f, ds = 0.f;
    bool see = false;
    if (j < a.rows) {
      const int pj = lm_pos(a, b, j);
      see = lm_visible(a, prefix, pi, di, pj, lm_doc(a, b, pj));
      if (see) lm_pair(a, slope, q, k + j * ld, g, v + j * ld, delta, lse, pi, pj, &p, &ds);
    }
    for (unsigned long long w = __ballot(see); w; w &= w - 1) {
      const int jj = __ffsll((long long)w) - 1;
      const float f = __shfl(ds, jj);
      const T* kr = k + (j0 + jj) * ld;
      if (lane < d) acc0 = fmaf(f, lm_load(kr + lane), acc0);
      if (lane + 64 < d) acc1 = fmaf(f, lm_load(kr + lane + 64), acc1);
    }
  }
  T* dq = (T*)a.out + (row0 + t) * ld + head * d;
  if (lane < d) lm_store(dq + lane, acc0);
  if (lane + 64 < d) lm_store(dq + lane + 64, acc1);
}

// dK and dV of key t of (sample b, key / value head kv), from query heads h0 .. h1 - 1
template <typename T>
__device__ void lm_backward_key(const MaskedAttention& a, int b, int kv, int h0, int h1, int t, int lane, float (&dk)[2], float (&dv)[2]) {
  const int d = a.d;
  const long long ld = (long long)(a.h + 2 * a.hk) * d, lda = (long long)a.h * d, row0 = (long long)b * a.rows;
  const T* k = (const T*)a.qkv + (row0 + t) * ld + (long long)(a.h + kv) * d;
  const T* v = k + (long long)a.hk * d;
  const int prefix = lm_prefix(a, b), pj = lm_pos(a, b, t), dj = lm_doc(a, b, pj);
  dk[0] = dk[1] = dv[0] = dv[1] = 0.f;
  for (int head = h0; head < h1; ++head) {
    const T* q = (const T*)a.qkv + row0 * ld + head * d;
    const T* g = (const T*)a.dA + row0 * lda + head * d;
    const T* o = (const T*)a.A + row0 * lda + head * d;
    const float slope = a.slopes ? a.slopes[head] : 0.f;
    for (int i0 = 0; i0 < a.rows; i0 += 64) {
      const int i = i0 + lane;
      float p = 0.f, ds = 0.f;
      bool see = false;
      if (i < a.rows) {
        const int pi = lm_pos(a, b, i);
        see = lm_visible(a, prefix, pi, lm_doc(a, b, pi), pj, dj);
        if (see)
          lm_pair(a, slope, q + i * ld, k, g + i * lda, v, lm_dot(g + i * lda, o + i * lda, d), a.lse[(row0 + i) * a.h + head], pi, pj, &p, &ds);
      }
      for (unsigned long long w = __ballot(see); w; w &= w - 1) {
        const int ii = __ffsll((long long)w) - 1;
        const float f = __shfl(ds, ii), fp = __shfl(p, ii);
        const T *qr = q + (i0 + ii) * ld, *gr = g + (i0 + ii) * lda;
        if (lane < d) { dk[0] = fmaf(f, lm_load(qr + lane), dk[0]); dv[0] = fmaf(fp, lm_load(gr + lane), dv[0]); }
        if (lane + 64 < d) { dk[1] = fmaf(f, lm_load(qr + lane + 64), dk[1]); dv[1] = fmaf(fp, lm_load(gr + lane + 64), dv[1]); }
      }
    }
  }
}

}  // namespace sbp
#endif
