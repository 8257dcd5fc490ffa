// The token table (sbp_lm.h): scaled lookup, and the table's gradient from the kept rows, grouped by token.
#include <algorithm>

#include "sbp_lm_internal.h"
#include "sbp_mfma_gemm.h"

namespace sbp {

template <typename T> struct EmPiece;                      // 16 bytes of a row as floats
template <> struct EmPiece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
    const float4 w = *reinterpret_cast<const float4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct EmPiece<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const uint16_t* p, float (&v)[8]) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = bf16_lo(x[e]); v[2 * e + 1] = bf16_hi(x[e]); }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
  }
};
__device__ __forceinline__ float em_get(const float* p) { return *p; }
__device__ __forceinline__ float em_get(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void em_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void em_put(uint16_t* p, float v) { *p = (uint16_t)bf16_pack(v, v); }

template <typename K>
__device__ __forceinline__ long long em_token(const K* tokens, const int32_t* idx, long long j) { return (long long)tokens[idx ? idx[j] : j]; }

// ---- lookup: one piece of 16 bytes (VEC) or one channel per thread and step ----------------------------------------
template <typename T, typename K, bool VEC>
__global__ void __launch_bounds__(256) embedding_forward_kernel(const K* __restrict__ tokens, const T* __restrict__ table, long long M, long long V,
                                                                int C, float scale, T* __restrict__ E) {
  constexpr int N = VEC ? EmPiece<T>::N : 1;
  const int per_row = C / N, lane = threadIdx.x & 63;
  // a wavefront takes a row
  for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); r < M; r += (long long)gridDim.x * 4) {
    const long long tok = (long long)tokens[r];
    const bool ok = tok >= 0 && tok < V;
    const T* src = table + (ok ? tok : 0) * C;
    for (int p = lane; p < per_row; p += 64) {
      if constexpr (VEC) {
        float v[N];
        EmPiece<T>::load(src + p * N, v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = ok ? v[e] * scale : 0.f;
        EmPiece<T>::store(E + r * C + p * N, v);
      } else {
        em_put(E + r * C + p, ok ? em_get(src + p) * scale : 0.f);
      }
    }
  }
}

// ---- gradient, without a sort: a workgroup owns one table row and looks through all kept tokens for it ------------
template <typename T, typename K, typename O>
__global__ void __launch_bounds__(256) embedding_scan_kernel(const T* __restrict__ dE, const K* __restrict__ tokens, const int32_t* __restrict__ idx,
                                                             long long Kn, int C, float scale, int compact, int accumulate, O* __restrict__ out) {
  const long long v = blockIdx.x;
  for (int c0 = 0; c0 < C; c0 += 256) {
    const int c = c0 + threadIdx.x;
    float s = 0.f;
    bool any = false;
    for (long long j0 = 0; j0 < Kn; j0 += 64) {
      const long long j = j0 + (threadIdx.x & 63);
      const bool hit = j < Kn && em_token(tokens, idx, j) == v;
      for (unsigned long long w = __ballot(hit); w; w &= w - 1) {
        const long long jj = j0 + __ffsll((long long)w) - 1, r = compact || !idx ? jj : idx[jj];
        any = true;
        if (c < C) s += em_get(dE + r * C + c);
      }
    }
    if (c < C) {
      O* o = out + v * C + c;
      if (!accumulate) em_put(o, s * scale);
      else if (any) em_put(o, em_get(o) + s * scale);
    }
  }
}

EmbeddingPlan plan_embedding_backward(int64_t K, int64_t V, int32_t C, int32_t dtype) { return EmbeddingPlan{}; }

template <typename T, typename K>
static void launch_em_fwd(const void* tokens, const void* table, int64_t M, int64_t V, int32_t C, float scale, void* E, hipStream_t s) {
  const bool vec = C % EmPiece<T>::N == 0 && ((uintptr_t)table | (uintptr_t)E) % 16 == 0;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(M, 4), 1 << 20));
  if (vec) SBP_LAUNCH(SBP_PROF_GATHER, s, (embedding_forward_kernel<T, K, true>), grid, dim3(256), 0, s, (const K*)tokens, (const T*)table, (long long)M, (long long)V, C, scale, (T*)E);
  else SBP_LAUNCH(SBP_PROF_GATHER, s, (embedding_forward_kernel<T, K, false>), grid, dim3(256), 0, s, (const K*)tokens, (const T*)table, (long long)M, (long long)V, C, scale, (T*)E);
}

int32_t launch_forward_embedding(const void* tokens, int32_t token_bytes, const void* table, int64_t M, int64_t V, int32_t C, float scale,
                                 int32_t dtype, void* E, hipStream_t s) {
  if (dtype == SBP_F32) { if (token_bytes == 4) launch_em_fwd<float, int32_t>(tokens, table, M, V, C, scale, E, s); else launch_em_fwd<float, int64_t>(tokens, table, M, V, C, scale, E, s); }
  else { if (token_bytes == 4) launch_em_fwd<uint16_t, int32_t>(tokens, table, M, V, C, scale, E, s); else launch_em_fwd<uint16_t, int64_t>(tokens, table, M, V, C, scale, E, s); }
  return check_launch("forward_embedding");
}

template <typename T, typename K, typename O>
static void launch_em_bwd(const EmbeddingPlan& p, const void* dE, const void* tokens, const int32_t* idx, int64_t Kn, int64_t V, int32_t C, float scale,
                          void* out, void* ws, uint32_t flags, hipStream_t s) {
  SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_scan_kernel<T, K, O>), dim3((unsigned)V), dim3(256), 0, s, (const T*)dE, (const K*)tokens, idx, (long long)Kn, C, scale,
             flags & SBP_FLAG_DY_COMPACT ? 1 : 0, flags & SBP_FLAG_ACCUMULATE_DW ? 1 : 0, (O*)out);
}
template <typename T, typename K>
static void launch_em_bwd_out(const EmbeddingPlan& p, const void* dE, const void* tokens, const int32_t* idx, int64_t Kn, int64_t V, int32_t C, float scale,
                              void* out, void* ws, uint32_t flags, hipStream_t s) {
  if (flags & SBP_FLAG_DW_OUT_BF16) launch_em_bwd<T, K, uint16_t>(p, dE, tokens, idx, Kn, V, C, scale, out, ws, flags, s);
  else launch_em_bwd<T, K, float>(p, dE, tokens, idx, Kn, V, C, scale, out, ws, flags, s);
}

int32_t launch_backward_embedding(const EmbeddingPlan& p, const void* dE, const void* tokens, int32_t token_bytes, const int32_t* idx, int64_t M,
                                  int64_t K, int64_t V, int32_t C, float scale, int32_t dtype, void* out, void* ws, uint32_t flags, hipStream_t s) {
  if (dtype == SBP_F32) { if (token_bytes == 4) launch_em_bwd_out<float, int32_t>(p, dE, tokens, idx, K, V, C, scale, out, ws, flags, s); else launch_em_bwd_out<float, int64_t>(p, dE, tokens, idx, K, V, C, scale, out, ws, flags, s); }
  else { if (token_bytes == 4) launch_em_bwd_out<uint16_t, int32_t>(p, dE, tokens, idx, K, V, C, scale, out, ws, flags, s); else launch_em_bwd_out<uint16_t, int64_t>(p, dE, tokens, idx, K, V, C, scale, out, ws, flags, s); }
  return check_launch("backward_embedding");
}

}  // namespace sbp
