// Masked attention (sbp_lm.h): forward over all tokens of a sample and backward on the kept ones.
#include "sbp_lm_attention_rows.h"

namespace sbp {

template <typename T>
__global__ void __launch_bounds__(256) masked_forward_rows_kernel(MaskedAttention a) {
  const int lane = threadIdx.x & 63, nb = (int)((a.rows + 31) / 32), unit = blockIdx.x, c = unit % nb, bh = unit / nb;
  for (int i = threadIdx.x >> 6; i < 32; i += 4) {
    const int t = c * 32 + i;
    if (t < a.rows) lm_forward_row<T>(a, bh / a.h, bh % a.h, t, lane);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) masked_backward_rows_kernel(MaskedAttention a) {
  const int lane = threadIdx.x & 63, nb = (int)((a.rows + 31) / 32), nq = a.B * a.h * nb;
  const bool key = (int)blockIdx.x >= nq;
  const int unit = key ? blockIdx.x - nq : blockIdx.x, c = unit % nb, bh = unit / nb;
  for (int i = threadIdx.x >> 6; i < 32; i += 4) {
    const int t = c * 32 + i;
    if (t >= a.rows) continue;
    if (!key) {
      lm_backward_query<T>(a, bh / a.h, bh % a.h, t, lane);
    } else {
      const int b = bh / a.hk, kv = bh % a.hk, g = a.h / a.hk;
      float dk[2], dv[2];
      lm_backward_key<T>(a, b, kv, kv * g, (kv + 1) * g, t, lane, dk, dv);
      T* o = (T*)a.out + ((long long)b * a.rows + t) * ((long long)(a.h + 2 * a.hk) * a.d) + (long long)(a.h + kv) * a.d;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < a.d) {
          lm_store(o + lane + 64 * e, dk[e]);
          lm_store(o + (long long)a.hk * a.d + lane + 64 * e, dv[e]);
        }
    }
  }
}

MaskedAttentionPlan plan_masked_attention_backward(const sbp_attention_desc&, int32_t, int32_t) { return MaskedAttentionPlan{0}; }

int32_t launch_forward_attention_masked(const MaskedAttention& a, int32_t dtype, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.B * a.h * ceil_div(a.rows, 32)));
  if (dtype == SBP_BF16) {
    if (a.d == 16) launch_masked_forward_bf16<16>(a, s);
    else if (a.d == 32) launch_masked_forward_bf16<32>(a, s);
    else if (a.d == 64) launch_masked_forward_bf16<64>(a, s);
    else launch_masked_forward_bf16<128>(a, s);
  } else SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_forward_rows_kernel<float>), grid, dim3(256), 0, s, a);
  return check_launch("forward_attention_masked");
}

int32_t launch_backward_attention_masked(const MaskedAttention& a, const MaskedAttentionPlan&, int32_t dtype, void*, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.B * (a.h + a.hk) * ceil_div(a.rows, 32)));
  if (dtype == SBP_BF16) SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_backward_rows_kernel<uint16_t>), grid, dim3(256), 0, s, a);
  else SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_backward_rows_kernel<float>), grid, dim3(256), 0, s, a);
  return check_launch("backward_attention_masked");
}

}  // namespace sbp
