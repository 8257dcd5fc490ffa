// Masked attention (sbp_lm.h): forward over all tokens of a sample and backward on the kept ones.
#include <algorithm>
#include <type_traits>

#include "sbp_lm_attention_tiles.h"

namespace sbp {

// What the backward's main kernel reads per token (LmTables).  Bound: the read of A and dA (4 x 12 heads of 64, 1024 kept tokens: 12.6 MB, 4.8 us of
// which most is the launch and one round trip to memory; 16 heads of 128, 4096 tokens: 33.5 MB, 8.3 us);
// all of a wavefront's loads are under way at once.
template <typename T, int D>
__global__ void __launch_bounds__(256) masked_prepare_kernel(MaskedAttention a, LmTables w) {
  // a workgroup per tile and head (head h: positions and documents)
  const int tiles = w.npad / kLmTile, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, b = bh / (a.h + 1), head = bh % (a.h + 1), t = tile * kLmTile + lane;
  const bool on = t < a.rows;
  if (head == a.h) {
    if (wave) return;
    const int p = on ? lm_pos(a, b, t) : 0, d = on ? lm_doc(a, b, p) : -1;
    w.pos[(long long)b * w.npad + t] = on ? (float)p : NAN;
    w.doc[(long long)b * w.npad + t] = d;
    LmDocs r;
    if (on) r.add(d);
    int p0 = on ? p : INT32_MAX, p1 = on ? p : INT32_MIN;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      r.join(m);
      p0 = min(p0, __shfl_xor(p0, m));
      p1 = max(p1, __shfl_xor(p1, m));
    }
    r.close();
    if (lane == 0) w.range[(long long)b * tiles + tile] = make_int4(p0, p1, r.lo, r.hi);
    return;
  }
  // delta of a row: D / 8 (bf16) or D / 4 (fp32) lanes of 16 bytes each
  constexpr int N = 16 / sizeof(T), PER = D / N, ROWS = 64 / PER < 16 ? 64 / PER : 16, IT = 16 / ROWS;
  const long long ld = (long long)a.h * D, row0 = (long long)b * a.rows, at = ((long long)b * a.h + head) * w.npad + tile * kLmTile;
  const float l = wave == 0 && on ? a.lse[(row0 + t) * a.h + head] : -INFINITY;
  uint4 x[IT], y[IT];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const long long off = (row0 + min(tile * kLmTile + 16 * wave + i * ROWS + min(lane / PER, ROWS - 1), a.rows - 1)) * ld + head * D + lane % PER * N;
    x[i] = *reinterpret_cast<const uint4*>((const T*)a.dA + off);
    y[i] = *reinterpret_cast<const uint4*>((const T*)a.A + off);
  }
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int row = 16 * wave + i * ROWS + lane / PER;
    float s = tile * kLmTile + row < a.rows ? lm_dot((const T*)&x[i], (const T*)&y[i], N) : 0.f;
#pragma unroll
    for (int m = 1; m < PER; m <<= 1) s += __shfl_xor(s, m);
    if (lane / PER < ROWS && lane % PER == 0) w.nd[at + row] = -s;
  }
  if (wave) return;
  w.l2[at + lane] = l == -INFINITY ? 1e30f : l * (sizeof(T) == 2 ? kLog2e : 1.f);      // (a weight of exp(score - 1e30) = 0)
}

// Adds the parts of dK and dV of shared heads in order and rounds once: four channels per thread.
template <typename T>
__global__ void __launch_bounds__(256) masked_join_kernel(MaskedAttention a, LmTables w) {
  const long long pieces = (long long)a.B * a.rows * a.hk * 2 * a.d / 4, i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= pieces) return;
  float4 s = reinterpret_cast<const float4*>(w.part)[i];
  for (int p = 1; p < w.parts; ++p) {
    const float4 v = reinterpret_cast<const float4*>(w.part)[p * pieces + i];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  const int c = (int)(i * 4 % (2 * a.d)), kv = (int)(i * 4 / (2 * a.d) % a.hk);
  const long long row = i * 4 / (2 * a.d) / a.hk, ld = (long long)(a.h + 2 * a.hk) * a.d;
  T* out = (T*)a.out + row * ld + (c < a.d ? (a.h + kv) * a.d + c : (a.h + a.hk + kv) * a.d + c - a.d);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(bf16_pack(s.x, s.y), bf16_pack(s.z, s.w));
  else *reinterpret_cast<float4*>(out) = s;
}

// Parts of a key / value head: its query heads follow one another in one workgroup per 128 keys (fp32: 32) unless that leaves fewer
// workgroups of this kind than CUs (256); then they are dealt to the smallest number of parts that does not, each one more set of fp32
// dK and dV.  (16 heads of 128 sharing 2, 4096 kept tokens: 4 parts 331 us, 2 parts 553, 8 parts 334 with twice the workspace.)
static int masked_parts(int64_t heads, int share, int nchunks) {
  int p = 1;
  while (p < share && heads * p * nchunks < 256) {
    ++p;
    while (share % p) ++p;
  }
  return p;
}

MaskedAttentionPlan plan_masked_attention_backward(const sbp_attention_desc& d, int32_t n_k, int32_t dtype) {
  MaskedAttentionPlan p = {};
  if (n_k == 0) return p;
  p.npad = (int)(ceil_div(n_k, kLmTile) * kLmTile);
  p.nchunks = (int)ceil_div(n_k, dtype == SBP_BF16 ? kLmChunk : 32);
  p.parts = masked_parts((int64_t)d.B * d.h_kv, d.h / d.h_kv, p.nchunks);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
  p.off_l2 = take((size_t)d.B * d.h * p.npad * 4);
  p.off_nd = take((size_t)d.B * d.h * p.npad * 4);
  p.off_pos = take((size_t)d.B * p.npad * 4);
  p.off_doc = take((size_t)d.B * p.npad * 4);
  p.off_range = take((size_t)d.B * (p.npad / kLmTile) * sizeof(int4));
  p.off_part = take(p.parts > 1 ? (size_t)p.parts * d.B * n_k * d.h_kv * 2 * d.d * 4 : 0);
  p.bytes = at;
  return p;
}

int32_t launch_forward_attention_masked(const MaskedAttention& a, int32_t dtype, hipStream_t s) {
  if (dtype != SBP_BF16) launch_masked_f32(a, nullptr, s);
  else if (a.d == 16) launch_masked_forward_bf16<16>(a, s);
  else if (a.d == 32) launch_masked_forward_bf16<32>(a, s);
  else if (a.d == 64) launch_masked_forward_bf16<64>(a, s);
  else launch_masked_forward_bf16<128>(a, s);
  return check_launch("forward_attention_masked");
}

int32_t launch_backward_attention_masked(const MaskedAttention& a, const MaskedAttentionPlan& p, int32_t dtype, void* ws_, hipStream_t s) {
  char* ws = (char*)ws_;
  const bool bf16 = dtype == SBP_BF16;
  const LmTables w{(float*)(ws + p.off_l2), (float*)(ws + p.off_nd), (float*)(ws + p.off_pos), (int32_t*)(ws + p.off_doc), (int4*)(ws + p.off_range),
                   p.parts > 1 ? (float*)(ws + p.off_part) : nullptr, p.npad, p.parts, p.nchunks};
  const dim3 prepare((unsigned)((int64_t)a.B * (a.h + 1) * (p.npad / kLmTile)));
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (bf16) SBP_LAUNCH(SBP_PROF_OTHER, s, (masked_prepare_kernel<uint16_t, D>), prepare, dim3(256), 0, s, a, w);
    else SBP_LAUNCH(SBP_PROF_OTHER, s, (masked_prepare_kernel<float, D>), prepare, dim3(256), 0, s, a, w);
  };
  if (a.d == 16) go(std::integral_constant<int, 16>{});
  else if (a.d == 32) go(std::integral_constant<int, 32>{});
  else if (a.d == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  if (!bf16) launch_masked_f32(a, &w, s);
  else if (a.d == 16) launch_masked_backward_bf16<16>(a, w, s);
  else if (a.d == 32) launch_masked_backward_bf16<32>(a, w, s);
  else if (a.d == 64) launch_masked_backward_bf16<64>(a, w, s);
  else launch_masked_backward_bf16<128>(a, w, s);
  if (p.parts > 1) {
    const dim3 join((unsigned)ceil_div((int64_t)a.B * a.rows * a.hk * 2 * a.d / 4, 256));
    if (bf16) SBP_LAUNCH(SBP_PROF_REDUCE, s, (masked_join_kernel<uint16_t>), join, dim3(256), 0, s, a, w);
    else SBP_LAUNCH(SBP_PROF_REDUCE, s, (masked_join_kernel<float>), join, dim3(256), 0, s, a, w);
  }
  return check_launch("backward_attention_masked");
}

}  // namespace sbp
