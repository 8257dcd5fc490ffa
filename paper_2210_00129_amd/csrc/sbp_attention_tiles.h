// Pieces of the attention kernels on the bf16 matrix cores: the layout of a tile of token rows in LDS, operands out of accumulators,
// rows out of accumulators.
#ifndef SBP_ATTENTION_TILES_H_
#define SBP_ATTENTION_TILES_H_

#include "sbp_mfma_gemm.h"

namespace sbp {

static constexpr float kLog2e = 1.4426950408889634f;

// Accumulated C registers 8 ks .. 8 ks + 7 as an operand: 16 contraction rows of the lane's column.
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t& c, int ks) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = bf16_pack(c[8 * ks + 2 * e], c[8 * ks + 2 * e + 1]);
  return __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
}

// AttnSwizzled: rows of 2 D bytes, 16-byte chunk c of row r at place c ^ swz(r), written by global -> LDS copies whose lanes
// choose the chunk they fetch (the copy fixes the LDS place by lane; a copy fills 1 KB, 512 / D rows).  By their addresses both
// kinds of reads meet all 64 banks once: a transposing read's half wavefront takes 64 bytes of each of 4 neighbouring rows, so these
// rows differ in the bits of the place above the chunks it takes (bit 2; D = 128: bits 2 and 3), and the 16-byte reads of 16
// neighbouring rows fall on different places because the copies within 16 rows lie 16 bytes further apart than their 1 KB (not for
// D = 32, whose 16 rows are one copy: rows r and r + 8 share banks, two turns).  That holds for 16 consecutive lanes to a turn; the
// counter still has conflicts in 31 % of the LDS cycles at D = 64, 44 before.  (With c ^ (r & 7) and no
// gaps rows r and r + 2 exchanged places within the same 64 bytes: every transposing read took two turns, D = 128 four.)
// D = 16: a copy is 32 rows of 32 bytes as they are; the 32 rows of a transposing operand are the 16 head dimensions twice.
template <int D>
struct AttnSwizzled {
  static constexpr int RB = 2 * D, CH = D / 8, KS = D / 16, DB = D < 32 ? 1 : D / 32;
  static constexpr int RPC = 512 / D, COPY = D <= 32 ? 1024 : 1040, G16 = D < 32 ? 16 * RB : (16 / RPC - 1) * COPY + 1024;   // rows of a copy, pitch of the copies, bytes of 16 rows
  static __device__ __forceinline__ int swz(int r) {
    return D < 32 ? 0 : D == 32 ? (r >> 1) & 3 : D == 64 ? (r & 2) << 1 | (r & 4) >> 1 : (r & 3) << 2;
  }
  static __device__ __forceinline__ int place(int r) { return D < 32 ? r * RB : (r >> 4) * G16 + ((r & 15) / RPC) * COPY + (r % RPC) * RB; }
  int foff[KS], toff[DB];
  __device__ __forceinline__ explicit AttnSwizzled(int lane) {
    const int g = lane >> 4, i = lane & 15, r = lane & 31, rt = 4 * (g >> 1) + (i >> 2);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) foff[ks] = place(r) + (((2 * ks + (lane >> 5)) ^ swz(r)) << 4);
#pragma unroll
    for (int x = 0; x < DB; ++x) toff[x] = place(rt) + ((((4 * x + 2 * (g & 1) + ((i & 3) >> 1)) ^ swz(rt)) & (CH - 1)) << 4) + 8 * (i & 1);
  }
  // row0: a multiple of 32
  __device__ __forceinline__ bf16x8_t row(const char* tile, int row0, int ks) const {
    return *reinterpret_cast<const bf16x8_t*>(tile + (row0 >> 4) * G16 + foff[ks]);
  }
  // row0: a multiple of 16; rows 8 further on lie 8 / RPC copies further on, with the same swz
  __device__ __forceinline__ bf16x8_t tr(const char* tile, int row0, int x) const {
    const char* p = tile + (row0 >> 4) * G16 + toff[x];
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SBP_LDS s16x4_t*)(p));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SBP_LDS s16x4_t*)(p + (D <= 32 ? 8 * RB : 8 / RPC * COPY)));
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// Writes an accumulated [head dim][32 tokens] block to the tokens' rows (out: row 0 of the head's columns) through LDS
// (one 32-row image of the wavefront's own, pitch 2 D + 16 bytes): whole 2 D-byte rows instead of 8-byte pieces; f: the lane's factor
template <int D>
__device__ __forceinline__ void attn_store_rows(char* image, const f32x16_t (&acc)[AttnSwizzled<D>::DB], float f, uint16_t* __restrict__ out, long long ld,
                                                int first, int n_k, int lane) {
  constexpr int PITCH = 2 * D + 16, LPR = D / 8;           // lanes per row
  char* row = image + (lane & 31) * PITCH + 8 * (lane >> 5);
#pragma unroll
  for (int x = 0; x < AttnSwizzled<D>::DB; ++x)
#pragma unroll
    for (int q4 = 0; q4 < (D < 32 ? D / 8 : 4); ++q4)
      *reinterpret_cast<uint2*>(row + 64 * x + 16 * q4) = make_uint2(bf16_pack(acc[x][4 * q4] * f, acc[x][4 * q4 + 1] * f),
                                                                     bf16_pack(acc[x][4 * q4 + 2] * f, acc[x][4 * q4 + 3] * f));
#pragma unroll
  for (int r = 0; r < 32 * LPR / 64; ++r) {                // (a wavefront's LDS accesses complete in order)
    const int tok = r * (64 / LPR) + lane / LPR, c = lane % LPR;
    const uint4 v = *reinterpret_cast<const uint4*>(image + tok * PITCH + 16 * c);
    if (first + tok < n_k) *reinterpret_cast<uint4*>(out + (first + tok) * ld + 8 * c) = v;
  }
}

__device__ __forceinline__ float attn_dot2(uint32_t a, uint32_t b, float c) {      // two exact products added in fp32
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, b), c, false);
}

}  // namespace sbp
#endif
