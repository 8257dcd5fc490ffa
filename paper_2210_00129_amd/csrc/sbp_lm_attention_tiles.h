// What the masked attention kernels on the matrix cores share: which pairs of blocks a wavefront has to look at, and the stream of key
// and value (or query and gradient) tiles through LDS.
#ifndef SBP_LM_ATTENTION_TILES_H_
#define SBP_LM_ATTENTION_TILES_H_

#include "sbp_lm_attention_rows.h"

namespace sbp {

// Positions and documents of some tokens, as ranges: positions p0 .. p1; documents d0 .. d1 of the tokens that belong to one (none:
// d0 > d1), made wider where others belong to none, so that d0 = d1 means that all of them belong to that one.
struct LmRange {
  int p0, p1, d0, d1;
};
struct LmDocs {
  int lo = INT32_MAX, hi = INT32_MIN, none = 0;
  __device__ __forceinline__ void add(int d) {
    none |= d < 0;
    if (d >= 0) { lo = min(lo, d); hi = max(hi, d); }
  }
  __device__ __forceinline__ void join(int mask) {           // with the lane `mask` away
    lo = min(lo, __shfl_xor(lo, mask));
    hi = max(hi, __shfl_xor(hi, mask));
    none |= __shfl_xor(none, mask);
  }
  __device__ __forceinline__ void close() {
    if (none && lo == hi) { if (hi < INT32_MAX) ++hi; else --lo; }
  }
};
// 0: no query of q sees a key of k; 2: every one sees every one; 1: in between (or not known from the ranges)
__device__ __forceinline__ int lm_class(const LmRange& q, const LmRange& k, bool causal, int prefix, bool docs) {
  if (docs && (k.d1 < q.d0 || k.d0 > q.d1 || k.d0 > k.d1)) return 0;
  if (causal && k.p0 > q.p1 && k.p0 >= prefix) return 0;
  const bool order = !causal || k.p1 <= q.p0 || k.p1 < prefix, same = !docs || (q.d0 == q.d1 && k.d0 == k.d1 && q.d0 == k.d0);
  return order && same ? 2 : 1;
}
// The unit of workgroup i: kinds of units of equal length share a rank, longest first; the samples and heads of one XCD stay on it
// where their number is a multiple of 8 (the tiles they stream are then in that XCD's L2 alone).
__device__ __forceinline__ void lm_unit(unsigned i, int heads, int* rank, int* head) {
  if (heads % 8 == 0) {
    const int per = heads / 8, x = i & 7, j = i >> 3;
    *rank = j / per;
    *head = x * per + j % per;
  } else {
    *rank = i / heads;
    *head = i % heads;
  }
}

// Copies straight into LDS (see async_copy16), 16 or 4 bytes per lane into 1 KB or 256 bytes at the wave-uniform LDS address `to`.
// Written as assembly because the compiler waits for every copy it knows of before the next transposing read of LDS, whatever the
// address: with the builtin each stage began by waiting for the copies of the next one.  The kernels order them by lm_copies_done()
// and barriers; both keep the compiler from moving LDS reads across them.  An address is read when its copy is issued; m0 is a register
// that the compiler sets right before each of its own uses.
__device__ __forceinline__ uint32_t lm_lds(const char* p) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uintptr_t)(SBP_LDS const char*)p); }
// base: wave-uniform; off: bytes, per lane
__device__ __forceinline__ void lm_copy16(const void* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(to) : "memory");
}
__device__ __forceinline__ void lm_copy4(const void* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(to) : "memory");
}
__device__ __forceinline__ void lm_copies_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Copies of a tile of kLmTile rows of 2 D bytes into an LDS image, shared out over NW wavefronts.
template <int D, int NW>
struct LmStream {
  using L = AttnSwizzled<D>;
  static constexpr int IMG = kLmTile / 16 * L::G16, COPIES = kLmTile / L::RPC, NI = (COPIES + NW - 1) / NW;
  static_assert(COPIES >= 1, "a copy is at most a tile");
  static __device__ __forceinline__ int image_place(int c) { return D < 32 ? c * 1024 : (c * L::RPC >> 4) * L::G16 + (c * L::RPC & 15) / L::RPC * L::COPY; }
  uint32_t off[NI];                // the lane's pieces of a whole tile, bytes from its first row
  int ld;                          // elements per row
  __device__ __forceinline__ LmStream(int ld_, int lane, int wave) : ld(ld_) {
#pragma unroll
    for (int n = 0; n < NI; ++n) off[n] = piece(n, kLmTile, lane, wave);
  }
  __device__ __forceinline__ uint32_t piece(int n, int rows, int lane, int wave) const {
    const int row = (wave + n * NW) * L::RPC + lane / L::CH, ch = (lane % L::CH) ^ L::swz(row);
    return (uint32_t)(min(row, rows - 1) * ld) * 2u + 16 * ch;
  }
  // src: row 0 of the tensor (bf16); tile rows t0 .. t0 + 63 of `rows` (past the end: the last row)
  __device__ __forceinline__ void issue(const uint16_t* src, int t0, int rows, uint32_t buf, int lane, int wave) const {
    const uint16_t* base = src + (long long)t0 * ld;
    if (rows - t0 >= kLmTile) {
#pragma unroll
      for (int n = 0; n < NI; ++n)
        if (COPIES % NW == 0 || wave + n * NW < COPIES) lm_copy16(base, off[n], buf + image_place(wave + n * NW));
    } else {
#pragma unroll
      for (int n = 0; n < NI; ++n)
        if (COPIES % NW == 0 || wave + n * NW < COPIES) lm_copy16(base, piece(n, rows - t0, lane, wave), buf + image_place(wave + n * NW));
    }
  }
};

}  // namespace sbp
#endif
