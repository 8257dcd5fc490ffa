// The token table (sbp_lm.h): scaled lookup, and the table's gradient from the kept rows, grouped by token.
#include <algorithm>
#include <type_traits>

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

// ---- lookup: a wavefront per row, a piece of 16 bytes (VEC) or one channel per lane and step.  Bound: HBM (32768 rows of 2048 channels, bf16,
// out of 50000: 256 MB in 48 us) ----------------------------------------
template <typename T, typename K, bool VEC>
__global__ void __launch_bounds__(256) embedding_forward_kernel(const K* __restrict__ tokens, const T* __restrict__ table, long long M, long long V,
                                                                int C, int slice, float scale, T* __restrict__ E) {
  constexpr int N = VEC ? EmPiece<T>::N : 1;
  const int lane = threadIdx.x & 63, first = blockIdx.y * slice, per_row = min(first + slice, C / N);
  // a wavefront takes a slice of a row
  for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); r < M; r += (long long)gridDim.x * 4) {
    const long long tok = (long long)tokens[r];
    const bool ok = tok >= 0 && tok < V;
    const T* src = table + (ok ? tok : 0) * C;
    for (int p = first + lane; p < per_row; p += 64) {
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

// ------------------------------------------------------------------------------------------------
// Gradient.  dtable[v] = scale * sum of the kept rows of dE whose token is v.  The floor is the read of the kept rows and the write
// of the whole table (dense, as the weight gradients of the other layers are); the grouping moves 8 bytes per kept row.
//
// Up to kEmScan kept rows one launch does it all: every workgroup owns some table rows and looks through the kept tokens for them.
// (1000 rows of 200 channels, fp32, 198 kept: 10 us with the lookup's 2, sorted 17.)
// More rows are sorted by token (stable least-significant-digit radix sort of (token, row) pairs): by one workgroup with the pairs in
// registers and LDS, all passes in one launch, or by 64 workgroups, one launch per pass.  The rest of the (first) launch zeroes the table.
// One workgroup: up to kEmOne rows, and up to kEmOneFill of them where zeroing kEmFill bytes or more hides a part of its time
// (2048 channels, lookup and gradient; one workgroup and 64: 4000 rows, 500 / 16000 / 32000 tokens: 29 and 28, 40 and 55, 65 and 84 us; 8000
// rows: 55 and 39, 71 and 74, 91 and 110; 16384 rows: 76 and 58, 122 and 119, 135 and 153).
// Then a wavefront sums chunks of kEmChunk sorted rows in order and writes the rows of the tokens that end there, and tokens that cross
// a chunk's border are joined from partial sums in chunk order: every sum runs in the order of idx whatever the grid does.
// 50000 tokens of 2048 channels, 16384 kept rows, bf16, V C 4 = 410 MB: sort and zeroing 58 us (7 TB/s), sums 42, joins 6.
// ------------------------------------------------------------------------------------------------
static constexpr int kEmScan = 256, kEmOne = 4096, kEmOneFill = 16384, kEmChunk = 32, kEmBins = 2048, kEmBlocks = 64;
static constexpr int64_t kEmFill = 100 << 20;

static int64_t em_fill_bytes(int64_t V, int32_t C, uint32_t flags) { return flags & SBP_FLAG_ACCUMULATE_DW ? 0 : V * C * (flags & SBP_FLAG_DW_OUT_BF16 ? 2 : 4); }

// A lane's columns of one row: a piece of 16 bytes of the input (VEC) or one column.
template <typename T, bool VEC>
struct EmCols {
  static constexpr int N = VEC ? EmPiece<T>::N : 1, SLICE = 64 * N;      // columns of a lane, of a wavefront
  using Raw = typename std::conditional<VEC, uint4, T>::type;            // as it lies in memory
  static __device__ __forceinline__ Raw load(const T* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void add(const Raw& w, float (&s)[N]) {
    if constexpr (!VEC) {
      s[0] += em_get(&w);
    } else {
      const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) s[e] += __uint_as_float(x[e]);
        else { s[2 * e] += bf16_lo(x[e]); s[2 * e + 1] += bf16_hi(x[e]); }
      }
    }
  }
  template <typename O>
  static __device__ __forceinline__ void put(O* o, const float (&s)[N], float scale, bool add) {
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = s[e] * scale;
    if (add)
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] += em_get(o + e);
    if constexpr (!VEC) em_put(o, v[0]);
    else if constexpr (sizeof(O) == 4)
#pragma unroll
      for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(o + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    else
#pragma unroll
      for (int e = 0; e < N; e += 4) *reinterpret_cast<uint2*>(o + e) = make_uint2(bf16_pack(v[e], v[e + 1]), bf16_pack(v[e + 2], v[e + 3]));
  }
};

// Zeroes the bytes from `begin` to `end` (multiples of sizeof(O)), thread `t` of `threads`: whole pieces of 16 bytes by their addresses, and
// what lies before and behind them.
template <typename O>
__device__ __forceinline__ void em_zero(char* begin, char* end, long long t, long long threads) {
  char *head = (char*)(((uintptr_t)begin + 15) & ~(uintptr_t)15), *tail = (char*)((uintptr_t)end & ~(uintptr_t)15);
  if (head > end) head = end;
  if (tail < head) tail = head;
  for (long long i = t; i < (tail - head) / 16; i += threads) reinterpret_cast<uint4*>(head)[i] = make_uint4(0, 0, 0, 0);
  if (t < 16 / (long long)sizeof(O)) {
    if (begin + t * sizeof(O) < head) reinterpret_cast<O*>(begin)[t] = 0;
    if (tail + t * sizeof(O) < end) reinterpret_cast<O*>(tail)[t] = 0;
  }
}

// A workgroup owns `rows` table rows and, of these, a slice of the columns (all of them where there are rows enough for every CU).  It zeroes
// its part, and sums the rows of the tokens that it finds among the kept ones, in their order.
template <typename T, typename K, typename O, bool VEC>
__global__ void __launch_bounds__(256) embedding_scan_kernel(const T* __restrict__ dE, const K* __restrict__ tokens, const int32_t* __restrict__ idx,
                                                             int Kn, long long V, int C, int rows, int slice, float scale, int compact, int accumulate,
                                                             O* __restrict__ out) {
  using Cols = EmCols<T, VEC>;
  constexpr int N = Cols::N, U = 8, Q = kEmScan / 64;
  __shared__ int tok_s[kEmScan], row_s[kEmScan], list_s[4][kEmScan];
  const int t = threadIdx.x, lane = t & 63;
  int* list = list_s[t >> 6];
  const int first = blockIdx.y * slice, last = min(first + slice, C);
  const long long v0 = (long long)blockIdx.x * rows, v1 = min(v0 + rows, V);
  if (t < Kn) {
    const long long tok = em_token(tokens, idx, t);
    tok_s[t] = tok >= v0 && tok < v1 ? (int)(tok - v0) : -1;
    row_s[t] = compact || !idx ? t : idx[t];
  } else {
    tok_s[t] = -1;
  }
  __syncthreads();
  int tk[Q];
  unsigned long long left[Q], any = 0;                     // the same for all wavefronts
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    tk[q] = tok_s[64 * q + lane];
    left[q] = __ballot(tk[q] >= 0);
    any |= left[q];
  }
  if (!accumulate && !(rows == 1 && any)) {                  // (a row alone whose token occurs is written below)
    if (slice >= C) em_zero<O>((char*)(out + v0 * C), (char*)(out + v1 * C), t, 256);
    else
      for (long long v = v0; v < v1; ++v) em_zero<O>((char*)(out + v * C + first), (char*)(out + v * C + last), t, 256);
    if (any) {                                               // other threads write some of these places again
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    }
  }
#pragma unroll
  for (int q0 = 0; q0 < Q; ++q0)
    while (left[q0]) {
      const int v = __builtin_amdgcn_readlane(tk[q0], __ffsll((long long)left[q0]) - 1);
      unsigned long long hit[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        hit[q] = __ballot(tk[q] == v);
        left[q] &= ~hit[q];
      }
      // the token's rows in order: a list of the wavefront's own (its LDS accesses complete in order)
      int count = 0;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (tk[q] == v) list[count + __popcll(hit[q] & ((1ull << lane) - 1))] = row_s[64 * q + lane];
        count += __popcll(hit[q]);
      }
      __builtin_amdgcn_wave_barrier();
      for (int c0 = first + t * N; c0 < last; c0 += 256 * N) {
        float s[N];
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = 0.f;
        for (int i = 0; i < count; i += U) {                 // U rows in flight (past the end the last one again, unused), added in order
          typename Cols::Raw x[U];
#pragma unroll
          for (int u = 0; u < U; ++u) x[u] = Cols::load(dE + (long long)list[min(i + u, count - 1)] * C + c0);
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (i + u < count) Cols::add(x[u], s);
        }
        Cols::put(out + (v0 + v) * C + c0, s, scale, accumulate != 0);
      }
      __builtin_amdgcn_wave_barrier();
    }
}

// ---- sort ----------------------------------------------------------------------------------------------------------
// The lanes whose element has the same digit as this lane's, among the lanes that have one.
__device__ __forceinline__ unsigned long long em_same(uint32_t digit, bool on, int bits) {
  unsigned long long same = __ballot(on);
  for (int bit = 0; bit < bits; ++bit) {
    const unsigned long long ones = __ballot(digit >> bit & 1);
    same &= digit >> bit & 1 ? ones : ~ones;
  }
  return same;
}

// One workgroup of 16 wavefronts, all passes: every wavefront holds a run of the elements in registers (R rounds of 64), finds an
// element's place among the wavefront's own, and after the counts of all wavefronts have been added up writes it to its place in LDS.
// The other workgroups of the launch zero the table.
template <typename K, typename O, int R>
__global__ void __launch_bounds__(1024) embedding_sort_kernel(const K* __restrict__ tokens, const int32_t* __restrict__ idx, int compact, int Kn,
                                                              long long V, int bits, int passes, uint32_t* __restrict__ keys_out,
                                                              int32_t* __restrict__ rows_out, char* __restrict__ table, long long table_bytes) {
  if (blockIdx.x) {
    em_zero<O>(table, table + table_bytes, (blockIdx.x - 1) * 1024LL + threadIdx.x, (gridDim.x - 1) * 1024LL);
    return;
  }
  extern __shared__ uint32_t em_lds[];
  uint32_t *skey = em_lds, *srow = skey + R * 1024, *count = srow + R * 1024;     // [16 * 64 * R] twice, [16][256]
  __shared__ uint32_t scan_s[4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, first = wave * 64 * R + lane, bins = 1 << bits;
  uint32_t key[R], row[R], at[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int j = first + 64 * r;
    row[r] = j < Kn ? (idx ? (uint32_t)idx[j] : (uint32_t)j) : 0u;
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int j = first + 64 * r;
    const long long tok = j < Kn ? (long long)tokens[row[r]] : V;
    key[r] = tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V;
    if (compact) row[r] = (uint32_t)j;
  }
  for (int p = 0; p < passes; ++p) {
    for (int i = t; i < 16 * bins; i += 1024) count[i] = 0;
    __syncthreads();
    uint32_t* mine = count + wave * bins;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool on = first + 64 * r < Kn;
      const uint32_t digit = key[r] >> (p * bits) & (bins - 1);
      const unsigned long long same = em_same(digit, on, bits);
      const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
      if (on) at[r] = mine[digit] + rank;
      __builtin_amdgcn_wave_barrier();                       // (a wavefront's LDS accesses complete in order)
      if (on && rank + 1 == (uint32_t)__popcll(same)) mine[digit] = at[r] + 1;
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // digit t: the elements of the wavefronts before each one, then those of the digits before it
    uint32_t total = 0, scan = 0;
    if (t < 256) {
      if (t < bins)
        for (int w = 0; w < 16; ++w) {
          const uint32_t n = count[w * bins + t];
          count[w * bins + t] = total;
          total += n;
        }
      scan = total;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const uint32_t o = __shfl_up(scan, m);
        scan += lane >= m ? o : 0;
      }
      if (lane == 63) scan_s[wave] = scan;
    }
    __syncthreads();
    if (t < bins) {
      scan -= total;
      for (int w = 0; w < wave; ++w) scan += scan_s[w];
      for (int w = 0; w < 16; ++w) count[w * bins + t] += scan;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (first + 64 * r < Kn) {
        const uint32_t to = at[r] + mine[key[r] >> (p * bits) & (bins - 1)];
        skey[to] = key[r];
        srow[to] = row[r];
      }
    __syncthreads();
    if (p + 1 < passes) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (first + 64 * r < Kn) { key[r] = skey[first + 64 * r]; row[r] = srow[first + 64 * r]; }
      __syncthreads();
    }
  }
  for (int i = t; i < Kn; i += 1024) { keys_out[i] = skey[i]; rows_out[i] = (int32_t)srow[i]; }
}

// 64 workgroups: kept row j belongs to block b = j / per.  hist[p][b][digit]: how many elements of block b (in the order before pass p)
// have the digit.  The workgroups behind the first nb zero the table.
template <typename K, typename O>
__global__ void __launch_bounds__(256) embedding_count_kernel(const K* __restrict__ tokens, const int32_t* __restrict__ idx, int Kn, long long V,
                                                              int per, int nb, int bits, int passes, uint32_t* __restrict__ hist,
                                                              char* __restrict__ table, long long table_bytes) {
  __shared__ uint32_t bins_s[kEmBins];
  if ((int)blockIdx.x >= nb) {
    em_zero<O>(table, table + table_bytes, (blockIdx.x - nb) * 256LL + threadIdx.x, (gridDim.x - nb) * 256LL);
    return;
  }
  const int t = threadIdx.x, bins = 1 << bits;
  for (int i = t; i < bins; i += 256) bins_s[i] = 0;
  for (int p = 1; p < passes; ++p)
    for (int i = t; i < bins; i += 256) hist[((long long)p * nb + blockIdx.x) * bins + i] = 0;
  __syncthreads();
  const long long j0 = (long long)blockIdx.x * per, j1 = min(j0 + per, (long long)Kn);
  for (long long j = j0 + t; j < j1; j += 256) {
    const long long tok = em_token(tokens, idx, j);
    atomicAdd(&bins_s[(tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int i = t; i < bins; i += 256) hist[(long long)blockIdx.x * bins + i] = bins_s[i];
}

// One pass: a block of four wavefronts moves its run of elements, every wavefront a quarter in order.  FIRST: the elements come from
// the tokens; later passes read the pairs of the pass before.
template <typename K, bool FIRST>
__global__ void __launch_bounds__(256) embedding_move_kernel(const K* __restrict__ tokens, const int32_t* __restrict__ idx, int compact,
                                                             const uint32_t* __restrict__ keys, const int32_t* __restrict__ rows, int Kn, long long V,
                                                             int per, int bits, int pass, int passes, uint32_t* __restrict__ hist,
                                                             uint32_t* __restrict__ keys_out, int32_t* __restrict__ rows_out) {
  __shared__ uint32_t place[4 * kEmBins];
  __shared__ uint32_t wave_total[4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, nb = gridDim.x, shift = pass * bits, bins = 1 << bits;
  const long long first = (long long)blockIdx.x * per + (long long)wave * (per / 4);
  const long long last = min(min(first + per / 4, (long long)(blockIdx.x + 1) * per), (long long)Kn);
  uint32_t* mine = place + wave * bins;
  for (int i = t; i < 4 * bins; i += 256) place[i] = 0;
  __syncthreads();
  auto key_at = [&](long long j) -> uint32_t {
    if constexpr (!FIRST) return keys[j];
    const long long tok = em_token(tokens, idx, j);
    return tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V;
  };
  for (long long j = first + lane; j < last; j += 64) atomicAdd(&mine[key_at(j) >> shift & (bins - 1)], 1u);
  __syncthreads();
  // where the block's elements of each digit go: the digits below it (runs of 256 digits in turn), the blocks before this one, the
  // wavefronts before each one
  uint32_t below = 0;
  for (int d0 = 0; d0 < bins; d0 += 256) {
    const int d = d0 + t;
    uint32_t total = 0, before = 0;
    if (d < bins) {
      const uint32_t* h = hist + (long long)pass * nb * bins + d;
#pragma unroll 16
      for (int b = 0; b < nb; ++b) {
        const uint32_t x = h[(long long)b * bins];
        before += b < (int)blockIdx.x ? x : 0;
        total += x;
      }
    }
    uint32_t scan = total;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const uint32_t o = __shfl_up(scan, m);
      scan += lane >= m ? o : 0;
    }
    if (lane == 63) wave_total[wave] = scan;
    __syncthreads();
    uint32_t p = below + scan - total + before;
    for (int w = 0; w < 4; ++w) {
      if (w < wave) p += wave_total[w];
      below += wave_total[w];
    }
    if (d < bins)
      for (int w = 0; w < 4; ++w) {
        const uint32_t n = place[w * bins + d];
        place[w * bins + d] = p;
        p += n;
      }
    __syncthreads();
  }
  for (long long j0 = first; j0 < last; j0 += 64) {          // (the same count for every lane)
    const long long j = j0 + lane;
    const bool on = j < last;
    const uint32_t key = on ? key_at(j) : 0, digit = key >> shift & (bins - 1);
    const int32_t row = !on ? 0 : FIRST ? (compact || !idx ? (int32_t)j : idx[j]) : rows[j];
    const unsigned long long same = em_same(digit, on, bits);
    const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
    uint32_t dest = 0;
    if (on) dest = mine[digit] + rank;
    __builtin_amdgcn_wave_barrier();                         // (a wavefront's LDS accesses complete in order)
    if (on && rank + 1 == (uint32_t)__popcll(same)) mine[digit] = dest + 1;
    __builtin_amdgcn_wave_barrier();
    if (on) {
      keys_out[dest] = key;
      rows_out[dest] = row;
      if (pass + 1 < passes) atomicAdd(&hist[((long long)(pass + 1) * nb + dest / per) * bins + (key >> (shift + bits) & (bins - 1))], 1u);
    }
  }
}

// ---- sums ----------------------------------------------------------------------------------------------------------
// A wavefront per (chunk, column slice).  A token that lies in the chunk altogether is finished here; one that began before it leaves
// its part in partial[chunk][0], one that begins here and goes on in partial[chunk][1].
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256) embedding_sum_kernel(const T* __restrict__ dE, const uint32_t* __restrict__ keys, const int32_t* __restrict__ rows,
                                                            int Kn, long long V, int C, int chunks, int slices, float scale, int accumulate,
                                                            float* __restrict__ partial, O* __restrict__ out) {
  using Cols = EmCols<T, VEC>;
  constexpr int N = Cols::N, U = 16;
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= (long long)chunks * slices) return;
  const int chunk = (int)(unit / slices), c0 = (int)(unit % slices) * Cols::SLICE + lane * N;
  const int i0 = chunk * kEmChunk, n = min(kEmChunk, Kn - i0);
  const bool on = c0 < C;
  const T* src = dE + (on ? c0 : 0);
  // keys of the chunk, of its neighbours, and the rows, one per lane: lane l has element i0 - 1 + l
  const int me = i0 - 1 + lane;
  const uint32_t key = me >= 0 && me < Kn && lane <= kEmChunk + 1 ? keys[me] : 0xffffffffu;
  const int row = me >= 0 && me < Kn && lane <= kEmChunk ? rows[me] : 0;
  const unsigned long long ends = __ballot(key != (uint32_t)__shfl_down((int)key, 1) || lane == 63);   // bit l: element l is its token's last
  const bool begun = !(ends & 1);                          // the element before the chunk has the first one's token
  float s[N];
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = 0.f;
  bool head = true;                                        // still in the chunk's first token
  for (int i = 0; i < n; i += U) {
    typename Cols::Raw x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {                            // (past the chunk's end its last row again, unused)
      const long long r = __builtin_amdgcn_readlane(row, min(i + u, n - 1) + 1);
      x[u] = Cols::load(src + r * C);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= n) break;
      Cols::add(x[u], s);
      const bool end = ends >> (i + u + 1) & 1;
      if (!end && i + u + 1 < n) continue;
      const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key, i + u + 1);
      if (k < (uint32_t)V && on) {
        if (end && !(head && begun)) {
          Cols::put(out + (long long)k * C + c0, s, scale, accumulate != 0);
        } else {
          float* p = partial + ((long long)chunk * 2 + (head && begun ? 0 : 1)) * C + c0;
#pragma unroll
          for (int e = 0; e < N; ++e) p[e] = s[e];
        }
      }
      head = false;
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.f;
    }
  }
}

// A token that begins in a chunk and goes on beyond it: its parts in chunk order.
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256) embedding_join_kernel(const uint32_t* __restrict__ keys, const float* __restrict__ partial, int Kn, long long V,
                                                             int C, int chunks, int slices, float scale, int accumulate, O* __restrict__ out) {
  using Cols = EmCols<T, VEC>;
  constexpr int N = Cols::N, U = 8;
  const int lane = threadIdx.x & 63;
  const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= (long long)(chunks - 1) * slices) return;
  const int chunk = (int)(unit / slices), c0 = (int)(unit % slices) * Cols::SLICE + lane * N;
  const int i0 = chunk * kEmChunk, i1 = i0 + kEmChunk;       // (not the last chunk: it is full, and element i1 exists)
  const uint32_t key = keys[i1 - 1];
  if (key != keys[i1] || key >= (uint32_t)V) return;
  if (key == keys[i0] && i0 > 0 && keys[i0 - 1] == key) return;        // it began before this chunk
  int m = 1;                                               // chunks after this one that hold some of it
  for (;;) {
    // lane l: does the token go on from chunk + m + l into the next one?
    const long long next = (long long)(chunk + m + lane + 1) * kEmChunk;
    const unsigned long long stop = __ballot(!(next < Kn && keys[next] == key));
    if (stop) { m += __ffsll((long long)stop) - 1; break; }
    m += 64;
  }
  if (c0 >= C) return;
  const float* p = partial + (long long)chunk * 2 * C + c0;
  float s[N];
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = p[C + e];
  for (int q = 1; q <= m; q += U) {
    float x[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) x[u][e] = p[(long long)min(q + u, m) * 2 * C + e];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q + u <= m)
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] += x[u][e];
  }
  Cols::put(out + (long long)key * C + c0, s, scale, accumulate != 0);
}

EmbeddingPlan plan_embedding_backward(int64_t K, int64_t V, int32_t C, uint32_t flags) {
  EmbeddingPlan p = {};
  p.sorted = K > kEmScan;
  if (!p.sorted) return p;
  int need = 1;                                             // bits of the keys 0 .. V
  while (V >> need) ++need;
  p.one = K <= kEmOne || (K <= kEmOneFill && em_fill_bytes(V, C, flags) >= kEmFill);
  if (p.one) {
    p.nblocks = 1;
    p.passes = (int)ceil_div(need, 8);
  } else {
    p.per = align_up((size_t)ceil_div(K, kEmBlocks), 256);
    p.nblocks = (int)ceil_div(K, p.per);
    p.passes = (int)ceil_div(need, 11);
  }
  p.bits = (int)ceil_div(need, p.passes);
  p.chunks = (int)ceil_div(K, kEmChunk);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
  for (int i = 0; i < 2; ++i) { p.off_keys[i] = take(4 * K); p.off_rows[i] = take(4 * K); }
  p.off_hist = take(p.one ? 0 : (size_t)p.passes * p.nblocks * (4 << p.bits));
  p.off_partial = take((size_t)p.chunks * 2 * C * 4);
  p.bytes = at;
  return p;
}

template <typename T, typename K>
static void launch_em_fwd(const void* tokens, const void* table, int64_t M, int64_t V, int32_t C, float scale, void* E, hipStream_t s) {
  const bool vec = C % EmPiece<T>::N == 0 && ((uintptr_t)table | (uintptr_t)E) % 16 == 0;
  // a wavefront per row; fewer than 2048 rows are cut into slices of 64 pieces or more (3 rows of 3493 channels: one wavefront each takes 55 turns)
  const int64_t pieces = vec ? C / EmPiece<T>::N : C, cuts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(pieces, 64), 2048 / std::max<int64_t>(M, 1)));
  const int slice = (int)align_up((size_t)ceil_div(pieces, cuts), 64);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(M, 4), 1 << 20), (unsigned)ceil_div(pieces, slice));
  if (vec) SBP_LAUNCH(SBP_PROF_GATHER, s, (embedding_forward_kernel<T, K, true>), grid, dim3(256), 0, s, (const K*)tokens, (const T*)table, (long long)M, (long long)V, C, slice, scale, (T*)E);
  else SBP_LAUNCH(SBP_PROF_GATHER, s, (embedding_forward_kernel<T, K, false>), grid, dim3(256), 0, s, (const K*)tokens, (const T*)table, (long long)M, (long long)V, C, slice, scale, (T*)E);
}

int32_t launch_forward_embedding(const void* tokens, int32_t token_bytes, const void* table, int64_t M, int64_t V, int32_t C, float scale,
                                 int32_t dtype, void* E, hipStream_t s) {
  if (dtype == SBP_F32) { if (token_bytes == 4) launch_em_fwd<float, int32_t>(tokens, table, M, V, C, scale, E, s); else launch_em_fwd<float, int64_t>(tokens, table, M, V, C, scale, E, s); }
  else { if (token_bytes == 4) launch_em_fwd<uint16_t, int32_t>(tokens, table, M, V, C, scale, E, s); else launch_em_fwd<uint16_t, int64_t>(tokens, table, M, V, C, scale, E, s); }
  return check_launch("forward_embedding");
}

template <typename T, typename O, bool VEC>
static void launch_em_sums(const EmbeddingPlan& p, const T* dE, const uint32_t* keys, const int32_t* rows, int64_t Kn, int64_t V, int32_t C, float scale,
                           O* out, char* ws, int accumulate, hipStream_t s) {
  const int slices = (int)ceil_div(C, EmCols<T, VEC>::SLICE);
  const long long units = (long long)p.chunks * slices;
  float* partial = (float*)(ws + p.off_partial);
  SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_sum_kernel<T, O, VEC>), dim3((unsigned)ceil_div(units, 4)), dim3(256), 0, s, dE, keys, rows, (int)Kn, (long long)V, C,
             p.chunks, slices, scale, accumulate, partial, out);
  if (p.chunks > 1)
    SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_join_kernel<T, O, VEC>), dim3((unsigned)ceil_div((long long)(p.chunks - 1) * slices, 4)), dim3(256), 0, s,
               keys, partial, (int)Kn, (long long)V, C, p.chunks, slices, scale, accumulate, out);
}

template <typename T, typename K, typename O>
static void launch_em_bwd(const EmbeddingPlan& p, const void* dE, const void* tokens, const int32_t* idx, int64_t Kn, int64_t V, int32_t C, float scale,
                          void* out, void* ws_, uint32_t flags, hipStream_t s) {
  const bool vec = C % EmPiece<T>::N == 0 && ((uintptr_t)dE | (uintptr_t)out) % 16 == 0;
  const int compact = flags & SBP_FLAG_DY_COMPACT ? 1 : 0, accumulate = flags & SBP_FLAG_ACCUMULATE_DW ? 1 : 0;
  if (!p.sorted) {
    // table rows per workgroup: at most 2048 workgroups read the tokens; fewer than 1024 rows are cut into slices of 256 pieces or more
    const int rows = (int)std::max<int64_t>(1, ceil_div(V, 2048));
    const int64_t n = vec ? EmPiece<T>::N : 1, cuts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(C, 256 * n), 1024 / V));
    const int slice = (int)std::min<int64_t>(C, align_up((size_t)ceil_div(C, cuts), 256 * (size_t)n));
    const dim3 grid((unsigned)ceil_div(V, rows), (unsigned)ceil_div(C, slice));
    if (vec) SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_scan_kernel<T, K, O, true>), grid, dim3(256), 0, s, (const T*)dE, (const K*)tokens, idx, (int)Kn, (long long)V, C, rows, slice, scale, compact, accumulate, (O*)out);
    else SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_scan_kernel<T, K, O, false>), grid, dim3(256), 0, s, (const T*)dE, (const K*)tokens, idx, (int)Kn, (long long)V, C, rows, slice, scale, compact, accumulate, (O*)out);
    return;
  }
  char* ws = (char*)ws_;
  const long long fill = em_fill_bytes(V, C, flags);
  const uint32_t* keys;
  const int32_t* rows;
  if (p.one) {
    uint32_t* ko = (uint32_t*)(ws + p.off_keys[0]);
    int32_t* ro = (int32_t*)(ws + p.off_rows[0]);
    // (a filling workgroup has one piece of 16 bytes per thread at least, and the chip holds about two of these workgroups per CU)
    const unsigned fillers = (unsigned)std::min<long long>(ceil_div(fill, 16 * 1024), 511);
    auto go = [&](auto r) {
      constexpr int R = decltype(r)::value;
      const size_t lds = (size_t)(2 * R * 1024 + 16 * 256) * 4;
      allow_dynamic_lds(reinterpret_cast<const void*>(embedding_sort_kernel<K, O, R>), lds);
      SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_sort_kernel<K, O, R>), dim3(1 + fillers), dim3(1024), lds, s, (const K*)tokens, idx, compact, (int)Kn, (long long)V,
                 p.bits, p.passes, ko, ro, (char*)out, fill);
    };
    if (Kn <= 1024) go(std::integral_constant<int, 1>{});
    else if (Kn <= 4096) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, 16>{});
    keys = ko; rows = ro;
  } else {
    uint32_t* hist = (uint32_t*)(ws + p.off_hist);
    const unsigned fillers = (unsigned)std::min<long long>(ceil_div(fill, 16 * 256), 2048);
    SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_count_kernel<K, O>), dim3(p.nblocks + fillers), dim3(256), 0, s, (const K*)tokens, idx, (int)Kn, (long long)V, (int)p.per,
               p.nblocks, p.bits, p.passes, hist, (char*)out, fill);
    for (int q = 0; q < p.passes; ++q) {
      uint32_t *ki = (uint32_t*)(ws + p.off_keys[(q + 1) & 1]), *ko = (uint32_t*)(ws + p.off_keys[q & 1]);
      int32_t *ri = (int32_t*)(ws + p.off_rows[(q + 1) & 1]), *ro = (int32_t*)(ws + p.off_rows[q & 1]);
      if (q == 0) SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_move_kernel<K, true>), dim3(p.nblocks), dim3(256), 0, s, (const K*)tokens, idx, compact, ki, ri, (int)Kn, (long long)V, (int)p.per, p.bits, q, p.passes, hist, ko, ro);
      else SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_move_kernel<K, false>), dim3(p.nblocks), dim3(256), 0, s, (const K*)tokens, idx, compact, ki, ri, (int)Kn, (long long)V, (int)p.per, p.bits, q, p.passes, hist, ko, ro);
    }
    keys = (const uint32_t*)(ws + p.off_keys[(p.passes + 1) & 1]);
    rows = (const int32_t*)(ws + p.off_rows[(p.passes + 1) & 1]);
  }
  if (vec) launch_em_sums<T, O, true>(p, (const T*)dE, keys, rows, Kn, V, C, scale, (O*)out, ws, accumulate, s);
  else launch_em_sums<T, O, false>(p, (const T*)dE, keys, rows, Kn, V, C, scale, (O*)out, ws, accumulate, s);
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
