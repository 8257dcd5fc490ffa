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

// ------------------------------------------------------------------------------------------------
// Gradient.  dtable[v] = scale * sum of the kept rows of dE whose token is v.  The floor is the read of the kept rows and the write
// of the whole table (dense, as the weight gradients of the other layers are); the grouping moves 8 bytes per kept row.
//
// Up to kEmScan kept rows one launch does it all: every wavefront owns some table rows and looks for each of them through the
// kept tokens in LDS.  More rows are sorted by token (stable least-significant-digit radix sort of (token, row) pairs, 11 bits a
// pass), then a wavefront sums chunks of kEmChunk sorted rows in order, and tokens that cross a chunk's border are joined from
// partial sums in chunk order: every sum runs in the order of idx whatever the grid does.  Table rows without a token are zeroed
// beside the sums, by a bitmap of the tokens that occur.
// ------------------------------------------------------------------------------------------------
// One launch costs less than the sort's four or five, but a token that all rows share is then summed by one wavefront.
static constexpr int kEmScan = 256, kEmChunk = 32, kEmDigit = 11, kEmBins = 1 << kEmDigit, kEmBlocks = 64;

// A lane's columns of one row: a piece of 16 bytes of the input (VEC) or one column.
template <typename T, bool VEC>
struct EmCols {
  static constexpr int N = VEC ? EmPiece<T>::N : 1, SLICE = 64 * N;      // columns of a lane, of a wavefront
  static __device__ __forceinline__ void load(const T* p, float (&v)[N]) {
    if constexpr (VEC) EmPiece<T>::load(p, v);
    else v[0] = em_get(p);
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

template <typename T, typename K, typename O, bool VEC>
__global__ void __launch_bounds__(256) embedding_scan_kernel(const T* __restrict__ dE, const K* __restrict__ tokens, const int32_t* __restrict__ idx,
                                                             int Kn, long long V, int C, int rows_per_wave, float scale, int compact, int accumulate,
                                                             O* __restrict__ out) {
  using Cols = EmCols<T, VEC>;
  constexpr int N = Cols::N, U = 4;
  __shared__ int tok_s[kEmScan], row_s[kEmScan];
  const int t = threadIdx.x, lane = t & 63;
  if (t < Kn) {
    const long long tok = em_token(tokens, idx, t);
    tok_s[t] = tok >= 0 && tok < V ? (int)tok : -1;
    row_s[t] = compact || !idx ? t : idx[t];
  } else {
    tok_s[t] = -1;
  }
  __syncthreads();
  const long long v0 = ((long long)blockIdx.x * 4 + (t >> 6)) * rows_per_wave, v1 = min(v0 + rows_per_wave, V);
  int tk[kEmScan / 64];
#pragma unroll
  for (int q = 0; q < kEmScan / 64; ++q) tk[q] = tok_s[64 * q + lane];
  for (long long v = v0; v < v1; ++v) {
    unsigned long long hit[kEmScan / 64], any = 0;
#pragma unroll
    for (int q = 0; q < kEmScan / 64; ++q) { hit[q] = __ballot(tk[q] == (int)v); any |= hit[q]; }
    if (accumulate && !any) continue;
    for (int c0 = lane * N; c0 < C; c0 += Cols::SLICE) {
      float s[N];
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.f;
      for (int q = 0; any && q < kEmScan / 64; ++q) {
        unsigned long long w = hit[q];
        while (w) {                                        // U rows in flight, added in order
          float x[U][N];
          int n = 0;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (!w) break;
            Cols::load(dE + (long long)row_s[64 * q + __ffsll((long long)w) - 1] * C + c0, x[u]);
            w &= w - 1;
            n = u + 1;
          }
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (u < n)
#pragma unroll
              for (int e = 0; e < N; ++e) s[e] += x[u][e];
        }
      }
      Cols::put(out + v * C + c0, s, scale, accumulate != 0);
    }
  }
}

// ---- sort ----------------------------------------------------------------------------------------------------------
// Kept row j of block b = j / per.  hist[p][b][digit]: how many elements of block b (in the order before pass p) have the digit.
template <typename K>
__global__ void __launch_bounds__(256) embedding_count_kernel(const K* __restrict__ tokens, const int32_t* __restrict__ idx, int Kn, long long V,
                                                              int per, int passes, uint32_t* __restrict__ hist, uint32_t* __restrict__ present,
                                                              int words) {
  __shared__ uint32_t bins[kEmBins];
  const int t = threadIdx.x, nb = gridDim.x;
  for (int i = t; i < kEmBins; i += 256) bins[i] = 0;
  for (int p = 1; p < passes; ++p)
    for (int i = t; i < kEmBins; i += 256) hist[((long long)p * nb + blockIdx.x) * kEmBins + i] = 0;
  for (int i = blockIdx.x * 256 + t; i < words; i += nb * 256) present[i] = 0;
  __syncthreads();
  const long long j0 = (long long)blockIdx.x * per, j1 = min(j0 + per, (long long)Kn);
  for (long long j = j0 + t; j < j1; j += 256) {
    const long long tok = em_token(tokens, idx, j);
    atomicAdd(&bins[(tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V) & (kEmBins - 1)], 1u);
  }
  __syncthreads();
  for (int i = t; i < kEmBins; i += 256) hist[(long long)blockIdx.x * kEmBins + i] = bins[i];
}

// One pass: a block of four wavefronts moves its run of elements, every wavefront a quarter in order.  FIRST: the elements come from
// the tokens, and the bitmap of those that occur is made; later passes read the pairs of the pass before.
template <typename K, bool FIRST>
__global__ void __launch_bounds__(256) embedding_move_kernel(const K* __restrict__ tokens, const int32_t* __restrict__ idx, int compact,
                                                             const uint32_t* __restrict__ keys, const int32_t* __restrict__ rows, int Kn, long long V,
                                                             int per, int pass, int passes, uint32_t* __restrict__ hist,
                                                             uint32_t* __restrict__ present, uint32_t* __restrict__ keys_out,
                                                             int32_t* __restrict__ rows_out) {
  __shared__ uint32_t place[4][kEmBins];
  __shared__ uint32_t wave_total[4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, nb = gridDim.x, shift = pass * kEmDigit;
  const long long first = (long long)blockIdx.x * per + (long long)wave * (per / 4);
  const long long last = min(min(first + per / 4, (long long)(blockIdx.x + 1) * per), (long long)Kn);
  for (int i = t; i < 4 * kEmBins; i += 256) (&place[0][0])[i] = 0;
  __syncthreads();
  auto key_at = [&](long long j) -> uint32_t {
    if constexpr (!FIRST) return keys[j];
    const long long tok = em_token(tokens, idx, j);
    return tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V;
  };
  for (long long j = first + lane; j < last; j += 64) atomicAdd(&place[wave][key_at(j) >> shift & (kEmBins - 1)], 1u);
  // where the block's elements of each digit go: digits below it, then the blocks before this one
  constexpr int PT = kEmBins / 256;
  const uint32_t* h = hist + (long long)pass * nb * kEmBins + t * PT;
  uint32_t total[PT], before[PT], sum = 0;
#pragma unroll
  for (int e = 0; e < PT; ++e) total[e] = before[e] = 0;
  for (int b = 0; b < nb; ++b) {
    uint32_t x[PT];
#pragma unroll
    for (int e = 0; e < PT; ++e) x[e] = h[(long long)b * kEmBins + e];
#pragma unroll
    for (int e = 0; e < PT; ++e) { before[e] += b < (int)blockIdx.x ? x[e] : 0; total[e] += x[e]; }
  }
#pragma unroll
  for (int e = 0; e < PT; ++e) sum += total[e];
  uint32_t scan = sum;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t o = __shfl_up(scan, m);
    scan += lane >= m ? o : 0;
  }
  if (lane == 63) wave_total[wave] = scan;
  __syncthreads();
  uint32_t at = scan - sum;
  for (int w = 0; w < wave; ++w) at += wave_total[w];
#pragma unroll
  for (int e = 0; e < PT; ++e) {
    uint32_t p = at + before[e];
    at += total[e];
    for (int w = 0; w < 4; ++w) {
      const uint32_t n = place[w][t * PT + e];
      place[w][t * PT + e] = p;
      p += n;
    }
  }
  __syncthreads();
  volatile uint32_t* mine = place[wave];
  for (long long j0 = first; j0 < last; j0 += 64) {          // (the same count for every lane)
    const long long j = j0 + lane;
    const bool on = j < last;
    const uint32_t key = on ? key_at(j) : 0, digit = key >> shift & (kEmBins - 1);
    const int32_t row = !on ? 0 : FIRST ? (compact || !idx ? (int32_t)j : idx[j]) : rows[j];
    unsigned long long same = __ballot(on);
#pragma unroll
    for (int bit = 0; bit < kEmDigit; ++bit) {
      const unsigned long long ones = __ballot(digit >> bit & 1);
      same &= digit >> bit & 1 ? ones : ~ones;
    }
    const uint32_t rank = __popcll(same & ((1ull << lane) - 1)), count = __popcll(same);
    uint32_t dest = 0;
    if (on) dest = mine[digit] + rank;
    if (on && rank == count - 1) mine[digit] = dest + 1;     // (a wavefront's LDS accesses complete in order)
    if (on) {
      keys_out[dest] = key;
      rows_out[dest] = row;
      if (FIRST && key < (uint32_t)V) atomicOr(&present[key >> 5], 1u << (key & 31));
      if (pass + 1 < passes) atomicAdd(&hist[((long long)(pass + 1) * nb + dest / per) * kEmBins + (key >> (shift + kEmDigit) & (kEmBins - 1))], 1u);
    }
  }
}

// ---- sums ----------------------------------------------------------------------------------------------------------
// Wavefronts: first (chunk, column slice) units, then runs of kEmFill table rows to be zeroed where no token occurs.  A token that lies
// in the chunk altogether is finished here; one that began before it leaves its part in partial[chunk][0], one that begins here
// and goes on in partial[chunk][1].
static constexpr int kEmFill = 8;

template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256) embedding_sum_kernel(const T* __restrict__ dE, const uint32_t* __restrict__ keys, const int32_t* __restrict__ rows,
                                                            const uint32_t* __restrict__ present, int Kn, long long V, int C, int chunks, int slices,
                                                            long long fills, float scale, int accumulate, float* __restrict__ partial,
                                                            O* __restrict__ out) {
  using Cols = EmCols<T, VEC>;
  constexpr int N = Cols::N, U = 8;
  const int lane = threadIdx.x & 63;
  long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= (long long)chunks * slices) {
    unit -= (long long)chunks * slices;
    if (unit >= fills) return;
    const float zero[N] = {};
    for (long long v = unit * kEmFill; v < min((unit + 1) * kEmFill, V); ++v) {
      if (present[v >> 5] >> (v & 31) & 1) continue;
      for (int c = lane * N; c < C; c += Cols::SLICE) Cols::put(out + v * C + c, zero, 1.f, false);
    }
    return;
  }
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
    float x[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {                            // (past the chunk's end its last row again, unused)
      const long long r = __builtin_amdgcn_readlane(row, min(i + u, n - 1) + 1);
      Cols::load(src + r * C, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= n) break;
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] += x[u][e];
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

EmbeddingPlan plan_embedding_backward(int64_t K, int64_t V, int32_t C, int32_t) {
  EmbeddingPlan p = {};
  p.sorted = K > kEmScan;
  if (!p.sorted) return p;
  p.nblocks = (int)std::min<int64_t>(kEmBlocks, ceil_div(K, 2048));
  p.per = align_up((size_t)ceil_div(K, p.nblocks), 256);
  p.nblocks = (int)ceil_div(K, p.per);
  for (p.passes = 1; (V >> (p.passes * kEmDigit)) != 0; ++p.passes) {}
  p.chunks = (int)ceil_div(K, kEmChunk);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
  for (int i = 0; i < 2; ++i) { p.off_keys[i] = take(4 * K); p.off_rows[i] = take(4 * K); }
  p.off_hist = take((size_t)p.passes * p.nblocks * kEmBins * 4);
  p.off_present = take((size_t)ceil_div(V, 32) * 4);
  p.off_partial = take((size_t)p.chunks * 2 * C * 4);
  p.bytes = at;
  return p;
}

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

template <typename T, typename O, bool VEC>
static void launch_em_sums(const EmbeddingPlan& p, const T* dE, const uint32_t* keys, const int32_t* rows, int64_t Kn, int64_t V, int32_t C, float scale,
                           O* out, char* ws, int accumulate, hipStream_t s) {
  const int slices = (int)ceil_div(C, EmCols<T, VEC>::SLICE);
  const long long fills = accumulate ? 0 : ceil_div(V, kEmFill), units = (long long)p.chunks * slices;
  float* partial = (float*)(ws + p.off_partial);
  SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_sum_kernel<T, O, VEC>), dim3((unsigned)ceil_div(units + fills, 4)), dim3(256), 0, s, dE, keys, rows,
             (const uint32_t*)(ws + p.off_present), (int)Kn, (long long)V, C, p.chunks, slices, fills, scale, accumulate, partial, out);
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
    const int rpw = (int)std::max<int64_t>(1, ceil_div(V, 4 * 2048));      // table rows per wavefront: at most 2048 workgroups read the tokens
    const dim3 grid((unsigned)ceil_div(V, 4 * rpw));
    if (vec) SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_scan_kernel<T, K, O, true>), grid, dim3(256), 0, s, (const T*)dE, (const K*)tokens, idx, (int)Kn, (long long)V, C, rpw, scale, compact, accumulate, (O*)out);
    else SBP_LAUNCH(SBP_PROF_REDUCE, s, (embedding_scan_kernel<T, K, O, false>), grid, dim3(256), 0, s, (const T*)dE, (const K*)tokens, idx, (int)Kn, (long long)V, C, rpw, scale, compact, accumulate, (O*)out);
    return;
  }
  char* ws = (char*)ws_;
  uint32_t *hist = (uint32_t*)(ws + p.off_hist), *present = (uint32_t*)(ws + p.off_present);
  SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_count_kernel<K>), dim3(p.nblocks), dim3(256), 0, s, (const K*)tokens, idx, (int)Kn, (long long)V, (int)p.per, p.passes,
             hist, present, (int)ceil_div(V, 32));
  for (int q = 0; q < p.passes; ++q) {
    uint32_t *ki = (uint32_t*)(ws + p.off_keys[(q + 1) & 1]), *ko = (uint32_t*)(ws + p.off_keys[q & 1]);
    int32_t *ri = (int32_t*)(ws + p.off_rows[(q + 1) & 1]), *ro = (int32_t*)(ws + p.off_rows[q & 1]);
    if (q == 0) SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_move_kernel<K, true>), dim3(p.nblocks), dim3(256), 0, s, (const K*)tokens, idx, compact, ki, ri, (int)Kn, (long long)V, (int)p.per, q, p.passes, hist, present, ko, ro);
    else SBP_LAUNCH(SBP_PROF_OTHER, s, (embedding_move_kernel<K, false>), dim3(p.nblocks), dim3(256), 0, s, (const K*)tokens, idx, compact, ki, ri, (int)Kn, (long long)V, (int)p.per, q, p.passes, hist, present, ko, ro);
  }
  const uint32_t* keys = (const uint32_t*)(ws + p.off_keys[(p.passes + 1) & 1]);
  const int32_t* rows = (const int32_t*)(ws + p.off_rows[(p.passes + 1) & 1]);
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
