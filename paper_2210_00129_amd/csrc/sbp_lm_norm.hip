// The step between two blocks (sbp_lm.h): norm after a block, gate, residual sum, norm before the next block; and its backward
// on the kept rows.
// A team of TS threads owns a row and keeps it in registers (E channels per thread: 8 up to 8192 channels, 16 beyond; in the backward 16 from 4097 on
// but for single channels without the sums of shifts), so that every tensor is read once and
// written once; the row's sums go over the wavefront and, for teams of several wavefronts, through LDS with one barrier per round.
// Bound: HBM.  16384 x 4096, bf16, both norms: forward 106 us for 537 MB (5.1 TB/s, what a copy of 1 GiB reaches); backward with half of
// the rows kept 122 us, 7 of them the sums of the partial sums (537 MB, 4.6 TB/s without them).
#include <algorithm>
#include <type_traits>

#include "sbp_lm_internal.h"
#include "sbp_mfma_gemm.h"

namespace sbp {

template <typename T> struct LmPiece;                      // 16 bytes of a row
template <> struct LmPiece<float> { static constexpr int N = 4; };
template <> struct LmPiece<uint16_t> { static constexpr int N = 8; };

// The channels of a thread: pieces of 16 bytes (PIECES), piece i at channel (i * TS + t) * N, or single channels i * TS + t.  VEC: the rows are
// whole pieces at multiples of 16 bytes.  Pieces without VEC lie at any multiple of an element, and the last one of a row goes element by
// element; that takes fewer addresses and more comparisons than single channels, and pays only where the registers are short: the backward
// of more than 8192 channels (4096 x 12001, half of the rows kept, fp32 423 us, single channels 2878; bf16 277 and 439; but 16384 x 4095,
// bf16, 243 and 175).
template <typename T, int TS, int E, bool VEC, bool PIECES = VEC>
struct LmRow {
  static constexpr int N = PIECES ? LmPiece<T>::N : 1, P = E / N;
  static_assert(E % N == 0, "whole pieces");
  int t, C;
  __device__ __forceinline__ int channel(int i) const { return (i / N * TS + t) * N + i % N; }
  __device__ __forceinline__ bool valid(int i) const { return (VEC ? (i / N * TS + t) * N : channel(i)) < C; }   // (VEC: C is a multiple of N)
  using Piece = typename std::conditional<PIECES, uint4, T>::type;
  struct Raw { Piece p[P]; };                              // the thread's part of a row as it lies in memory (zeros past C)
  __device__ __forceinline__ void load(const T* row, Raw& w) const {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * TS + t) * N;
      if constexpr (VEC || !PIECES) {
        w.p[p] = c < C ? *reinterpret_cast<const Piece*>(row + c) : Piece{};
      } else {
        uint32_t v[4] = {0, 0, 0, 0};
        if (c + N <= C) {
          __builtin_memcpy(v, row + c, 16);
        } else if (c < C) {
#pragma unroll
          for (int e = 0; e < N - 1; ++e)
            if (c + e < C) {
              if constexpr (sizeof(T) == 4) v[e] = __float_as_uint(row[c + e]);
              else v[e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
            }
        }
        w.p[p] = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
  }
  static __device__ __forceinline__ void widen(const Raw& w, float (&v)[E]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if constexpr (!PIECES) {
        if constexpr (sizeof(T) == 4) v[p] = w.p[p];
        else v[p] = __uint_as_float((uint32_t)w.p[p] << 16);
      } else {
        const uint32_t x[4] = {w.p[p].x, w.p[p].y, w.p[p].z, w.p[p].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 4) v[4 * p + e] = __uint_as_float(x[e]);
          else { v[8 * p + 2 * e] = bf16_lo(x[e]); v[8 * p + 2 * e + 1] = bf16_hi(x[e]); }
        }
      }
    }
  }
  __device__ __forceinline__ void store(T* row, const float (&v)[E]) const {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * TS + t) * N;
      if (c >= C) continue;
      if constexpr (!PIECES) {
        if constexpr (sizeof(T) == 4) row[c] = v[p];
        else row[c] = (uint16_t)bf16_pack(v[p], v[p]);
      } else {
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 4) x[e] = __float_as_uint(v[4 * p + e]);
          else x[e] = bf16_pack(v[8 * p + 2 * e], v[8 * p + 2 * e + 1]);
        }
        if constexpr (VEC) {
          *reinterpret_cast<uint4*>(row + c) = make_uint4(x[0], x[1], x[2], x[3]);
        } else if (c + N <= C) {
          __builtin_memcpy(row + c, x, 16);
        } else {
#pragma unroll
          for (int e = 0; e < N - 1; ++e)
            if (c + e < C) {
              if constexpr (sizeof(T) == 4) row[c + e] = __uint_as_float(x[e]);
              else row[c + e] = (uint16_t)(x[e >> 1] >> (16 * (e & 1)));
            }
        }
      }
    }
  }
  __device__ __forceinline__ void param(const float* v, float def, float (&out)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) out[i] = v && valid(i) ? v[channel(i)] : def;
  }
};

// v + v of the lane that a row operation names
template <int CTRL>
__device__ __forceinline__ float lm_dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over the wavefront, the same bits in every lane: each step adds a value and its mirror image, so both sides round alike.  Neighbours
// by row operations, then 16 and 32 lanes apart by swaps of rows: 6 steps of a few cycles, where a shuffle through LDS takes some 100.
__device__ __forceinline__ float lm_sum64(float v) {
  v = lm_dpp_add<0xB1>(v);                                  // lane ^ 1
  v = lm_dpp_add<0x4E>(v);                                  // lane ^ 2
  v = lm_dpp_add<0x141>(v);                                 // mirrored within 8
  v = lm_dpp_add<0x140>(v);                                 // mirrored within 16
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  v = __int_as_float(a[0]) + __int_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(b[0]) + __int_as_float(b[1]);
}

// Sums of R values over the team, the same in every thread of it.  `slot` alternates between two LDS areas, so that one barrier
// per round is enough: a wavefront writes an area again only after the barrier of the round in between.
template <int TS, int R>
__device__ __forceinline__ void lm_team_sum(float (&v)[R], float* red, int& slot) {
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = lm_sum64(v[r]);
  if constexpr (TS > 64) {
    constexpr int W = TS / 64;
    float* at = red + slot * (4 * W);
    slot ^= 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
#pragma unroll
      for (int r = 0; r < R; ++r) at[r * W + wave] = v[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += at[r * W + w];
      v[r] = s;
    }
  }
}

struct LmNormFwd {
  const void *x, *y;
  void *x_out, *z;
  const float *gate, *gamma_post, *beta_post, *gamma_pre, *beta_pre;
  long long M, rows_per_gate;
  int C;
  float alpha, eps;
};

// v <- normalised v (zeros past C stay whatever they are: they are never stored nor summed)
template <typename T, int TS, int E, bool VEC, bool LAYER>
__device__ __forceinline__ void lm_normalise(const LmRow<T, TS, E, VEC>& io, float (&v)[E], float eps, float* red, int& slot) {
  float s[1] = {0.f};
  const float inv = 1.f / (float)io.C;
  if constexpr (LAYER) {
#pragma unroll
    for (int i = 0; i < E; ++i) s[0] += v[i];
    lm_team_sum<TS, 1>(s, red, slot);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = io.valid(i) ? v[i] - mean : 0.f;
  }
#pragma unroll
  for (int i = 0; i < E; ++i) s[0] = fmaf(v[i], v[i], s[0]);
  lm_team_sum<TS, 1>(s, red, slot);
  const float r = 1.f / sqrtf(s[0] * inv + eps);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] *= r;
}

// Workgroups: four teams of one wavefront, or one team.
template <int TS> struct LmTeams { static constexpr int N = TS == 64 ? 4 : 1, THREADS = TS == 64 ? 256 : TS; };

template <typename T, int TS, int E, bool VEC, bool LAYER>
__global__ void __launch_bounds__(LmTeams<TS>::THREADS) residual_norm_forward_kernel(LmNormFwd a) {
  constexpr int TEAMS = LmTeams<TS>::N;
  using Row = LmRow<T, TS, E, VEC>;
  __shared__ float red[TS > 64 ? 8 * (TS / 64) : 1];
  int slot = 0;
  const int team = TEAMS > 1 ? threadIdx.x / TS : 0;
  const Row io{TEAMS > 1 ? (int)threadIdx.x % TS : (int)threadIdx.x, a.C};
  long long r = (long long)blockIdx.x * TEAMS + team;
  const long long step = (long long)gridDim.x * TEAMS;
  typename Row::Raw rx, ry;                                // the next row, under way while this one is worked on
  if (r < a.M) {
    io.load((const T*)a.x + r * a.C, rx);
    if (a.y) io.load((const T*)a.y + r * a.C, ry);
  }
  float gp[E], bp[E], gn[E], bn[E], gate[E];
  io.param(a.gamma_post, 1.f, gp); io.param(a.beta_post, 0.f, bp);
  io.param(a.gamma_pre, 1.f, gn); io.param(a.beta_pre, 0.f, bn);
  io.param(nullptr, 1.f, gate);
  long long group = -1;
  // (teams of several wavefronts: the whole workgroup is one team, so every thread meets every barrier)
  for (; r < a.M; r += step) {
    float x[E], u[E];
    Row::widen(rx, x);
    if (a.y) Row::widen(ry, u);
    if (r + step < a.M) {
      io.load((const T*)a.x + (r + step) * a.C, rx);
      if (a.y) io.load((const T*)a.y + (r + step) * a.C, ry);
    }
    if (a.gate && r / a.rows_per_gate != group) {
      group = r / a.rows_per_gate;
      io.param(a.gate + group * a.C, 1.f, gate);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] *= a.alpha;
    if (a.y) {
      if (a.gamma_post) {
        lm_normalise<T, TS, E, VEC, LAYER>(io, u, a.eps, red, slot);
#pragma unroll
        for (int i = 0; i < E; ++i) u[i] = fmaf(u[i], gp[i], bp[i]);
      }
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = io.valid(i) ? fmaf(gate[i], u[i], x[i]) : 0.f;
    }
    if (a.x_out) io.store((T*)a.x_out + r * a.C, x);
    if (a.z) {
      lm_normalise<T, TS, E, VEC, LAYER>(io, x, a.eps, red, slot);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = fmaf(x[i], gn[i], bn[i]);
      io.store((T*)a.z + r * a.C, x);
    }
  }
}

struct LmNormBwd {
  const void *dx_out, *dz, *x_out, *y;
  void *dx, *dy;
  const int32_t *idx, *inv;
  const float *gate, *gamma_post, *gamma_pre;
  float* partial;                // [G][nblocks][2 or 4][C]: sums of dz xhat, t yhat and, with SHIFT, dz, t;  NULL: no parameter gradient wanted
  long long M, K, per_group;     // kept rows per group
  int C, nblocks, row_blocks, drop_blocks, compact;
  float alpha, eps;
};

// Blocks 0 .. row_blocks - 1 own kept rows (block b of group g: rows b, b + nblocks, ... of the group), the others the dropped
// rows of dx.  Per kept row, with the row's tensors in registers: the two sums each norm's backward needs come with the sums
// of its statistics, so a layer norm takes three rounds of sums for both norms, a root-mean-square norm two.  The gate is
// constant within a group, so the four sums over rows serve all five parameter gradients: with S1 = sum t yhat, S2 = sum t,
// dgate = gamma S1 + beta S2, dgamma = gate S1, dbeta = gate S2.
// SHIFT: the sums of dz and t are wanted as well (some beta's gradient, or dgate with a beta_post).
template <typename T, int TS, int E, bool VEC, bool LAYER, bool SHIFT>
__global__ void __launch_bounds__(LmTeams<TS>::THREADS) residual_norm_backward_kernel(LmNormBwd a) {
  constexpr int TEAMS = LmTeams<TS>::N, Q = SHIFT ? 4 : 2;
  using Row = LmRow<T, TS, E, VEC, VEC || (E == 16 && TS == 1024)>;
  __shared__ float red[TS > 64 ? 8 * (TS / 64) : 1];
  int slot = 0;
  const int team = TEAMS > 1 ? threadIdx.x / TS : 0;
  const Row io{TEAMS > 1 ? (int)threadIdx.x % TS : (int)threadIdx.x, a.C};
  const float inv_c = 1.f / (float)a.C;
  if ((int)blockIdx.x >= a.row_blocks) {
    // a run of rows per team: every wavefront looks up 64 of them at a time
    const long long teams = (long long)a.drop_blocks * TEAMS, me = (long long)(blockIdx.x - a.row_blocks) * TEAMS + team;
    const long long first = a.M * me / teams, end = a.M * (me + 1) / teams;
    for (long long r0 = first; r0 < end; r0 += 64) {
      const long long mine = r0 + (threadIdx.x & 63);
      bool dropped = false;
      if (mine < end) {
        const int j = a.inv[mine];
        dropped = !(j >= 0 && j < a.K && a.idx[j] == mine);
      }
      for (unsigned long long m = __ballot(dropped); m; m &= m - 1) {
        const long long r = r0 + __ffsll((long long)m) - 1;
        typename Row::Raw w = {};
        if (a.dx_out) io.load((const T*)a.dx_out + r * a.C, w);
        float v[E];
        Row::widen(w, v);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = a.dx_out ? v[i] * a.alpha : 0.f;
        io.store((T*)a.dx + r * a.C, v);
      }
    }
    return;
  }
  const int group = blockIdx.x / a.nblocks, blk = blockIdx.x % a.nblocks;
  const long long j_end = (group + 1) * a.per_group, step = (long long)a.nblocks * TEAMS;
  long long j = group * a.per_group + (long long)blk * TEAMS + team;
  float gn[E], gg[E];                                      // gamma_pre; gate * gamma_post
  io.param(a.gamma_pre, 0.f, gn);
  {
    float gp[E];
    io.param(a.gamma_post, 1.f, gp);
    io.param(a.gate ? a.gate + (long long)group * a.C : nullptr, 1.f, gg);
#pragma unroll
    for (int i = 0; i < E; ++i) gg[i] *= gp[i];
  }
  float acc[Q][E];                                         // sums of dz xhat, t yhat, dz, t
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int i = 0; i < E; ++i) acc[q][i] = 0.f;
  for (; j < j_end; j += step) {
    const long long r = a.compact || !a.idx ? j : a.idx[j];
    typename Row::Raw rt = {}, ry = {}, rz = {}, rx = {};
    if (a.y) io.load((const T*)a.y + j * a.C, ry);
    if (a.dz) {
      io.load((const T*)a.dz + j * a.C, rz);
      io.load((const T*)a.x_out + j * a.C, rx);
    }
    if (a.dx_out) io.load((const T*)a.dx_out + r * a.C, rt);
    float t[E], y[E], dz[E], x[E];
    Row::widen(ry, y);
    Row::widen(rz, dz);
    Row::widen(rx, x);
    float ry1 = 1.f;
    if constexpr (LAYER) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < E; ++i) { s[0] += x[i]; s[1] += y[i]; }
      lm_team_sum<TS, 2>(s, red, slot);
      const float mx = s[0] * inv_c, my = a.gamma_post ? s[1] * inv_c : 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = io.valid(i) ? x[i] - mx : 0.f;
        y[i] = io.valid(i) ? y[i] - my : 0.f;
      }
    }
    float s[LAYER ? 4 : 3];
#pragma unroll
    for (int q = 0; q < (LAYER ? 4 : 3); ++q) s[q] = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float g = dz[i] * gn[i];
      s[0] = fmaf(x[i], x[i], s[0]);
      s[1] = fmaf(y[i], y[i], s[1]);
      s[2] = fmaf(g, x[i], s[2]);
      if constexpr (LAYER) s[3] += g;
    }
    lm_team_sum<TS, (LAYER ? 4 : 3)>(s, red, slot);
    const float rx1 = 1.f / sqrtf(s[0] * inv_c + a.eps);
    if (a.gamma_post) ry1 = 1.f / sqrtf(s[1] * inv_c + a.eps);
    const float mgx = s[2] * inv_c * rx1;
    float mg = 0.f;
    if constexpr (LAYER) mg = s[3] * inv_c;
    Row::widen(rt, t);
    if (a.dz) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float hat = x[i] * rx1;
        acc[0][i] = fmaf(dz[i], hat, acc[0][i]);
        if constexpr (SHIFT) acc[2][i] += dz[i];
        t[i] = fmaf(rx1, dz[i] * gn[i] - mg - hat * mgx, t[i]);
      }
    }
    if (a.dx) {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = a.alpha * t[i];
      io.store((T*)a.dx + r * a.C, x);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      y[i] *= ry1;
      acc[1][i] = fmaf(t[i], y[i], acc[1][i]);
      if constexpr (SHIFT) acc[3][i] += t[i];
    }
    if (a.dy) {
      if (a.gamma_post) {
        float h[LAYER ? 2 : 1];
        h[0] = 0.f;
        if constexpr (LAYER) h[1] = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          t[i] = io.valid(i) ? t[i] * gg[i] : 0.f;
          h[0] = fmaf(t[i], y[i], h[0]);
          if constexpr (LAYER) h[1] += t[i];
        }
        lm_team_sum<TS, (LAYER ? 2 : 1)>(h, red, slot);
        const float mhy = h[0] * inv_c;
        float mh = 0.f;
        if constexpr (LAYER) mh = h[1] * inv_c;
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = ry1 * (t[i] - mh - y[i] * mhy);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] *= gg[i];
      }
      io.store((T*)a.dy + j * a.C, t);
    }
  }
  if (!a.partial) return;
  // teams of one workgroup join in order through LDS
  if constexpr (TEAMS > 1) {
    __shared__ float join[(TEAMS - 1) * TS * E];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (team)
#pragma unroll
        for (int i = 0; i < E; ++i) join[((team - 1) * E + i) * TS + io.t] = acc[q][i];
      __syncthreads();
      if (team == 0)
        for (int w = 0; w < TEAMS - 1; ++w)
#pragma unroll
          for (int i = 0; i < E; ++i) acc[q][i] += join[(w * E + i) * TS + io.t];
      __syncthreads();
    }
    if (team) return;
  }
  float* p = a.partial + (long long)blockIdx.x * Q * a.C;
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (io.valid(i)) p[(long long)q * a.C + io.channel(i)] = acc[q][i];
}

// Sums of the partial sums in order: 32 channels per workgroup, 32 slices of the blocks.  blockIdx.y = 0: the sums over all groups;
// blockIdx.y = 1 + g: dgate of group g.
template <int Q>
__global__ void __launch_bounds__(1024) residual_norm_reduce_kernel(const float* __restrict__ partial, int G, int nblocks, int C, const float* gate,
                                                                    const float* gamma_post, const float* beta_post, sbp_residual_norm_grads g,
                                                                    int accumulate) {
  __shared__ float join[32][Q][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, own = (int)blockIdx.y - 1;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < C) {
    const int b0 = own < 0 ? 0 : own * nblocks, b1 = own < 0 ? G * nblocks : b0 + nblocks;
#pragma unroll 4
    for (int b = b0 + slice; b < b1; b += 32) {
      const float* p = partial + (long long)b * Q * C + c;
      const float f = own < 0 && gate ? gate[(long long)(b / nblocks) * C + c] : 1.f;
      s[0] += p[0];
      s[1] = fmaf(f, p[C], s[1]);
      if constexpr (Q == 4) {
        s[2] += p[2LL * C];
        s[3] = fmaf(f, p[3LL * C], s[3]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < Q; ++q) join[slice][q][lane] = s[q];
  __syncthreads();
  if (slice || c >= C) return;
#pragma unroll 8
  for (int w = 1; w < 32; ++w)
#pragma unroll
    for (int q = 0; q < Q; ++q) s[q] += join[w][q][lane];
  auto put = [&](float* out, long long at, float v) { if (out) out[at] = accumulate ? out[at] + v : v; };
  if (own < 0) {
    put(g.dgamma_pre, c, s[0]);
    put(g.dgamma_post, c, s[1]);
    put(g.dbeta_pre, c, s[2]);
    put(g.dbeta_post, c, s[3]);
  } else {
    put(g.dgate, (long long)own * C + c, (gamma_post ? gamma_post[c] : 1.f) * s[1] + (beta_post ? beta_post[c] : 0.f) * s[3]);
  }
}

// ------------------------------------------------------------------------------------------------
// host side: the smallest team whose registers hold the row
// ------------------------------------------------------------------------------------------------
// Eight channels per thread leave the registers for many wavefronts: bf16, 16384 x 4096, forward 109 us with teams of 512, 126 us with
// 256 threads of 16 channels.
static int lm_team(int C) { return C <= 512 ? 64 : C <= 1024 ? 128 : C <= 2048 ? 256 : C <= 4096 ? 512 : C <= 8192 ? 1024 : 0; }
static int lm_rows_per_block(int team) { return team == 64 ? 4 : 1; }
static int lm_threads(int team) { return team == 64 ? 256 : team ? team : 1024; }

template <typename F>
static void lm_for_team(int team, const F& f) {
  switch (team) {
    case 64: f(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{}); break;
    case 128: f(std::integral_constant<int, 128>{}, std::integral_constant<int, 8>{}); break;
    case 256: f(std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{}); break;
    case 512: f(std::integral_constant<int, 512>{}, std::integral_constant<int, 8>{}); break;
    case 1024: f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{}); break;
    default: f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 16>{}); break;
  }
}
static bool lm_vec(int C, int32_t dtype, uintptr_t all) { return C % (dtype == SBP_F32 ? 4 : 8) == 0 && all % 16 == 0; }

template <typename T, bool LAYER>
static void launch_norm_fwd(const LmNormFwd& a, bool vec, hipStream_t s) {
  const int team = lm_team(a.C), rpb = lm_rows_per_block(team);
  const unsigned blocks = (unsigned)std::min<long long>(ceil_div(a.M, rpb), 2048);
  lm_for_team(team, [&](auto ts, auto e) {
    constexpr int TS = decltype(ts)::value, E = decltype(e)::value;
    const dim3 block(LmTeams<TS>::THREADS);
    if (vec) SBP_LAUNCH(SBP_PROF_OTHER, s, (residual_norm_forward_kernel<T, TS, E, true, LAYER>), dim3(blocks), block, 0, s, a);
    else SBP_LAUNCH(SBP_PROF_OTHER, s, (residual_norm_forward_kernel<T, TS, E, false, LAYER>), dim3(blocks), block, 0, s, a);
  });
}

int32_t launch_forward_residual_norm(const sbp_residual_norm_desc& d, const void* x, const void* y, int32_t dtype, void* x_out, void* z,
                                     hipStream_t s) {
  const LmNormFwd a{x, y, x_out, z, d.gate, d.gamma_post, d.beta_post, d.gamma_pre, d.beta_pre, d.M, d.M / d.G, d.C, d.alpha, d.eps};
  const bool vec = lm_vec(d.C, dtype, (uintptr_t)x | (uintptr_t)y | (uintptr_t)x_out | (uintptr_t)z), layer = d.kind == SBP_NORM_LAYER;
  if (dtype == SBP_F32) { if (layer) launch_norm_fwd<float, true>(a, vec, s); else launch_norm_fwd<float, false>(a, vec, s); }
  else { if (layer) launch_norm_fwd<uint16_t, true>(a, vec, s); else launch_norm_fwd<uint16_t, false>(a, vec, s); }
  return check_launch("forward_residual_norm");
}

ResidualNormPlan plan_residual_norm_backward(const sbp_residual_norm_desc& a, int64_t K, int32_t dtype, uint32_t flags) {
  ResidualNormPlan p;
  // no more workgroups than the chip holds at 16 wavefronts per CU: each writes partial sums
  const int team = lm_team(a.C);
  p.nblocks = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(K / a.G, lm_rows_per_block(team)), std::max<int64_t>(1, 262144 / lm_threads(team) / a.G)));
  p.off_partial = 0;
  p.off_inv = align_up((size_t)a.G * p.nblocks * 4 * a.C * sizeof(float), 256);
  p.bytes = p.off_inv + (flags & SBP_FLAG_DX_COMPACT ? 0 : align_up((size_t)a.M * sizeof(int32_t), 256));
  return p;
}

template <typename T, bool LAYER, bool SHIFT>
static void launch_norm_bwd(const LmNormBwd& a, bool vec, hipStream_t s) {
  const unsigned blocks = (unsigned)(a.row_blocks + a.drop_blocks);
  if (!blocks) return;
  auto go = [&](auto ts, auto e, auto v) {
    constexpr int TS = decltype(ts)::value, E = decltype(e)::value;
    SBP_LAUNCH(SBP_PROF_OTHER, s, (residual_norm_backward_kernel<T, TS, E, decltype(v)::value, LAYER, SHIFT>), dim3(blocks), dim3(LmTeams<TS>::THREADS), 0, s, a);
  };
  // 1024 threads have 128 registers each: rows of 4097 .. 8192 channels go to 512 threads of 16 channels where that saves enough of them (bf16,
  // 16384 x 8192: 247 -> 224 us; layer norms with betas, 8192 x 5120: 224 -> 109), not where single channels need many addresses besides
  // (16384 x 8191: 351, 388 so)
  lm_for_team(lm_team(a.C), [&](auto ts, auto e) {
    if constexpr (decltype(ts)::value == 1024 && decltype(e)::value == 8) {
      constexpr std::integral_constant<int, 512> half{};
      constexpr std::integral_constant<int, 16> twice{};
      if (vec) go(half, twice, std::true_type{});
      else if constexpr (SHIFT) go(half, twice, std::false_type{});
      else go(ts, e, std::false_type{});
    } else {
      if (vec) go(ts, e, std::true_type{});
      else go(ts, e, std::false_type{});
    }
  });
}

int32_t launch_backward_residual_norm(const ResidualNormPlan& p, const sbp_residual_norm_desc& d, const void* dx_out, const void* dz,
                                      const void* x_out, const void* y, const int32_t* idx, const int32_t* inv, int64_t K, int32_t dtype,
                                      void* dx, void* dy, const sbp_residual_norm_grads& g, void* ws, uint32_t flags, hipStream_t s) {
  const bool compact = flags & SBP_FLAG_DX_COMPACT, wants = g.dgate || g.dgamma_post || g.dbeta_post || g.dgamma_pre || g.dbeta_pre;
  const bool drop = dx && !compact && K < d.M && !(dx == dx_out && d.alpha == 1.f);
  const bool rows = (dx && K > 0) || (dy && K > 0) || wants;
  if (drop && !inv) {
    int32_t* own = (int32_t*)((char*)ws + p.off_inv);
    if (K > 0) launch_build_inverse(idx, K, own, s);
    inv = own;
  }
  LmNormBwd a = {};
  a.dx_out = dx_out; a.dz = K > 0 ? dz : nullptr; a.x_out = x_out; a.y = y; a.dx = dx; a.dy = dy; a.idx = idx; a.inv = inv;
  a.gate = d.gate; a.gamma_post = d.gamma_post; a.gamma_pre = d.gamma_pre;
  a.partial = wants ? (float*)((char*)ws + p.off_partial) : nullptr;
  a.M = d.M; a.K = K; a.per_group = K / d.G; a.C = d.C; a.nblocks = p.nblocks;
  a.row_blocks = rows ? d.G * p.nblocks : 0;
  const int team = lm_team(d.C);
  a.drop_blocks = drop ? (int)std::min<int64_t>(ceil_div(d.M, lm_rows_per_block(team)), 262144 / lm_threads(team)) : 0;
  a.compact = compact; a.alpha = d.alpha; a.eps = d.eps;
  const bool vec = lm_vec(d.C, dtype, (uintptr_t)dx_out | (uintptr_t)dz | (uintptr_t)x_out | (uintptr_t)y | (uintptr_t)dx | (uintptr_t)dy);
  const bool layer = d.kind == SBP_NORM_LAYER;
  const bool shift = g.dbeta_pre || g.dbeta_post || (g.dgate && d.beta_post);
  auto go = [&](auto t) {
    using T = decltype(t);
    if (layer) { if (shift) launch_norm_bwd<T, true, true>(a, vec, s); else launch_norm_bwd<T, true, false>(a, vec, s); }
    else { if (shift) launch_norm_bwd<T, false, true>(a, vec, s); else launch_norm_bwd<T, false, false>(a, vec, s); }
  };
  if (dtype == SBP_F32) go(float{}); else go(uint16_t{});
  if (wants) {
    const dim3 grid((unsigned)ceil_div(d.C, 32), (unsigned)(1 + (g.dgate ? d.G : 0)));
    const int accumulate = flags & SBP_FLAG_ACCUMULATE_DW ? 1 : 0;
    if (shift) SBP_LAUNCH(SBP_PROF_REDUCE, s, (residual_norm_reduce_kernel<4>), grid, dim3(1024), 0, s, a.partial, d.G, p.nblocks, d.C, d.gate, d.gamma_post, d.beta_post, g, accumulate);
    else SBP_LAUNCH(SBP_PROF_REDUCE, s, (residual_norm_reduce_kernel<2>), grid, dim3(1024), 0, s, a.partial, d.G, p.nblocks, d.C, d.gate, d.gamma_post, d.beta_post, g, accumulate);
  }
  return check_launch("backward_residual_norm");
}

}  // namespace sbp
