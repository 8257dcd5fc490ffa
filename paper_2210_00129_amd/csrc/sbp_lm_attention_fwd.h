// Forward of the masked attention on the bf16 matrix cores.
//
// A workgroup of NW wavefronts owns 32 NW queries of one (sample, query head), every wavefront 32 of them, with the q fragments, the
// output accumulators and the softmax statistics in registers; the rows of k and v stream through LDS in tiles of 64, one pass.
//   S^T = K Q^T: rows j, column i = lane (v_mfma_f32_32x32x16_bf16, layouts at sbp_attention.hip).  A query's scores of a block of 32
//   keys are 16 registers in each of lanes i and i + 32, so its maximum and sum need one exchange between the halves, and P^T is,
//   packed to bf16, the B operand of O^T += V^T P^T as it is; V^T comes out of LDS with transposing reads.
// P is rounded to bf16 (2^-8 of the weight) because the matrix cores multiply bf16; its sum l is taken before the rounding.  Where no maximum is
// taken out (LM_CAP_FIXED), A is divided by the sum of the rounded weights instead: a row's largest weight is then not 1, and what its rounding
// does to sum and products alike cancels (one key: A = v as it is; error against 64 bits, documents of 9 tokens on average 0.0021 -> 0.0017,
// 500 tokens 0.0023 -> 0.0021; the long text 308 -> 314 us, 4 x 12 heads of 64 sharing 4, 2048 tokens 55 -> 56).
// The running maximum moves only when a block's maximum is more than kLmSlack above it (weights up to 2^kLmSlack instead of 1: no loss
// in a floating format), so that the accumulators are rescaled rarely.
// A stage of the loop has a product part M(t) = {O += V(t-1) P(t-1); S(t) = K(t) Q} and an arithmetic part A(t) = softmax of S(t), in
// LDS K(t) and V(t-1).  With 8 wavefronts there are two on every SIMD, and left to themselves they do their products at the same time
// and then their arithmetic at the same time (matrix cores busy 31 %, vector arithmetic 60 % of the cycles, next to no overlap).
// So wavefronts 4 .. 7 run half a stage behind the others, held there by a second barrier per stage: one half's products run under
// the other half's arithmetic.
// Tiles that no query of the workgroup can see are never copied: with documents, a list of the others is made from the documents'
// ranges per tile; without, they are a run of tiles.  A wavefront works from the first to the last of them that it sees itself, and
// masks element by element only where a tile is not visible altogether.
// A value that is not finite in a row of v whose weight is 0 turns into NaN in the product.  Where the result of a query is not
// finite, its row is computed again without the keys it does not see (sbp_lm_attention_rows.h).
// Bound, d = 128: the products of one half against the vector arithmetic of the other, at the clock that the card keeps under them (counted over the
// busy cycles of a CU, capped: matrix cores 40 %, vector units 64 %, LDS 31 %, 1.9 GHz; uncapped 50, 45, 39 %, 1.95 GHz); 16 heads sharing
// 2, 8192 tokens, causal, capped: 300 .. 325 us (275 GFLOP counted, 0.85 .. 0.92 PFLOP/s; up to 355 at lower clocks), uncapped 267 (1.03).
// d = 64: vector arithmetic, and for short documents the chain of a workgroup's few tiles (1.25 us each with one workgroup on a CU, some 8 us
// before and after them) and their unequal number (a CU is busy half of the time on average); 4 x 12 heads of 64, 2048 tokens in documents of
// 500 on average, biased: 33 .. 37 us; without documents and bias 44 us (0.59 PFLOP/s), 16 samples of it 144 (0.72).
#ifndef SBP_LM_ATTENTION_FWD_H_
#define SBP_LM_ATTENTION_FWD_H_

#include "sbp_lm_attention_tiles.h"

namespace sbp {

// Score arithmetic: plain (scale > 0), with the distance bias (any scale), capped with |score| <= cap <= 60 and no bias (weights
// exp(score) themselves: no maximum is needed, exp(-60) .. exp(60) and their sums stay within fp32), capped otherwise; short samples, capped in any
// way: with tanh right to a step of fp32 of the value, where the others' is right to some 2^-22 of the cap.  That error averages out in the lse of
// many keys, not of few (samples of 1 .. 26 tokens, cap 50: lse off by 1 .. 3e-6 of its size, so below 1e-7).  It takes a fifth more time where many
// such samples fill the card (400 samples of 32 tokens, 8 heads of 64: 25 -> 30 us), 0.3 us for one.
enum LmMode { LM_PLAIN = 0, LM_BIAS = 1, LM_CAP_FIXED = 2, LM_CAP = 3, LM_CAP_SHORT = 4 };
static constexpr int kLmShort = 32;                        // tokens: one block of keys
// (Fixed, cap 50: the long text 310 us, with the running maximum 368.  Products of a weight and a value below 2^-126 are lost, so
// a row whose weights sum to less than kLmFixedSum, all scores below -41, is computed again with its maximum, and no other loses more than 2^-66 of A.)
static constexpr float kLmSlack = 6.f, kLmFixedCap = 60.f, kLmFixedSum = 0x1p-60f;
static constexpr uint32_t kLmOnes = 0x3f803f80u;           // two ones
static constexpr int kLmAhead = 6;                         // (the long text uncapped 267 us; 2: 269)
static constexpr int kLmList = 128;                        // tiles per list (8192 tokens); longer samples take several

// max(a, b, c); of the numbers where some are NaN.  (fmaxf() first makes every operand that the compiler does not know to be a quiet
// one quiet, which doubles the steps.)  The operands must not be results of a matrix instruction under way.
__device__ __forceinline__ float lm_max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

template <int D, int NW>
struct LmFwd {
  using L = AttnSwizzled<D>;
  using S = LmStream<D, NW>;
  static constexpr int STAGE = 2 * S::IMG, DOCS = 2 * STAGE;      // two stages of a k and a v tile; documents of the tokens of four k tiles
  static constexpr int OUT = NW * 32 * (2 * D + 16);        // the output images
  static constexpr size_t LDS = DOCS + 4 * 4 * kLmTile > OUT ? DOCS + 4 * 4 * kLmTile : OUT;
};

// (workgroups per CU of 4 wavefronts: what the loops leave room for; without the bias d <= 32 for four)
template <int D, int NW, int MODE>
__global__ void __launch_bounds__(64 * NW, D == 128 ? 2 : D < 64 && (MODE == LM_PLAIN || MODE == LM_CAP_FIXED) ? 4 : 3) masked_forward_kernel(MaskedAttention a, int nchunks) {
  using L = AttnSwizzled<D>;
  using F = LmFwd<D, NW>;
  constexpr int KS = L::KS, DB = L::DB;
  constexpr bool PAIR = NW == 8, CAP = MODE == LM_CAP || MODE == LM_CAP_FIXED || MODE == LM_CAP_SHORT,
                 BIAS = MODE == LM_CAP || MODE == LM_CAP_SHORT || MODE == LM_BIAS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int4 list_s[kLmList];                           // a tile to look at, the documents in it
  __shared__ int range_s[2 * NW + 1];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), u = lane >> 5;
  int rank, bh;
  lm_unit(blockIdx.x, a.B * a.h, &rank, &bh);
  const int chunk = a.causal ? nchunks - 1 - rank : rank;   // causal: the last queries see the most
  const int b = bh / a.h, head = bh - b * a.h, kv = head / (a.h / a.hk), n = a.n;
  const int ld = (a.h + 2 * a.hk) * D;
  const uint16_t* base = (const uint16_t*)a.qkv + (long long)b * n * ld;
  const uint16_t *k0 = base + (a.h + kv) * D, *v0 = k0 + a.hk * D;
  const int first = chunk * 32 * NW + wave * 32, mine = first + (lane & 31), own = min(mine, n - 1);
  const bool busy = first < n;
  const bool docs = a.doc != nullptr;
  const int prefix = lm_prefix(a, b);
  const int32_t* doc = docs ? a.doc + (long long)b * n : nullptr;
  const int di = docs ? doc[own] : 0;
  int dv[4] = {0, 0, 0, 0};                                 // documents of four tokens of tile t / 16, for the first list
  if (docs)
#pragma unroll
    for (int e = 0; e < 4; ++e) dv[e] = doc[min((t >> 4) * kLmTile + (t & 15) * 4 + e, n - 1)];
  const L lay(lane);
  const uint32_t lds0 = lm_lds(smem);
  const typename F::S st(ld, lane, wave);
  bf16x8_t qf[KS];
  {
    const uint16_t* q = base + (long long)own * ld + head * D + 8 * u;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(q + 16 * ks);
  }
  LmRange wq;                                               // of the wavefront's queries
  wq.p0 = first; wq.p1 = min(first + 31, n - 1); wq.d0 = wq.d1 = 0;
  if (docs) {
    LmDocs r;
    r.add(di);
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) r.join(m);
    r.close();
    wq.d0 = __builtin_amdgcn_readfirstlane(r.lo);
    wq.d1 = __builtin_amdgcn_readfirstlane(r.hi);
  }
  const bool strays = __ballot(di < 0) != 0;                // queries of no document
  LmRange gq;                                               // ... of the workgroup's
  gq.p0 = chunk * 32 * NW; gq.p1 = min(gq.p0 + 32 * NW - 1, n - 1); gq.d0 = gq.d1 = 0;
  if (docs) {
    if (lane == 0) { range_s[wave] = wq.d0; range_s[NW + wave] = wq.d1; }
    __syncthreads();
    gq.d0 = range_s[0]; gq.d1 = range_s[NW];
#pragma unroll
    for (int w = 1; w < NW; ++w) { gq.d0 = min(gq.d0, range_s[w]); gq.d1 = max(gq.d1, range_s[NW + w]); }
  }
  const float slope2 = BIAS && a.slopes ? a.slopes[head] * kLog2e : 0.f;
  float c2 = a.scale * kLog2e;
  if constexpr (BIAS) asm("" : "+v"(c2));                    // (a fused product reads one scalar register: the bias)
  const float cap2 = a.cap * kLog2e;
  float ct = 2.f * kLog2e * a.per_cap;
  if constexpr (CAP) asm("" : "+v"(ct));
  float ahead[BIAS ? 16 : 1];                                // bias of a block's keys relative to the lane's first one (wave-uniform: scalar registers)
  if constexpr (BIAS)
#pragma unroll
    for (int e = 0; e < 16; ++e) ahead[e] = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(slope2 * (float)(8 * (e >> 2) + (e & 3)))));
  const bool forward_only = a.causal && prefix == 0;         // no visible key stands behind its query

  f32x16_t o[DB];
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[x][e] = 0.f;
  float m2 = MODE == LM_CAP_FIXED ? 0.f : -INFINITY, l = 0.f;      // the maximum in units of log2, the half's share of the sum
  float lr[4] = {0.f, 0.f, 0.f, 0.f};                       // LM_CAP_FIXED: the same of the rounded weights (four sums: one waits for itself)

  f32x16_t sc[2];                                            // scores of the tile's two blocks of 32 keys
  bf16x8_t pw[2][2];                                         // their weights
  // M(t): the products of a stage, P V of one tile and K Q of the next (either may be left out), with every operand read kLmAhead
  // products before it is multiplied (the compiler by itself reads it right before, or two products ahead: a product takes 32 cycles, a
  // read under way some 150).
  auto multiply = [&](auto pv_, auto kq_, const char* tv, const char* tk) {
    constexpr int NP = decltype(pv_)::value ? 4 * DB : 0, N = NP + (decltype(kq_)::value ? 2 * KS : 0), AHEAD = kLmAhead < N ? kLmAhead : N;
    const f32x16_t zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto operand = [&](int i) { return i < NP ? lay.tr(tv, 16 * (i / DB), i % DB) : lay.row(tk, 32 * ((i - NP) & 1), (i - NP) >> 1); };
    bf16x8_t f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = operand(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i < NP) {
        const int g = i / DB, x = i % DB;
        o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], pw[g >> 1][g & 1], o[x], 0, 0, 0);
      } else {
        const int y = (i - NP) & 1, ks = (i - NP) >> 1;
        sc[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], qf[ks], ks ? sc[y] : zero, 0, 0, 0);
      }
      if (i + AHEAD < N) f[i % AHEAD] = operand(i + AHEAD);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  // Scores of a tile into weights; r: its positions and documents, td: the documents of its keys.
  // Bias: where no visible key stands behind its query, slope |pos_i - pos_j| is linear, and what the lane's keys have in common of it
  // joins the maximum's subtraction.
  auto weigh = [&](const LmRange& r, const int* td) {
    const int p = r.p0, rel = mine - p - 4 * u;              // rel: distance to the lane's key of register 0
    float common[2] = {0.f, 0.f};
    if constexpr (MODE != LM_PLAIN) {
      const float relf = (float)rel;
      const bool linear = BIAS && (forward_only || r.p1 <= wq.p0);
      if (linear) {
        common[0] = -slope2 * relf;
        common[1] = -slope2 * (relf - 32.f);
      }
      if constexpr (MODE == LM_CAP_SHORT) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          sc[0][e] = cap2 * lm_tanh(sc[0][e] * a.per_cap);
          sc[1][e] = -INFINITY;                              // (one tile, whose second block is past the end)
        }
      } else if constexpr (CAP) {
        // cap tanh(z / cap) by one exponential and a reciprocal (a polynomial for small arguments has more steps than these: 19 % more time
        // for the long text)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[y][e] = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(sc[y][e] * ct) + 1.f), cap2);
      }
      if constexpr (BIAS) {
        if (linear) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if constexpr (CAP) sc[y][e] += ahead[e];
              else sc[y][e] = fmaf(sc[y][e], c2, ahead[e]);
            }
        } else {
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float v = CAP ? sc[y][e] : sc[y][e] * c2;
              sc[y][e] = fmaf(-slope2, fabsf(relf - (float)(32 * y + 8 * (e >> 2) + (e & 3))), v);
            }
        }
      }
    }
    // element by element only what the ranges leave open
    if (r.p1 >= n || strays || (a.causal && r.p1 > wq.p0 && r.p1 >= prefix)) {
      // the lane's keys of registers with row < lim are seen: up to the query's own position or the end of the prefix, and of the sample
      int lim = n - p - 4 * u;
      if (a.causal) lim = min(lim, max(rel + 1, prefix - p - 4 * u));
      if (di < 0) lim = 0;
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[y][e] = 32 * y + 8 * (e >> 2) + (e & 3) < lim ? sc[y][e] : -INFINITY;
    }
    if (docs && !(r.d0 == r.d1 && wq.d0 == wq.d1 && r.d0 == wq.d0)) {
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int4 dj = *reinterpret_cast<const int4*>(td + 32 * y + 4 * u + 8 * q4);
          const int dk[4] = {dj.x, dj.y, dj.z, dj.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[y][4 * q4 + e] = dk[e] == di ? sc[y][4 * q4 + e] : -INFINITY;
        }
    }
    if constexpr (MODE != LM_CAP_FIXED) {
      // (plain scores come from the matrix cores as they are: 24 cycles let the last product finish)
      if constexpr (MODE == LM_PLAIN) asm volatile("s_nop 15\n\ts_nop 7" : "+v"(sc[0]), "+v"(sc[1]));
      float top[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        top[y] = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; e += 2) top[y] = lm_max3(top[y], sc[y][e], sc[y][e + 1]);
        if constexpr (BIAS) top[y] += common[y];
      }
      float mx = fmaxf(top[0], top[1]);
      if constexpr (MODE == LM_PLAIN) mx *= c2;
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (__ballot(mx > m2 + kLmSlack)) {
        const float mn = mx > m2 + kLmSlack ? mx : m2, f = mn > m2 ? __builtin_amdgcn_exp2f(m2 - mn) : 1.f;
        m2 = mn;
        l *= f;
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[x][e] *= f;
      }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const float ms = (m2 == -INFINITY ? 0.f : m2) - (BIAS ? common[y] : 0.f);      // (nothing seen so far: every weight is 0)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if constexpr (MODE == LM_PLAIN) sc[y][e] = __builtin_amdgcn_exp2f(fmaf(sc[y][e], c2, -ms));
        else if constexpr (MODE == LM_CAP_FIXED) sc[y][e] = __builtin_amdgcn_exp2f(sc[y][e]);
        else sc[y][e] = __builtin_amdgcn_exp2f(sc[y][e] - ms);
        l += sc[y][e];
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        pw[y][ks] = pack8(sc[y], ks);
        if constexpr (MODE == LM_CAP_FIXED) {
          const uint4 w = __builtin_bit_cast(uint4, pw[y][ks]);
          lr[0] = attn_dot2(w.x, kLmOnes, lr[0]);
          lr[1] = attn_dot2(w.y, kLmOnes, lr[1]);
          lr[2] = attn_dot2(w.z, kLmOnes, lr[2]);
          lr[3] = attn_dot2(w.w, kLmOnes, lr[3]);
        }
      }
    }
  };

  const int ntiles = (n + kLmTile - 1) / kLmTile;
  const int reach = a.causal ? min(ntiles, max(gq.p1 / kLmTile + 1, (min(prefix, n) + kLmTile - 1) / kLmTile)) : ntiles;
  for (int base_tile = 0; base_tile < reach; base_tile += kLmList) {
    const int here = min(kLmList, reach - base_tile);
    int ns = here;
    if (docs) {
      // document ranges of the tiles, four lanes to a tile, and the list of those to look at
      __syncthreads();
      for (int i0 = 0; i0 < here; i0 += 4 * NW) {            // 16 lanes to a tile, 4 tokens to a lane
        const int i = i0 + (t >> 4), at = (base_tile + i) * kLmTile + (t & 15) * 4;
        LmDocs r;
        if (i < here) {
          if (base_tile + i0)
#pragma unroll
            for (int e = 0; e < 4; ++e) dv[e] = doc[min(at + e, n - 1)];
#pragma unroll
          for (int e = 0; e < 4; ++e) r.add(dv[e]);
        }
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) r.join(m);
        r.close();
        if (i < here && (t & 15) == 0) list_s[i] = make_int4(i, r.lo, r.hi, 0);
      }
      __syncthreads();
      if (wave == 0) {
        int count = 0;
        for (int i0 = 0; i0 < here; i0 += 64) {
          const int i = i0 + lane, p = (base_tile + i) * kLmTile;
          const int4 e = i < here ? list_s[i] : make_int4(0, 0, 0, 0);
          const bool on = i < here && lm_class(gq, LmRange{p, p + kLmTile - 1, e.y, e.z}, a.causal, prefix, true) != 0;
          const unsigned long long w = __ballot(on);
          if (on) list_s[count + __popcll(w & ((1ull << lane) - 1))] = e;      // (in place: no entry moves up past one not yet read)
          count += __popcll(w);
        }
        if (lane == 0) range_s[2 * NW] = count;
      }
      __syncthreads();
      ns = __builtin_amdgcn_readfirstlane(range_s[2 * NW]);
    }
    auto entry = [&](int s) { return docs ? list_s[min(s, kLmList - 1)] : make_int4(s, 0, 0, 0); };
    // copies of stage s: the k tile of entry s, the v tile of the entry before it
    auto issue = [&](int s, int tile, int before) {
      const uint32_t buf = lds0 + (s & 1) * F::STAGE;
      if (s < ns) {
        const int t0 = (base_tile + tile) * kLmTile;
        st.issue(k0, t0, n, buf, lane, wave);
        if (docs && wave == s % NW) lm_copy4(doc + t0, 4u * min(lane, n - 1 - t0), lds0 + F::DOCS + (s & 3) * (4 * kLmTile));
      }
      if (s > 0 && s <= ns) st.issue(v0, (base_tile + before) * kLmTile, n, buf + F::S::IMG, lane, wave);
    };
    int copied = __builtin_amdgcn_readfirstlane(entry(0).x), coming = __builtin_amdgcn_readfirstlane(entry(1).x);
    issue(0, copied, 0);
    const bool late = PAIR && wave >= NW / 2;                // this wavefront runs half a stage behind
    // the meeting before stage s: its copies have arrived everywhere, the places of stage s - 1 are free; and the one half a stage later
    auto meet = [&](bool first_half, int s) {
      if (first_half) lm_copies_done();
      lds_barrier();
      if (first_half) {
        issue(s + 1, coming, copied);
        copied = coming;
        coming = __builtin_amdgcn_readfirstlane(entry(s + 2).x);
      }
    };
    auto top = [&](int t) { meet(!late, t); };
    auto mid = [&](int t) { if (PAIR) meet(late, t + 1); };
    auto idle = [&](int from, int to) {
#pragma unroll 1
      for (int t = from; t < to; ++t) { top(t); mid(t); }
    };
    // the entries s0 .. s1 - 1 hold all that the wavefront sees
    int s0 = 0, s1 = busy ? ns : 0;
    if (docs) {
      s0 = ns; s1 = 0;
      for (int i0 = 0; busy && i0 < ns; i0 += 64) {
        const int4 e = list_s[min(i0 + lane, kLmList - 1)];
        const int p = (base_tile + e.x) * kLmTile;
        const unsigned long long w = __ballot(i0 + lane < ns && lm_class(wq, LmRange{p, p + kLmTile - 1, e.y, e.z}, a.causal, prefix, true) != 0);
        if (w) {
          s0 = min(s0, i0 + __ffsll((long long)w) - 1);
          s1 = i0 + 64 - __clzll((long long)w);
        }
      }
    } else if (a.causal && busy) {
      s1 = min(ns, max(max(wq.p1 / kLmTile + 1, (min(prefix, n) + kLmTile - 1) / kLmTile) - base_tile, 0));
    }
    auto stage_at = [&](int t) { return smem + (t & 1) * F::STAGE; };
    auto weights_of = [&](int t) {
      const int4 e = entry(t);
      LmRange r;
      r.p0 = (base_tile + __builtin_amdgcn_readfirstlane(e.x)) * kLmTile; r.p1 = r.p0 + kLmTile - 1;
      r.d0 = __builtin_amdgcn_readfirstlane(e.y); r.d1 = __builtin_amdgcn_readfirstlane(e.z);
      weigh(r, reinterpret_cast<const int*>(smem + F::DOCS + (t & 3) * (4 * kLmTile)));
    };
    wait_async_copies<0>();                                  // (the queries' loads too, lest the loop waits for them)
    if (late) meet(true, 0);
    if (s0 < s1) {
      idle(0, s0);
      top(s0);
      multiply(No{}, Yes{}, nullptr, stage_at(s0));
      mid(s0);
      weights_of(s0);
#pragma unroll 1
      for (int t = s0 + 1; t < s1; ++t) {
        top(t);
        multiply(Yes{}, Yes{}, stage_at(t) + F::S::IMG, stage_at(t));
        mid(t);
        weights_of(t);
      }
      top(s1);
      multiply(Yes{}, No{}, stage_at(s1) + F::S::IMG, nullptr);
      mid(s1);
      idle(s1 + 1, ns + 1);
    } else {
      idle(0, ns + 1);
    }
    if (PAIR && !late) meet(false, 0);
    lds_barrier();                                           // the tiles have been consumed: their places are free for the next list or the output
  }
  if (!busy) return;
  l += __shfl_xor(l, 32);
  const bool empty = l == 0.f;
  float total = l;
  if constexpr (MODE == LM_CAP_FIXED) {
    total = (lr[0] + lr[1]) + (lr[2] + lr[3]);
    total += __shfl_xor(total, 32);
  }
  const float f = empty ? 0.f : 1.f / total;
  bool fine = true;
#pragma unroll
  for (int x = 0; x < DB; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (D >= 32 || e < 8) fine = fine && lm_finite(o[x][e]);
  fine = fine || !lm_finite(l);                              // (a sum of weights has seen scores alone: this row is NaN as it should be)
  if constexpr (MODE == LM_CAP_FIXED) fine = fine && !(l > 0.f && l < kLmFixedSum);
  uint16_t* out = (uint16_t*)a.out + (long long)b * n * (a.h * D) + head * D;
  attn_store_rows<D>(smem + wave * (32 * (2 * D + 16)), o, f, out, (long long)a.h * D, first, n, lane);
  if (a.lse_out && u == 0 && mine < n)
    a.lse_out[((long long)b * n + mine) * a.h + head] = empty ? -INFINITY : (m2 + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  const unsigned long long bad = __ballot(!fine);
  const uint32_t again = (uint32_t)(bad | bad >> 32);
  if (__builtin_expect(again != 0, 0)) lm_forward_again<uint16_t, D>(a, b, head, first, again, lane);
}

template <int D, int NW, int MODE>
static void launch_masked_forward(const MaskedAttention& a, hipStream_t s) {
  const int nchunks = (int)ceil_div(a.n, 32 * NW);
  constexpr size_t lds = LmFwd<D, NW>::LDS;
  allow_dynamic_lds(reinterpret_cast<const void*>(masked_forward_kernel<D, NW, MODE>), lds);
  SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_forward_kernel<D, NW, MODE>), dim3((unsigned)((int64_t)a.B * a.h * nchunks)), dim3(64 * NW), lds, s, a, nchunks);
}
template <int D, int NW>
static void launch_masked_forward_mode(const MaskedAttention& a, hipStream_t s) {
  const bool bias = a.slopes != nullptr;
  if (a.cap > 0.f && !bias && a.cap <= kLmFixedCap) launch_masked_forward<D, NW, LM_CAP_FIXED>(a, s);
  else if (a.cap > 0.f) launch_masked_forward<D, NW, LM_CAP>(a, s);
  else if (bias || !(a.scale > 0.f)) launch_masked_forward<D, NW, LM_BIAS>(a, s);
  else launch_masked_forward<D, NW, LM_PLAIN>(a, s);
}
template <int D>
void launch_masked_forward_bf16(const MaskedAttention& a, hipStream_t s) {
  if (a.cap > 0.f && a.n <= kLmShort) return launch_masked_forward<D, 4, LM_CAP_SHORT>(a, s);
  // Pairs of wavefronts half a stage apart pay where the products of a stage are many (d = 128: the long text 310 us, with 4 wavefronts
  // 335, uncapped 267 and 294; with the running maximum and the cap, whose arithmetic is the most, 367 and 363) and there is more than one workgroup
  // of 4 to a head; for smaller d the meetings cost more than they hide (4 x 12 heads of 64, 2048 packed tokens: 35 us with 4 wavefronts, 50
  // with 8; 16 samples of them 94 and 159).
  if constexpr (D == 128) {
    if (a.n > 128) return launch_masked_forward_mode<D, 8>(a, s);
  }
  launch_masked_forward_mode<D, 4>(a, s);
}

}  // namespace sbp
#endif
