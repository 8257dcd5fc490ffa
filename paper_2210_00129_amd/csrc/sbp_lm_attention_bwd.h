// Backward of the masked attention on the kept tokens, on the bf16 matrix cores.
//
// A small kernel first makes what the others read per token: lse log2(e) and -delta = -dA.A per head (padded to whole tiles of 64 with
// weights of 0), positions and documents per sample, and their ranges per tile.
// A workgroup of 4 wavefronts owns 128 tokens of one sample, every wavefront 32, in one of two roles: as keys of a key / value head (dK,
// dV; the rows of q and dA of its query heads stream through LDS) or as queries of a query head (dQ; k and v stream).  Layouts as in
// sbp_attention.hip: own tokens are the columns (lanes) of every product, streamed ones the rows (registers), so that P and dM are,
// packed to bf16 (one rounding of 2^-8, the matrix cores multiply bf16), the B operands of the products that follow.  Recomputing S and
// dP in the second role costs 2 of 7 products and saves every sum across workgroups: no atomics, deterministic.
// Query heads that share a key / value head follow one another in the stream of its key role; where that leaves too few workgroups, they
// are dealt to several whose dK and dV, in fp32, a last small kernel adds in order.
// The loop is a pipeline over blocks of 32 streamed tokens: while the scores of block b turn into weights on the vector units, the matrix
// cores multiply the weights of block b - 1 and the scores of block b + 1, instruction by instruction in turn.  A tile of two blocks
// stays three tiles long in a ring of three; one barrier per tile.
// Tiles of which the workgroup sees nothing are left out of the list (ranges of positions and documents per tile; any order of the kept
// tokens is right, ascending order makes it short).  Tiles that are visible altogether come first, in a loop without mask arithmetic.
// Where a result is not finite, its row is computed again without the tokens it does not see (sbp_lm_attention_rows.h).
// Bound, d = 128 (one wavefront per SIMD): what one wavefront can issue; counted over the busy cycles of a CU, capped, the matrix cores are busy
// 35 %, the vector units 49 %, the LDS 31 % (a layout without its conflicts: no gain), uncapped 44, 33 and 38 %, at a clock of 2.1 GHz.
// 16 heads sharing 2, 4096 of 8192 tokens, causal, capped: 330 .. 350 us with the first kernel's 8 and the last one's 7 (up to 380 at lower clocks),
// uncapped 277.  d = 64: vector arithmetic and the chain of a workgroup's tiles; 4 x 12 heads of 64, 1024 of 2048 tokens in documents of
// 500 on average, biased: 35 .. 39 us (a CU is busy 63 % of it on average); 16 samples of it 110.
#ifndef SBP_LM_ATTENTION_BWD_H_
#define SBP_LM_ATTENTION_BWD_H_

#include "sbp_lm_attention_tiles.h"

namespace sbp {

static constexpr int kLmBwdList = 256;                     // tiles per list (16384 tokens); longer samples take several

enum { LM_BWD_CAP = 1, LM_BWD_BIAS = 2 };

template <int D>
struct LmBwd {
  using L = AttnSwizzled<D>;
  using S = LmStream<D, 4>;
  static constexpr int TABLE = 2 * S::IMG, STAGE = TABLE + 4 * 4 * kLmTile;   // two images, then l2, nd, pos, doc of the tile's tokens
  static constexpr int OUT = 4 * 2 * 32 * (2 * D + 16);
  static constexpr size_t LDS = 3 * STAGE > OUT ? 3 * STAGE : OUT;
};

template <int D, bool KEY, int MODE>
__device__ __forceinline__ void masked_backward_body(char* smem, int* list_s, int* count_s, const MaskedAttention& a, const LmTables& w, int b, int group,
                                                     int chunk) {
  using F = LmBwd<D>;
  using L = AttnSwizzled<D>;
  constexpr int KS = L::KS, DB = L::DB;
  constexpr bool CAP = MODE & LM_BWD_CAP, BIAS = MODE & LM_BWD_BIAS;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), u = lane >> 5;
  const int rows = a.rows, tiles = w.npad / kLmTile, ld = (a.h + 2 * a.hk) * D, lda = a.h * D, share = a.h / a.hk;
  // heads of the stream (KEY) or the head of the queries
  const int nh = KEY ? share / w.parts : 1;
  const int kv = KEY ? group / w.parts : group / share;
  const int h0 = KEY ? kv * share + group % w.parts * nh : group;
  const long long row0 = (long long)b * rows;
  const uint16_t* qkv = (const uint16_t*)a.qkv + row0 * ld;
  const uint16_t* dA = (const uint16_t*)a.dA + row0 * lda;
  const int first = chunk * kLmChunk + wave * 32, mine = first + (lane & 31), own = min(mine, rows - 1);
  const bool busy = first < rows, docs = a.doc != nullptr;
  const int prefix = lm_prefix(a, b);
  const L lay(lane);
  const uint32_t lds0 = lm_lds(smem);
  const typename F::S st1(ld, lane, wave), st2(lda, lane, wave);
  const char* tables[4] = {(const char*)w.l2, (const char*)w.nd, (const char*)w.pos, (const char*)w.doc};
  const uint32_t table_off = (uint32_t)(tables[lane >> 4] - tables[0]) + 16 * (lane & 15);

  bf16x8_t f1[KS], f2[KS];                                  // k, v (KEY) or q, dA of the own token
  {
    const uint16_t* p1 = qkv + (long long)own * ld + (KEY ? a.h + kv : h0) * D + 8 * u;
    const uint16_t* p2 = KEY ? p1 + a.hk * D : dA + (long long)own * lda + h0 * D + 8 * u;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      f1[ks] = *reinterpret_cast<const bf16x8_t*>(p1 + 16 * ks);
      f2[ks] = *reinterpret_cast<const bf16x8_t*>(p2 + 16 * ks);
    }
  }
  const float own_pos = w.pos[(long long)b * w.npad + own];
  const int own_doc = w.doc[(long long)b * w.npad + own];
  // streamed positions >= bound (KEY) or <= bound are visible
  float bound = KEY ? -3e38f : 3e38f;
  if (a.causal) bound = KEY ? (own_pos < (float)prefix ? -3e38f : own_pos) : fmaxf(own_pos, (float)prefix - 1.f);
  if (docs && own_doc < 0) bound = KEY ? 3e38f : -3e38f;
  float own_l2 = 0.f;
  f32x16_t nd;                                              // QUERY: -delta in every register
  if constexpr (!KEY) {
    own_l2 = w.l2[((long long)b * a.h + h0) * w.npad + own];
    const float v = w.nd[((long long)b * a.h + h0) * w.npad + own];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      nd[e] = v;
      asm("" : "+v"(nd[e]));                                // (16 registers for good: as one value it would be copied 16 times per block)
    }
  }
  const float c2 = a.scale * kLog2e, cap2 = a.cap * kLog2e;
  float ct = 2.f * kLog2e * a.per_cap;
  if constexpr (CAP) asm("" : "+v"(ct));                     // (in a vector register: 12 heads of 64 sharing 4, 2000 tokens 210 us, from a scalar one 218)

  constexpr int NACC = KEY ? 2 : 1;
  f32x16_t acc[NACC][DB];                                   // dK, dV or dQ: rows head dim, columns own tokens
#pragma unroll
  for (int q = 0; q < NACC; ++q)
#pragma unroll
    for (int x = 0; x < DB; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[q][x][e] = 0.f;
  f32x16_t sc, dp;                                          // scores and dP of the block whose weights come next
  bf16x8_t pw[2], ds[2];                                    // P and dM of the block before

  // One turn of the pipeline: products of the block before (in tile pt, first row pj), weights of the block whose scores are there (wt, wj:
  // half 0 or 1 of its tile), scores of the next one (st, sj).  Operands are read AHEAD
  // products before they are multiplied, the first ones of a turn (and the first rows of its table) at the end of the turn before: a
  // product takes 32 cycles, a read of LDS under way some 150.
  // (d = 64 with the bias: 4 ahead leave more in memory, 16 samples of the packed documents 115 us, 2 ahead 110)
  constexpr int NP = 2 * DB * NACC, N = NP + 2 * KS, AHEAD = D == 128 ? 8 : D == 64 && !BIAS ? 4 : 2;
  static_assert(AHEAD <= NP && N % AHEAD == 0, "the operands read ahead are products' and keep their places from turn to turn");
  bf16x8_t f[AHEAD];
  f32x4_t tl[2], tp[2];                                     // the tokens' table, four rows at a time: lse, positions, documents
  int4 td[2];
  auto product_operand = [&](int i, const char* tile, int row) {
    const int x = i % DB, q = i / DB % NACC, ks = i / DB / NACC;
    return lay.tr(tile + (q ? F::S::IMG : 0), row + 16 * ks, x);
  };
  auto table = [&](bool masked, const char* tile, int row, int q4) {
    const float* tab = reinterpret_cast<const float*>(tile + F::TABLE) + row + 4 * u + 8 * q4;
    if constexpr (KEY) tl[q4 & 1] = *reinterpret_cast<const f32x4_t*>(tab);
    if (BIAS || masked) tp[q4 & 1] = *reinterpret_cast<const f32x4_t*>(tab + 2 * kLmTile);
    if (masked) td[q4 & 1] = *reinterpret_cast<const int4*>(tab + 3 * kLmTile);
  };
  auto turn = [&](auto masked_, auto half_, const char* pt, const char* wt, float slope2, const char* st) {
    constexpr bool MASKED = decltype(masked_)::value;
    constexpr int wj = 32 * decltype(half_)::value, pj = 32 - wj, sj = 32 - wj;
    auto operand = [&](int i) {                              // (from N on: of the next turn, whose block before is this one's)
      if (i < NP) return product_operand(i, pt, pj);
      if (i >= N) return product_operand(i - N, wt, wj);
      const int j = i - NP;
      return lay.row(st + (j & 1 ? F::S::IMG : 0), sj, j >> 1);
    };
    f32x16_t sn, dn;
    if constexpr (KEY) {
      const float* nt = reinterpret_cast<const float*>(st + F::TABLE) + kLmTile + sj + 4 * u;
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(nt + 8 * q4);
#pragma unroll
        for (int e = 0; e < 4; ++e) dn[4 * q4 + e] = v[e];
      }
    } else {
      dn = nd;
    }
    const f32x16_t zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    bf16x8_t pn[2], mn[2];
    // the weights, register e: 16 steps dealt out over the products
    auto weight = [&](int e) {
      const int q4 = e >> 2, i = e & 3;
      if (i == 0) {                                          // the next rows: of this block, or of the next one (in tile st)
        if (q4 < 3) table(MASKED, wt, wj, q4 + 1);
        else table(MASKED, st, sj, 0);
      }
      const float l2 = KEY ? tl[q4 & 1][i] : own_l2;
      float x, slope = 1.f;
      if constexpr (CAP) {
        const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(sc[e] * ct) + 1.f);
        x = fmaf(-2.f * cap2, r, cap2) - l2;                 // cap tanh(z / cap)
        slope = fmaf(-r, r, r);                              // (1 - tanh^2) / 4
      } else {
        x = fmaf(sc[e], c2, -l2);
      }
      if constexpr (BIAS) x = fmaf(-slope2, fabsf(tp[q4 & 1][i] - own_pos), x);
      float p = __builtin_amdgcn_exp2f(x), m = p * dp[e];
      if constexpr (CAP) m *= slope;
      if constexpr (MASKED) {
        const int dj = i == 0 ? td[q4 & 1].x : i == 1 ? td[q4 & 1].y : i == 2 ? td[q4 & 1].z : td[q4 & 1].w;
        const bool see = (KEY ? tp[q4 & 1][i] >= bound : tp[q4 & 1][i] <= bound) && dj == own_doc;
        p = see ? p : 0.f;
        m = see ? m : 0.f;
      }
      sc[e] = p;
      dp[e] = m;
      if (e == 7 || e == 15) {
        if constexpr (KEY) pn[e >> 3] = pack8(sc, e >> 3);
        mn[e >> 3] = pack8(dp, e >> 3);
      }
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i < NP) {
        const int x = i % DB, q = i / DB % NACC, ks = i / DB / NACC;
        acc[q][x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], q ? pw[ks] : ds[ks], acc[q][x], 0, 0, 0);
      } else {
        const int j = i - NP;
        if (j & 1) dn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], f2[j >> 1], dn, 0, 0, 0);
        else sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % AHEAD], f1[j >> 1], j ? sn : zero, 0, 0, 0);
      }
      f[i % AHEAD] = operand(i + AHEAD);
#pragma unroll
      for (int e = 16 * i / N; e < 16 * (i + 1) / N; ++e) weight(e);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      if constexpr (KEY) pw[ks] = pn[ks];
      ds[ks] = mn[ks];
    }
    sc = sn;
    dp = dn;
  };

  const int4* ranges = w.range + (long long)b * tiles;
  LmRange mr[2];                                            // the two halves of the chunk
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int4 r = ranges[min(2 * chunk + y, tiles - 1)];
    mr[y] = LmRange{r.x, r.y, r.z, r.w};
  }
  for (int base = 0; base < tiles; base += kLmBwdList) {
    const int here = min(kLmBwdList, tiles - base);
    // the list: first the tiles that are visible altogether, from its front, then the others, from its back
    if (wave == 0) {
      int count = 0, back = 0;
      for (int i0 = 0; i0 < here; i0 += 64) {
        const int i = i0 + lane;
        const int4 e = ranges[base + min(i, here - 1)];
        const LmRange r{e.x, e.y, e.z, e.w};
        int cls[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) cls[y] = KEY ? lm_class(r, mr[y], a.causal, prefix, docs) : lm_class(mr[y], r, a.causal, prefix, docs);
        const bool on = i < here && (cls[0] | cls[1]), full = on && cls[0] == 2 && cls[1] == 2 && (base + i + 1) * kLmTile <= rows;
        const unsigned long long m = __ballot(full), v = __ballot(on && !full), below = (1ull << lane) - 1;
        if (full) list_s[count + __popcll(m & below)] = base + i;
        else if (on) list_s[kLmBwdList - 1 - back - __popcll(v & below)] = base + i;
        count += __popcll(m);
        back += __popcll(v);
      }
      if (lane == 0) { count_s[0] = count; count_s[1] = back; }
    }
    __syncthreads();
    const int nf = __builtin_amdgcn_readfirstlane(count_s[0]), nm = __builtin_amdgcn_readfirstlane(count_s[1]), total = (nf + nm) * nh;
    if (total > 0) {
      // the stream: the visible tiles for every head, then the masked ones for every head
      struct Place { int head, i, masked; };
      auto entry = [&](const Place& p) { return __builtin_amdgcn_readfirstlane(list_s[p.masked ? kLmBwdList - 1 - p.i : p.i]); };
      auto advance = [&](Place& p) {
        if (++p.i < (p.masked ? nm : nf)) return;
        p.i = 0;
        if (++p.head < h0 + nh) return;
        p.head = h0;
        p.masked = 1;
      };
      auto issue = [&](int s, const Place& p) {             // into the place at byte s of the ring
        const int t0 = entry(p) * kLmTile, head = p.head;
        const uint32_t buf = lds0 + (uint32_t)s;
        st1.issue(qkv + (KEY ? head : a.h + kv) * D, t0, rows, buf, lane, wave);
        if constexpr (KEY) st2.issue(dA + head * D, t0, rows, buf + F::S::IMG, lane, wave);
        else st1.issue(qkv + (a.h + a.hk + kv) * D, t0, rows, buf + F::S::IMG, lane, wave);
        if (wave == 3) {
          // (every place in the tables is less than 2^32 bytes behind l2, and the copies take their offsets as unsigned: the limit on
          // B h n / 32 leaves each of the four tables less than 2^30 bytes)
          const uint32_t th = 4u * (uint32_t)((b * a.h + head) * w.npad + t0), tb = 4u * (uint32_t)(b * w.npad + t0);
          lm_copy16(w.l2, table_off + (lane < 32 ? th : tb), buf + F::TABLE);
        }
      };
      Place coming{h0, 0, nf == 0}, at = coming;            // of the next tile to copy, of the one whose weights come next
      issue(0, coming);
      advance(coming);
      if (total > 1) { issue(F::STAGE, coming); advance(coming); }
      wait_async_copies<0>();
      lm_copies_done();
      lds_barrier();
      if (busy) {
        // the pipeline's first scores; the products of the turn before them are of weights 0
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int e = 0; e < 8; ++e) pw[ks][e] = ds[ks][e] = (__bf16)0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = 0.f;
        if constexpr (KEY) {
          const float* nt = reinterpret_cast<const float*>(smem + F::TABLE) + kLmTile + 4 * u;
#pragma unroll
          for (int e = 0; e < 16; ++e) dp[e] = nt[8 * (e >> 2) + (e & 3)];
        } else {
          dp = nd;
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lay.row(smem, 0, ks), f1[ks], sc, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lay.row(smem + F::S::IMG, 0, ks), f2[ks], dp, 0, 0, 0);
        }
      }
      int before = 0, now = 0, after = F::STAGE, left = total;      // places of the tile before (at first: any), of this one, of the next
      auto tile = [&](auto masked_) {
        const float slope2 = BIAS ? a.slopes[at.head] * kLog2e : 0.f;
        if (busy) turn(masked_, std::integral_constant<int, 0>{}, smem + before, smem + now, slope2, smem + now);
        lm_copies_done();                                   // the next tile ...
        lds_barrier();                                      // ... everywhere; the place of the one before is free
        const int over = 3 * F::STAGE - now - after;
        if (left > 2) { issue(over, coming); advance(coming); }
        // (after the last block its tile's own rows stand for the next scores, which nothing uses)
        if (busy) turn(masked_, std::integral_constant<int, 1>{}, smem + now, smem + now, slope2, smem + (left > 1 ? after : now));
        before = now; now = after; after = over;
        --left;
        advance(at);
      };
      if (busy) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f[i] = product_operand(i, smem, 32);
        table(true, smem, 0, 0);
      }
#pragma unroll 1
      for (int s = 0; s < nf * nh; ++s) tile(std::false_type{});
      if (busy && nf) table(true, smem + now, 0, 0);         // (the loop before read less of it)
#pragma unroll 1
      for (int s = 0; s < nm * nh; ++s) tile(std::true_type{});
      if (busy) {
        const char* last = smem + before;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int x = 0; x < DB; ++x) {
            acc[0][x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lay.tr(last, 32 + 16 * ks, x), ds[ks], acc[0][x], 0, 0, 0);
            if constexpr (KEY) acc[1][x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lay.tr(last + F::S::IMG, 32 + 16 * ks, x), pw[ks], acc[1][x], 0, 0, 0);
          }
      }
    }
    __syncthreads();                                        // the tiles and the list have been consumed
  }
  if (!busy) return;
  bool fine = true;
#pragma unroll
  for (int q = 0; q < NACC; ++q)
#pragma unroll
    for (int x = 0; x < DB; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (D >= 32 || e < 8) fine = fine && lm_finite(acc[q][x][e]);
  const unsigned long long bad = __ballot(!fine);
  const uint32_t again = (uint32_t)(bad | bad >> 32);
  const float dscale = CAP ? 4.f * a.scale : a.scale;
  uint16_t* out = (uint16_t*)a.out + row0 * ld;
  char* img = smem + wave * (2 * 32 * (2 * D + 16));
  if constexpr (!KEY) {
    attn_store_rows<D>(img, acc[0], dscale, out + h0 * D, ld, first, rows, lane);
    if (__builtin_expect(again != 0, 0)) lm_backward_again<uint16_t, D, false>(a, w, b, kv, h0, 1, first, again, lane, nullptr);
  } else {
    float* part = w.part ? w.part + (((long long)(group % w.parts) * a.B + b) * rows * a.hk + kv) * (2 * D) : nullptr;
    if (!part) {
      attn_store_rows<D>(img, acc[0], dscale, out + (a.h + kv) * D, ld, first, rows, lane);
      attn_store_rows<D>(img + 32 * (2 * D + 16), acc[1], 1.f, out + (a.h + a.hk + kv) * D, ld, first, rows, lane);
    } else if (mine < rows) {
      float* p = part + (long long)mine * (a.hk * 2 * D) + 4 * u;
#pragma unroll
      for (int x = 0; x < DB; ++x)
#pragma unroll
        for (int q4 = 0; q4 < (D < 32 ? D / 8 : 4); ++q4) {
          *reinterpret_cast<float4*>(p + 32 * x + 8 * q4) = make_float4(acc[0][x][4 * q4] * dscale, acc[0][x][4 * q4 + 1] * dscale, acc[0][x][4 * q4 + 2] * dscale, acc[0][x][4 * q4 + 3] * dscale);
          *reinterpret_cast<float4*>(p + D + 32 * x + 8 * q4) = make_float4(acc[1][x][4 * q4], acc[1][x][4 * q4 + 1], acc[1][x][4 * q4 + 2], acc[1][x][4 * q4 + 3]);
        }
    }
    if (__builtin_expect(again != 0, 0)) lm_backward_again<uint16_t, D, true>(a, w, b, kv, h0, nh, first, again, lane, part);
  }
}

template <int D, int MODE>
__global__ void __launch_bounds__(256, D == 128 ? 1 : 2) masked_backward_kernel(MaskedAttention a, LmTables w) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int list_s[kLmBwdList], count_s[2];
  // Units: the key groups and the query heads of all samples, each for every rank; those of one XCD stay on it where both divide by 8.
  // d = 128 (one workgroup on a CU): all key units first, the longer kind (the long text 331 us, mixed by rank 348).  Smaller heads (two): mixed,
  // since a key and a query unit share a CU better than two key units (packed documents 37 us, key units first 41).
  const int nk = a.B * a.hk * w.parts, nq = a.B * a.h, x8 = nk % 8 == 0 && nq % 8 == 0 ? 8 : 1, pk = nk / x8, pq = nq / x8;
  const int x = blockIdx.x % x8, j = blockIdx.x / x8;
  int rank, k;
  if (D == 128) {
    const int q = j - pk * w.nchunks;
    rank = q < 0 ? j / pk : q / pq;
    k = q < 0 ? x * pk + j % pk : nk + x * pq + q % pq;
  } else {
    rank = j / (pk + pq);
    k = j % (pk + pq);
    k = k < pk ? x * pk + k : nk + x * pq + k - pk;
  }
  // causal: the first keys are seen by the most queries, the last queries see the most keys
  if (k < nk) masked_backward_body<D, true, MODE>(smem, list_s, count_s, a, w, k / (a.hk * w.parts), k % (a.hk * w.parts), rank);
  else masked_backward_body<D, false, MODE>(smem, list_s, count_s, a, w, (k - nk) / a.h, (k - nk) % a.h, a.causal ? w.nchunks - 1 - rank : rank);
}

template <int D, int MODE>
static void launch_masked_backward(const MaskedAttention& a, const LmTables& w, hipStream_t s) {
  constexpr size_t lds = LmBwd<D>::LDS;
  allow_dynamic_lds(reinterpret_cast<const void*>(masked_backward_kernel<D, MODE>), lds);
  SBP_LAUNCH(SBP_PROF_ATTENTION, s, (masked_backward_kernel<D, MODE>), dim3((unsigned)((int64_t)w.nchunks * a.B * (a.hk * w.parts + a.h))), dim3(256), lds, s,
             a, w);
}
template <int D>
void launch_masked_backward_bf16(const MaskedAttention& a, const LmTables& w, hipStream_t s) {
  const bool cap = a.cap > 0.f, bias = a.slopes != nullptr;
  if (cap && bias) launch_masked_backward<D, LM_BWD_CAP | LM_BWD_BIAS>(a, w, s);
  else if (cap) launch_masked_backward<D, LM_BWD_CAP>(a, w, s);
  else if (bias) launch_masked_backward<D, LM_BWD_BIAS>(a, w, s);
  else launch_masked_backward<D, 0>(a, w, s);
}

}  // namespace sbp
#endif
