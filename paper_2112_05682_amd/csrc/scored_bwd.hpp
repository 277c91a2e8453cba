// Backward of attention with modified scores (scored.hpp), recomputing each tile's
// scores from the forward's log-sum-exp (arXiv 2112.05682, Section 5.2):
//   P_ij = exp(s_ij - lse_i),  dP_ij = dO_i . v_j,  D_i = dO_i . o_i,
//   dS_ij = P_ij (dP_ij - D_i),              dV_j = sum_i P_ij dO_i,
//   dX_ij = dS_ij (1 - (y_ij / cap)^2),      dK_j = scale sum_i dX_ij q_i,
//   dtable[t, h] = sum dS_ij over the pairs  dQ_i = scale sum_j dX_ij k_j.
//   of bucket t (all batches),
// Three passes, and no atomics in memory, so that results do not depend on timing:
//   pre  : lse and D of every row;
//   dkdv : a wave per 32 keys of a key head (K, V in registers), over the queries of
//          every head that shares it, so that shared heads' gradients add up in
//          registers; a key on each lane;
//   dq   : a wave per 32 queries (Q, dO in registers) over the keys; a query on each
//          lane.  Its dS also gives the bias gradient: per lane one sum for each
//          side beyond the span, and within it sums of each tile's diagonals.
// dkdv and dq both make the scores and dP again, 14 d a pair for the 10 d it needs:
// in one pass dQ's sums would cross workgroups.
//
// What bounds it: vector instructions next to the products in two waves per SIMD
// (registers; counters at d = 128 with a cap VALU 60 %, MFMA 37 %, at d = 64 with a learned
// bias 48 %, 32 %).  All passes, causal, 16-bit: cap, 2x16 heads on 4, 4096, d = 128 628 us, 547
// TFLOP/s of what it needs; learned bias with its gradient, 4x16x4096, d = 64 647 us, 531.  The
// pre pass reads at 5.5 TB/s (18 us there).
#pragma once

#include "scored.hpp"

namespace mea {

// ------------------------------------------------------------------- pre
template <typename T, int D>
__global__ __launch_bounds__(256) void scored_bwd_pre_kernel(ScoredBwdParams p) {
  constexpr int E = sizeof(T), W = 16 / E, TPR = D / W, RPB = 256 / TPR;
  const int64_t rows = (int64_t)p.n_b * p.s.heads * p.n_q_pad;
  const int64_t prow = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  const int64_t bh = prow / p.n_q_pad, i = prow % p.n_q_pad;
  const bool real = prow < rows && i < p.n_q;
  const int part = threadIdx.x % TPR;
  float acc = 0.0f;
  if (real) {
    typedef T vec __attribute__((ext_vector_type(W)));
    const int64_t b = bh / p.s.heads, hd = bh % p.s.heads;
    const vec o = *reinterpret_cast<const vec*>(static_cast<const T*>(p.o) + b * p.so.b + hd * p.so.h + i * p.so.r + part * W);
    const vec g = *reinterpret_cast<const vec*>(static_cast<const T*>(p.d_o) + b * p.sdo.b + hd * p.sdo.h + i * p.sdo.r + part * W);
    float of[W];
#pragma unroll
    for (int e = 0; e < W; ++e) of[e] = (float)o[e];
    if constexpr (E == 2) {
      // o + o_lo carries about 16 bits of the unrounded output; D is subtracted from
      // sums it nearly equals, where o's own rounding would show.
      if (p.o_lo) {
        const vec lo = *reinterpret_cast<const vec*>(static_cast<const T*>(p.o_lo) + (bh * p.n_q + i) * D + part * W);
#pragma unroll
        for (int e = 0; e < W; ++e) of[e] += (float)lo[e];
      }
    }
#pragma unroll
    for (int e = 0; e < W; ++e) acc = fmaf(of[e], (float)g[e], acc);
  }
#pragma unroll
  for (int off = TPR / 2; off > 0; off >>= 1) acc += __shfl_xor(acc, off, TPR);
  if (prow < rows && part == 0) {
    const float lse = real ? p.lse[bh * p.n_q + i] : -INFINITY;
    const bool live = lse != -INFINITY;
    p.lse2[prow] = live ? lse * kLog2eF : INFINITY;
    p.neg_d[prow] = live ? -acc : 0.0f;
  }
}

// 1 - tanh^2 of a score that is still the tanh, or hidden (-inf, whose weight is 0).
__device__ __forceinline__ float cap_grad(float t) {
  t = fmaxf(t, -1.0f);
  return fmaf(-t, t, 1.0f);
}

// ------------------------------------------------------------------- dK, dV
template <typename T, int D>
struct ScoredKvTile {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NT = 256, BKG = 128;              // keys of a workgroup
  static constexpr int QS = D == 64 ? 2 : 1, BQ = 32 * QS;  // queries of a staged tile
  static constexpr int NP = Planes<T>::NP;
  static constexpr int RS = D + 8, TILE = BQ * RS;       // float32: padded rows of three planes
  static constexpr int TILE_BYTES = F32 ? NP * TILE * 2 : BQ * D * 2;
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES + 2 * BQ * 4;  // Q, dO, lse2, -D
  static constexpr int OCC = F32 ? 1 : 2;
  // 16-bit, d = 128: the K fragments of every lane wait in LDS (32 registers less).
  static constexpr bool K_LDS = !F32 && D == 128;
  static constexpr int KSLOT_BYTES = K_LDS ? NT * (D / 16) * 16 : 0;
  static constexpr int kBiasMax = 4 * (2 * kMaxBiasSpan + 1 + 2 * kPad) + 16;
  static constexpr int NBUF = 2 * STAGE_BYTES + KSLOT_BYTES + kBiasMax <= 160 * 1024 / OCC - 1280 ? 2 : 1;
  static constexpr int LDS_BYTES = NBUF * STAGE_BYTES + KSLOT_BYTES;
  static constexpr int CPR = D / 8, CHUNKS = 2 * BQ * CPR, CPT = CHUNKS / NT;
  static_assert(CHUNKS % NT == 0, "tile shapes");
  static_assert(F32 || NBUF == 2, "asynchronous copies need two stages");
};

// Workgroup `block` of n_blocks.
template <typename T, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void dkdv_workgroup(const ScoredBwdParams& p, int block, int n_blocks) {
  using C = ScoredKvTile<T, D>;
  using LE = typename Planes<T>::E;
  constexpr bool F32 = C::F32;
  constexpr bool KEEP = CAP && (BIAS || D == 64);  // 1 - tanh^2 is kept, else (registers) made again from the score
  constexpr int BQ = C::BQ, QS = C::QS, KC = D / 16, NDT = D / 32, NBUF = C::NBUF;

  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* const lds_bias = smem + C::LDS_BYTES;
  __shared__ int4 wave_ids[4];
  __shared__ __align__(16) int tile_ids[4][32];

  const ScoreArgs& sa = p.s;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int h = lane >> 5, c = lane & 31;

  const TileItem item = tile_item(block, n_blocks, p.n_ktiles, sa.causal ? p.tile_order : 0);
  const int b = item.group % p.n_b, kvh = item.group / p.n_b % p.heads_kv;
  // This part's heads and its share of the tiles of queries.
  const int part = item.group / (p.n_b * p.heads_kv);
  const int part_h = part % p.kv_heads_parts, part_q = part / p.kv_heads_parts;
  const int g0 = p.heads_per_kv * part_h / p.kv_heads_parts, g_end = p.heads_per_kv * (part_h + 1) / p.kv_heads_parts;
  const int64_t k0 = (int64_t)item.tile * C::BKG, kw = k0 + 32 * wave, key = kw + c;

  const int64_t n_kv = batch_keys(sa, b, p.n_k), pos0 = first_pos(sa, b);
  const int64_t reach = key_reach(sa, b, p.n_k);
  bool live = key < n_kv;
  int doc = -2;
  int4 ids = make_int4(0, 0, 0, 0);
  if (sa.q_doc) {
    doc = key < p.n_k ? sa.k_doc[(int64_t)b * p.n_k + key] : -1;
    if (doc < 0) {
      doc = -2;
      live = false;
    }
    ids = workgroup_ids(doc, wave, lane, wave_ids);
  }
  // The first query that sees this lane's key, and (uniform) the first one of the
  // workgroup's first key, of its last, and of the wave's first.
  auto first_query = [&](int64_t j) { return j < reach || j <= pos0 ? (int64_t)0 : j - pos0; };
  const int min_q = live ? (int)first_query(key) : 0;
  const int64_t q_begin = first_query(k0), q_full = first_query(k0 + C::BKG - 1), qw_begin = first_query(kw);

  const T* __restrict__ kg = static_cast<const T*>(p.k) + (int64_t)b * p.sk.b + (int64_t)kvh * p.sk.h;
  const T* __restrict__ vg = static_cast<const T*>(p.v) + (int64_t)b * p.sv.b + (int64_t)kvh * p.sv.h;

  // ---- the stream: for each head of the key head its query tiles.
  const int n_units = (int)((p.n_q + 31) / 32);
  const int2* const ranges = sa.q_range ? sa.q_range + (int64_t)b * n_units : nullptr;
  DocTiles<QS> docs(ranges, n_units, ids.x, ids.y);
  const int t_all = k0 < n_kv ? (int)((p.n_q + BQ - 1) / BQ) : 0;
  const int64_t t_see = q_begin / BQ < t_all ? q_begin / BQ : t_all;
  const int t_begin = (int)(t_see + (t_all - t_see) * part_q / p.kv_query_parts);
  const int t_end = (int)(t_see + (t_all - t_see) * (part_q + 1) / p.kv_query_parts);
  int g = g0, t = 0;  // current head and tile
  auto first_tile = [&]() {
    docs.base = -64;
    return docs.next(t_begin, t_end);
  };
  // The tile after (g_, t_); g_ = g_end at the end.
  auto advance = [&](int& g_, int& t_) {
    t_ = docs.next(t_ + 1, t_end);
    if (t_ >= t_end) {
      ++g_;
      t_ = first_tile();
    }
  };
  t = first_tile();
  if (t >= t_end) g = g_end;  // no query sees these keys

  constexpr int CPR = C::CPR;
  const TileCopy<std::conditional_t<F32, __bf16, T>, D, BQ, false> copies(wave, lane, p.sq.r, p.sdo.r);
  auto head_of = [&](int g_) { return kvh * p.heads_per_kv + g_; };
  float stage_f = 0.0f;
  auto load_rows = [&](int g_, int t_) __attribute__((always_inline)) {
    if (tid < 2 * BQ) {
      const int64_t at = ((int64_t)b * sa.heads + head_of(g_)) * p.n_q_pad + (int64_t)t_ * BQ + tid % BQ;
      stage_f = tid < BQ ? p.lse2[at] : p.neg_d[at];
    }
  };
  auto store_rows = [&](int buf) __attribute__((always_inline)) {
    if (tid < 2 * BQ) reinterpret_cast<float*>(smem + buf * C::STAGE_BYTES + 2 * C::TILE_BYTES)[tid] = stage_f;
  };
  // 16-bit: asynchronous copies into swizzled rows; rows past n_q repeat the last.
  auto copy_tile = [&](int g_, int t_, int buf) __attribute__((always_inline)) {
    if constexpr (!F32)
      copies(static_cast<const T*>(p.q) + (int64_t)b * p.sq.b + (int64_t)head_of(g_) * p.sq.h, p.sq.r,
             static_cast<const T*>(p.d_o) + (int64_t)b * p.sdo.b + (int64_t)head_of(g_) * p.sdo.h, p.sdo.r,
             (int64_t)t_ * BQ, p.n_q, __builtin_amdgcn_readfirstlane(lds_addr(smem + buf * C::STAGE_BYTES)), wave);
  };
  Range<T, false> range;
  Chunk8<T> stage[F32 ? C::CPT : 1];
  auto load_stage = [&](int g_, int t_) __attribute__((always_inline)) {
    if constexpr (F32) {
      const T* qg = static_cast<const T*>(p.q) + (int64_t)b * p.sq.b + (int64_t)head_of(g_) * p.sq.h;
      const T* og = static_cast<const T*>(p.d_o) + (int64_t)b * p.sdo.b + (int64_t)head_of(g_) * p.sdo.h;
#pragma unroll
      for (int i = 0; i < C::CPT; ++i) {
        const int chunk = tid + i * C::NT;
        const bool is_o = chunk >= BQ * CPR;
        const int rem = is_o ? chunk - BQ * CPR : chunk;
        const int r = rem / CPR, col = rem % CPR;
        const int64_t qi = (int64_t)t_ * BQ + r;
        const T* src = is_o ? og + qi * p.sdo.r : qg + qi * p.sq.r;
        stage[i] = qi < p.n_q ? ld_chunk8<T, T>(src + 8 * col) : zero_chunk8<T>();
      }
    }
  };
  auto store_stage = [&](int buf) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < C::CPT; ++i) {
        const int chunk = tid + i * C::NT;
        const bool is_o = chunk >= BQ * CPR;
        const int rem = is_o ? chunk - BQ * CPR : chunk;
        st_chunk8<T>(reinterpret_cast<LE*>(smem + buf * C::STAGE_BYTES + (is_o ? C::TILE_BYTES : 0)) + rem / CPR * C::RS +
                         8 * (rem % CPR),
                     C::TILE, stage[i], range);
      }
    }
  };

  // The first tile is on its way while K and V are read.
  if (g < g_end) {
    load_rows(g, t);
    if constexpr (!F32) copy_tile(g, t, 0);
  }

  // K^T and V^T as B operands: lane (h, key c) holds features 16 kc + 8 h ..
  T* const kslot = reinterpret_cast<T*>(smem + NBUF * C::STAGE_BYTES) + 8 * tid;
  Frag<T> kf[C::K_LDS ? 1 : KC], vf[KC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const Frag<T> f = live ? ld_frag_as<T, T>(kg + key * p.sk.r + 16 * kc + 8 * h, range) : zero_frag<T>();
    if constexpr (C::K_LDS) *reinterpret_cast<Frag<T>*>(kslot + 8 * C::NT * kc) = f;
    else kf[kc] = f;
    vf[kc] = live ? ld_frag_as<T, T>(vg + key * p.sv.r + 16 * kc + 8 * h, range) : zero_frag<T>();
  }
  auto kfrag = [&](int kc) __attribute__((always_inline)) {
    if constexpr (C::K_LDS) return lds_frag<T>(kslot + 8 * C::NT * kc);
    else return kf[kc];
  };

  f32x16 dk[NDT], dv[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[dt][r] = dv[dt][r] = 0.0f;

  const int qrow = perm32(c);
  const float unit = sa.unit;
  float slope = 0.0f;

  // One tile of queries: masked, some query sees some key of the workgroup not; by_doc,
  // documents differ (uniform branches of one copy of the code, as in the forward).
  auto compute = [&](int t_, int buf, bool masked, bool by_doc) __attribute__((always_inline)) {
    const int64_t q0t = (int64_t)t_ * BQ;
    if (q0t + BQ <= qw_begin || kw >= n_kv) return;  // none of the wave's keys is seen
    const unsigned char* st = smem + buf * C::STAGE_BYTES;
#pragma unroll 1
    for (int qs = 0; qs < QS; ++qs) {
      const int64_t q0 = q0t + 32 * qs;
      const unsigned char* qt = st + qs * 32 * (2 * D);
      const unsigned char* ot = qt + C::TILE_BYTES;
      const LE* qt32 = reinterpret_cast<const LE*>(st) + qs * 32 * C::RS;
      const LE* ot32 = reinterpret_cast<const LE*>(st + C::TILE_BYTES) + qs * 32 * C::RS;
      const float* lse_s = reinterpret_cast<const float*>(st + 2 * C::TILE_BYTES) + 32 * qs + 8 * h;
      f32x16 s, dp;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 d = *reinterpret_cast<const f32x4*>(lse_s + BQ + 16 * (j >> 1) + 4 * (j & 1));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[4 * j + e] = 0.0f;
          dp[4 * j + e] = d[e];
        }
      }
      if constexpr (F32) {
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          s = mma(lds_frag_planes<T>(qt32 + qrow * C::RS + 16 * kc + 8 * h, C::TILE), kfrag(kc), s);
          dp = mma(lds_frag_planes<T>(ot32 + qrow * C::RS + 16 * kc + 8 * h, C::TILE), vf[kc], dp);
        }
      } else {
        // Fragments are read one chunk before their MFMAs, and not earlier (registers).
        Frag<T> fa[2], fg[2];
        fa[0] = row_frag<T, D>(qt, qrow, h);
        fg[0] = row_frag<T, D>(ot, qrow, h);
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          if (kc + 1 < KC) {
            fa[(kc + 1) & 1] = row_frag<T, D>(qt, qrow, 2 * (kc + 1) + h);
            fg[(kc + 1) & 1] = row_frag<T, D>(ot, qrow, 2 * (kc + 1) + h);
          }
          s = mma(fa[kc & 1], kfrag(kc), s);
          dp = mma(fg[kc & 1], vf[kc], dp);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      float grad[KEEP ? 16 : 1];
      if constexpr (CAP) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = cap_tanh<T>(sa, s[r]);
          if constexpr (KEEP) grad[r] = fmaf(-s[r], s[r], 1.0f);
        }
      }
      float add = 0.0f;  // what every pair gets
      if constexpr (BIAS) {
        const int off = (int)key - (int)(pos0 + q0) - 8 * h;  // distance to the tile's first query, less 8 h
        const int64_t p_lo = pos0 + q0, p_hi = p_lo + 31;
        if (sa.slopes) {
          if (kw + 31 <= p_lo) {
            add = (float)off * slope;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf((float)permuted_row(r, 0), -slope, s[r]);
          } else {
            float d0 = (float)off;
            stay(d0);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf(-fabsf(d0 - (float)permuted_row(r, 0)), slope, s[r]);
          }
        }
        if (sa.table) {
          const int hi = bias_ahead(sa);
          if (kw + 31 <= p_lo - sa.span || kw >= p_hi + hi) {
            add += reinterpret_cast<const float*>(lds_bias)[kw >= p_hi + hi ? bias_places(sa) - 1 : 0];
          } else {
            int from = off + sa.span + kPad;
            stay(from);
            const float* at = reinterpret_cast<const float*>(lds_bias) + from;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] += at[-permuted_row(r, 0)];
          }
        }
      }
      if (masked) {
        int m = min_q - (int)q0 - 8 * h;
        stay(m);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (permuted_row(r, 0) < m) s[r] = -INFINITY;
      }
      if (by_doc) {
        const int mine = q0 + c < p.n_q ? sa.q_doc[(int64_t)b * p.n_q + q0 + c] : -1;
        hide_documents(s, doc, mine, tile_ids[wave], lane);
      }
      // dV^T += dO^T P and dK^T += Q^T dX, P and dX rounded to their operands.
      const float base = BIAS ? add * unit : 0.0f;
      auto weight = [&](int r, float l2, float& x, float& y) __attribute__((always_inline)) {
        x = fast_exp2(fmaf(s[r], unit, BIAS ? base - l2 : -l2));
        y = x * dp[r];
        if constexpr (KEEP) y *= grad[r];
        else if constexpr (CAP) y *= cap_grad(s[r]);
      };
      if constexpr (F32) {
        Frag<T> pf[2], sf[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          float x[8], y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) weight(8 * m + e, lse_s[16 * m + e], x[e], y[e]);
          pf[m] = to_frag<T>(x);
          sf[m] = to_frag<T>(y);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            dv[dt] = mma(lds_col_frag_planes<T>(ot32, C::TILE, C::RS, 16 * m, 32 * dt, lane), pf[m], dv[dt]);
            dk[dt] = mma(lds_col_frag_planes<T>(qt32, C::TILE, C::RS, 16 * m, 32 * dt, lane), sf[m], dk[dt]);
          }
      } else {
        // The second 16 rows' weights are made between the first ones' products, a share
        // a step, and each step's fragments are read one step ahead.
        typedef uint32_t u32x4w __attribute__((ext_vector_type(4)));
        constexpr int PER = 8 / NDT;
        u32x4w pw, dw;
        auto pair = [&](int m, int e) __attribute__((always_inline)) {
          const f32x2 l2 = *reinterpret_cast<const f32x2*>(lse_s + 16 * m + e);
          float x0, y0, x1, y1;
          weight(8 * m + e, l2[0], x0, y0);
          weight(8 * m + e + 1, l2[1], x1, y1);
          pw[e / 2] = pack2<T>(x0, x1);
          dw[e / 2] = pack2<T>(y0, y1);
        };
#pragma unroll
        for (int e = 0; e < 8; e += 2) pair(0, e);
        Frag<T> pa = __builtin_bit_cast(Frag<T>, pw), da = __builtin_bit_cast(Frag<T>, dw);
        Frag<T> bo = col_frag<T, D>(ot, 0, 0, lane), bq = col_frag<T, D>(qt, 0, 0, lane);
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const bool last = dt + 1 == NDT;
            Frag<T> bo_n = bo, bq_n = bq;
            if (!last || m == 0) {
              bo_n = col_frag<T, D>(ot, 16 * (last ? m + 1 : m), last ? 0 : 32 * (dt + 1), lane);
              bq_n = col_frag<T, D>(qt, 16 * (last ? m + 1 : m), last ? 0 : 32 * (dt + 1), lane);
            }
            dv[dt] = mma(bo, pa, dv[dt]);
            dk[dt] = mma(bq, da, dk[dt]);
            if (m == 0)
#pragma unroll
              for (int e = PER * dt; e < PER * dt + PER; e += 2) pair(1, e);
            bo = bo_n;
            bq = bq_n;
            __builtin_amdgcn_sched_barrier(0);
          }
          pa = __builtin_bit_cast(Frag<T>, pw);
          da = __builtin_bit_cast(Frag<T>, dw);
        }
      }
    }
  };

  int buf = 0, g_bias = -1;
  if (g < g_end) {
    if constexpr (F32) {
      load_stage(g, t);
      store_stage(0);
    }
    store_rows(0);
  }
  if constexpr (F32) __syncthreads();
  while (g < g_end) {
    const bool masked = (int64_t)t * BQ < q_full;
    bool by_doc = false, absent = false;
    if (sa.q_doc) {
      const int2 of = docs.of_tile(t);
      by_doc = ids.z || docs.mixed(of);
      absent = of.x < 0;
    }
    int gn = g, tn = t;
    advance(gn, tn);
    const bool more = gn < g_end;
    if constexpr (!F32) {
      wait_global_loads();
      __syncthreads();
    }
    if constexpr (BIAS) {
      if (g != g_bias) {  // the heads' biases take turns
        if (sa.slopes) slope = sa.slopes[head_of(g)] * (kLog2eF / unit);
        if (sa.table) {
          fill_bias(sa, lds_bias, 1, head_of(g), tid, C::NT);
          __syncthreads();
        }
        g_bias = g;
      }
    }
    if (more) {
      load_rows(gn, tn);
      if constexpr (F32) load_stage(gn, tn);
      else copy_tile(gn, tn, buf ^ 1);
    }
    if (absent) {
      LE* st = reinterpret_cast<LE*>(smem + buf * C::STAGE_BYTES);
      constexpr int RS = F32 ? C::RS : D, PL = F32 ? C::TILE : 0;
      zero_absent<LE, D, RS, RS, PL, PL, F32 ? C::NP : 1>(st, st + C::TILE_BYTES / 2, sa.q_doc + (int64_t)b * p.n_q, (int64_t)t * BQ,
                                                         p.n_q, 0, BQ, tid, C::NT);
      __syncthreads();
    }
    compute(t, buf, masked, by_doc);
    const int nb = NBUF == 2 ? buf ^ 1 : 0;
    if constexpr (F32) {
      if (NBUF == 1) __syncthreads();
      if (more) {
        store_stage(nb);
        store_rows(nb);
      }
      __syncthreads();
    } else {
      if (more) store_rows(nb);
    }
    buf = nb;
    g = gn;
    t = tn;
  }

  if (key >= p.n_k) return;
  if (p.dk_part) {
    const int64_t at = ((((int64_t)part * p.n_b + b) * p.heads_kv + kvh) * p.n_k + key) * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int a4 = 0; a4 < 4; ++a4) {
        f32x4 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = live ? dk[dt][4 * a4 + e] : 0.0f;
          y[e] = live ? dv[dt][4 * a4 + e] : 0.0f;
        }
        *reinterpret_cast<f32x4*>(p.dk_part + at + 32 * dt + 8 * a4 + 4 * h) = x;
        *reinterpret_cast<f32x4*>(p.dv_part + at + 32 * dt + 8 * a4 + 4 * h) = y;
      }
    return;
  }
  T* dkg = static_cast<T*>(p.dk) + (int64_t)b * p.sdk.b + (int64_t)kvh * p.sdk.h + key * p.sdk.r;
  T* dvg = static_cast<T*>(p.dv) + (int64_t)b * p.sdv.b + (int64_t)kvh * p.sdv.h + key * p.sdv.r;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int a4 = 0; a4 < 4; ++a4) {
      typename FragT<T>::half x, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = (T)(live ? dk[dt][4 * a4 + e] * p.scale : 0.0f);
        y[e] = (T)(live ? dv[dt][4 * a4 + e] : 0.0f);
      }
      *reinterpret_cast<typename FragT<T>::half*>(dkg + 32 * dt + 8 * a4 + 4 * h) = x;
      *reinterpret_cast<typename FragT<T>::half*>(dvg + 32 * dt + 8 * a4 + 4 * h) = y;
    }
}

// ------------------------------------------------------------------- dQ
template <typename T, int D>
struct ScoredDqTile {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NT = 256, ROWS = kScoredDqRows;
  static constexpr int BK = !F32 && D == 64 ? 64 : 32;
  static constexpr int NP = Planes<T>::NP;
  static constexpr int RS = D + 8, TILE = BK * RS;
  static constexpr int TILE_BYTES = F32 ? NP * TILE * 2 : BK * D * 2;
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
  static constexpr int OCC = F32 && D == 128 ? 1 : 2;
  // The bias by place; its gradient takes 4 waves' sums by place and 32 KiB more.
  static constexpr int kBiasMax = 4 * (2 * kMaxBiasSpan + 1 + 2 * kPad) + 16;
  static constexpr int NBUF = 2 * STAGE_BYTES + 5 * kBiasMax + 32768 <= 160 * 1024 - 1280 ? 2 : 1;
  static constexpr int LDS_BYTES = NBUF * STAGE_BYTES;
  static constexpr int CPR = D / 8, CHUNKS = 2 * BK * CPR, CPT = CHUNKS / NT;
  static_assert(CHUNKS % NT == 0, "tile shapes");
  static_assert(F32 || NBUF == 2, "asynchronous copies need two stages");
};

template <typename T, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void dq_workgroup(const ScoredBwdParams& p, int block, int n_blocks) {
  using C = ScoredDqTile<T, D>;
  using LE = typename Planes<T>::E;
  constexpr bool F32 = C::F32;
  constexpr bool KEEP = CAP && (BIAS || D == 64);  // 1 - tanh^2 is kept, else (registers) made again from the score
  constexpr int BK = C::BK, KC = D / 16, NKT = BK / 32, NDT = D / 32, NBUF = C::NBUF;

  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* const lds_bias = smem + C::LDS_BYTES;
  __shared__ int4 wave_ids[4];
  __shared__ __align__(16) int tile_ids[4][32];
  __shared__ float far_sums[8];

  const ScoreArgs& sa = p.s;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int h = lane >> 5, c = lane & 31;

  const TileItem item = tile_item(block, n_blocks, p.n_qtiles, sa.causal ? p.tile_order : 0);
  const int qtile = sa.causal ? p.n_qtiles - 1 - item.tile : item.tile;
  // Heads that share a key head are neighbours, then batches.
  const int gi = item.group / p.heads_per_kv;
  const int b = gi % p.n_b, kvh = gi / p.n_b % p.heads_kv, part = gi / (p.n_b * p.heads_kv);
  const int head = kvh * p.heads_per_kv + item.group % p.heads_per_kv;
  const int64_t q0 = (int64_t)qtile * C::ROWS, qw = q0 + 32 * wave, qi = qw + c;
  const int64_t q_last = (q0 + C::ROWS < p.n_q ? q0 + C::ROWS : p.n_q) - 1;

  const int64_t n_kv = batch_keys(sa, b, p.n_k), pos0 = first_pos(sa, b);
  const int64_t row = ((int64_t)b * sa.heads + head) * p.n_q_pad + qi;
  const bool in_rows = qi < p.n_q;
  const float l2 = in_rows ? p.lse2[row] : INFINITY, neg_d = in_rows ? p.neg_d[row] : 0.0f;
  const int64_t reach = key_reach(sa, b, p.n_k);
  const int pos = (int)(pos0 + qi);
  int lim = in_rows && l2 != INFINITY ? (int)key_limit(n_kv, reach, pos0 + qi) : 0;
  const int64_t lim_hi = key_limit(n_kv, reach, pos0 + q_last), lim_lo = key_limit(n_kv, reach, pos0 + q0);
  const int64_t w_last = qw + 31 < p.n_q ? qw + 31 : p.n_q - 1;
  const int64_t w_lim = qw < p.n_q ? key_limit(n_kv, reach, pos0 + w_last) : 0;

  int doc = -2;
  int4 ids = make_int4(0, 0, 0, 0);
  if (sa.q_doc) {
    doc = in_rows ? sa.q_doc[(int64_t)b * p.n_q + qi] : -1;
    if (doc < 0) {
      doc = -2;
      lim = 0;
    }
    ids = workgroup_ids(doc, wave, lane, wave_ids);
  }
  const bool live = lim > 0;
  const int n_units = (int)((p.n_k + 31) / 32);
  DocTiles<BK / 32> docs(sa.k_range ? sa.k_range + (int64_t)b * n_units : nullptr, n_units, ids.x, ids.y);

  const T* __restrict__ kg = static_cast<const T*>(p.k) + (int64_t)b * p.sk.b + (int64_t)kvh * p.sk.h;
  const T* __restrict__ vg = static_cast<const T*>(p.v) + (int64_t)b * p.sv.b + (int64_t)kvh * p.sv.h;
  constexpr int CPR = C::CPR;
  const TileCopy<std::conditional_t<F32, __bf16, T>, D, BK, false> copies(wave, lane, p.sk.r, p.sv.r);
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
    if constexpr (!F32)
      copies(kg, p.sk.r, vg, p.sv.r, (int64_t)t * BK, lim_hi,
             __builtin_amdgcn_readfirstlane(lds_addr(smem + buf * C::STAGE_BYTES)), wave);
  };
  Range<T, false> range;
  Chunk8<T> stage[F32 ? C::CPT : 1];
  auto load_stage = [&](int t) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < C::CPT; ++i) {
        const int chunk = tid + i * C::NT;
        const bool is_v = chunk >= BK * CPR;
        const int rem = is_v ? chunk - BK * CPR : chunk;
        const int r = rem / CPR, col = rem % CPR;
        const int64_t key = (int64_t)t * BK + r;
        const T* src = is_v ? vg + key * p.sv.r : kg + key * p.sk.r;
        stage[i] = key < lim_hi ? ld_chunk8<T, T>(src + 8 * col) : zero_chunk8<T>();
      }
    }
  };
  auto store_stage = [&](int buf) __attribute__((always_inline)) {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < C::CPT; ++i) {
        const int chunk = tid + i * C::NT;
        const bool is_v = chunk >= BK * CPR;
        const int rem = is_v ? chunk - BK * CPR : chunk;
        st_chunk8<T>(reinterpret_cast<LE*>(smem + buf * C::STAGE_BYTES + (is_v ? C::TILE_BYTES : 0)) + rem / CPR * C::RS +
                         8 * (rem % CPR),
                     C::TILE, stage[i], range);
      }
    }
  };

  // The first tile is on its way while the rest is set up.
  const int64_t t_all = (lim_hi + BK - 1) / BK;
  const int t_end = (int)(t_all * (part + 1) / p.dq_parts);
  int t = docs.next((int)(t_all * part / p.dq_parts), t_end), buf = 0;
  if constexpr (!F32)
    if (t < t_end) copy_tile(t, 0);

  const float unit = sa.unit;
  const float slope = BIAS && sa.slopes ? sa.slopes[head] * (kLog2eF / unit) : 0.0f;
  const int places = BIAS ? bias_places(sa) : 0;
  const bool sums = BIAS && p.table_part;
  // For the bias gradient: sums by place of each wave, and each wave's 32 x 64 skewed
  // tile: dS of row c and key x at column x - c + 31, so that a column is a diagonal;
  // the places that no pair has stay 0.
  float* const bins = reinterpret_cast<float*>(lds_bias + bias_lds_bytes(sa, 1));
  float* const my_bins = bins + wave * places;
  float* const skew = bins + 4 * places + 2048 * wave;
  if (BIAS && sa.table) {
    fill_bias(sa, lds_bias, 1, head, tid, C::NT);
    if (sums)
      for (int x = tid; x < places + 2048; x += C::NT) reinterpret_cast<f32x4*>(bins)[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  Frag<T> qf[KC], gf[KC];
  {
    const T* qg = static_cast<const T*>(p.q) + (int64_t)b * p.sq.b + (int64_t)head * p.sq.h + qi * p.sq.r;
    const T* og = static_cast<const T*>(p.d_o) + (int64_t)b * p.sdo.b + (int64_t)head * p.sdo.h + qi * p.sdo.r;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      qf[kc] = live ? ld_frag_as<T, T>(qg + 16 * kc + 8 * h, range) : zero_frag<T>();
      gf[kc] = live ? ld_frag_as<T, T>(og + 16 * kc + 8 * h, range) : zero_frag<T>();
    }
  }
  f32x16 acc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[dt][r] = 0.0f;
  float far_lo = 0.0f, far_hi = 0.0f;
  __syncthreads();  // the bias is there

  const int krow = perm32(c);
  const int64_t p_lo = pos0 + qw, p_hi = pos0 + w_last;  // the wave's positions

  auto tile = [&](int t, int buf, bool masked, bool by_doc) __attribute__((always_inline)) {
    const unsigned char* st = smem + buf * C::STAGE_BYTES;
#pragma unroll 1
    for (int kt = 0; kt < NKT; ++kt) {
      const int64_t k0 = (int64_t)t * BK + 32 * kt;
      if (k0 >= w_lim) return;
      const unsigned char* kt16 = st + kt * 32 * (2 * D);
      const unsigned char* vt16 = kt16 + C::TILE_BYTES;
      const LE* kt32 = reinterpret_cast<const LE*>(st) + kt * 32 * C::RS;
      const LE* vt32 = reinterpret_cast<const LE*>(st + C::TILE_BYTES) + kt * 32 * C::RS;
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = 0.0f;
        dp[r] = neg_d;
      }
      if constexpr (F32) {
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          s = mma(lds_frag_planes<T>(kt32 + krow * C::RS + 16 * kc + 8 * h, C::TILE), qf[kc], s);
          dp = mma(lds_frag_planes<T>(vt32 + krow * C::RS + 16 * kc + 8 * h, C::TILE), gf[kc], dp);
        }
      } else {
        Frag<T> fa[2], fg[2];
        fa[0] = row_frag<T, D>(kt16, krow, h);
        fg[0] = row_frag<T, D>(vt16, krow, h);
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          if (kc + 1 < KC) {
            fa[(kc + 1) & 1] = row_frag<T, D>(kt16, krow, 2 * (kc + 1) + h);
            fg[(kc + 1) & 1] = row_frag<T, D>(vt16, krow, 2 * (kc + 1) + h);
          }
          s = mma(fa[kc & 1], qf[kc], s);
          dp = mma(fg[kc & 1], gf[kc], dp);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      float grad[KEEP ? 16 : 1];
      if constexpr (CAP) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = cap_tanh<T>(sa, s[r]);
          if constexpr (KEEP) grad[r] = fmaf(-s[r], s[r], 1.0f);
        }
      }
      float add = 0.0f;  // what every pair gets
      const int off = BIAS ? (int)k0 - pos + 8 * h : 0;  // distance of the lane's first key
      const int hi = bias_ahead(sa);
      const bool far = BIAS && (k0 + 31 <= p_lo - sa.span || k0 >= p_hi + hi);
      if constexpr (BIAS) {
        if (sa.slopes) {
          if (k0 + 31 <= p_lo) {
            add = (float)off * slope;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf((float)permuted_row(r, 0), slope, s[r]);
          } else {
            float d0 = (float)off;
            stay(d0);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = fmaf(-fabsf(d0 + (float)permuted_row(r, 0)), slope, s[r]);
          }
        }
        if (sa.table) {
          if (far) {
            add += reinterpret_cast<const float*>(lds_bias)[k0 >= p_hi + hi ? places - 1 : 0];
          } else {
            int from = off + sa.span + kPad;
            stay(from);
            const float* at = reinterpret_cast<const float*>(lds_bias) + from;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] += at[permuted_row(r, 0)];
          }
        }
      }
      if (masked) {
        int m = lim - (int)k0 - 8 * h;
        stay(m);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (permuted_row(r, 0) >= m) s[r] = -INFINITY;
      }
      if (by_doc) {
        const int mine = k0 + c < p.n_k ? sa.k_doc[(int64_t)b * p.n_k + k0 + c] : -1;
        hide_documents(s, doc, mine, tile_ids[wave], lane);
      }
      const float neg = BIAS ? fmaf(add, unit, -l2) : -l2;
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] *= fast_exp2(fmaf(s[r], unit, neg));  // dS
      if constexpr (BIAS) {
        if (sums) {
          if (far) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = dp[e] + dp[8 + e];
            const float x = tree_sum<8>(y, 0.0f);
            if (k0 >= p_hi + hi) far_hi += x;
            else far_lo += x;
          } else {
            // A lane adds a diagonal of the wave's tile.  (LDS atomics by distance took 166
            // cycles an instruction; this takes 48 reads and writes for 16 of them.)
            float* const to = skew + 63 * c + 31 + 8 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) to[permuted_row(r, 0)] = dp[r];
            float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int x = 0; x < 32; ++x) y[x & 3] += skew[64 * x + lane];
            my_bins[(int)(k0 - p_lo) + lane - 31 + sa.span + kPad] += (y[0] + y[1]) + (y[2] + y[3]);
          }
        }
      }
      if constexpr (CAP)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if constexpr (KEEP) dp[r] *= grad[r];
          else dp[r] *= cap_grad(s[r]);
        }
      Frag<T> sf[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = dp[8 * m + e];
        sf[m] = to_frag<T>(x);
      }
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          if constexpr (F32) acc[dt] = mma(lds_col_frag_planes<T>(kt32, C::TILE, C::RS, 16 * m, 32 * dt, lane), sf[m], acc[dt]);
          else acc[dt] = mma(col_frag<T, D>(kt16, 16 * m, 32 * dt, lane), sf[m], acc[dt]);
        }
    }
  };

  if constexpr (F32) {
    if (t < t_end) {
      load_stage(t);
      store_stage(0);
    }
    __syncthreads();
  }
  while (t < t_end) {
    const int tn = docs.next(t + 1, t_end);
    const bool masked = (int64_t)(t + 1) * BK > lim_lo;
    bool by_doc = false, absent = false;
    if (sa.q_doc) {
      const int2 of = docs.of_tile(t);
      by_doc = ids.z || docs.mixed(of);
      absent = of.x < 0;
    }
    if constexpr (F32) {
      if (tn < t_end) load_stage(tn);
    } else {
      wait_global_loads();
      __syncthreads();
      if (tn < t_end) copy_tile(tn, buf ^ 1);
    }
    if (absent) {
      LE* st = reinterpret_cast<LE*>(smem + buf * C::STAGE_BYTES);
      constexpr int RS = F32 ? C::RS : D, PL = F32 ? C::TILE : 0;
      zero_absent<LE, D, RS, RS, PL, PL, F32 ? C::NP : 1>(st, st + C::TILE_BYTES / 2, sa.k_doc + (int64_t)b * p.n_k, (int64_t)t * BK,
                                                         lim_hi, 0, BK, tid, C::NT);
      __syncthreads();
    }
    tile(t, buf, masked, by_doc);
    const int nb = NBUF == 2 ? buf ^ 1 : 0;
    if constexpr (F32) {
      if (NBUF == 1) __syncthreads();
      if (tn < t_end) store_stage(nb);
      __syncthreads();
    }
    buf = nb;
    t = tn;
  }

  if (in_rows && p.dq_part) {
    float* to = p.dq_part + ((((int64_t)part * p.n_b + b) * sa.heads + head) * p.n_q + qi) * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int a4 = 0; a4 < 4; ++a4) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = live ? acc[dt][4 * a4 + e] : 0.0f;
        *reinterpret_cast<f32x4*>(to + 32 * dt + 8 * a4 + 4 * h) = x;
      }
  } else if (in_rows) {
    T* dqg = static_cast<T*>(p.dq) + (int64_t)b * p.sdq.b + (int64_t)head * p.sdq.h + qi * p.sdq.r;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int a4 = 0; a4 < 4; ++a4) {
        typename FragT<T>::half x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (T)(live ? acc[dt][4 * a4 + e] * p.scale : 0.0f);
        *reinterpret_cast<typename FragT<T>::half*>(dqg + 32 * dt + 8 * a4 + 4 * h) = x;
      }
  }

  if constexpr (BIAS) {
    if (!sums) return;
    // The workgroup's sums by bucket: by place over the waves in order, then
    // a bucket's places in order.  Places beyond the span belong to the last bucket of
    // their side, as do the far sums (with keys ahead at distance 0: to bucket 0).
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      far_lo += __shfl_xor(far_lo, o);
      far_hi += __shfl_xor(far_hi, o);
    }
    if (lane == 0) {
      far_sums[wave] = far_lo;
      far_sums[4 + wave] = far_hi;
    }
    __syncthreads();
    for (int x = tid; x < places; x += C::NT) {
      float y = bins[x];
#pragma unroll
      for (int w = 1; w < 4; ++w) y += bins[w * places + x];
      if (x == 0) y += (far_sums[0] + far_sums[1]) + (far_sums[2] + far_sums[3]);
      if (x == places - 1) y += (far_sums[4] + far_sums[5]) + (far_sums[6] + far_sums[7]);
      bins[x] = y;
    }
    __syncthreads();
    const int nb = sa.n_edges * (sa.two_sided ? 2 : 1), zero = sa.span + kPad;  // place of distance 0
    // Workgroups of one head are neighbours in table_part: [head][batch][query tile][part].
    float* const to = p.table_part + ((((int64_t)head * p.n_b + b) * p.n_qtiles + qtile) * p.dq_parts + part) * nb;
    // 8 lanes a bucket: a chain of reads by one took 3 us where a bucket has 100 places.
    for (int e0 = 0; e0 < nb; e0 += C::NT / 8) {
      const int e = e0 + tid / 8;
      const bool ahead = e >= sa.n_edges;
      const int s = e >= nb ? 0 : (ahead ? e - sa.n_edges : e);
      // Its places [lo, end).
      int lo = s + 1 < sa.n_edges ? sa.edges[s] : sa.span, end = s + 1 < sa.n_edges ? sa.edges[s + 1] : sa.span + 1 + kPad;
      if (ahead) {
        lo = zero + (lo > 0 ? lo : 1);  // distance 0 is behind
        end = zero + end;
      } else {
        const int from = zero - end + 1;
        end = s == 0 && !sa.two_sided ? places : zero - lo + 1;
        lo = from;
      }
      if (e >= nb) end = lo;
      float y = 0.0f;
      for (int x = lo + (tid & 7); x < end; x += 8) y += bins[x];
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) y += __shfl_xor(y, o);
      if (e < nb && (tid & 7) == 0) to[e] = y;
    }
  }
}

// dK/dV (the first n_kv workgroups) and dQ in one launch, where each fills what the
// other leaves of the chip.  PARTS 1 and 2, a launch each, for larger float32 grids at
// d = 64, where dQ alone has two workgroups per CU and dK/dV one.  Backward in us, two
// launches / one: bf16 d = 64 4x16 heads, 4096 causal 676 / 657, 16x12, 512 121 / 99, 15x15
// on 5, 1199 518 / 497; d = 128 2x16 on 4, 4096 causal 673 / 655, 3x24 on 3, 897 129 / 121,
// 2x32 on 8, 4096 1032 / 1050; float32 d = 64 1x4, 64 39 / 24, 2x8 on 4, 700 75 / 79, 4x8, 2000
// 381 / 436; d = 128 4x8, 2000 952 / 929.
template <typename T, int D, bool CAP, bool BIAS, int PARTS>
__global__ __launch_bounds__(256, PARTS == 2 ? (ScoredDqTile<T, D>::OCC) : (ScoredKvTile<T, D>::OCC))
void scored_bwd_kernel(ScoredBwdParams p, int n_kv) {
  const int block = (int)blockIdx.x;
  if constexpr (PARTS & 1)
    if (block < n_kv) dkdv_workgroup<T, D, CAP, BIAS>(p, block, n_kv);
  if constexpr (PARTS & 2)
    if (block >= n_kv) dq_workgroup<T, D, CAP, BIAS>(p, block - n_kv, (int)gridDim.x - n_kv);
}

// The parts' sums, added in order, scaled and rounded: blocks of rows of dK, of dV, of
// dQ; a thread per row and 4 features.
template <typename T, int D>
__global__ __launch_bounds__(256) void scored_bwd_sum_kernel(ScoredBwdParams p, int64_t kv_blocks) {
  constexpr int G4 = D / 4;
  int64_t block = blockIdx.x;
  const int which = p.dk_part ? (block < kv_blocks ? 0 : (block < 2 * kv_blocks ? 1 : 2)) : 2;
  if (p.dk_part) block -= which * kv_blocks;
  const int heads = which == 2 ? p.s.heads : p.heads_kv, parts = which == 2 ? p.dq_parts : p.kv_heads_parts * p.kv_query_parts;
  const int64_t n = which == 2 ? p.n_q : p.n_k, rows = (int64_t)p.n_b * heads * n;
  const int64_t gid = block * 256 + threadIdx.x, row = gid / G4;
  const int f0 = 4 * (int)(gid % G4);
  if (row >= rows) return;
  const float* from = (which == 0 ? p.dk_part : which == 1 ? p.dv_part : p.dq_part) + row * D + f0;
  f32x4 x = *reinterpret_cast<const f32x4*>(from);
  for (int i = 1; i < parts; ++i) x += *reinterpret_cast<const f32x4*>(from + (int64_t)i * rows * D);
  const TensorStrides st = which == 0 ? p.sdk : which == 1 ? p.sdv : p.sdq;
  T* to = static_cast<T*>(which == 0 ? p.dk : which == 1 ? p.dv : p.dq) + row / n / heads * st.b + row / n % heads * st.h +
          row % n * st.r + f0;
  const float f = which == 1 ? 1.0f : p.scale;
  typename FragT<T>::half y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (T)(x[e] * f);
  *reinterpret_cast<typename FragT<T>::half*>(to) = y;
}

// ------------------------------------------------------------------ launchers
template <typename T, int D>
static hipError_t launch_scored_sum(const ScoredBwdParams& p, hipStream_t stream) {
  ScoredBwdParams a = p;
  auto blocks = [](int64_t rows) { return (rows * (D / 4) + 255) / 256; };
  int64_t kv = blocks((int64_t)p.n_b * p.heads_kv * p.n_k);
  const int64_t grid = (p.dk_part ? 2 * kv : 0) + (p.dq_part ? blocks((int64_t)p.n_b * p.s.heads * p.n_q) : 0);
  if (!grid) return hipSuccess;
  void* args[] = {&a, &kv};
  return hipLaunchKernel(reinterpret_cast<const void*>(scored_bwd_sum_kernel<T, D>), dim3((unsigned)grid), dim3(256), args, 0,
                         stream);
}
template <typename T, int D, bool CAP, bool BIAS>
static hipError_t launch_scored_bwd_kernels(const ScoredBwdParams& p, hipStream_t stream) {
  using K = ScoredKvTile<T, D>;
  using Q = ScoredDqTile<T, D>;
  ScoredBwdParams a = p;
  a.n_ktiles = (int)((p.n_k + K::BKG - 1) / K::BKG);
  a.n_qtiles = (int)((p.n_q + Q::ROWS - 1) / Q::ROWS);
  const int64_t kv_wgs = p.dk ? (int64_t)a.n_ktiles * p.n_b * p.heads_kv * p.kv_heads_parts * p.kv_query_parts : 0;
  const int64_t q_wgs = p.dq ? (int64_t)a.n_qtiles * p.n_b * p.s.heads * p.dq_parts : 0;
  const int bias = bias_lds_bytes(p.s, 1), bins = p.table_part ? (4 * bias_places(p.s) + 8192) * 4 : 0;
  const int kv_lds = K::LDS_BYTES + bias, q_lds = Q::LDS_BYTES + bias + bins;
  int n_kv = (int)kv_wgs;
  void* args[] = {&a, &n_kv};
  static_assert(Q::OCC >= K::OCC, "one launch has dK/dV's registers");
  auto launch = [&](auto parts, int64_t grid, int lds) {
    return hipLaunchKernel(reinterpret_cast<const void*>(scored_bwd_kernel<T, D, CAP, BIAS, decltype(parts)::value>),
                           dim3((unsigned)grid), dim3(256), args, lds, stream);
  };
  hipError_t e = hipSuccess;
  bool one = true;
  if constexpr (Q::OCC > K::OCC) {
    one = kv_wgs && q_wgs && kv_wgs + q_wgs <= 256;
    if (!one && kv_wgs) e = launch(std::integral_constant<int, 1>{}, kv_wgs, kv_lds);
    n_kv = one ? n_kv : 0;
    if (!one && q_wgs && e == hipSuccess) e = launch(std::integral_constant<int, 2>{}, q_wgs, q_lds);
  }
  if (one) {
    const int lds = !q_wgs || (kv_wgs && kv_lds > q_lds) ? kv_lds : q_lds;
    e = launch(std::integral_constant<int, 3>{}, kv_wgs + q_wgs, lds);
  }
  if (e == hipSuccess && p.table_part) e = launch_scored_table(a, stream);
  return e != hipSuccess ? e : launch_scored_sum<T, D>(a, stream);
}
template <typename T, int D>
static hipError_t launch_scored_bwd_d(const ScoredBwdParams& p, hipStream_t stream) {
  ScoredBwdParams a = p;
  void* args[] = {&a};
  constexpr int RPB = 256 / (D * (int)sizeof(T) / 16);
  const int64_t rows = (int64_t)p.n_b * p.s.heads * p.n_q_pad;
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(scored_bwd_pre_kernel<T, D>),
                                       dim3((unsigned)((rows + RPB - 1) / RPB)), dim3(256), args, 0, stream);
  if (e != hipSuccess) return e;
  const bool cap = p.s.capped, bias = p.s.slopes || p.s.table;
  if (cap)
    return bias ? launch_scored_bwd_kernels<T, D, true, true>(p, stream)
                : launch_scored_bwd_kernels<T, D, true, false>(p, stream);
  return bias ? launch_scored_bwd_kernels<T, D, false, true>(p, stream)
              : launch_scored_bwd_kernels<T, D, false, false>(p, stream);
}
template <typename T>
hipError_t launch_scored_bwd(const ScoredBwdParams& p, int d, hipStream_t stream) {
  return d == 64 ? launch_scored_bwd_d<T, 64>(p, stream) : launch_scored_bwd_d<T, 128>(p, stream);
}

}  // namespace mea
