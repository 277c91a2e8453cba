// The stream kernel: rows of queries against keys with the lazy softmax
// (arXiv 2112.05682, Sections 2-4) of modified scores (scored.hpp).
//
// A workgroup is 4 waves.  RW of them own 32 rows each, and with RW < 4 the
// others take shares of the same rows' keys (KW = 4 / RW), whose summaries are
// combined in LDS.  S^T = K Q^T puts a row on each lane, so that a row's limit,
// position, document, slope and softmax state are scalars of the lane.  16-bit
// K and V tiles go to LDS by asynchronous copies into swizzled rows, two stages;
// with RW = 1 a wave copies the keys it reads, so that the waves run without a
// barrier.  float32 tiles are split into their three parts on the way.
//
// What bounds it: many rows, the vector unit (exponentials, with a cap two and a
// reciprocal a pair; counters: VALU 72 %, MFMA 33 % of the time with work).  Causal, 16-bit: cap,
// 2x16 heads on 4, 4096, d = 128 212 us, 650 TFLOP/s; learned bias, 4x16x4096, d = 64 194 us,
// 710 TFLOP/s.  32 keys a tile, or other workgroups per CU, took 209-234 us for the former.
// Few rows, memory: 16x32 heads on 8, 32768 keys of d = 128 232 us, 5.9 TB/s (a read
// alone: 6.9); 8x32 on 8, 65536 of d = 64 162 us, 6.6 TB/s.
#pragma once

#include "scored.hpp"
#include "scored_few.hpp"

namespace mea {

template <typename T, int D, int RW>
struct StreamTile {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NT = 256, KW = 4 / RW, ROWS = 32 * RW;
  static constexpr int BK = stream_tile(!F32, RW), BKW = BK / KW;
  static constexpr int NP = Planes<T>::NP;
  // float32: padded rows of three bf16 planes (the pads as in FwdTile).
  static constexpr int RSK = D + 8, RSV = D + 32;
  static constexpr int TILEK = BK * RSK, TILEV = BK * RSV;
  static constexpr int STAGE_BYTES = F32 ? NP * (TILEK + TILEV) * 2 : 2 * BK * D * 2;
  // Workgroups per CU that the registers are kept to.
  static constexpr int OCC = F32 ? (D == 64 && RW == 4 ? 2 : 1) : (RW == 1 ? (D == 64 ? 2 : 1) : (D == 64 ? 3 : 2));
  static constexpr int kBiasMax = 4 * (2 * kMaxBiasSpan + 1 + 2 * kPad) + 16;
  static constexpr int NBUF = 2 * STAGE_BYTES + kBiasMax <= 160 * 1024 / OCC ? 2 : 1;
  static constexpr int ML_BYTES = 2 * 4 * 32 * 4;
  static constexpr int RED_BYTES = KW > 1 ? ML_BYTES + RW * (D / 32) * (KW - 1) * 4096 : 0;
  static constexpr int LDS_BYTES = NBUF * STAGE_BYTES > RED_BYTES ? NBUF * STAGE_BYTES : RED_BYTES;
  // Chunks a thread stages (float32).
  static constexpr int CPR = D / 8, CHUNKS = 2 * BK * CPR, CPT = CHUNKS / NT;
  static_assert(CHUNKS % NT == 0 && BKW % 32 == 0, "tile shapes");
  static_assert(F32 || NBUF == 2, "asynchronous copies need two stages");
  static_assert((LDS_BYTES + kBiasMax + 1280) * OCC <= 160 * 1024, "LDS");
};

// Workgroup `block` of n_blocks.
template <typename T, int D, int RW, bool CAP, bool BIAS>
__device__ __forceinline__ void stream_workgroup(const StreamParams& p, int block, int n_blocks) {
  using C = StreamTile<T, D, RW>;
  using LE = typename Planes<T>::E;
  constexpr bool F32 = C::F32;
  constexpr int KW = C::KW, BK = C::BK, BKW = C::BKW, KC = D / 16, NKT = BKW / 32, NPC = BKW / 16, NDT = D / 32;

  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* const lds_bias = smem + C::LDS_BYTES;
  __shared__ int4 wave_ids[4];
  __shared__ __align__(16) int tile_ids[4][32];

  const ScoreArgs& sa = p.s;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int h = lane >> 5, c = lane & 31;
  const int wave_q = RW == 4 ? wave : wave % RW, wave_k = RW == 4 ? 0 : wave / RW;

  // ---- workgroup -> row tile, group, key range.
  const TileItem item = tile_item(block, n_blocks, p.n_rtiles, p.tile_order);
  const int rtile = sa.causal ? p.n_rtiles - 1 - item.tile : item.tile;  // longest rows first
  const int split = item.group / p.n_groups;
  int gi = item.group % p.n_groups;
  const int sub = gi % p.groups_per_kv;
  gi /= p.groups_per_kv;
  const int b0 = gi % p.n_b, kvh = gi / p.n_b;
  const int head0 = kvh * p.heads_per_kv + sub * p.fold;

  // ---- this lane's row.  Rows of a group, keys and positions are below 2^31.
  const uint32_t n_rows = (uint32_t)p.group_rows, fold = (uint32_t)p.fold;
  const uint32_t row0 = (uint32_t)rtile * C::ROWS;
  const uint32_t row_last = (row0 + C::ROWS < n_rows ? row0 + C::ROWS : n_rows) - 1;
  const uint32_t row = row0 + 32 * wave_q + c;
  const bool in_rows = row < n_rows;
  const uint32_t rr = in_rows ? row : row_last;
  uint32_t g = 0, qu = rr;
  int b = b0;
  if (fold > 1) {
    qu = rr / fold;
    g = rr - qu * fold;
  }
  if (p.batches > 1) {
    const uint32_t x = qu / (uint32_t)p.n_q;
    qu -= x * (uint32_t)p.n_q;
    b = (int)x;
  }
  const int64_t qi = qu;
  const int head = head0 + (int)g;

  const int64_t n_kv = batch_keys(sa, b0, p.n_k);
  const int64_t pos0 = first_pos(sa, b0), reach = key_reach(sa, b0, p.n_k);
  const int pos = (int)(pos0 + qi);
  int lim = in_rows ? (int)key_limit(n_kv, reach, pos0 + qi) : 0;
  // Limits grow with the query, so the tile's first and last rows bound them (a
  // group of several batches has no positional mask: every limit is n_kv).
  auto pos_of = [&](uint32_t r) { return pos0 + (fold > 1 ? r / fold : r); };
  const int64_t lim_hi = key_limit(n_kv, reach, pos_of(row_last)), lim_lo = key_limit(n_kv, reach, pos_of(row0));
  const uint32_t w_row0 = row0 + 32 * wave_q;
  const bool wave_rows = w_row0 < n_rows;
  // The wave's first and last position (uniform), and its limit.
  const int64_t wq_lo = pos_of(w_row0), wq_hi = pos_of(w_row0 + 31 < n_rows ? w_row0 + 31 : n_rows - 1);
  const int64_t w_lim = wave_rows ? key_limit(n_kv, reach, wq_hi) : 0;

  int doc = -2;
  int4 ids = make_int4(0, 0, 0, 0);
  if (sa.q_doc) {
    if (in_rows) doc = sa.q_doc[(int64_t)b * p.n_q + qi];
    if (doc < 0) {
      doc = -2;
      lim = 0;
    }
    ids = workgroup_ids(doc, wave, lane, wave_ids);
  }
  constexpr int UNITS = BK / 32;
  const int n_units = (int)((p.n_k + 31) / 32);
  DocTiles<UNITS> docs(sa.k_range ? sa.k_range + (int64_t)b0 * n_units : nullptr, n_units, ids.x, ids.y);

  // ---- keys of this range: the visible tiles dealt evenly.
  const int all_tiles = (int)((lim_hi + BK - 1) / BK);
  const int per = (all_tiles + p.n_splits - 1) / p.n_splits;
  const int t0 = split * per;
  const int t1 = t0 + per < all_tiles ? t0 + per : all_tiles;
  const int64_t kb = p.batches > 1 ? 0 : (int64_t)b0;
  const T* __restrict__ kg = static_cast<const T*>(p.k) + kb * p.sk.b + (int64_t)kvh * p.sk.h;
  const T* __restrict__ vg = static_cast<const T*>(p.v) + kb * p.sv.b + (int64_t)kvh * p.sv.h;

  // ---- staging.  16-bit: copies of 1 KiB, rows past the last visible key repeat
  // it (finite, and masked); with RW = 1 each wave copies its own keys.
  constexpr int CPR = C::CPR;
  constexpr bool OWN = RW == 1;
  const TileCopy<std::conditional_t<F32, __bf16, T>, D, BK, OWN> copies(wave, lane, p.sk.r, p.sv.r);
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
      LE* base = reinterpret_cast<LE*>(smem + buf * C::STAGE_BYTES);
#pragma unroll
      for (int i = 0; i < C::CPT; ++i) {
        const int chunk = tid + i * C::NT;
        const bool is_v = chunk >= BK * CPR;
        const int rem = is_v ? chunk - BK * CPR : chunk;
        const int r = rem / CPR, col = rem % CPR;
        st_chunk8<T>(base + (is_v ? C::NP * C::TILEK + r * C::RSV : r * C::RSK) + 8 * col, is_v ? C::TILEV : C::TILEK,
                     stage[i], range);
      }
    }
  };

  // The first tile is on its way while the rest is set up.
  int t = docs.next(t0, t1), buf = 0;
  if constexpr (!F32)
    if (t < t1) copy_tile(t, 0);

  const float unit = sa.unit;
  const float slope = BIAS && sa.slopes ? sa.slopes[head] * (kLog2eF / unit) : 0.0f;
  if (BIAS && sa.table) fill_bias(sa, lds_bias, p.fold, head0, tid, C::NT);

  // ---- Q^T as B operands: lane (h, row c) holds features 16 kc + 8 h ..
  Frag<T> qf[KC];
  {
    const T* qg = static_cast<const T*>(p.q) + (int64_t)b * p.sq.b + (int64_t)head * p.sq.h + qi * p.sq.r;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
      qf[kc] = lim > 0 ? ld_frag_as<T, T>(qg + 16 * kc + 8 * h, range) : zero_frag<T>();
  }

  f32x16 acc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[dt][r] = 0.0f;
  float m_ref = -INFINITY, l_run = 0.0f;
  __syncthreads();  // the bias is there

  const int krow = perm32(c);

  // One tile: masked, some key is beyond some row's limit; by_doc, documents differ.
  // The masks are uniform branches of one copy of the code: with a copy each for plain
  // and masked tiles the d = 64 kernels spilled 84-173 registers in the loop.
  auto tile = [&](int t, int buf, bool masked, bool by_doc) __attribute__((always_inline)) {
    const int64_t k0 = (int64_t)t * BK + BKW * wave_k;
    if (k0 >= w_lim) return;  // all keys beyond this wave's rows
    const unsigned char* st = smem + buf * C::STAGE_BYTES;
    const LE* ks = reinterpret_cast<const LE*>(st) + BKW * wave_k * C::RSK;             // float32
    const LE* vs = reinterpret_cast<const LE*>(st) + C::NP * C::TILEK + BKW * wave_k * C::RSV;
    const unsigned char* kt16 = st + BKW * wave_k * (2 * D);                            // 16-bit
    const unsigned char* vt16 = st + BK * D * 2 + BKW * wave_k * (2 * D);

    f32x16 s[NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt][r] = 0.0f;
    f32x16 rest[F32 ? NKT : 1] = {};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        if constexpr (F32) {
          const Frag<T> a = lds_frag_planes<T>(ks + (32 * kt + krow) * C::RSK + 16 * kc + 8 * h, C::TILEK);
          rest[kt] = mma_rest(a, qf[kc], rest[kt]);
          s[kt] = mma(lead(a), lead(qf[kc]), s[kt]);
        } else {
          s[kt] = mma(row_frag<T, D>(kt16, 32 * kt + krow, 2 * kc + h), qf[kc], s[kt]);
        }
      }
    if constexpr (F32)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) s[kt] += rest[kt];

    // Cap and bias.  add: what every key of the tile gets.
    if constexpr (CAP) {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][r] = cap_tanh<T>(sa, s[kt][r]);
    }
    float add = 0.0f;
    if constexpr (BIAS) {
      const int off = (int)k0 - pos + 8 * h;  // distance of the lane's first key
      if (sa.slopes) {
        if (k0 + BKW - 1 <= wq_lo) {  // no key is ahead: -|d| = d
          add = (float)off * slope;
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = fmaf((float)(32 * kt + permuted_row(r, 0)), slope, s[kt][r]);
        } else {
          float d0 = (float)off;
          stay(d0);
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(-fabsf(d0 + (float)(32 * kt + permuted_row(r, 0))), slope, s[kt][r]);
        }
      }
      if (sa.table) {
        const int hi = bias_ahead(sa), last = bias_places(sa) - 1;
        if (k0 + BKW - 1 <= wq_lo - sa.span || k0 >= wq_hi + hi) {  // one value for every key of a row
          add += bias_at(sa, lds_bias, p.fold, (int)g, k0 >= wq_hi + hi ? last : 0);
        } else {
          int at_off = off;
          stay(at_off);
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt) {
            const int64_t ka = k0 + 32 * kt;
            if (ka + 31 <= wq_lo - sa.span || ka >= wq_hi + hi) {
              const float v = bias_at(sa, lds_bias, p.fold, (int)g, ka >= wq_hi + hi ? last : 0);
#pragma unroll
              for (int r = 0; r < 16; ++r) s[kt][r] += v;
            } else if (p.fold == 1) {
              const float* at = reinterpret_cast<const float*>(lds_bias) + (at_off + 32 * kt + sa.span + kPad);
#pragma unroll
              for (int r = 0; r < 16; ++r) s[kt][r] += at[permuted_row(r, 0)];
            } else {
#pragma unroll
              for (int r = 0; r < 16; ++r)
                s[kt][r] += bias_at(sa, lds_bias, p.fold, (int)g, at_off + 32 * kt + permuted_row(r, 0) + sa.span + kPad);
            }
          }
        }
      }
    }

    // Masks.
    if (masked) {
      int l = lim - (int)k0 - 8 * h;
      stay(l);
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kt + permuted_row(r, 0) >= l) s[kt][r] = -INFINITY;
    }
    if (by_doc) {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const int64_t key = k0 + 32 * kt + c;
        const int mine = key < p.n_k ? sa.k_doc[(int64_t)b0 * p.n_k + key] : -1;
        hide_documents(s[kt], doc, mine, tile_ids[wave], lane);
      }
    }

    // Lazy softmax, one row per lane (both halves hold keys of the same row).
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kt][r]);
    const float mx_c = xhalf_max(mx + add) * unit;  // (the halves' add differs with slopes)
    const bool raise = mx_c > m_ref + p.slack;
    if (__builtin_amdgcn_ballot_w64(raise)) {
      const float m_new = raise ? mx_c : m_ref;
      const float alpha = raise ? fast_exp2(m_ref - m_new) : 1.0f;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] *= alpha;
      m_ref = m_new;
    }
    // A row with no visible key so far: its exponents (all -inf, or add is) get weight 0.
    const float neg = m_ref == -INFINITY ? add : fmaf(add, unit, -m_ref);
    auto weight = [&](int pc, int e) __attribute__((always_inline)) {
      return fast_exp2(fmaf(s[pc >> 1][8 * (pc & 1) + e], unit, neg));
    };
    // O^T += V^T P^T.
    if constexpr (F32 || NDT > 2) {
      Frag<T> pf[NPC];
#pragma unroll
      for (int pc = 0; pc < NPC; ++pc) {
        float e8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) e8[e] = weight(pc, e);
        pf[pc] = to_frag<T>(e8);
        l_run = tree_sum<8>(e8, l_run);
      }
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        f32x16 sum = {};
#pragma unroll
        for (int pc = 0; pc < NPC; ++pc) {
          if constexpr (F32) sum = mma(lds_col_frag_planes<T>(vs, C::TILEV, C::RSV, 16 * pc, 32 * dt, lane), pf[pc], sum);
          else acc[dt] = mma(col_frag<T, D>(vt16, 16 * pc, 32 * dt, lane), pf[pc], acc[dt]);
        }
        if constexpr (F32) acc[dt] += sum;  // a tile's products are added once
      }
    } else {
      // 16 keys at a time; the next ones' weights are made between their products, a
      // share a step, and each step's fragment is read one step ahead (4x16 heads, 4096
      // causal, learned bias: 205 -> 194 us; at d = 128, whose products take longer, it took
      // 3 % more).
      constexpr int PER = 8 / NDT;
      float e8[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) e8[e] = weight(0, e);
      Frag<T> a = col_frag<T, D>(vt16, 0, 0, lane);
#pragma unroll
      for (int pc = 0; pc < NPC; ++pc) {
        const Frag<T> pf = to_frag<T>(e8);
        l_run = tree_sum<8>(e8, l_run);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          const bool last = dt + 1 == NDT;
          Frag<T> a_n = a;
          if (!last || pc + 1 < NPC) a_n = col_frag<T, D>(vt16, 16 * (last ? pc + 1 : pc), last ? 0 : 32 * (dt + 1), lane);
          acc[dt] = mma(a, pf, acc[dt]);
          if (pc + 1 < NPC)
#pragma unroll
            for (int e = PER * dt; e < PER * dt + PER; ++e) e8[e] = weight(pc + 1, e);
          a = a_n;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };

  // ---- the loop over the visible tiles of this range.
  if constexpr (F32) {
    if (t < t1) {
      load_stage(t);
      store_stage(0);
    }
    __syncthreads();
  }
  while (t < t1) {
    const int tn = docs.next(t + 1, t1);
    const bool masked = (int64_t)(t + 1) * BK > lim_lo;
    bool by_doc = false, absent = false;
    if (sa.q_doc) {
      const int2 of = docs.of_tile(t);
      by_doc = ids.z || docs.mixed(of);
      absent = of.x < 0;
    }
    if constexpr (F32) {
      if (tn < t1) load_stage(tn);
    } else {
      wait_global_loads();
      if constexpr (!OWN) __syncthreads();
      else wait_lds_reads();
      if (tn < t1) copy_tile(tn, buf ^ 1);
    }
    if (absent) {
      const int* kd = sa.k_doc + (int64_t)b0 * p.n_k;
      LE* st = reinterpret_cast<LE*>(smem + buf * C::STAGE_BYTES);
      if constexpr (F32)
        zero_absent<LE, D, C::RSK, C::RSV, C::TILEK, C::TILEV, C::NP>(st, st + C::NP * C::TILEK, kd, (int64_t)t * BK, lim_hi, 0, BK,
                                                                      tid, C::NT);
      else
        zero_absent<LE, D, D, D, 0, 0, 1>(st, st + BK * D, kd, (int64_t)t * BK, lim_hi, OWN ? BKW * wave : 0, OWN ? BKW : BK,
                                          OWN ? lane : tid, OWN ? 64 : C::NT);
      if constexpr (!OWN) __syncthreads();
    }
    tile(t, buf, masked, by_doc);
    if constexpr (F32) {
      if (C::NBUF == 1) __syncthreads();
      if (tn < t1) store_stage(C::NBUF == 1 ? 0 : buf ^ 1);
      __syncthreads();
    }
    if (C::NBUF == 2) buf ^= 1;
    t = tn;
  }

  // ---- KW > 1: one summary of the waves that share the rows, in their order.
  float l_sum = xhalf_sum(l_run);
  if constexpr (KW > 1) {
    __syncthreads();  // every wave is done with the stages
    float* red_m = reinterpret_cast<float*>(smem);
    float* red_l = red_m + 128;
    float* red_o = red_m + C::ML_BYTES / 4 + wave_q * NDT * (KW - 1) * 1024 + lane;
    if (h == 0) {
      red_m[wave * 32 + c] = m_ref;
      red_l[wave * 32 + c] = l_sum;
    }
    __syncthreads();
    float m_g = -INFINITY, l_g = 0.0f;
#pragma unroll
    for (int y = 0; y < KW; ++y) m_g = fmaxf(m_g, red_m[(wave_q + y * RW) * 32 + c]);
#pragma unroll
    for (int y = 0; y < KW; ++y) {
      const float m_y = red_m[(wave_q + y * RW) * 32 + c];
      l_g += (m_y == -INFINITY ? 0.0f : fast_exp2(m_y - m_g)) * red_l[(wave_q + y * RW) * 32 + c];
    }
    const float f = m_ref == -INFINITY ? 0.0f : fast_exp2(m_ref - m_g);
    m_ref = m_g;
    l_sum = l_g;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] *= f;
      if (dt % KW != wave_k)
#pragma unroll
        for (int r = 0; r < 16; ++r) red_o[((dt * (KW - 1) + wave_k - (wave_k > dt % KW)) * 16 + r) * 64] = acc[dt][r];
    }
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
      if (dt % KW == wave_k)
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
          for (int y = 0; y < KW - 1; ++y) acc[dt][r] += red_o[((dt * (KW - 1) + y) * 16 + r) * 64];
  }

  // ---- epilogue.
  if (!in_rows) return;
  const int64_t out_row = ((int64_t)b * sa.heads + head) * p.n_q + qi;
  if (p.direct) {
    const float inv = l_sum == 0.0f ? 0.0f : 1.0f / l_sum;  // no visible key: o = 0
    T* og = static_cast<T*>(p.o) + (int64_t)b * p.so.b + (int64_t)head * p.so.h + qi * p.so.r;
    T* gl = p.o_lo ? static_cast<T*>(p.o_lo) + out_row * D : nullptr;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      if (KW > 1 && dt % KW != wave_k) continue;
#pragma unroll
      for (int a4 = 0; a4 < 4; ++a4) {
        float x4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x4[e] = acc[dt][4 * a4 + e] * inv;
        const int f = 32 * dt + 8 * a4 + 4 * h;
        store_out4<T>(og + f, gl ? gl + f : nullptr, x4);
      }
    }
    if (h == 0 && wave_k == 0 && p.lse) p.lse[out_row] = l_sum == 0.0f ? -INFINITY : (m_ref + __log2f(l_sum)) * kLn2F;
  } else {
    const int64_t prow = (int64_t)(p.split0 + split) * p.out_rows + out_row;
    float* po = p.part_o + prow * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      if (KW > 1 && dt % KW != wave_k) continue;
#pragma unroll
      for (int a4 = 0; a4 < 4; ++a4) {
        f32x4 v4;
#pragma unroll
        for (int e = 0; e < 4; ++e) v4[e] = acc[dt][4 * a4 + e];
        *reinterpret_cast<f32x4*>(po + 32 * dt + 8 * a4 + 4 * h) = v4;
      }
    }
    if (h == 0 && wave_k == 0) {
      p.part_m[prow] = m_ref;
      p.part_l[prow] = l_sum;
    }
  }
}

template <typename T, int D, int RW, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, (StreamTile<T, D, RW>::OCC)) void scored_stream_kernel(StreamParams p) {
  stream_workgroup<T, D, RW, CAP, BIAS>(p, (int)blockIdx.x, (int)gridDim.x);
}

// A shared prefix (the first n_a workgroups) and the own keys in one launch, so that
// the one fills what the other leaves of the chip.
template <typename T, int D, int RWA, int RWB>
__global__ __launch_bounds__(256, (StreamTile<T, D, RWA>::OCC)) void scored_pair_kernel(StreamParams a, StreamParams b, int n_a) {
  if ((int)blockIdx.x < n_a) stream_workgroup<T, D, RWA, false, false>(a, (int)blockIdx.x, n_a);
  else stream_workgroup<T, D, RWB, false, false>(b, (int)blockIdx.x - n_a, (int)gridDim.x - n_a);
}

// Combine of the summaries of n_parts key ranges (Section 4): rescaled to the
// common maximum, added, divided.  A thread per row and 4 features; with SHARES > 1 the
// threads of a row take a share of the ranges each (of few rows and many ranges, a
// chain of loads is all it takes), whose sums meet in LDS, in order.
template <typename T, int D, int SHARES>
__global__ __launch_bounds__(256) void scored_combine_kernel(StreamParams p, int n_parts) {
  constexpr int G4 = D / 4, NT = 256 / SHARES, N = SHARES > 1 ? 4 : 8;
  const int share = threadIdx.x / NT, t = threadIdx.x % NT;
  const int64_t gid = (int64_t)blockIdx.x * NT + t;
  const bool in_rows = gid < p.out_rows * G4;
  const int64_t row = in_rows ? gid / G4 : 0;
  const int f0 = 4 * (int)(gid % G4);
  float m = -INFINITY, l = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](float mi, float li, f32x4 oi, float mx) {
    // (0 times a NaN denominator, a range of NaN scores only, stays NaN)
    const float w = mi == -INFINITY ? 0.0f : fast_exp2(mi - mx);
    l = fmaf(w, li, l);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(w, oi[e], o[e]);
  };
  auto rescale = [&](float mx) {
    const float a = m == -INFINITY ? 0.0f : fast_exp2(m - mx);
    l *= a;
    o *= a;
    m = mx;
  };
  // N ranges at a time, their loads in flight together.
  for (int s0 = share; s0 < n_parts; s0 += N * SHARES) {
    float ms[N], ls[N];
    f32x4 os[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool in = s0 + i * SHARES < n_parts;
      const int64_t at = (int64_t)(in ? s0 + i * SHARES : s0) * p.out_rows + row;
      ms[i] = p.part_m[at];
      ls[i] = p.part_l[at];
      os[i] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + f0);
      if (!in) ms[i] = -INFINITY;
    }
    float mx = m;
#pragma unroll
    for (int i = 0; i < N; ++i) mx = fmaxf(mx, ms[i]);
    rescale(mx);
#pragma unroll
    for (int i = 0; i < N; ++i) add(ms[i], ls[i], os[i], mx);
  }
  if constexpr (SHARES > 1) {
    __shared__ __align__(16) f32x4 os[SHARES][NT];
    __shared__ float ms[SHARES][NT], ls[SHARES][NT];
    os[share][t] = o;
    ms[share][t] = m;
    ls[share][t] = l;
    __syncthreads();
    if (share) return;
    float mx = m;
#pragma unroll
    for (int i = 1; i < SHARES; ++i) mx = fmaxf(mx, ms[i][t]);
    rescale(mx);
#pragma unroll
    for (int i = 1; i < SHARES; ++i) add(ms[i][t], ls[i][t], os[i][t], mx);
  }
  if (!in_rows) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  float x4[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) x4[e] = o[e] * inv;
  const int64_t qi = row % p.n_q, bh = row / p.n_q;
  T* og = static_cast<T*>(p.o) + bh / p.s.heads * p.so.b + bh % p.s.heads * p.so.h + qi * p.so.r;
  T* gl = p.o_lo ? static_cast<T*>(p.o_lo) + row * D : nullptr;
  store_out4<T>(og + f0, gl ? gl + f0 : nullptr, x4);
  if (f0 == 0 && p.lse) p.lse[row] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2F;
}

// ------------------------------------------------------------------ launchers
template <typename T, int D, int RWA, int RWB>
static hipError_t launch_pair_kernel(const StreamParams& a, const StreamParams& b, hipStream_t stream) {
  using A = StreamTile<T, D, RWA>;
  using B = StreamTile<T, D, RWB>;
  StreamParams x = a, y = b;
  x.n_rtiles = (int)((a.group_rows + A::ROWS - 1) / A::ROWS);
  y.n_rtiles = (int)((b.group_rows + B::ROWS - 1) / B::ROWS);
  constexpr int lds = A::LDS_BYTES > B::LDS_BYTES ? A::LDS_BYTES : B::LDS_BYTES;
  const int64_t n_a = (int64_t)x.n_rtiles * a.n_groups * a.n_splits, n_b = (int64_t)y.n_rtiles * b.n_groups * b.n_splits;
  if (n_a < 1 || n_b < 1 || n_a + n_b >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  int na = (int)n_a;
  void* args[] = {&x, &y, &na};
  return hipLaunchKernel(reinterpret_cast<const void*>(scored_pair_kernel<T, D, RWA, RWB>), dim3((unsigned)(n_a + n_b)),
                         dim3(256), args, lds, stream);
}
template <typename T, int D>
static hipError_t launch_pair_rows(const StreamParams& a, const StreamParams& b, int rwa, int rwb, hipStream_t stream) {
  if (rwa == 4 && rwb == 4) return launch_pair_kernel<T, D, 4, 4>(a, b, stream);
  if (rwa == 4 && rwb == 2) return launch_pair_kernel<T, D, 4, 2>(a, b, stream);
  if constexpr (sizeof(T) == 2) {
    if (rwa == 1 && rwb == 1) return launch_pair_kernel<T, D, 1, 1>(a, b, stream);
  } else {
    if (rwa == 2 && rwb == 2) return launch_pair_kernel<T, D, 2, 2>(a, b, stream);
  }
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t launch_stream_pair(const StreamParams& a, const StreamParams& b, int d, int rwa, int rwb, hipStream_t stream) {
  return d == 64 ? launch_pair_rows<T, 64>(a, b, rwa, rwb, stream) : launch_pair_rows<T, 128>(a, b, rwa, rwb, stream);
}

template <typename T, int D, int RW, bool CAP, bool BIAS>
static hipError_t launch_stream_kernel(const StreamParams& p, hipStream_t stream) {
  using C = StreamTile<T, D, RW>;
  StreamParams q = p;
  q.n_rtiles = (int)((p.group_rows + C::ROWS - 1) / C::ROWS);
  const int lds = C::LDS_BYTES + bias_lds_bytes(p.s, p.fold);
  const int64_t grid = (int64_t)q.n_rtiles * p.n_groups * p.n_splits;
  if (grid < 1 || grid >= ((int64_t)1 << 31) || lds > 160 * 1024 - 1280) return hipErrorInvalidValue;
  void* args[] = {&q};
  return hipLaunchKernel(reinterpret_cast<const void*>(scored_stream_kernel<T, D, RW, CAP, BIAS>), dim3((unsigned)grid),
                         dim3(C::NT), args, lds, stream);
}
template <typename T, int D, int RW>
static hipError_t launch_stream_mods(const StreamParams& p, hipStream_t stream) {
  const bool cap = p.s.capped, bias = p.s.slopes || p.s.table;
  if (cap)
    return bias ? launch_stream_kernel<T, D, RW, true, true>(p, stream)
                : launch_stream_kernel<T, D, RW, true, false>(p, stream);
  return bias ? launch_stream_kernel<T, D, RW, false, true>(p, stream)
              : launch_stream_kernel<T, D, RW, false, false>(p, stream);
}
template <typename T, int D>
static hipError_t launch_stream_rows(const StreamParams& p, int row_waves, hipStream_t stream) {
  switch (row_waves) {
    case 4: return launch_stream_mods<T, D, 4>(p, stream);
    case 2: return launch_stream_mods<T, D, 2>(p, stream);
    case 1:
      if constexpr (sizeof(T) == 2) return launch_stream_mods<T, D, 1>(p, stream);
      break;
    case 0:
      if constexpr (sizeof(T) == 4) return launch_stream_few<D>(p, stream);
  }
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t launch_stream(const StreamParams& p, int d, int row_waves, hipStream_t stream) {
  return d == 64 ? launch_stream_rows<T, 64>(p, row_waves, stream) : launch_stream_rows<T, 128>(p, row_waves, stream);
}
template <typename T>
hipError_t launch_scored_combine(const StreamParams& p, int d, int n_parts, hipStream_t stream) {
  StreamParams q = p;
  void* args[] = {&q, &n_parts};
  const void* k;
  if (combine_shares(n_parts) > 1)
    k = d == 64 ? reinterpret_cast<const void*>(scored_combine_kernel<T, 64, kCombineShares>)
                : reinterpret_cast<const void*>(scored_combine_kernel<T, 128, kCombineShares>);
  else
    k = d == 64 ? reinterpret_cast<const void*>(scored_combine_kernel<T, 64, 1>)
                : reinterpret_cast<const void*>(scored_combine_kernel<T, 128, 1>);
  return hipLaunchKernel(k, dim3((unsigned)combine_blocks(p.out_rows, d, n_parts)), dim3(256), args, 0, stream);
}

}  // namespace mea
