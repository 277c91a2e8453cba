// Attention with modified scores: what the forward, the backward and the
// shared-prefix kernels have in common.
//
//   x_ij = scale q_i . k_j
//   y_ij = cap tanh(x_ij / cap)                       (x_ij without a cap)
//   s_ij = y_ij - slope_h |pos_i - j| + table[bucket(j - pos_i), h]
//   visible(i, j): j < lim_i and, with documents, q_doc_i = k_doc_j >= 0
//   lim_i = valid keys of the batch; causal: and at most max(pos_i + 1, prefix)
//   o_i = sum_j softmax_j(s_ij) v_j over the visible keys; none: o_i = 0, lse_i = -inf
//
// Every positional mask is one limit per query, so a tile of keys is plain (below
// every limit of the workgroup), masked, or not visited.  Documents are told apart
// by the smallest and largest id of every 32 tokens (doc_range_kernel): tiles whose
// ranges do not meet are not visited, tiles of one document need no test.  The
// learned bias is a function of the distance alone that is constant beyond its
// span, so only the tiles within the span of the diagonal read it element by
// element (from LDS); the others add one value.
//
// Scores are kept in units of `unit` powers of two until their exponential: raw
// products (unit = scale log2 e), or tanh (unit = cap log2 e).  Biases are divided by
// it, so that one FMA makes the exponent whatever came before, and a bias that is
// the same for all keys of a tile joins the row's offset in that FMA.
#pragma once

#include <type_traits>

#include "device.hpp"
#include "kernels.hpp"

namespace mea {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxSideBuckets = 64;  // MEA_MAX_SIDE_BUCKETS
constexpr int kMaxBiasSpan = 512;    // MEA_MAX_BIAS_SPAN
constexpr float kLog2eF = 1.4426950408889634f, kLn2F = 0.6931471805599453f;

// What changes the scores (see mea_score in mea.h).
struct ScoreArgs {
  const float* slopes;   // [H] or null
  const void* table;     // [buckets, H] or null
  const int* q_doc;      // [B, n_q] or null
  const int* k_doc;      // [B, n_k]
  const int* q_pos;      // [B] or null
  const int* prefix;     // [B] or null
  const int* kv_len;     // [B] or null
  const int2* q_range;   // smallest and largest id of every 32 queries, [B, ceil(n_q / 32)]
  const int2* k_range;   // of every 32 keys
  float unit;            // powers of two of a score's unit: cap * log2 e, or scale * log2 e
  int capped;
  float cap_in;          // scores to the argument of the cap's 2^x: 2 log2 e scale / cap
  float cap_small;       // scores to the argument of tanh: scale / cap
  int causal;
  int table_dtype;       // mea_dtype
  int heads;             // H
  int n_edges, two_sided, span;
  int edges[kMaxSideBuckets];  // smallest distance of each bucket of a side
  int n_buckets() const { return n_edges * (two_sided ? 2 : 1); }
};

// Arguments of the stream kernel: rows (queries of the heads that share a key
// head, of one batch or of all) against keys.
struct StreamParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;     // [B, H, n_q] or null
  void* o_lo;     // contiguous [B, H, n_q, D] or null
  float* part_o;  // summaries of the key ranges, [n_parts, B * H * n_q, D] and two of [n_parts, B * H * n_q]
  float* part_m;
  float* part_l;
  int64_t n_q, n_k;
  int64_t out_rows;    // B * H * n_q
  int64_t group_rows;  // rows of a group: batches * n_q * fold
  int fold;            // heads of a group, whose rows alternate: row r is head r % fold of query r / fold
  int batches;         // batches of a group (1, or all of a shared prefix)
  int n_b;             // batches over the groups (B, or 1)
  int groups_per_kv;   // groups that share a key head: (H / H_kv) / fold
  int heads_per_kv;    // H / H_kv
  int n_groups, n_rtiles, n_splits;
  int split0;          // first summary of this launch
  int direct;          // 1: one range, o and lse are written; 0: summaries
  int tile_order;
  // The reference maximum is raised by a score that exceeds it by more than this
  // many powers of two: kRescaleSlack where only o is wanted, 0 where a backward will
  // follow.  A row's largest weight is then exactly 1 when it is rounded to 16 bits, and
  // D_i = dO_i . o_i, which that row's dS is a small difference from, is not off by its
  // rounding (scores of standard deviation 4, causal 2048 keys, in float64 with these
  // roundings: dS off by 5e-4 of itself, 2.1e-3 with weights up to 2^8; dQ 2.46e-3 and
  // 3.28e-3, of which 2.40e-3 are the roundings of dS and of dQ itself).
  float slack;
  TensorStrides sq, sk, sv, so;
  ScoreArgs s;
};

// Chunk swizzle of a row of D 16-bit features: physical 16-byte chunk x ^ swz(r).
// Rows of 256 bytes (one LDS line) spread 16 consecutive rows over 16 chunks and 4
// consecutive rows over the 4 groups of 4; rows of 128 bytes (two to a line) spread
// 8 pairs of rows over 8 chunks and neighbouring pairs over the 2 groups of 4: row
// reads and transposing reads of the same tile are both free of bank conflicts.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
template <typename T, int D>
__device__ __forceinline__ Frag<T> row_frag(const unsigned char* tile, int r, int x) {
  return *reinterpret_cast<const Frag<T>*>(tile + r * (2 * D) + ((x ^ swz<D>(r)) << 4));
}
template <typename T, int D>
__device__ __forceinline__ Frag<T> col_frag(const unsigned char* tile, int row0, int col0, int lane) {
  const int g = lane >> 4, i = lane & 15;
  const int row = row0 + 8 * (g >> 1) + (i >> 2);
  const int col = col0 + 16 * (g & 1) + 4 * (i & 3);
  const int off = (col & 7) << 1;
  const v4s_t lo = lds_read_tr16(tile + row * (2 * D) + (((col >> 3) ^ swz<D>(row)) << 4) + off);
  const v4s_t hi = lds_read_tr16(tile + (row + 4) * (2 * D) + (((col >> 3) ^ swz<D>(row + 4)) << 4) + off);
  typedef short v8s_t __attribute__((ext_vector_type(8)));
  v8s_t r8;
  r8[0] = lo[0]; r8[1] = lo[1]; r8[2] = lo[2]; r8[3] = lo[3];
  r8[4] = hi[0]; r8[5] = hi[1]; r8[6] = hi[2]; r8[7] = hi[3];
  return __builtin_bit_cast(Frag<T>, r8);
}

// Asynchronous copies of ROWS rows of two 16-bit tensors into swizzled LDS tiles,
// by 4 waves, 1 KiB (64 / CPR rows) an instruction.  A whole tile's copies take one
// byte offset per lane and tensor, computed once, and scalar bases: wave w copies
// units w, w + 4, .., rows that share their swizzle.  OWN: a wave copies its quarter
// of the rows (which it alone reads), whose swizzle repeats every 16 rows.  Rows from
// `end` on repeat the last one before it.
template <typename T, int D, int ROWS, bool OWN>
struct TileCopy {
  static constexpr int CPR = D / 8, RPU = 64 / CPR, UPW = ROWS / RPU / 4;
  static constexpr int NV = OWN ? 16 / RPU : 1;  // offsets
  static constexpr int STEP = OWN ? 16 : 4 * RPU;  // rows between units of one offset
  static_assert(UPW % NV == 0 && (OWN || 4 * RPU % 16 == 0), "swizzle period");
  unsigned va[NV], vb[NV];
  int first, lane_chunk;  // this lane's first row, and its physical chunk
  __device__ __forceinline__ TileCopy(int wave, int lane, int64_t row_a, int64_t row_b) {
    first = (OWN ? wave * (ROWS / 4) : wave * RPU) + lane / CPR;
    lane_chunk = lane % CPR;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int r = lane / CPR + RPU * i;  // from the wave's first row
      const unsigned ch = 16u * (unsigned)(lane_chunk ^ swz<D>(first + RPU * i));
      va[i] = 2u * (unsigned)r * (unsigned)row_a + ch;
      vb[i] = 2u * (unsigned)r * (unsigned)row_b + ch;
    }
  }
  __device__ __forceinline__ void operator()(const T* a, int64_t row_a, const T* b, int64_t row_b, int64_t r0, int64_t end,
                                             unsigned lds, int wave) const {
    const int w0 = OWN ? wave * (ROWS / 4) : wave * RPU;  // uniform
    const unsigned dst = lds + (unsigned)(w0 * 2 * D);
    constexpr unsigned TILE = ROWS * D * 2;
    if (r0 + ROWS <= end) {
      const T* pa = a + (r0 + w0) * row_a;
      const T* pb = b + (r0 + w0) * row_b;
#pragma unroll
      for (int j = 0; j < UPW; ++j) {
        const int rows = j / NV * STEP;
        const unsigned at = dst + (unsigned)((rows + j % NV * RPU) * 2 * D);
        copy_to_lds16_sb<OWN>(pa + rows * row_a, va[j % NV], at);
        copy_to_lds16_sb<OWN>(pb + rows * row_b, vb[j % NV], at + TILE);
      }
    } else {
#pragma unroll
      for (int j = 0; j < UPW; ++j) {
        const int rows = j / NV * STEP + j % NV * RPU, r = first + rows;
        int64_t at = r0 + r;
        if (at > end - 1) at = end - 1;
        const int ch = 8 * (lane_chunk ^ swz<D>(r));
        copy_to_lds16<OWN>(a + at * row_a + ch, dst + (unsigned)(rows * 2 * D));
        copy_to_lds16<OWN>(b + at * row_b + ch, dst + (unsigned)(rows * 2 * D) + TILE);
      }
    }
  }
};

// A value of the bias table, in score units.
__device__ __forceinline__ float table_value(const ScoreArgs& s, int bucket, int head, float per_unit) {
  const int64_t at = (int64_t)bucket * s.heads + head;
  float x;
  if (s.table_dtype == 0) x = static_cast<const float*>(s.table)[at];
  else if (s.table_dtype == 1) x = (float)static_cast<const _Float16*>(s.table)[at];
  else x = (float)static_cast<const __bf16*>(s.table)[at];
  return x * per_unit;
}
// The edges across a wave's lanes, and the bucket of a side for a distance >= 0 (the
// last one that starts at most there).  All lanes have to be active: edges are read
// from other lanes' registers, as a chain of scalar loads took 2 us a workgroup.
__device__ __forceinline__ int lane_edge(const ScoreArgs& s, int lane) { return s.edges[lane < s.n_edges ? lane : 0]; }
__device__ __forceinline__ int side_bucket(const ScoreArgs& s, int edge, int distance) {
  int n = 0;
  for (int e = 0; e < s.n_edges; ++e) n += __builtin_amdgcn_readlane(edge, e) <= distance;
  return n - 1;
}
// The bias by place: place x stands for the distance j - pos = x - span - kPad.  Where
// it is beyond the span (or ahead, with keys ahead at distance 0) the value repeats; a
// tile of 32 x 32 pairs that is not all beyond the span stays within the kPad places
// beyond it, so that its places are one address per lane and constant offsets.
constexpr int kPad = 64;
__host__ __device__ __forceinline__ int bias_ahead(const ScoreArgs& s) { return s.two_sided ? s.span : 0; }
__host__ __device__ __forceinline__ int bias_places(const ScoreArgs& s) {
  return s.table ? s.span + bias_ahead(s) + 1 + 2 * kPad : 0;
}
__device__ __forceinline__ int place_bucket(const ScoreArgs& s, int edge, int x) {
  int d = x - s.span - kPad;
  if (d > bias_ahead(s)) d = bias_ahead(s);
  return side_bucket(s, edge, d < 0 ? -d : d) + (d > 0 ? s.n_edges : 0);
}
// LDS bytes of the bias for fold heads: the values by place, or (several heads)
// each place's bucket and the heads' buckets.
__host__ __device__ __forceinline__ int bias_lds_bytes(const ScoreArgs& s, int fold) {
  const int n = bias_places(s);
  if (!n) return 0;
  if (fold == 1) return (4 * n + 15) / 16 * 16;
  return (n + 15) / 16 * 16 + (4 * fold * s.n_edges * (s.two_sided ? 2 : 1) + 15) / 16 * 16;
}
__device__ __forceinline__ void fill_bias(const ScoreArgs& s, unsigned char* lds, int fold, int head0, int tid, int nt) {
  const int n = bias_places(s), edge = lane_edge(s, tid & 63);
  const float per_unit = kLog2eF / s.unit;
  for (int x0 = 0; x0 < n; x0 += nt) {
    const int x = x0 + tid, bucket = place_bucket(s, edge, x);
    if (x >= n) continue;
    if (fold == 1) reinterpret_cast<float*>(lds)[x] = table_value(s, bucket, head0, per_unit);
    else lds[x] = (unsigned char)bucket;
  }
  if (fold == 1) return;
  const int nb = s.n_edges * (s.two_sided ? 2 : 1);
  float* tab = reinterpret_cast<float*>(lds + (n + 15) / 16 * 16);
  for (int e = tid; e < fold * nb; e += nt) tab[e] = table_value(s, e % nb, head0 + e / nb, per_unit);
}
// The bias at a place for head g of the fold.
__device__ __forceinline__ float bias_at(const ScoreArgs& s, const unsigned char* lds, int fold, int g, int x) {
  if (fold == 1) return reinterpret_cast<const float*>(lds)[x];
  const int n = bias_places(s);
  return reinterpret_cast<const float*>(lds + (n + 15) / 16 * 16)[g * s.n_edges * (s.two_sided ? 2 : 1) + lds[x]];
}

// tanh of scale x / cap.  With e = 2^(2 log2 e scale x / cap) it is 1 - 2 / (1 + e),
// off by a few 2^-24 in all; float32 scores, whose small values are exact to 2^-24 of
// themselves, take the series of small arguments instead.
template <typename T>
__device__ __forceinline__ float cap_tanh(const ScoreArgs& s, float x) {
  const float e = fast_exp2(x * s.cap_in);
  float t = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + e), 1.0f);
  if constexpr (sizeof(T) == 4) {
    // y - y^3/3 + 2 y^5/15 - 17 y^7/315 + 62 y^9/2835 - 1382 y^11/155925: below 0.35
    // the next term is under 2^-26 of y.
    const float y = x * s.cap_small, z = y * y;
    const float a = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -8.863235e-3f, 2.1869488e-2f), -5.3968254e-2f),
                                             1.3333333e-1f), -3.3333333e-1f), 1.0f);
    t = fabsf(y) < 0.35f ? a : t;
  }
  return t;
}

// A value that the compiler takes as made here: what depends on it is not computed
// ahead of the branch that it stands in (masks of a few tiles, in every tile's code).
__device__ __forceinline__ void stay(int& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void stay(float& x) { asm volatile("" : "+v"(x)); }

// Keys visible to a query by position: [0, lim).  reach: keys that every query sees
// (a prefix; all of them without the causal mask).
__device__ __forceinline__ int64_t key_limit(int64_t n_kv, int64_t reach, int64_t pos) {
  const int64_t lim = pos + 1 > reach ? pos + 1 : reach;
  return lim < n_kv ? lim : n_kv;
}
__device__ __forceinline__ int64_t first_pos(const ScoreArgs& s, int b) {
  const int p = s.q_pos ? s.q_pos[b] : 0;
  return p > 0 ? p : 0;
}
__device__ __forceinline__ int64_t key_reach(const ScoreArgs& s, int b, int64_t n_k) {
  if (!s.causal) return n_k;
  const int p = s.prefix ? s.prefix[b] : 0;
  return p > 0 ? p : 0;
}
__device__ __forceinline__ int64_t batch_keys(const ScoreArgs& s, int b, int64_t n_k) {
  if (!s.kv_len) return n_k;
  const int64_t l = s.kv_len[b];
  return l < 0 ? 0 : (l > n_k ? n_k : l);
}
// Smallest and largest id of a wave's 64 lanes.
__device__ __forceinline__ int2 wave_range(int lo, int hi) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const int a = __shfl_xor(lo, o), b = __shfl_xor(hi, o);
    lo = a < lo ? a : lo;
    hi = b > hi ? b : hi;
  }
  return make_int2(__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi));
}

// Smallest and largest id of a workgroup's tokens and (z) whether one of them has
// none; id < 0: none.  Every thread of the 4 waves calls it.
__device__ __forceinline__ int4 workgroup_ids(int id, int wave, int lane, int4* lds) {
  const int2 w = wave_range(id < 0 ? 0x7fffffff : id, id);
  const int none = __builtin_amdgcn_ballot_w64(id < 0) != 0;
  if (lane == 0) lds[wave] = make_int4(w.x, w.y, none, 0);
  __syncthreads();
  int4 a = lds[0];
#pragma unroll
  for (int y = 1; y < 4; ++y) {
    const int4 o = lds[y];
    a.x = o.x < a.x ? o.x : a.x;
    a.y = o.y > a.y ? o.y : a.y;
    a.z |= o.z;
  }
  return make_int4(__builtin_amdgcn_readfirstlane(a.x), __builtin_amdgcn_readfirstlane(a.y),
                   __builtin_amdgcn_readfirstlane(a.z), 0);
}

// Hides the pairs of other documents than the lane's.  mine: the ids of the 32 tokens
// across, one on each lane of a half, which go by way of 32 words of LDS of this wave's
// own: a write and 4 reads of 16 bytes that all lanes of a half share, a group at a
// time (registers).
__device__ __forceinline__ void hide_documents(f32x16& s, int doc, int mine, int* lds, int lane) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  if (lane < 32) lds[lane] = mine;
  const int* at = lds + 8 * (lane >> 5);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const i32x4 x = *reinterpret_cast<const i32x4*>(at + 16 * (j >> 1) + 4 * (j & 1));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (x[e] != doc) s[4 * j + e] = -INFINITY;
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Zeroes the rows of two staged tiles whose tokens have no document (the tiles' rows
// are tokens r0 .., from `end` on the last one before it again), so that whatever they
// hold meets weights of 0 as a number.  nt threads, for rows [first, first + rows); the caller synchronises.
template <typename T, int D, int RSA, int RSB, int PA, int PB, int NP>
__device__ __forceinline__ void zero_absent(T* a, T* b, const int* ids, int64_t r0, int64_t end, int first, int rows, int tid,
                                            int nt) {
  for (int i = tid; i < rows * (D / 8); i += nt) {
    const int r = first + i / (D / 8), x = 8 * (i % (D / 8));
    if (ids[r0 + r < end ? r0 + r : end - 1] < 0) {
#pragma unroll
      for (int y = 0; y < NP; ++y) {
        st16(a + y * PA + r * RSA + x, u32x4{0, 0, 0, 0});
        st16(b + y * PB + r * RSB + x, u32x4{0, 0, 0, 0});
      }
    }
  }
}

// Tiles of one side that may meet the ids [lo, hi]: 64 tiles at a time, a bit each.
// Ranges are of 32 tokens, UNITS of them a tile.
template <int UNITS>
struct DocTiles {
  const int2* range;  // of this batch, or null: every tile is visited
  int n_units, lo, hi, base;
  uint64_t bits;
  __device__ __forceinline__ DocTiles(const int2* r, int n, int l, int h_) : range(r), n_units(n), lo(l), hi(h_), base(-64), bits(0) {}
  __device__ __forceinline__ int2 of_tile(int t) const {
    int2 x = make_int2(0x7fffffff, -1);
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
      if (t * UNITS + u < n_units) {
        const int2 y = range[t * UNITS + u];
        x.x = y.x < x.x ? y.x : x.x;
        x.y = y.y > x.y ? y.y : x.y;
      }
    return x;
  }
  // The first tile >= t and < end to visit, or end.  t never decreases.
  __device__ __forceinline__ int next(int t, int end) {
    if (!range) return t;
    while (t < end) {
      if (t >= base + 64 || base < 0) {
        base = t;
        const int mine = t + (int)(threadIdx.x & 63);
        const int2 x = of_tile(mine);
        bits = __builtin_amdgcn_ballot_w64(mine < end && x.x <= hi && x.y >= lo);
      }
      const uint64_t left = bits >> (t - base);
      if (left) {
        const int at = t + __builtin_ctzll(left);
        return at < end ? at : end;
      }
      t = base + 64;
    }
    return end;
  }
  // Whether a tile holds other ids than [lo, hi], all the same; and one below 0.
  __device__ __forceinline__ bool mixed(int2 of) const { return !(lo == hi && of.x == lo && of.y == lo); }
};

// Arguments of the backward kernels.
struct ScoredBwdParams {
  const void* q;
  const void* k;
  const void* v;
  const void* o;
  const void* o_lo;  // residual of a 16-bit o (contiguous [B, H, n_q, D]) or null
  const void* d_o;
  const float* lse;
  void* dq;
  void* dk;
  void* dv;
  // Per row, [B * H, n_q_pad], written by the preprocess: lse log2 e (inf for a row
  // with no visible key and for padding, whose weights are then 0) and -D_i.
  float* lse2;
  float* neg_d;
  float* table_part;  // dS sums by bucket of each dQ workgroup, [n_wgs, buckets], or null
  // Float32 sums of each part, where a pass has several (BwdParts): [part, B, H_kv, n_k, D]
  // twice, and [part, B, H, n_q, D].
  float* dk_part;
  float* dv_part;
  float* dq_part;
  int kv_heads_parts, kv_query_parts, dq_parts;
  void* d_table;      // [buckets, H], the table's type
  int64_t n_q, n_k, n_q_pad;
  int n_b, heads_kv, heads_per_kv;
  int n_ktiles, n_qtiles, tile_order;
  float scale;
  TensorStrides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  ScoreArgs s;
};

// Into how many parts dK/dV workgroups split their heads and their queries, and dQ
// workgroups their keys, where the tiles alone would leave places on the chip empty
// (the parts' float32 sums are added afterwards, in order).  The two kinds run in one
// launch, so each is to fill half the chip's places; with the causal mask, whose tiles
// differ in length, all of them, 16-bit one and a half times over.  Heads before queries, as
// a part of a head reads the same keys again, and a number of heads that leaves
// no part more than another.  Backward in us at 1 / 0.75 / 0.5 of twice that (causal 16-bit:
// of 1.33 times), bf16 d = 64 2x8 heads, 1000 unmasked 56 / 55 / 45; 4x12, 1999 causal 156 /
// 140 / 140; d = 128 4x8, 1000 unmasked 128 / 100 / 100; causal 3x2 on 1, 3761 156 / 145 / 154;
// 3x24 on 3, 897 120 / 120 / 145; 10x8 on 2, 1309 210 / 204 / 199; float32 d = 128 2x4 on 2,
// 1000 causal 148 / 136 / 116.  Forward + backward without parts and with them: causal
// bf16 d = 128 2x16 on 4, 4096 1380 / 862, 3x2 on 1, 3761 644 / 248; float32 d = 64 2x8 on 4, 700
// 219 / 122.
struct BwdParts {
  int kv_heads, kv_queries, dq;
};
inline BwdParts bwd_parts(bool is16, bool causal, int d, int64_t n_q, int64_t n_k, int64_t batch, int64_t heads,
                          int64_t heads_kv) {
  const int64_t G = heads / heads_kv, kv_wgs = batch * heads_kv * ((n_k + 127) / 128), q_wgs = batch * heads * ((n_q + 127) / 128);
  const int64_t kv_places = is16 ? 512 : 256, q_places = is16 || d == 64 ? 512 : 256;
  const double fill = !causal ? 0.5 : (is16 ? 1.5 : 1.0);
  const int64_t q_tiles = (n_q + 127) / 128, k_tiles = (n_k + 127) / 128;
  BwdParts r = {1, 1, 1};
  int64_t want = (int64_t)(fill * (double)kv_places / (double)kv_wgs);
  if (want > 1) {
    int64_t ph = want < G ? want : G;
    while (G % ph) ++ph;
    int64_t pq = want / ph;
    if (pq > q_tiles) pq = q_tiles;
    r.kv_heads = (int)ph;
    r.kv_queries = pq < 1 ? 1 : (int)pq;
  }
  want = (int64_t)(fill * (double)q_places / (double)q_wgs);
  if (want > k_tiles) want = k_tiles;
  if (want > 1) r.dq = (int)want;
  return r;
}

hipError_t launch_scored_table(const ScoredBwdParams& p, hipStream_t stream);
hipError_t launch_doc_ranges(const int* ids, int64_t n, int64_t batches, int2* out, hipStream_t stream);

// Rows per workgroup: 32 for each of 4 waves, or 2 or 1 (the other waves take
// shares of the keys), or 0: at most kFewRows float32 rows (scored_few.hpp).
constexpr int kFewRows = 8;
template <typename T> hipError_t launch_stream(const StreamParams& p, int d, int row_waves, hipStream_t stream);
// Two key sets in one launch: row waves 4 and 4 or 2, or 1 and 1 (float32: 2 and 2).
template <typename T>
hipError_t launch_stream_pair(const StreamParams& a, const StreamParams& b, int d, int rwa, int rwb, hipStream_t stream);
// Threads that share a row's ranges in the combine, and its workgroups.
constexpr int kCombineShares = 8;
inline int combine_shares(int64_t n_parts) { return n_parts > 8 ? kCombineShares : 1; }
inline int64_t combine_blocks(int64_t rows, int64_t d, int64_t n_parts) {
  return (rows * (d / 4) * combine_shares(n_parts) + 255) / 256;
}
template <typename T>
hipError_t launch_scored_combine(const StreamParams& p, int d, int n_parts, hipStream_t stream);
template <typename T> hipError_t launch_scored_bwd(const ScoredBwdParams& p, int d, hipStream_t stream);
// Rows of a dQ workgroup (the plan sizes table_part by it), and the row padding.
constexpr int kScoredDqRows = 128, kScoredRowPad = 64;
// Keys of a staged tile.
__host__ __device__ constexpr int stream_tile(bool is16, int row_waves) {
  return is16 ? (row_waves == 1 ? 128 : 64) : (row_waves == 4 ? 32 : 64);
}

}  // namespace mea
