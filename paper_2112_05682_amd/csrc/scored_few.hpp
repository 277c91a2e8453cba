// The stream kernel of a few float32 rows (a step of decoding) on the vector unit.
//
// Up to 8 rows share every key, so that products are 2 flop for each byte read, and
// tiles of matrix instructions would be split into three bf16 planes for rows that are
// padding.  Here D / 4 lanes hold a key (16 bytes each), a wave 256 / D keys, whose
// scores are dot products reduced across those lanes; each group of lanes keeps its own
// softmax of the keys that it met, and the groups' summaries meet in LDS.  What bounds
// it: memory, with 8 loads of 1 KiB in flight a wave; from 5 rows on the vector unit.
// us, as tiles / here: d = 128 32x16 heads, 8000 keys, a row 1229 / 634 (6.6 TB/s); 8x16, 4000 170 /
// 84; 11x6, 6700, 4 rows, learned bias 190 / 102; 8x4 of 8 rows, 16000, cap 187 / 163; d = 64 16x8, up to
// 5000, 2 rows 112 / 47; 4x4, 8000, 4 rows 31 / 21; 4x8, 10000, 8 rows, slopes 65 / 67.
#pragma once

#include "scored.hpp"

namespace mea {

template <int N>
__device__ __forceinline__ float rotated16(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + N, 0xf, 0xf, true));
}
// The sum over LANES (16 or 32) neighbouring lanes, the same bits on each.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  x += rotated16<8>(x);
  x += rotated16<4>(x);
  x += rotated16<2>(x);
  x += rotated16<1>(x);
  if constexpr (LANES == 32) x += __shfl_xor(x, 16);
  return x;
}

template <int D, int ROWS>
struct FewTile {
  static constexpr int LPK = D / 4, KPW = 64 / LPK, U = 4;  // lanes of a key, keys of a wave's load, loads of a step
  static constexpr int STEP = 4 * U * KPW;                  // keys of a workgroup's step
  static constexpr int GROUPS = 4 * KPW;
  static constexpr int LDS_BYTES = GROUPS * ROWS * (D + 2) * 4;
  static_assert(64 % STEP == 0 && LDS_BYTES % 16 == 0, "ranges are whole steps");
};

template <int D, int ROWS, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, ROWS == 8 ? 2 : 4) void scored_few_kernel(StreamParams p) {
  using C = FewTile<D, ROWS>;
  constexpr int U = C::U, KPW = C::KPW, LPK = C::LPK;
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* const lds_bias = smem + C::LDS_BYTES;
  const ScoreArgs& sa = p.s;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int sub = lane / LPK, c4 = 4 * (lane % LPK);

  const int block = tile_item((int)blockIdx.x, (int)gridDim.x, 1, 0).group;
  const int split = block / p.n_groups;
  int gi = block % p.n_groups;
  const int part_of_kv = gi % p.groups_per_kv;
  gi /= p.groups_per_kv;
  const int b = gi % p.n_b, kvh = gi / p.n_b, head0 = kvh * p.heads_per_kv + part_of_kv * p.fold;
  const int n_rows = (int)p.group_rows;

  const int64_t n_kv = batch_keys(sa, b, p.n_k), pos0 = first_pos(sa, b), reach = key_reach(sa, b, p.n_k);
  const int64_t lim_hi = key_limit(n_kv, reach, pos0 + (n_rows - 1) / p.fold);
  if (BIAS && sa.table) fill_bias(sa, lds_bias, p.fold, head0, tid, 256);

  // ---- the rows, all of them on every lane: 4 features of q, and scalars.
  const float unit = sa.unit;
  f32x4 q[ROWS], acc[ROWS];
  float m[ROWS], l[ROWS], slope[ROWS];
  int lim[ROWS], pos[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const bool in = r < n_rows;
    const int qi = in ? r / p.fold : 0, head = head0 + (in ? r % p.fold : 0);
    const float* qg = static_cast<const float*>(p.q) + (int64_t)b * p.sq.b + (int64_t)head * p.sq.h + qi * p.sq.r + c4;
    pos[r] = (int)(pos0 + qi);
    lim[r] = in ? (int)key_limit(n_kv, reach, pos0 + qi) : 0;
    q[r] = lim[r] > 0 ? *reinterpret_cast<const f32x4*>(qg) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    slope[r] = BIAS && sa.slopes ? sa.slopes[head] * (kLog2eF / unit) : 0.0f;
    acc[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m[r] = -INFINITY;
    l[r] = 0.0f;
  }
  const int places = BIAS ? bias_places(sa) : 0;
  __syncthreads();  // the bias is there

  // ---- keys of this range, in units of 64.
  const int64_t units = (lim_hi + 63) / 64, per = (units + p.n_splits - 1) / p.n_splits;
  const int64_t k_begin = 64 * per * split, k_all = k_begin + 64 * per, k_end = k_all < lim_hi ? k_all : lim_hi;
  const float* __restrict__ kg = static_cast<const float*>(p.k) + (int64_t)b * p.sk.b + (int64_t)kvh * p.sk.h + c4;
  const float* __restrict__ vg = static_cast<const float*>(p.v) + (int64_t)b * p.sv.b + (int64_t)kvh * p.sv.h + c4;
  for (int64_t k0 = k_begin + wave * (U * KPW); k0 < k_end; k0 += C::STEP) {
    f32x4 kx[U], vx[U];
    // (keys from lim_hi on repeat the last one before it, and are masked)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t key = k0 + u * KPW + sub, at = key < lim_hi ? key : lim_hi - 1;
      kx[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(kg + at * p.sk.r));
      vx[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(vg + at * p.sv.r));
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float s[U], mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x = q[r][0] * kx[u][0];
#pragma unroll
        for (int e = 1; e < 4; ++e) x = fmaf(q[r][e], kx[u][e], x);
        x = lanes_sum<LPK>(x);
        if constexpr (CAP) x = cap_tanh<float>(sa, x);
        const int key = (int)k0 + u * KPW + sub;
        if constexpr (BIAS) {
          const int off = key - pos[r];
          x = fmaf(-fabsf((float)off), slope[r], x);
          if (sa.table) {
            int at = off + sa.span + kPad;
            at = at < 0 ? 0 : (at < places ? at : places - 1);
            x += bias_at(sa, lds_bias, p.fold, r < n_rows ? r % p.fold : 0, at);
          }
        }
        s[u] = key < lim[r] ? x : -INFINITY;
        mx = fmaxf(mx, s[u]);
      }
      const float m_new = fmaxf(m[r], mx * unit);
      const float a = m[r] == -INFINITY ? 0.0f : fast_exp2(m[r] - m_new), neg = m_new == -INFINITY ? 0.0f : -m_new;
      m[r] = m_new;
      l[r] *= a;
      acc[r] *= a;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = fast_exp2(fmaf(s[u], unit, neg));
        l[r] += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][e] = fmaf(w, vx[u][e], acc[r][e]);
      }
    }
  }

  // ---- the groups' summaries, in order.
  float* const red_o = reinterpret_cast<float*>(smem);
  float* const red_m = red_o + C::GROUPS * ROWS * D;
  float* const red_l = red_m + C::GROUPS * ROWS;
  const int grp = wave * KPW + sub;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    *reinterpret_cast<f32x4*>(red_o + (grp * ROWS + r) * D + c4) = acc[r];
    if (c4 == 0) {
      red_m[grp * ROWS + r] = m[r];
      red_l[grp * ROWS + r] = l[r];
    }
  }
  __syncthreads();
  const int r = tid / LPK, f = 4 * (tid % LPK);
  if (r >= n_rows || r >= ROWS) return;
  float mg = -INFINITY, lg = 0.0f;
#pragma unroll
  for (int y = 0; y < C::GROUPS; ++y) mg = fmaxf(mg, red_m[y * ROWS + r]);
  f32x4 og = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int y = 0; y < C::GROUPS; ++y) {
    const float my = red_m[y * ROWS + r], w = my == -INFINITY ? 0.0f : fast_exp2(my - mg);
    lg = fmaf(w, red_l[y * ROWS + r], lg);
    const f32x4 oy = *reinterpret_cast<const f32x4*>(red_o + (y * ROWS + r) * D + f);
#pragma unroll
    for (int e = 0; e < 4; ++e) og[e] = fmaf(w, oy[e], og[e]);
  }
  const int64_t qi = r / p.fold, head = head0 + r % p.fold, out_row = ((int64_t)b * sa.heads + head) * p.n_q + qi;
  if (p.direct) {
    const float inv = lg == 0.0f ? 0.0f : 1.0f / lg;
    *reinterpret_cast<f32x4*>(static_cast<float*>(p.o) + (int64_t)b * p.so.b + head * p.so.h + qi * p.so.r + f) = og * inv;
    if (f == 0 && p.lse) p.lse[out_row] = lg == 0.0f ? -INFINITY : (mg + __log2f(lg)) * kLn2F;
  } else {
    const int64_t row = (int64_t)(p.split0 + split) * p.out_rows + out_row;
    *reinterpret_cast<f32x4*>(p.part_o + row * D + f) = og;
    if (f == 0) {
      p.part_m[row] = mg;
      p.part_l[row] = lg;
    }
  }
}

template <int D, int ROWS, bool CAP, bool BIAS>
static hipError_t launch_few_kernel(const StreamParams& p, hipStream_t stream) {
  StreamParams q = p;
  void* args[] = {&q};
  return hipLaunchKernel(reinterpret_cast<const void*>(scored_few_kernel<D, ROWS, CAP, BIAS>),
                         dim3((unsigned)(p.n_groups * p.n_splits)), dim3(256), args,
                         FewTile<D, ROWS>::LDS_BYTES + bias_lds_bytes(p.s, p.fold), stream);
}
template <int D, int ROWS>
static hipError_t launch_few_mods(const StreamParams& p, hipStream_t stream) {
  const bool bias = p.s.slopes || p.s.table;
  if (p.s.capped)
    return bias ? launch_few_kernel<D, ROWS, true, true>(p, stream) : launch_few_kernel<D, ROWS, true, false>(p, stream);
  return bias ? launch_few_kernel<D, ROWS, false, true>(p, stream) : launch_few_kernel<D, ROWS, false, false>(p, stream);
}
// Groups of at most kFewRows rows, no documents.
template <int D>
static hipError_t launch_stream_few(const StreamParams& p, hipStream_t stream) {
  if (p.group_rows > kFewRows || p.s.q_doc) return hipErrorInvalidValue;
  if (p.group_rows <= 1) return launch_few_mods<D, 1>(p, stream);
  if (p.group_rows <= 2) return launch_few_mods<D, 2>(p, stream);
  if (p.group_rows <= 4) return launch_few_mods<D, 4>(p, stream);
  return launch_few_mods<D, 8>(p, stream);
}

}  // namespace mea
