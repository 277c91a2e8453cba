// Entry points of attention with modified scores and of attention over a shared
// prefix: argument checks, work planning and dispatch.  Nothing here allocates
// device memory or synchronises.
#include <string.h>

#include "checks.hpp"
#include "scored.hpp"

namespace {

using namespace mea_host;
using mea::ScoreArgs;
using mea::ScoredBwdParams;
using mea::StreamParams;

static_assert(mea::kMaxSideBuckets == MEA_MAX_SIDE_BUCKETS && mea::kMaxBiasSpan == MEA_MAX_BIAS_SPAN, "limits");

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
// Whether a table's address is a multiple of its elements' size.
bool table_aligned(const void* p, int32_t dtype) { return (uintptr_t)p % elem_size(dtype) == 0; }
int64_t kv_heads_of(const mea_problem* p, int64_t given) { return given ? given : p->heads; }

mea_status check_base(const mea_problem* p, int64_t kv_heads) {
  const mea_status st = check_problem(p);
  if (st != MEA_OK) return st;
  if (kv_heads < 0 || (kv_heads && p->heads % kv_heads)) return MEA_ERR_INVALID_ARG;
  if (p->out_f32 && p->dtype != MEA_F32) return MEA_ERR_UNSUPPORTED;
  if (dv_of(p) != p->d) return MEA_ERR_UNSUPPORTED;
  return MEA_OK;
}

mea_status check_score(const mea_problem* p, const mea_score* s) {
  if (!s) return MEA_ERR_INVALID_ARG;
  const mea_status st = check_base(p, s->kv_heads);
  if (st != MEA_OK) return st;
  if (!(s->softcap >= 0.0f) || !isfinite(s->softcap)) return MEA_ERR_INVALID_ARG;
  if (s->softcap > 0.0f && !(s->softcap * kLog2e > 0.0f && isfinite(s->softcap * kLog2e) && isfinite(2.0f * kLog2e * p->scale / s->softcap)))
    return MEA_ERR_INVALID_ARG;
  if (!aligned4(s->slopes) || !aligned4(s->q_doc) || !aligned4(s->k_doc) || !aligned4(s->prefix_len) || !aligned4(s->q_pos))
    return MEA_ERR_INVALID_ARG;
  if ((s->q_doc == nullptr) != (s->k_doc == nullptr)) return MEA_ERR_INVALID_ARG;
  if (s->prefix_len && !p->causal) return MEA_ERR_INVALID_ARG;
  if (s->table) {
    if (s->table_dtype != MEA_F32 && s->table_dtype != MEA_F16 && s->table_dtype != MEA_BF16) return MEA_ERR_UNSUPPORTED;
    if (!table_aligned(s->table, s->table_dtype)) return MEA_ERR_INVALID_ARG;
    if (s->two_sided != 0 && s->two_sided != 1) return MEA_ERR_INVALID_ARG;
    if (!s->edges || s->n_edges < 2 || s->edges[0] != 0) return MEA_ERR_INVALID_ARG;
    if (s->n_edges > MEA_MAX_SIDE_BUCKETS) return MEA_ERR_UNSUPPORTED;
    for (int i = 1; i < s->n_edges; ++i)
      if (s->edges[i] < s->edges[i - 1]) return MEA_ERR_INVALID_ARG;
    if (s->edges[s->n_edges - 1] < 1) return MEA_ERR_INVALID_ARG;
    if (s->edges[s->n_edges - 1] > MEA_MAX_BIAS_SPAN) return MEA_ERR_UNSUPPORTED;
  }
  return MEA_OK;
}

ScoreArgs score_args(const mea_problem* p, const mea_score* s) {
  ScoreArgs a = {};
  a.kv_len = p->kv_len;
  a.causal = p->causal;
  a.heads = (int)p->heads;
  a.unit = p->scale * kLog2e;
  if (!s) return a;
  a.slopes = s->slopes;
  a.q_doc = s->q_doc;
  a.k_doc = s->k_doc;
  a.q_pos = s->q_pos;
  a.prefix = s->prefix_len;
  if (s->softcap > 0.0f) {
    a.capped = 1;
    a.unit = s->softcap * kLog2e;
    a.cap_in = 2.0f * kLog2e * p->scale / s->softcap;
    a.cap_small = p->scale / s->softcap;
  }
  if (s->table) {
    a.table = s->table;
    a.table_dtype = s->table_dtype;
    a.n_edges = s->n_edges;
    a.two_sided = s->two_sided;
    a.span = s->edges[s->n_edges - 1];
    memcpy(a.edges, s->edges, sizeof(int) * (size_t)s->n_edges);
  }
  return a;
}

size_t round256(size_t b) { return (b + 255) / 256 * 256; }
size_t range_bytes(int64_t batch, int64_t n) { return round256((size_t)batch * (size_t)((n + 31) / 32) * sizeof(int2)); }

// How rows meet keys in the stream kernel.
struct StreamPlan {
  int row_waves;
  int64_t fold, groups, rows, rtiles, splits;  // rows of a group
};

// Workgroups of these row waves that the chip holds at once.
int64_t places_of(const mea_problem* p, int row_waves) {
  if (p->dtype == MEA_F32 && row_waves == 0) return 1024;
  if (p->dtype == MEA_F32) return row_waves == 4 && p->d == 64 ? 512 : 256;
  return 256 * (row_waves == 1 && p->d == 128 ? 1 : 2);
}
// Row tiles, and key ranges for the places that `taken` workgroups leave.  At most 256
// ranges; us at 64 / 128 / 256 of them, one token, 8 heads of one key head: bf16 d = 128
// 131072 keys 30 / 23 / 22, d = 64 65536 keys 18 / 15 / 15, float32 65536 keys 85 / 50 / 36.
// A range has two tiles and more; of float32, whose tiles take longer than the combine
// (about 2 us each), one of 64 keys or four of 32: us in 1 / 2 / 3 / 4 / 6 ranges, causal
// d = 64, 4 heads, 300 (5 tiles of 64) 19 / 17 / 15 / 15 / 13, 2x8 heads, 700 (22 of 32) 48 / 34 /
// 29 / 27 / 28.  fill: workgroups wanted for each place.
void set_tiles(StreamPlan* pl, const mea_problem* p, int rw, int64_t n_keys, int64_t taken, double fill = 1.0) {
  pl->row_waves = rw;
  pl->rtiles = rw ? (pl->rows + 32 * rw - 1) / (32 * rw) : 1;
  const bool is16 = p->dtype != MEA_F32;
  const int64_t wgs = pl->groups * pl->rtiles, tile = mea::stream_tile(is16, rw);
  const int64_t key_tiles = (n_keys + tile - 1) / tile, places = (int64_t)(fill * (double)places_of(p, rw));
  const int64_t most = is16 || rw == 0 ? key_tiles / 2 : (rw == 4 ? key_tiles / 4 : (key_tiles > 2 ? key_tiles : 1));
  int64_t splits = (places - (taken < places / 2 ? taken : places / 2)) / wgs;
  if (splits > most) splits = most;
  if (splits > 256) splits = 256;
  pl->splits = splits < 1 ? 1 : splits;
}

// What a 16-bit stream kernel with many row tiles takes: us to start and end, us per
// 1000 keys of the workgroups of a CU (of the fullest without the causal mask, of the
// average with it) and of the longest workgroup, and, of several ranges, us of the
// combine and per million numbers of the parts.  Fitted to 68 shapes of 1-64 heads and
// 512-16384 tokens, d = 64 and 128, in up to 4 ranges (errors 5-10 %); what it chooses
// takes 1.01 times the best of those measured on average and 1.19 at most, where fixed
// numbers of row tiles (128 and 256) for 1, 2 and 4 row waves took 1.17 and 2.1 times.
struct StreamRate {
  double fixed, load[2], longest[2], combine, part;  // [with the causal mask]
};
StreamRate stream_rate(int64_t d, int row_waves) {
  if (d == 64)
    return row_waves == 1   ? StreamRate{11.5, {3.81, 4.33}, {0, 0}, 0, 0}
           : row_waves == 2 ? StreamRate{8.2, {4.86, 3.19}, {3.27, 7.14}, 3.7, 1.72}
                            : StreamRate{7.7, {7.34, 4.40}, {5.85, 11.4}, 3.6, 1.38};
  return row_waves == 1   ? StreamRate{19.5, {8.22, 9.97}, {0, 0}, 0, 0}
         : row_waves == 2 ? StreamRate{10.5, {9.72, 7.65}, {0, 6.63}, 2.1, 1.87}
                          : StreamRate{10.4, {14.2, 9.53}, {3.94, 13.6}, 0.5, 1.51};
}

// Fold: with few queries (a 32-row tile of one head would be padding) the heads that share a key head are rows of the same
// tile, so that the keys are read once for all of them; with many, each head has
// tiles of its own (the keys are then found in L2).  Row waves: as few as hold
// the rows, and on small grids fewer still, so that the waves without rows of
// their own take shares of the keys instead.  Splits: enough key ranges for about
// one workgroup for each place on the chip, of at least two tiles each.  16 bits, about 128
// row tiles and more (on long keys, 64): what stream_rate says is fastest, in ranges of 256 keys and
// more (documents, of whose keys a row tile sees a part: one range).  us, before / with it
// on 64-128 row tiles: d = 64 2x8192 causal 65 / 42, 1x16384 124 / 60; d = 128 1x8192 72 / 43, 2x4096
// 40 / 32.
StreamPlan plan_stream(const mea_problem* p, const ScoreArgs& s, int64_t kv_heads) {
  StreamPlan pl;
  const bool is16 = p->dtype != MEA_F32;
  const int64_t G = p->heads / kv_heads;
  pl.fold = p->n_q <= 32 || G * p->n_q <= 64 ? G : 1;
  // The biases of the folded heads have to fit beside the stages.
  if (pl.fold > 1 && mea::bias_lds_bytes(s, (int)pl.fold) > 24 * 1024) pl.fold = 1;
  pl.rows = p->n_q * pl.fold;
  pl.groups = p->heads / pl.fold * p->batch;
  const int64_t tiles128 = pl.groups * ((pl.rows + 127) / 128);
  const int64_t longest = p->causal && !s.q_pos && p->n_q < p->n_k ? p->n_q : p->n_k;
  const bool many = tiles128 > (p->d == 64 ? 128 : 127);
  if (is16 && pl.rows > 64 && !s.q_doc && (many || (tiles128 >= 64 && longest >= (p->d == 64 ? 6000 : 3000)))) {
    const double mean = (double)longest - (p->causal ? 0.5 * (double)(p->n_q < longest ? p->n_q : longest) : 0.0);
    const int masked = mean < 0.75 * (double)longest;
    double best = 0.0;
    for (int rw = many ? 1 : 2; rw <= 4; rw *= 2) {
      const StreamRate r = stream_rate(p->d, rw);
      const int64_t tiles = pl.groups * ((pl.rows + 32 * rw - 1) / (32 * rw));
      for (int64_t n = 1; n <= 8; n += n < 4 ? 1 : 2) {
        if (n > 1 && (rw == 1 || longest < 256 * n)) break;
        const double wgs = masked ? (double)tiles / 256.0 : (double)((tiles * n + 255) / 256) / (double)n;
        double t = r.fixed + (r.load[masked] * wgs * mean + r.longest[masked] * (double)longest / (double)n) / 1000.0;
        if (n > 1) t += r.combine + r.part * 1e-6 * (double)(n * pl.groups * pl.rows * p->d);
        if (rw < 4) t *= 1.1;  // caps and biases cost fewer row waves more: us at 2 / 4, slopes 48x1999 64 / 49
        if (best == 0.0 || t < best) {
          best = t;
          pl.row_waves = rw;
          pl.rtiles = tiles / pl.groups;
          pl.splits = n;
        }
      }
    }
    return pl;
  }
  int rw = tiles128 <= 128 ? 1 : (tiles128 <= 256 ? 2 : 4);
  if (pl.rows <= 32) rw = 1;
  else if (pl.rows <= 64 && rw > 2) rw = 2;
  if (!is16) rw = pl.rows <= mea::kFewRows && !s.q_doc ? 0 : (pl.rows <= 64 || tiles128 <= 32 ? 2 : 4);
  // Causal float32 row tiles differ in length: us at 1 / 1.25 of the places, d = 64 16 heads, 1500
  // 63 / 51; d = 128 12 heads on 4, 900 65 / 52.
  set_tiles(&pl, p, rw, p->n_k, 0, !is16 && p->causal && p->n_q > 128 ? 1.25 : 1.0);
  if (is16 && many && s.q_doc) pl.splits = 1;
  // Two workgroups on a CU that one fills hardly: us in 1 / 2 ranges, 16x512 10 / 13, 8x1024
  // 12 / 15, 4x2048 18 / 17, 2x4096 32 / 23.
  if (is16 && rw == 1 && p->d == 64 && pl.rows > 64) {
    const int64_t most = p->n_k < 1536 ? 1 : p->n_k / 768;
    if (pl.splits > most) pl.splits = most;
  }
  return pl;
}

size_t part_bytes(const mea_problem* p, int64_t parts) {
  const size_t rows = (size_t)parts * (size_t)p->batch * (size_t)p->heads * (size_t)p->n_q;
  return round256(rows * (size_t)p->d * 4) + 2 * round256(rows * 4);
}
void carve_parts(StreamParams* q, const mea_problem* p, int64_t parts, float* at) {
  const size_t rows = (size_t)parts * (size_t)q->out_rows;
  q->part_o = at;
  q->part_m = at + round256(rows * (size_t)p->d * 4) / 4;
  q->part_l = q->part_m + round256(rows * 4) / 4;
}

struct FwdWork {
  StreamPlan pl;
  size_t ranges, total;
};
FwdWork plan_scored_fwd(const mea_problem* p, const mea_score* s) {
  FwdWork w;
  w.pl = plan_stream(p, score_args(p, s), kv_heads_of(p, s->kv_heads));
  w.ranges = s->q_doc ? range_bytes(p->batch, p->n_k) : 0;
  w.total = w.ranges + (w.pl.splits > 1 ? part_bytes(p, w.pl.splits) : 0);
  if (w.total) w.total += 256;
  return w;
}

StreamParams stream_params(const mea_problem* p, const ScoreArgs& s, int64_t kv_heads, const StreamPlan& pl) {
  StreamParams q = {};
  q.s = s;
  q.n_q = p->n_q;
  q.n_k = p->n_k;
  q.out_rows = p->batch * p->heads * p->n_q;
  q.group_rows = pl.rows;
  q.fold = (int)pl.fold;
  q.batches = 1;
  q.n_b = (int)p->batch;
  q.heads_per_kv = (int)(p->heads / kv_heads);
  q.groups_per_kv = q.heads_per_kv / q.fold;
  q.n_groups = (int)pl.groups;
  q.n_splits = (int)pl.splits;
  q.slack = mea::kRescaleSlack;
  return q;
}

hipError_t run_stream(const StreamParams& q, const mea_problem* p, int row_waves, hipStream_t stream) {
  const int d = (int)p->d;
  switch (p->dtype) {
    case MEA_F32: return mea::launch_stream<float>(q, d, row_waves, stream);
    case MEA_F16: return mea::launch_stream<_Float16>(q, d, row_waves, stream);
    default: return mea::launch_stream<__bf16>(q, d, row_waves, stream);
  }
}
hipError_t run_combine(const StreamParams& q, const mea_problem* p, int parts, hipStream_t stream) {
  const int d = (int)p->d;
  switch (p->dtype) {
    case MEA_F32: return mea::launch_scored_combine<float>(q, d, parts, stream);
    case MEA_F16: return mea::launch_scored_combine<_Float16>(q, d, parts, stream);
    default: return mea::launch_scored_combine<__bf16>(q, d, parts, stream);
  }
}

mea_status status_of(hipError_t e) { return e == hipSuccess ? MEA_OK : MEA_ERR_HIP; }

// Whether one launch holds that many workgroups of 256 threads (2^32 threads).
bool fits_launch(int64_t wgs) { return wgs < ((int64_t)1 << 24); }

struct BwdWork {
  int64_t n_q_pad, n_qtiles;
  mea::BwdParts parts;
  size_t rows, ranges_q, ranges_k, table, kv_sums, q_sums, total;
};
BwdWork plan_scored_bwd(const mea_problem* p, const mea_score* s) {
  BwdWork w = {};
  w.n_q_pad = (p->n_q + mea::kScoredRowPad - 1) / mea::kScoredRowPad * mea::kScoredRowPad;
  w.n_qtiles = (p->n_q + mea::kScoredDqRows - 1) / mea::kScoredDqRows;
  const int64_t kv = kv_heads_of(p, s->kv_heads);
  w.parts = mea::bwd_parts(p->dtype != MEA_F32, p->causal != 0, (int)p->d, p->n_q, p->n_k, p->batch, p->heads, kv);
  const int kv_parts = w.parts.kv_heads * w.parts.kv_queries;
  if (kv_parts > 1) w.kv_sums = round256((size_t)kv_parts * (size_t)(p->batch * kv) * (size_t)p->n_k * (size_t)p->d * 4);
  if (w.parts.dq > 1) w.q_sums = round256((size_t)w.parts.dq * (size_t)(p->batch * p->heads) * (size_t)p->n_q * (size_t)p->d * 4);
  w.rows = round256((size_t)p->batch * (size_t)p->heads * (size_t)w.n_q_pad * 4);
  if (s->q_doc) {
    w.ranges_q = range_bytes(p->batch, p->n_q);
    w.ranges_k = range_bytes(p->batch, p->n_k);
  }
  if (s->table)
    w.table = round256((size_t)p->batch * (size_t)p->heads * (size_t)w.n_qtiles * (size_t)w.parts.dq *
                       (size_t)s->n_edges * (s->two_sided ? 2 : 1) * 4);
  w.total = 2 * w.rows + w.ranges_q + w.ranges_k + w.table + 2 * w.kv_sums + w.q_sums + 256;
  return w;
}

mea_status check_prefix(const mea_problem* p, const mea_shared_prefix* x) {
  if (!x) return MEA_ERR_INVALID_ARG;
  const mea_status st = check_base(p, x->kv_heads);
  if (st != MEA_OK) return st;
  if (x->n_p < 1 || x->n_p >= kMaxSeq || !aligned4(x->q_pos)) return MEA_ERR_INVALID_ARG;
  int64_t rows;
  if (!mul_ok(p->batch * p->heads, p->n_q, &rows) || rows >= kMaxSeq) return MEA_ERR_INVALID_ARG;
  return MEA_OK;
}
struct PrefixWork {
  StreamPlan shared, own;
  size_t total;
};
PrefixWork plan_prefix(const mea_problem* p, const mea_shared_prefix* x) {
  PrefixWork w;
  const bool is16 = p->dtype != MEA_F32;
  const int64_t kv = kv_heads_of(p, x->kv_heads), G = p->heads / kv;
  // Both key sets fold the heads of a key head; the prefix also all sequences.
  w.shared.fold = w.own.fold = G;
  w.shared.groups = kv;
  w.shared.rows = p->batch * p->n_q * G;
  w.own.groups = kv * p->batch;
  w.own.rows = p->n_q * G;
  // Four row waves read the prefix a quarter as often as one does, which pays on large
  // ones; short or few rows rather share the keys of a tile.  us, row waves 1 / 4, at the
  // best number of ranges each, bf16 d = 128: 256 rows of 8 key heads on 16384 keys 73 / 64,
  // 800 of 8 on 30000 281 / 134, 864 of 3 on 1329 30 / 32, 64 of 8 on 8192 30 / 31; d = 64: 512
  // of 4 on 4000 24 / 27.
  const bool large = w.shared.rows > 64 && (double)(kv * w.shared.rows) * (double)x->n_p > 16e6;
  const int own_least = w.own.rows <= 64 ? 2 : 4;
  const int rwa = large || w.own.rows > 64 ? 4 : (is16 && w.own.rows <= 32 ? 1 : (is16 ? 4 : 2));
  const int rwb = rwa == 4 ? own_least : rwa;
  set_tiles(&w.own, p, rwb, p->n_k, 0);
  // Ranges of the own keys have 4 tiles and more: in shorter ones the parts cost more than
  // they spare (27 sequences of 650, d = 128: 19 us in one range, 26 in more).
  const int64_t long_tiles = p->n_k / (4 * mea::stream_tile(is16, rwb));
  if (w.own.splits > long_tiles) w.own.splits = long_tiles;
  if (w.own.splits > 8) w.own.splits = 8;
  if (w.own.splits < 1) w.own.splits = 1;
  // The own keys' workgroups take places from the prefix: as many as they are, of a large
  // prefix their share of the work (800 rows of 8 on 30000: 134 us, 172 the other way).
  int64_t taken = w.own.groups * w.own.rtiles * w.own.splits;
  if (large) {
    const double own = (double)(w.own.groups * w.own.rtiles * 32 * rwb) * (double)p->n_k;
    const double pre = (double)(w.shared.groups * ((w.shared.rows + 127) / 128 * 128)) * (double)x->n_p;
    taken = (int64_t)(own / (own + pre) * (double)places_of(p, rwa));
  }
  set_tiles(&w.shared, p, rwa, x->n_p, taken);
  w.total = part_bytes(p, w.shared.splits + w.own.splits) + 256;
  return w;
}

}  // namespace

extern "C" {

mea_status mea_scored_attention_fwd_workspace_size(const mea_problem* p, const mea_score* s, size_t* bytes) {
  const mea_status st = check_score(p, s);
  if (st != MEA_OK) return st;
  if (!bytes) return MEA_ERR_INVALID_ARG;
  *bytes = plan_scored_fwd(p, s).total;
  return MEA_OK;
}

mea_status mea_scored_attention_bwd_workspace_size(const mea_problem* p, const mea_score* s, size_t* bytes) {
  const mea_status st = check_score(p, s);
  if (st != MEA_OK) return st;
  if (!bytes) return MEA_ERR_INVALID_ARG;
  *bytes = plan_scored_bwd(p, s).total;
  return MEA_OK;
}

mea_status mea_scored_attention_fwd(const mea_problem* p, const mea_score* s, const void* q, const void* k, const void* v,
                                    void* o, float* lse, void* o_lo, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
  const mea_status st = check_score(p, s);
  if (st != MEA_OK) return st;
  if (!dev_ptr_ok(q) || !dev_ptr_ok(k) || !dev_ptr_ok(v) || !dev_ptr_ok(o)) return MEA_ERR_INVALID_ARG;
  if (lse && !aligned16(lse)) return MEA_ERR_INVALID_ARG;
  if (o_lo && (!aligned16(o_lo) || p->dtype == MEA_F32)) return MEA_ERR_INVALID_ARG;
  const int64_t kv = kv_heads_of(p, s->kv_heads);
  const FwdWork w = plan_scored_fwd(p, s);
  if (w.total && (!workspace || workspace_bytes < w.total)) return MEA_ERR_WORKSPACE;
  StreamParams a = stream_params(p, score_args(p, s), kv, w.pl);
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = lse;
  a.o_lo = o_lo;
  if (o_lo) a.slack = 0.0f;
  {
    const mea_strides* t = p->strides;
    const size_t e = elem_size(p->dtype);
    a.sq = strides_of(t ? &t->q : nullptr, p->heads, p->n_q, p->d);
    a.sk = strides_of(t ? &t->k : nullptr, kv, p->n_k, p->d);
    a.sv = strides_of(t ? &t->v : nullptr, kv, p->n_k, p->d);
    a.so = strides_of(t ? &t->o : nullptr, p->heads, p->n_q, p->d);
    if (!strides_ok(p->batch, p->heads, a.sq, p->n_q, false, e, p->d) || !strides_ok(p->batch, kv, a.sk, p->n_k, false, e, p->d) ||
        !strides_ok(p->batch, kv, a.sv, p->n_k, false, e, p->d) || !strides_ok(p->batch, p->heads, a.so, p->n_q, true, e, p->d))
      return MEA_ERR_INVALID_ARG;
  }
  const int64_t grid = w.pl.rtiles * w.pl.groups * w.pl.splits;
  if (!fits_launch(grid) || (w.pl.splits > 1 && !fits_launch(mea::combine_blocks(a.out_rows, p->d, w.pl.splits))) ||
      (s->q_doc && !fits_launch(p->batch * ((p->n_k + 31) / 32))))
    return MEA_ERR_INVALID_ARG;
  if (p->causal)
    a.tile_order = mea::causal_tile_order(p->batch * kv * p->n_k * 2 * p->d * (int64_t)elem_size(p->dtype), grid, true);
  float* at = align256(workspace, 0);
  if (s->q_doc) {
    int2* r = reinterpret_cast<int2*>(at);
    a.s.k_range = r;
    const hipError_t e = mea::launch_doc_ranges(s->k_doc, p->n_k, p->batch, r, stream);
    if (e != hipSuccess) return MEA_ERR_HIP;
  }
  a.direct = w.pl.splits == 1;
  if (!a.direct) carve_parts(&a, p, w.pl.splits, at + w.ranges / 4);
  const hipError_t e = run_stream(a, p, w.pl.row_waves, stream);
  if (e != hipSuccess || a.direct) return status_of(e);
  return status_of(run_combine(a, p, (int)w.pl.splits, stream));
}

mea_status mea_scored_attention_bwd(const mea_problem* p, const mea_score* s, const void* q, const void* k, const void* v,
                                    const void* o, const void* o_lo, const void* d_o, const float* lse, void* dq, void* dk,
                                    void* dv, void* d_table, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const mea_status st = check_score(p, s);
  if (st != MEA_OK) return st;
  if (!dev_ptr_ok(q) || !dev_ptr_ok(k) || !dev_ptr_ok(v) || !dev_ptr_ok(o) || !dev_ptr_ok(d_o) || !dev_ptr_ok(lse))
    return MEA_ERR_INVALID_ARG;
  if (o_lo && (!aligned16(o_lo) || p->dtype == MEA_F32)) return MEA_ERR_INVALID_ARG;
  if (!aligned16(dq) || !aligned16(dk) || !aligned16(dv) || (dk == nullptr) != (dv == nullptr) || (!dq && !dk))
    return MEA_ERR_INVALID_ARG;
  if (d_table && (!s->table || !dq || !table_aligned(d_table, s->table_dtype))) return MEA_ERR_INVALID_ARG;
  const BwdWork w = plan_scored_bwd(p, s);
  if (!workspace || workspace_bytes < w.total) return MEA_ERR_WORKSPACE;
  const int64_t kv = kv_heads_of(p, s->kv_heads);
  ScoredBwdParams a = {};
  a.s = score_args(p, s);
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.o_lo = o_lo;
  a.d_o = d_o;
  a.lse = lse;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.d_table = d_table;
  a.n_q = p->n_q;
  a.n_k = p->n_k;
  a.n_q_pad = w.n_q_pad;
  a.n_b = (int)p->batch;
  a.heads_kv = (int)kv;
  a.heads_per_kv = (int)(p->heads / kv);
  a.scale = p->scale;
  {
    const mea_strides* t = p->strides;
    const size_t e = elem_size(p->dtype);
    const int64_t d = p->d, B = p->batch, H = p->heads;
    a.sq = strides_of(t ? &t->q : nullptr, H, p->n_q, d);
    a.sk = strides_of(t ? &t->k : nullptr, kv, p->n_k, d);
    a.sv = strides_of(t ? &t->v : nullptr, kv, p->n_k, d);
    a.so = strides_of(t ? &t->o : nullptr, H, p->n_q, d);
    a.sdo = strides_of(t ? &t->d_o : nullptr, H, p->n_q, d);
    a.sdq = strides_of(t ? &t->dq : nullptr, H, p->n_q, d);
    a.sdk = strides_of(t ? &t->dk : nullptr, kv, p->n_k, d);
    a.sdv = strides_of(t ? &t->dv : nullptr, kv, p->n_k, d);
    if (!strides_ok(B, H, a.sq, p->n_q, false, e, d) || !strides_ok(B, kv, a.sk, p->n_k, false, e, d) ||
        !strides_ok(B, kv, a.sv, p->n_k, false, e, d) || !strides_ok(B, H, a.so, p->n_q, false, e, d) ||
        !strides_ok(B, H, a.sdo, p->n_q, false, e, d) || (dq && !strides_ok(B, H, a.sdq, p->n_q, true, e, d)) ||
        (dk && (!strides_ok(B, kv, a.sdk, p->n_k, true, e, d) || !strides_ok(B, kv, a.sdv, p->n_k, true, e, d))))
      return MEA_ERR_INVALID_ARG;
  }
  const int64_t rows_wg = 256 / (p->d * (int64_t)elem_size(p->dtype) / 16);
  const int64_t wgs = p->batch * (kv * w.parts.kv_heads * w.parts.kv_queries * ((p->n_k + 127) / 128) +
                                  p->heads * w.parts.dq * w.n_qtiles);
  if (!fits_launch(p->batch * p->heads * w.n_q_pad / rows_wg + 1) || !fits_launch(wgs) ||
      ((w.kv_sums || w.q_sums) && !fits_launch((p->batch * (p->heads * p->n_q + 2 * kv * p->n_k) + 24) * p->d / 4 / 256)) ||
      (s->q_doc && !fits_launch(p->batch * ((p->n_k > p->n_q ? p->n_k : p->n_q) + 31) / 32)))
    return MEA_ERR_INVALID_ARG;
  if (p->causal)
    a.tile_order = mea::causal_tile_order(p->batch * kv * p->n_k * 2 * p->d * (int64_t)elem_size(p->dtype), 0, false);
  float* at = align256(workspace, 0);
  a.lse2 = at;
  a.neg_d = at + w.rows / 4;
  at += 2 * w.rows / 4;
  if (s->q_doc) {
    int2* rq = reinterpret_cast<int2*>(at);
    int2* rk = reinterpret_cast<int2*>(at + w.ranges_q / 4);
    a.s.q_range = rq;
    a.s.k_range = rk;
    at += (w.ranges_q + w.ranges_k) / 4;
    hipError_t e = mea::launch_doc_ranges(s->q_doc, p->n_q, p->batch, rq, stream);
    if (s->q_doc == s->k_doc && p->n_q == p->n_k) a.s.k_range = rq;
    else if (e == hipSuccess) e = mea::launch_doc_ranges(s->k_doc, p->n_k, p->batch, rk, stream);
    if (e != hipSuccess) return MEA_ERR_HIP;
  }
  if (d_table) a.table_part = at;
  at += w.table / 4;
  a.kv_heads_parts = w.parts.kv_heads;
  a.kv_query_parts = w.parts.kv_queries;
  a.dq_parts = w.parts.dq;
  if (w.kv_sums && dk) {
    a.dk_part = at;
    a.dv_part = at + w.kv_sums / 4;
  }
  if (w.q_sums && dq) a.dq_part = at + 2 * w.kv_sums / 4;
  const int d = (int)p->d;
  switch (p->dtype) {
    case MEA_F32: return status_of(mea::launch_scored_bwd<float>(a, d, stream));
    case MEA_F16: return status_of(mea::launch_scored_bwd<_Float16>(a, d, stream));
    default: return status_of(mea::launch_scored_bwd<__bf16>(a, d, stream));
  }
}

mea_status mea_prefix_attention_fwd_workspace_size(const mea_problem* p, const mea_shared_prefix* x, size_t* bytes) {
  const mea_status st = check_prefix(p, x);
  if (st != MEA_OK) return st;
  if (!bytes) return MEA_ERR_INVALID_ARG;
  *bytes = plan_prefix(p, x).total;
  return MEA_OK;
}

mea_status mea_prefix_attention_fwd(const mea_problem* p, const mea_shared_prefix* x, const void* q, const void* k,
                                    const void* v, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
  const mea_status st = check_prefix(p, x);
  if (st != MEA_OK) return st;
  if (!dev_ptr_ok(q) || !dev_ptr_ok(k) || !dev_ptr_ok(v) || !dev_ptr_ok(o) || !dev_ptr_ok(x->k) || !dev_ptr_ok(x->v))
    return MEA_ERR_INVALID_ARG;
  if (lse && !aligned16(lse)) return MEA_ERR_INVALID_ARG;
  const PrefixWork w = plan_prefix(p, x);
  if (!workspace || workspace_bytes < w.total) return MEA_ERR_WORKSPACE;
  const int64_t kv = kv_heads_of(p, x->kv_heads), d = p->d;
  const size_t e = elem_size(p->dtype);
  ScoreArgs sa = score_args(p, nullptr);
  sa.q_pos = x->q_pos;
  StreamParams own = stream_params(p, sa, kv, w.own);
  const mea_strides* t = p->strides;
  own.q = q;
  own.k = k;
  own.v = v;
  own.o = o;
  own.lse = lse;
  own.sq = strides_of(t ? &t->q : nullptr, p->heads, p->n_q, d);
  own.sk = strides_of(t ? &t->k : nullptr, kv, p->n_k, d);
  own.sv = strides_of(t ? &t->v : nullptr, kv, p->n_k, d);
  own.so = strides_of(t ? &t->o : nullptr, p->heads, p->n_q, d);
  auto shared_strides = [&](const mea_tensor_strides& s) {
    return s.row ? mea::TensorStrides{0, s.head, s.row} : mea::TensorStrides{0, x->n_p * d, d};
  };
  const mea::TensorStrides spk = shared_strides(x->k_strides), spv = shared_strides(x->v_strides);
  if (!strides_ok(p->batch, p->heads, own.sq, p->n_q, false, e, d) || !strides_ok(p->batch, kv, own.sk, p->n_k, false, e, d) ||
      !strides_ok(p->batch, kv, own.sv, p->n_k, false, e, d) || !strides_ok(p->batch, p->heads, own.so, p->n_q, true, e, d) ||
      !strides_ok(1, kv, spk, x->n_p, false, e, d) || !strides_ok(1, kv, spv, x->n_p, false, e, d))
    return MEA_ERR_INVALID_ARG;
  const int64_t parts = w.shared.splits + w.own.splits;
  if (!fits_launch(w.own.rtiles * w.own.groups * w.own.splits + w.shared.rtiles * w.shared.groups * w.shared.splits) ||
      !fits_launch(mea::combine_blocks(own.out_rows, d, parts)))
    return MEA_ERR_INVALID_ARG;
  carve_parts(&own, p, parts, align256(workspace, 0));
  own.split0 = (int)w.shared.splits;
  StreamParams pre = stream_params(p, score_args(p, nullptr), kv, w.shared);
  pre.s.causal = 0;  // every query sees the whole prefix
  pre.s.kv_len = nullptr;
  pre.q = q;
  pre.sq = own.sq;
  pre.k = x->k;
  pre.v = x->v;
  pre.sk = spk;
  pre.sv = spv;
  pre.n_k = x->n_p;
  pre.batches = (int)p->batch;
  pre.n_b = 1;
  pre.part_o = own.part_o;
  pre.part_m = own.part_m;
  pre.part_l = own.part_l;
  const int dd = (int)d, ra = w.shared.row_waves, rb = w.own.row_waves;
  hipError_t err;
  switch (p->dtype) {
    case MEA_F32: err = mea::launch_stream_pair<float>(pre, own, dd, ra, rb, stream); break;
    case MEA_F16: err = mea::launch_stream_pair<_Float16>(pre, own, dd, ra, rb, stream); break;
    default: err = mea::launch_stream_pair<__bf16>(pre, own, dd, ra, rb, stream);
  }
  if (err == hipSuccess) err = run_combine(own, p, (int)parts, stream);
  return status_of(err);
}

}  // extern "C"
