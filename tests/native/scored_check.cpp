// Host code of attention with modified scores and over a shared prefix
// (scored_api.hip) under sanitizers, with the launchers replaced by recorders: over a range
// of shapes every buffer that a launch gets lies inside the workspace that the size call
// asked for, none overlap, and grids, folds and parts are what the kernels assume.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "../../paper_2112_05682_amd/csrc/scored.hpp"
#include "../../include/mea.h"

namespace {
struct Span {
  const char* name;
  uintptr_t at;
  size_t bytes;
};
std::vector<Span> g_spans;
bool g_bad = false;
int g_streams, g_combines, g_bwds;

void fail(const char* what) {
  fprintf(stderr, "scored_check: %s\n", what);
  g_bad = true;
}
void expect(bool ok, const char* what) {
  if (!ok) fail(what);
}
void use(const char* name, const void* p, size_t bytes) {
  if (p) g_spans.push_back({name, (uintptr_t)p, bytes});
}
void stream_parts(const mea::StreamParams& p, int d, int rw, bool is16) {
  expect(rw == 4 || rw == 2 || (rw == 1 && is16) || (rw == 0 && !is16 && p.group_rows <= mea::kFewRows && !p.s.q_doc),
         "row waves");
  expect(p.fold >= 1 && p.heads_per_kv % p.fold == 0, "fold");
  expect(p.groups_per_kv * p.fold == p.heads_per_kv, "groups of a key head");
  expect(p.n_splits >= 1 && p.n_groups >= 1, "grid");
  expect(p.group_rows == (int64_t)p.batches * p.n_q * p.fold, "rows");
  const int64_t covered = (int64_t)p.n_groups * p.group_rows;
  expect(covered == p.out_rows, "every output row has one group");
  if (!p.direct) {
    use("m", p.part_m + (int64_t)p.split0 * p.out_rows, (size_t)p.n_splits * p.out_rows * 4);
    use("l", p.part_l + (int64_t)p.split0 * p.out_rows, (size_t)p.n_splits * p.out_rows * 4);
    use("o", p.part_o + (int64_t)p.split0 * p.out_rows * d, (size_t)p.n_splits * p.out_rows * d * 4);
  } else {
    expect(p.n_splits == 1, "direct output");
  }
}
}  // namespace

namespace mea {
hipError_t launch_doc_ranges(const int*, int64_t n, int64_t batches, int2* out, hipStream_t) {
  use("ranges", out, (size_t)batches * ((n + 31) / 32) * 8);
  return hipSuccess;
}
hipError_t launch_scored_table(const ScoredBwdParams&, hipStream_t) { return hipSuccess; }
template <typename T>
hipError_t launch_stream(const StreamParams& p, int d, int rw, hipStream_t) {
  ++g_streams;
  stream_parts(p, d, rw, sizeof(T) == 2);
  return hipSuccess;
}
template <typename T>
hipError_t launch_stream_pair(const StreamParams& a, const StreamParams& b, int d, int rwa, int rwb, hipStream_t) {
  g_streams += 2;
  stream_parts(a, d, rwa, sizeof(T) == 2);
  stream_parts(b, d, rwb, sizeof(T) == 2);
  expect((rwa == 4 && (rwb == 4 || rwb == 2)) || (rwa == rwb && rwa == (sizeof(T) == 2 ? 1 : 2)), "pair of row waves");
  return hipSuccess;
}
template <typename T>
hipError_t launch_scored_combine(const StreamParams& p, int, int n_parts, hipStream_t) {
  ++g_combines;
  expect(n_parts >= 2 && p.part_o, "combine");
  return hipSuccess;
}
template <typename T>
hipError_t launch_scored_bwd(const ScoredBwdParams& p, int d, hipStream_t) {
  ++g_bwds;
  const int64_t rows = (int64_t)p.n_b * p.s.heads * p.n_q_pad;
  use("lse", p.lse2, rows * 4);
  use("d", p.neg_d, rows * 4);
  const int kv_parts = p.kv_heads_parts * p.kv_query_parts;
  expect(kv_parts >= 1 && p.dq_parts >= 1 && p.heads_per_kv % p.kv_heads_parts == 0, "parts");
  expect((p.dk_part != nullptr) == (kv_parts > 1 && p.dk) && (p.dq_part != nullptr) == (p.dq_parts > 1 && p.dq), "sums of parts");
  const size_t kv = (size_t)kv_parts * p.n_b * p.heads_kv * p.n_k * d * 4;
  use("dk", p.dk_part, kv);
  use("dv", p.dv_part, kv);
  use("dq", p.dq_part, (size_t)p.dq_parts * p.n_b * p.s.heads * p.n_q * d * 4);
  use("table", p.table_part,
      (size_t)p.n_b * p.s.heads * ((p.n_q + kScoredDqRows - 1) / kScoredDqRows) * p.dq_parts * p.s.n_buckets() * 4);
  return hipSuccess;
}
#define INSTANCES(T)                                                                                       \
  template hipError_t launch_stream<T>(const StreamParams&, int, int, hipStream_t);                        \
  template hipError_t launch_stream_pair<T>(const StreamParams&, const StreamParams&, int, int, int, hipStream_t); \
  template hipError_t launch_scored_combine<T>(const StreamParams&, int, int, hipStream_t);                \
  template hipError_t launch_scored_bwd<T>(const ScoredBwdParams&, int, hipStream_t);
INSTANCES(float)
INSTANCES(_Float16)
INSTANCES(__bf16)
}  // namespace mea

static void check_spans(uintptr_t ws, size_t bytes) {
  for (size_t i = 0; i < g_spans.size(); ++i) {
    const Span& a = g_spans[i];
    if (a.at < ws || a.at + a.bytes > ws + bytes) {
      fprintf(stderr, "%s outside the workspace\n", a.name);
      g_bad = true;
    }
    for (size_t j = 0; j < i; ++j)
      if (a.at < g_spans[j].at + g_spans[j].bytes && g_spans[j].at < a.at + a.bytes) {
        fprintf(stderr, "%s and %s overlap\n", a.name, g_spans[j].name);
        g_bad = true;
      }
  }
  g_spans.clear();
}

int main() {
  int n = 0;
  int32_t edges[16];
  for (int i = 0; i < 16; ++i) edges[i] = i * 3;
  float dev_mem[4];
  (void)dev_mem;
  void* const fake = reinterpret_cast<void*>((uintptr_t)0x100000);
  const int64_t sizes[] = {1, 3, 31, 64, 65, 200, 1000, 4096, 33000};
  for (int dtype = 0; dtype < 3; ++dtype)
    for (int64_t d : {64, 128})
      for (int64_t B : {1, 3, 40})
        for (int64_t kv : {1, 2, 8})
          for (int64_t G : {1, 3, 8})
            for (int64_t nq : sizes)
              for (int64_t nk : sizes) {
                if ((double)B * kv * G * nq * d > 4e9 || (double)B * kv * nk * d > 4e9) continue;
                for (int mods = 0; mods < 4; ++mods) {
                  mea_problem p = {};
                  p.batch = B;
                  p.heads = kv * G;
                  p.n_q = nq;
                  p.n_k = nk;
                  p.d = d;
                  p.dtype = dtype;
                  p.causal = mods & 1;
                  p.scale = 0.125f;
                  mea_score s = {};
                  s.kv_heads = kv;
                  if (mods & 2) {
                    s.q_doc = s.k_doc = static_cast<const int32_t*>(fake);
                    s.table = fake;
                    s.edges = edges;
                    s.n_edges = 16;
                    s.two_sided = !p.causal;
                    s.softcap = 30.0f;
                  }
                  size_t bytes = 0;
                  expect(mea_scored_attention_fwd_workspace_size(&p, &s, &bytes) == MEA_OK, "forward size");
                  const uintptr_t ws = 0x7000000010;  // not aligned to 256
                  expect(mea_scored_attention_fwd(&p, &s, fake, fake, fake, fake, (float*)fake, nullptr, (void*)ws, bytes, nullptr) ==
                             MEA_OK,
                         "forward");
                  check_spans(ws, bytes);
                  expect(mea_scored_attention_bwd_workspace_size(&p, &s, &bytes) == MEA_OK, "backward size");
                  expect(mea_scored_attention_bwd(&p, &s, fake, fake, fake, fake, nullptr, fake, (float*)fake, fake, fake, fake,
                                                  s.table ? fake : nullptr, (void*)ws, bytes, nullptr) == MEA_OK,
                         "backward");
                  check_spans(ws, bytes);
                  if (!(mods & 2)) {
                    mea_shared_prefix x = {};
                    x.kv_heads = kv;
                    x.n_p = 1 + nk * 7 / 3;
                    x.k = x.v = fake;
                    expect(mea_prefix_attention_fwd_workspace_size(&p, &x, &bytes) == MEA_OK, "prefix size");
                    expect(mea_prefix_attention_fwd(&p, &x, fake, fake, fake, fake, nullptr, (void*)ws, bytes, nullptr) == MEA_OK,
                           "prefix");
                    check_spans(ws, bytes);
                  }
                  ++n;
                  if (g_bad) {
                    fprintf(stderr, "dtype %d d %d B %d kv %d G %d nq %d nk %d mods %d\n", dtype, (int)d, (int)B, (int)kv, (int)G,
                            (int)nq, (int)nk, mods);
                    return 1;
                  }
                }
              }
  expect(g_streams > 0 && g_combines > 0 && g_bwds > 0 && n > 1000, "cases");
  if (g_bad) return 1;
  printf("scored_check ok: %d problems\n", n);
  return 0;
}
