// C entry points of the attention over packed sequences: argument checks, sizes, and the buckets of the position bias.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include "../../include/lynx.h"
#include "kernels.h"

namespace {

using lynx::PackedAttn;

bool aligned(const void* p, uintptr_t to) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool stride_ok(int64_t stride, int64_t width) { return stride >= width && stride % 8 == 0 && stride <= LYNX_ATTENTION_MAX_STRIDE; }

// The shape's part of the kernels' arguments.
lynx_status make_args(const lynx_attention_config* c, bool backward, PackedAttn* g) {
  if (c == nullptr) return LYNX_ERR_INVALID_ARG;
  if (!(c->scale > 0.0f) || !isfinite(c->scale) || (c->num_buckets > 0 && c->bucket_starts == nullptr)) return LYNX_ERR_INVALID_ARG;
  if (c->dtype != LYNX_F32 && c->dtype != LYNX_BF16) return LYNX_ERR_SHAPE;
  if (c->heads <= 0 || c->kv_heads <= 0 || c->heads % c->kv_heads != 0 || c->heads > LYNX_ATTENTION_MAX_STRIDE / 8) return LYNX_ERR_SHAPE;
  if (c->head_dim <= 0 || c->head_dim % 8 != 0 || c->head_dim > LYNX_ATTENTION_MAX_HEAD_DIM) return LYNX_ERR_SHAPE;
  if (c->tokens <= 0 || c->tokens > (1 << 24) || c->sequences <= 0 || c->sequences > (1 << 20)) return LYNX_ERR_SHAPE;
  if (c->num_buckets < 0 || c->num_buckets > LYNX_MAX_BUCKETS) return LYNX_ERR_SHAPE;
  const int64_t q_width = static_cast<int64_t>(c->heads) * c->head_dim, kv_width = static_cast<int64_t>(c->kv_heads) * c->head_dim;
  if (!stride_ok(c->q_stride, q_width) || !stride_ok(c->k_stride, kv_width) || !stride_ok(c->v_stride, kv_width) || !stride_ok(c->out_stride, q_width))
    return LYNX_ERR_SHAPE;
  if (backward && (!stride_ok(c->dq_stride, q_width) || !stride_ok(c->dk_stride, kv_width) || !stride_ok(c->dv_stride, kv_width))) return LYNX_ERR_SHAPE;
  *g = PackedAttn{};
  g->sequences = c->sequences; g->tokens = c->tokens; g->heads = c->heads; g->kv_heads = c->kv_heads; g->d = c->head_dim;
  g->scale = c->scale;
  g->q_stride = c->q_stride; g->k_stride = c->k_stride; g->v_stride = c->v_stride; g->out_stride = c->out_stride;
  g->dq_stride = c->dq_stride; g->dk_stride = c->dk_stride; g->dv_stride = c->dv_stride;
  g->buckets = c->num_buckets;
  for (int i = 0; i < c->num_buckets; ++i) {
    if (c->bucket_starts[i] < (i == 0 ? 0 : c->bucket_starts[i - 1]) || (i == 0 && c->bucket_starts[0] != 0)) return LYNX_ERR_INVALID_ARG;
    if (c->bucket_starts[i] > LYNX_MAX_DISTANCE) return LYNX_ERR_SHAPE;
    g->starts[i] = c->bucket_starts[i];
  }
  for (int i = c->num_buckets; i < lynx::kMaxBuckets; ++i) g->starts[i] = INT32_MAX;
  g->far = c->num_buckets > 0 && g->starts[c->num_buckets - 1] > 1 ? g->starts[c->num_buckets - 1] : 1;
  lynx::attn_packed_choose(c->dtype == LYNX_BF16 ? 1 : 0, g);
  return lynx::attn_packed_fits(*g) ? LYNX_OK : LYNX_ERR_SHAPE;
}

size_t round_up(size_t n) { return (n + 255) / 256 * 256; }
size_t delta_bytes(const PackedAttn& g) { return round_up(static_cast<size_t>(g.heads) * g.tokens * sizeof(float)); }
size_t partials_bytes(const PackedAttn& g) { return round_up(static_cast<size_t>(g.row_slots) * g.heads * g.buckets * sizeof(float)); }

// (a b)^.. in whole numbers, for the borders of the buckets: at most 64 factors below 2^12
struct Whole {
  static constexpr int kWords = 32;
  uint32_t w[kWords] = {1};
  void times(uint32_t f) {
    uint64_t carry = 0;
    for (uint32_t& x : w) {
      carry += static_cast<uint64_t>(x) * f;
      x = static_cast<uint32_t>(carry);
      carry >>= 32;
    }
  }
  void times(uint32_t f, int n) {
    for (int i = 0; i < n; ++i) times(f);
  }
  bool operator<(const Whole& o) const {
    for (int i = kWords - 1; i >= 0; --i)
      if (w[i] != o.w[i]) return w[i] < o.w[i];
    return false;
  }
};

}  // namespace

namespace lynx {
lynx_status attention_check(const lynx_attention_config* cfg) {
  PackedAttn g;
  return make_args(cfg, true, &g);
}
}  // namespace lynx

extern "C" {

lynx_status lynx_position_buckets(int num_buckets, int max_distance, int32_t* starts_out) {
  if (starts_out == nullptr || num_buckets < 2 || num_buckets > LYNX_MAX_BUCKETS) return LYNX_ERR_INVALID_ARG;
  const int exact = num_buckets / 2, steps = num_buckets - exact;
  if (max_distance <= exact || max_distance > LYNX_MAX_DISTANCE) return LYNX_ERR_INVALID_ARG;
  for (int b = 0; b < exact; ++b) starts_out[b] = b;
  // Bucket exact + b starts at the least n with log(n / exact) / log(max_distance / exact) steps >= b, that is
  // n^steps exact^b >= max_distance^b exact^steps: no rounding decides on which side of a border a distance lies.
  for (int b = 0; b < steps; ++b) {
    Whole least;
    least.times(static_cast<uint32_t>(max_distance), b);
    least.times(static_cast<uint32_t>(exact), steps);
    int lo = exact, hi = max_distance;  // the answer lies in between
    while (lo < hi) {
      const int n = (lo + hi) / 2;
      Whole x;
      x.times(static_cast<uint32_t>(n), steps);
      x.times(static_cast<uint32_t>(exact), b);
      if (x < least) lo = n + 1;
      else hi = n;
    }
    starts_out[exact + b] = lo;
  }
  return LYNX_OK;
}

lynx_status lynx_attention_forward(const lynx_attention_config* cfg, const void* q, const void* k, const void* v, const int32_t* offsets,
                                   const void* bias_table, void* out, float* lse, void* hip_stream) {
  PackedAttn g;
  const lynx_status s = make_args(cfg, false, &g);
  if (s != LYNX_OK) return s;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(offsets, 4) || !aligned(lse, 4)) return LYNX_ERR_INVALID_ARG;
  if (g.buckets > 0 && !aligned(bias_table, 16)) return LYNX_ERR_INVALID_ARG;
  g.q = q; g.k = k; g.v = v; g.offsets = offsets; g.out = out; g.lse = lse;
  if (g.buckets > 0) g.table = bias_table;
  return lynx::attn_packed_fwd(cfg->dtype, g, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? LYNX_OK : LYNX_ERR_HIP;
}

size_t lynx_attention_backward_bytes(const lynx_attention_config* cfg) {
  PackedAttn g;
  if (make_args(cfg, true, &g) != LYNX_OK) return 0;
  return 2 * delta_bytes(g) + (g.buckets > 0 ? partials_bytes(g) : 0);
}

lynx_status lynx_attention_backward(const lynx_attention_config* cfg, const void* q, const void* k, const void* v, const int32_t* offsets,
                                    const void* bias_table, const void* out, const float* lse, const void* d_out, void* d_q, void* d_k,
                                    void* d_v, void* d_bias_table, void* workspace, size_t workspace_bytes, void* hip_stream) {
  PackedAttn g;
  const lynx_status s = make_args(cfg, true, &g);
  if (s != LYNX_OK) return s;
  const void* const device[] = {q, k, v, out, d_out, d_q, d_k, d_v};
  for (const void* p : device)
    if (!aligned(p, 16)) return LYNX_ERR_INVALID_ARG;
  if (!aligned(offsets, 4) || !aligned(lse, 4) || !aligned(workspace, 256)) return LYNX_ERR_INVALID_ARG;
  if (g.buckets > 0 && (!aligned(bias_table, 16) || !aligned(d_bias_table, 16))) return LYNX_ERR_INVALID_ARG;
  if (workspace_bytes < lynx_attention_backward_bytes(cfg)) return LYNX_ERR_OOM;
  g.q = q; g.k = k; g.v = v; g.offsets = offsets; g.out = const_cast<void*>(out); g.lse = const_cast<float*>(lse);
  g.d_out = d_out; g.dq = d_q; g.dk = d_k; g.dv = d_v;
  g.delta = static_cast<float*>(workspace);
  g.offset = g.delta + delta_bytes(g) / sizeof(float);
  if (g.buckets > 0) {
    g.table = bias_table;
    g.d_table = d_bias_table;
    g.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * delta_bytes(g));
  }
  return lynx::attn_packed_bwd(cfg->dtype, g, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? LYNX_OK : LYNX_ERR_HIP;
}

}  // extern "C"
