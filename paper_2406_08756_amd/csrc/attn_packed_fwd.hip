// Causal attention over packed sequences with grouped heads, forward: out = softmax(scale Q K^T + bias) V, one pass over the
// keys with a running maximum and sum; no seq x seq tensor.
#include "attn_packed.h"

namespace lynx {
namespace {

template <typename T, int DP> struct Fwd {
  static constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;  // keys per tile
  static constexpr size_t kTileBytes = static_cast<size_t>(kKeys) * DP * sizeof(T);
  static constexpr size_t kLds = 4 * kTileBytes;  // K and V, two of each
};

// One row again, pair by pair: lanes take keys for the scores and columns for the sum.
template <typename T>
__device__ void sum_row_forward(const PackedAttn& g, const T* q, const T* k, const T* v, int tok, float max2, float total, float scale2,
                                const float* bias, T* out) {
  const int lane = threadIdx.x & (kWave - 1);
  bool clean = true;
  float acc[2] = {0.f, 0.f};
  for (int j0 = 0; j0 <= tok; j0 += kWave) {
    const int j = j0 + lane;
    float p = 0.f;
    if (j <= tok) {
      clean = clean && row_finite(v + j * g.v_stride, g.d);
      float z = row_dot(q, k + j * g.k_stride, g.d) * scale2;
      if (bias != nullptr) z += bias[min(tok - j, g.far) + kPad];
      p = exp2_fast(z - max2) / total;
    }
    const int n = min(kWave, tok + 1 - j0);
    for (int i = 0; i < n; ++i) {
      const float pi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), i));
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (lane + kWave * c < g.d) acc[c] = __builtin_fmaf(pi, load1(v + (j0 + i) * g.v_stride + lane + kWave * c), acc[c]);
    }
  }
  if (__all(clean)) return;  // the values it sees are finite: the tile's own result stands
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + kWave * c < g.d) store1(out + lane + kWave * c, acc[c]);
}

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(kThreads, 2) void attn_packed_fwd_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Fwd<T, DP> S;
  constexpr int kKeys = S::kKeys, kBlocks = kKeys / 32;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  constexpr int kTileElems = kKeys * DP;
  float* const bias = reinterpret_cast<float*>(smem_raw + S::kLds);

  const int subs = g.heads >> g.pack;
  const int head0 = (static_cast<int>(blockIdx.x) % subs) << g.pack;
  SeqTile w;
  if (!find_tile</*LAST_FIRST=*/true>(g, static_cast<int>(blockIdx.x) / subs, kRowsLog, g.pack, &w)) return;
  if (BIAS) fill_bias<T, kThreads>(g, head0, bias);

  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = 1 << g.pack;
  const int kv = head0 / (g.heads / g.kv_heads);
  const T* const q = static_cast<const T*>(g.q) + w.start * g.q_stride + static_cast<long long>(head0) * g.d;
  const T* const k = static_cast<const T*>(g.k) + w.start * g.k_stride + static_cast<long long>(kv) * g.d;
  const T* const v = static_cast<const T*>(g.v) + w.start * g.v_stride + static_cast<long long>(kv) * g.d;
  T* const out = static_cast<T*>(g.out) + w.start * g.out_stride + static_cast<long long>(head0) * g.d;

  const int row0 = (w.tile << kRowsLog) + 32 * wave;  // this wavefront's
  const int row = row0 + (lane & 31), tok = row >> g.pack, hp = row & (heads - 1);
  const int first_tok = row0 >> g.pack, last_tok = first_tok < w.len ? min((row0 + 31) >> g.pack, w.len - 1) : -1;
  const bool there = tok < w.len;
  const float scale2 = g.scale * kLog2e;

  typename Op::Frag qf[L::kSteps];
  {
    const int left = min(w.len - first_tok, 32);
    const RowBuffer b = row_buffer(q + first_tok * g.q_stride,
                                   left > 0 ? static_cast<uint32_t>((left - 1) * g.q_stride + heads * g.d) * static_cast<uint32_t>(sizeof(T)) : 0u);
    load_row_frags<T, DP>(b, (static_cast<uint32_t>(tok - first_tok) * static_cast<uint32_t>(g.q_stride) + hp * g.d) * static_cast<uint32_t>(sizeof(T)), g.d, lane, qf);
  }
  const int end_tok = min(((w.tile + 1) << kRowsLog) >> g.pack, w.len);  // of the workgroup: the keys it sees
  const int tiles = (end_tok + kKeys - 1) / kKeys;
  const float* const my_bias = BIAS ? bias + hp * table_stride(g) + kPad : nullptr;

  Stage<T, DP, kKeys, kThreads> sk, sv;
  floatx16_t o[DP / 32];
  float m, total;
  bool spoilt = false;
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) o[b] = floatx16_t{};
    m = -kInf;       // maximum of the logits so far, times log2 e
    total = 0.f;     // this half's share of the sum
    sk.load_keys(k, g.k_stride, 0, w.len, g.d);
    sv.load_keys(v, g.v_stride, 0, w.len, g.d);
    for (int t = 0; t < tiles; ++t) {
      T* const kt = lds + (t & 1) * 2 * kTileElems;
      T* const vt = kt + kTileElems;
      sk.template store<false>(kt);
      if (clean) sv.template store<true>(vt);
      else sv.template store<false>(vt);
      __syncthreads();
      if (t + 1 < tiles) {
        sk.load_keys(k, g.k_stride, (t + 1) * kKeys, w.len, g.d);
        sv.load_keys(v, g.v_stride, (t + 1) * kKeys, w.len, g.d);
      }
      const int key0 = t * kKeys;
      if (key0 > last_tok) continue;
      floatx16_t s[kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        s[b] = floatx16_t{};
#pragma unroll
        for (int c = 0; c < L::kSteps; ++c) Op::mma(s[b], L::row_frag(kt, 32 * b, c, lane), qf[c]);
      }
      float top = -kInf;
      const bool edge = key0 + kKeys - 1 > first_tok;
      if (BIAS) {
        const int apart = tok - key0 - 4 * half;
        if (first_tok - (key0 + kKeys - 1) < g.far) {
          const float* const at = my_bias + apart;
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              // (masked by a choice: the sum would be NaN where the score is)
              const float z = __builtin_fmaf(s[b][i], scale2, at[-(32 * b + acc_row(i, 0))]);
              s[b][i] = apart >= 32 * b + acc_row(i, 0) ? z : -kInf;
              top = fmaxf(top, s[b][i]);
            }
        } else {
          const float far = my_bias[g.far];
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              s[b][i] = __builtin_fmaf(s[b][i], scale2, far);
              top = fmaxf(top, s[b][i]);
            }
        }
      } else {
        if (edge) {
          const int apart = tok - key0 - 4 * half;
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (apart < 32 * b + acc_row(i, 0)) s[b][i] = -kInf;
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top *= scale2;
      }
      top = fmaxf(top, other_half(top));
      if (__any(top > m)) {
        const float now = fmaxf(top, m);
        const float shrink = now == -kInf ? 1.f : exp2_fast(m - now);
        m = now;
        total *= shrink;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[b][i] *= shrink;
      }
      const float base = m == -kInf ? 0.f : m;  // (a row that has seen nothing yet: every probability 0)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[b][i] = exp2_fast(BIAS ? s[b][i] - base : __builtin_fmaf(s[b][i], scale2, -base));
          total += s[b][i];
        }
#pragma unroll
        for (int c = 0; c < L::kGroups; ++c) {
          const typename Op::Frag p = Op::from_acc(s[b], c);
#pragma unroll
          for (int e = 0; e < DP / 32; ++e) Op::mma(o[e], L::col_frag(vt, 32 * b, c, 32 * e, lane), p);
        }
      }
    }
    total += other_half(total);
    if (clean) break;
    float check = total * 0.f;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) check = __builtin_fmaf(o[b][i], 0.f, check);
    check += other_half(check);
    spoilt = there && check != 0.f;
    if (!__syncthreads_or(spoilt)) break;
  }
  const float inverse = total == 0.f ? 0.f : 1.f / total;
  T* const mine = out + tok * g.out_stride + hp * g.d;
  if (there) {
    if (half == 0) g.lse[static_cast<long long>(head0 + hp) * g.tokens + w.start + tok] = (m + __builtin_log2f(total)) * kLn2;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = 32 * b + acc_row(i, half);
        if (col < g.d) store4(mine + col, o[b][i] * inverse, o[b][i + 1] * inverse, o[b][i + 2] * inverse, o[b][i + 3] * inverse);
      }
  }
  if (__any(spoilt)) __threadfence();
  for (uint32_t rows = static_cast<uint32_t>(__ballot(spoilt)); rows != 0; rows &= rows - 1) {
    const int r = __builtin_ctz(rows), t = (row0 + r) >> g.pack, h = (row0 + r) & (heads - 1);
    sum_row_forward(g, q + t * g.q_stride + h * g.d, k, v, t, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), r)),
                    __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(total), r)), scale2,
                    BIAS ? bias + h * table_stride(g) : nullptr, out + t * g.out_stride + h * g.d);
  }
}

template <typename T, int DP, bool BIAS>
hipError_t launch_fwd(const PackedAttn& g, hipStream_t st) {
  const size_t lds = Fwd<T, DP>::kLds + (BIAS ? static_cast<size_t>(table_floats(g)) * sizeof(float) : 0);
  const auto kern = attn_packed_fwd_kernel<T, DP, BIAS>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(attn_packed_row_slots(g) * (g.heads >> g.pack))), dim3(kThreads), lds, st, g);
  return hipGetLastError();
}
template <typename T, int DP>
hipError_t launch_fwd(const PackedAttn& g, hipStream_t st) {
  return g.table != nullptr ? launch_fwd<T, DP, true>(g, st) : launch_fwd<T, DP, false>(g, st);
}
template <typename T>
hipError_t launch_fwd(const PackedAttn& g, hipStream_t st) {
  return g.d <= 64 ? launch_fwd<T, 64>(g, st) : launch_fwd<T, 128>(g, st);
}

}  // namespace

// As many heads of a group as are a power of two, up to 8; fewer where their biases by distance would take more than 24 KB
// of LDS (with the histograms of the backward pass in fp32, what is left of it).
void attn_packed_choose_pack(PackedAttn* g) {
  const int group = g->heads / g->kv_heads;
  g->pack = 0;
  while (g->pack < 3 && (group >> g->pack) % 2 == 0 && (g->buckets == 0 || table_stride(*g) << (g->pack + 1) <= 6144)) ++g->pack;
}
bool attn_packed_fits(const PackedAttn& g) {
  const long long slots = static_cast<long long>(attn_packed_row_slots(g));
  return fits_grid(slots * (g.heads >> g.pack), kThreads) && slots < (1ll << 31);
}
size_t attn_packed_row_slots(const PackedAttn& g) {
  return ((static_cast<size_t>(g.tokens) << g.pack) >> kRowsLog) + static_cast<size_t>(g.sequences);
}
hipError_t attn_packed_fwd(int dtype, const PackedAttn& g, hipStream_t st) {
  return dtype == 1 ? launch_fwd<bf16_t>(g, st) : launch_fwd<float>(g, st);
}

}  // namespace lynx
