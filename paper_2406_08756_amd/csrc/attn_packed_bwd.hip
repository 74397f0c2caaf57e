// Causal attention over packed sequences with grouped heads, backward: probabilities are formed again from the row statistic
// of the forward pass, p = exp(z - lse).
//   rows:  ds = p (d_out V^T - delta), dQ = scale ds K, and the gradient of the position bias, sums of ds by bucket
//   keys:  dV = P^T d_out and dK = scale dS^T Q, over all rows of all heads of the group that see the key
// Each result is summed by one workgroup in one order: no atomics between workgroups, the same bits every time.  The price is
// that both kernels form the scores and d_out V^T: seven products instead of five.
#include "attn_packed.h"

namespace lynx {
namespace {

constexpr int kHistStride = kThreads + 1;  // a column of the histogram: one float per thread

template <typename T, int DP, bool BIAS> struct Rows {
  static constexpr int kKeys = sizeof(T) == 2 && !BIAS ? 64 : 32;
  static constexpr size_t kLds = 4 * static_cast<size_t>(kKeys) * DP * sizeof(T);
};
template <typename T, int DP> struct Keys {
  static constexpr int kRows = sizeof(T) == 2 ? 64 : 32;
  static constexpr size_t kTiles = 4 * static_cast<size_t>(kRows) * DP * sizeof(T);
  static constexpr size_t kLds = kTiles + 4 * kRows * sizeof(float);
};

// The statistic as the exponent's offset; a row that sees nothing but minus infinity has probabilities of zero.
__device__ __forceinline__ float offset2(float lse) { return lse == -kInf ? kInf : lse * kLog2e; }

// One row's dQ again, pair by pair, if it sees an infinity or NaN in K.
template <typename T>
__device__ void sum_row_dq(const PackedAttn& g, const T* q, const T* d_out, const T* k, const T* v, int tok, float lse2, float delta,
                           float scale2, const float* bias, T* dq) {
  const int lane = threadIdx.x & (kWave - 1);
  bool clean = true;
  float acc[2] = {0.f, 0.f};
  for (int j0 = 0; j0 <= tok; j0 += kWave) {
    const int j = j0 + lane;
    float ds = 0.f;
    if (j <= tok) {
      clean = clean && row_finite(k + j * g.k_stride, g.d);
      float z = row_dot(q, k + j * g.k_stride, g.d) * scale2;
      if (bias != nullptr) z += bias[min(tok - j, g.far) + kPad];
      ds = exp2_fast(z - lse2) * (row_dot(d_out, v + j * g.v_stride, g.d) - delta);
    }
    const int n = min(kWave, tok + 1 - j0);
    for (int i = 0; i < n; ++i) {
      const float x = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ds), i));
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (lane + kWave * c < g.d) acc[c] = __builtin_fmaf(x, load1(k + (j0 + i) * g.k_stride + lane + kWave * c), acc[c]);
    }
  }
  if (__all(clean)) return;
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + kWave * c < g.d) store1(dq + lane + kWave * c, acc[c] * g.scale);
}

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 || DP == 64 ? 2 : 1) void attn_packed_rows_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Rows<T, DP, BIAS> S;
  constexpr int kKeys = S::kKeys;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  constexpr int kTileElems = kKeys * DP;
  float* const bias = reinterpret_cast<float*>(smem_raw + S::kLds);
  float* const hist = bias + (BIAS ? table_floats(g) : 0);
  unsigned char* const bucket = reinterpret_cast<unsigned char*>(hist + (BIAS ? g.buckets * kHistStride : 0));  // by distance

  const int subs = g.heads >> g.pack, slot = static_cast<int>(blockIdx.x) / subs;
  const int head0 = (static_cast<int>(blockIdx.x) % subs) << g.pack;
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = 1 << g.pack;
  SeqTile w;
  if (!find_tile</*LAST_FIRST=*/true>(g, slot, kRowsLog, g.pack, &w)) {
    if (BIAS)
      for (int x = threadIdx.x; x < heads * g.buckets; x += kThreads)
        g.partials[(static_cast<long long>(slot) * g.heads + head0) * g.buckets + x] = 0.f;
    return;
  }
  if (BIAS) {
    fill_bias<T, kThreads>(g, head0, bias);
    for (int x = threadIdx.x; x < table_stride(g); x += kThreads) bucket[x] = static_cast<unsigned char>(bucket_of(g, x - kPad));
    for (int x = threadIdx.x; x < g.buckets * kHistStride; x += kThreads) hist[x] = 0.f;
  }

  const int kv = head0 / (g.heads / g.kv_heads);
  const T* const q = static_cast<const T*>(g.q) + w.start * g.q_stride + static_cast<long long>(head0) * g.d;
  const T* const k = static_cast<const T*>(g.k) + w.start * g.k_stride + static_cast<long long>(kv) * g.d;
  const T* const v = static_cast<const T*>(g.v) + w.start * g.v_stride + static_cast<long long>(kv) * g.d;
  const T* const out = static_cast<const T*>(g.out) + w.start * g.out_stride + static_cast<long long>(head0) * g.d;
  const T* const d_out = static_cast<const T*>(g.d_out) + w.start * g.out_stride + static_cast<long long>(head0) * g.d;
  T* const dq = static_cast<T*>(g.dq) + w.start * g.dq_stride + static_cast<long long>(head0) * g.d;

  const int row0 = (w.tile << kRowsLog) + 32 * wave;
  const int row = row0 + (lane & 31), tok = row >> g.pack, hp = row & (heads - 1);
  const int first_tok = row0 >> g.pack, last_tok = first_tok < w.len ? min((row0 + 31) >> g.pack, w.len - 1) : -1;
  const bool there = tok < w.len;
  const float scale2 = g.scale * kLog2e;

  typename Op::Frag qf[L::kSteps], gf[L::kSteps];  // Q and d_out
  float delta = 0.f, lse2 = kInf;
  {
    const int left = min(w.len - first_tok, 32);
    const auto buffer = [&](const T* base, long long stride) {
      return row_buffer(base + first_tok * stride, left > 0 ? static_cast<uint32_t>((left - 1) * stride + heads * g.d) * static_cast<uint32_t>(sizeof(T)) : 0u);
    };
    const auto at = [&](long long stride) {
      return (static_cast<uint32_t>(tok - first_tok) * static_cast<uint32_t>(stride) + hp * g.d) * static_cast<uint32_t>(sizeof(T));
    };
    load_row_frags<T, DP>(buffer(out, g.out_stride), at(g.out_stride), g.d, lane, qf);
    load_row_frags<T, DP>(buffer(d_out, g.out_stride), at(g.out_stride), g.d, lane, gf);
#pragma unroll
    for (int s = 0; s < L::kSteps; ++s) delta += Op::dot(qf[s], gf[s]);
    delta += other_half(delta);
    load_row_frags<T, DP>(buffer(q, g.q_stride), at(g.q_stride), g.d, lane, qf);
    if (there) {
      const long long stat = static_cast<long long>(head0 + hp) * g.tokens + w.start + tok;
      lse2 = offset2(g.lse[stat]);
      if (half == 0) g.delta[stat] = delta;
    }
  }
  const int end_tok = min(((w.tile + 1) << kRowsLog) >> g.pack, w.len);
  const int tiles = (end_tok + kKeys - 1) / kKeys;
  const float* const my_bias = BIAS ? bias + hp * table_stride(g) + kPad : nullptr;
  float far_sum = 0.f;

  Stage<T, DP, kKeys, kThreads> sk, sv;
  floatx16_t acc[DP / 32];
  bool spoilt = false;
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) acc[b] = floatx16_t{};
    sk.load_keys(k, g.k_stride, 0, w.len, g.d);
    sv.load_keys(v, g.v_stride, 0, w.len, g.d);
    for (int t = 0; t < tiles; ++t) {
      T* const kt = lds + (t & 1) * 2 * kTileElems;
      T* const vt = kt + kTileElems;
      if (clean) sk.template store<true>(kt);
      else sk.template store<false>(kt);
      sv.template store<false>(vt);
      __syncthreads();
      if (t + 1 < tiles) {
        sk.load_keys(k, g.k_stride, (t + 1) * kKeys, w.len, g.d);
        sv.load_keys(v, g.v_stride, (t + 1) * kKeys, w.len, g.d);
      }
#pragma unroll
      for (int b = 0; b < kKeys / 32; ++b) {
        const int key0 = t * kKeys + 32 * b;
        if (key0 > last_tok) continue;
        floatx16_t s{}, dp{};
#pragma unroll
        for (int c = 0; c < L::kSteps; ++c) Op::mma(s, L::row_frag(kt, 32 * b, c, lane), qf[c]);
#pragma unroll
        for (int c = 0; c < L::kSteps; ++c) Op::mma(dp, L::row_frag(vt, 32 * b, c, lane), gf[c]);
        const int apart = tok - key0 - 4 * half;
        const bool near = BIAS && first_tok - (key0 + 31) < g.far, edge = key0 + 31 > first_tok;
        const float offset = BIAS && !near ? lse2 - my_bias[g.far] : lse2;
        if (BIAS && near) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], scale2, my_bias[apart - acc_row(i, 0)] - lse2);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(s[i], scale2, -offset);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = exp2_fast(s[i]) * (dp[i] - delta);
        if (edge) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (apart < acc_row(i, 0)) s[i] = 0.f;
        }
        if (!there) s = floatx16_t{};
        if (BIAS && !clean) {
          if (near) {
            // (each thread adds to a column of its own, in program order)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              __hip_atomic_fetch_add(hist + bucket[apart - acc_row(i, 0) + kPad] * kHistStride + threadIdx.x, s[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) far_sum += s[i];
          }
        }
#pragma unroll
        for (int c = 0; c < L::kGroups; ++c) {
          const typename Op::Frag ds = Op::from_acc(s, c);
#pragma unroll
          for (int e = 0; e < DP / 32; ++e) Op::mma(acc[e], L::col_frag(kt, 32 * b, c, 32 * e, lane), ds);
        }
      }
    }
    if (clean) break;
    float check = 0.f;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) check = __builtin_fmaf(acc[b][i], 0.f, check);
    check += other_half(check);
    spoilt = there && check != 0.f;
    if (!__syncthreads_or(spoilt)) break;
  }
  if (there) {
    T* const mine = dq + tok * g.dq_stride + hp * g.d;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = 32 * b + acc_row(i, half);
        if (col < g.d) store4(mine + col, acc[b][i] * g.scale, acc[b][i + 1] * g.scale, acc[b][i + 2] * g.scale, acc[b][i + 3] * g.scale);
      }
  }
  if (__any(spoilt)) __threadfence();
  for (uint32_t rows = static_cast<uint32_t>(__ballot(spoilt)); rows != 0; rows &= rows - 1) {
    const int r = __builtin_ctz(rows), t = (row0 + r) >> g.pack, h = (row0 + r) & (heads - 1);
    sum_row_dq(g, q + t * g.q_stride + h * g.d, d_out + t * g.out_stride + h * g.d, k, v, t,
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lse2), r)),
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(delta), r)), scale2, BIAS ? bias + h * table_stride(g) : nullptr,
               dq + t * g.dq_stride + h * g.d);
  }
  if (BIAS) {
    hist[(g.buckets - 1) * kHistStride + threadIdx.x] += far_sum;
    __syncthreads();
    for (int x = threadIdx.x; x < heads * g.buckets; x += kThreads) {
      const int h = x / g.buckets, b = x % g.buckets;
      float sum = 0.f;
      for (int r = h; r < kThreads; r += heads) sum += hist[b * kHistStride + r];  // (a thread's head: its number modulo the heads)
      g.partials[(static_cast<long long>(slot) * g.heads + head0 + h) * g.buckets + b] = sum;
    }
  }
}

// One key's dK and dV again, pair by pair, if a row that sees it has an infinity or NaN in Q or d_out.
template <typename T>
__device__ void sum_key(const PackedAttn& g, const SeqTile& w, int kv, int key, const float* bias, T* dk, T* dv) {
  const int lane = threadIdx.x & (kWave - 1), group = g.heads / g.kv_heads;
  const T* const k = static_cast<const T*>(g.k) + (w.start + key) * g.k_stride + static_cast<long long>(kv) * g.d;
  const T* const v = static_cast<const T*>(g.v) + (w.start + key) * g.v_stride + static_cast<long long>(kv) * g.d;
  bool clean = true;
  float ak[2] = {0.f, 0.f}, av[2] = {0.f, 0.f};
  for (int h = kv * group; h < (kv + 1) * group; ++h) {
    const T* const q = static_cast<const T*>(g.q) + w.start * g.q_stride + static_cast<long long>(h) * g.d;
    const T* const d_out = static_cast<const T*>(g.d_out) + w.start * g.out_stride + static_cast<long long>(h) * g.d;
    for (int t0 = key; t0 < w.len; t0 += kWave) {
      const int t = t0 + lane;
      float p = 0.f, ds = 0.f;
      if (t < w.len) {
        const long long stat = static_cast<long long>(h) * g.tokens + w.start + t;
        clean = clean && row_finite(q + t * g.q_stride, g.d) && row_finite(d_out + t * g.out_stride, g.d);
        float z = row_dot(q + t * g.q_stride, k, g.d) * (g.scale * kLog2e);
        if (bias != nullptr) z += load1(static_cast<const T*>(g.table) + static_cast<long long>(bucket_of(g, t - key)) * g.heads + h) * kLog2e;
        p = exp2_fast(z - offset2(g.lse[stat]));
        ds = p * (row_dot(d_out + t * g.out_stride, v, g.d) - g.delta[stat]);
      }
      const int n = min(kWave, w.len - t0);
      for (int i = 0; i < n; ++i) {
        const float pi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), i));
        const float di = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ds), i));
#pragma unroll
        for (int c = 0; c < 2; ++c)
          if (lane + kWave * c < g.d) {
            av[c] = __builtin_fmaf(pi, load1(d_out + (t0 + i) * g.out_stride + lane + kWave * c), av[c]);
            ak[c] = __builtin_fmaf(di, load1(q + (t0 + i) * g.q_stride + lane + kWave * c), ak[c]);
          }
      }
    }
  }
  if (__all(clean)) return;
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + kWave * c < g.d) {
      store1(dv + lane + kWave * c, av[c]);
      store1(dk + lane + kWave * c, ak[c] * g.scale);
    }
}

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(kThreads, DP == 64 ? 2 : 1) void attn_packed_keys_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Keys<T, DP> S;
  constexpr int kRows = S::kRows;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  constexpr int kTileElems = kRows * DP;
  float* const stats = reinterpret_cast<float*>(smem_raw + S::kTiles);  // offsets and deltas, two of each
  float* const bias = stats + 4 * kRows;

  const int kv = static_cast<int>(blockIdx.x) % g.kv_heads;
  SeqTile w;
  if (!find_tile</*LAST_FIRST=*/false>(g, static_cast<int>(blockIdx.x) / g.kv_heads, kRowsLog, 0, &w)) return;

  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = 1 << g.pack, group = g.heads / g.kv_heads, subs = group >> g.pack;
  const T* const k = static_cast<const T*>(g.k) + w.start * g.k_stride + static_cast<long long>(kv) * g.d;
  const T* const v = static_cast<const T*>(g.v) + w.start * g.v_stride + static_cast<long long>(kv) * g.d;
  const T* const q = static_cast<const T*>(g.q) + w.start * g.q_stride + static_cast<long long>(kv * group) * g.d;
  const T* const d_out = static_cast<const T*>(g.d_out) + w.start * g.out_stride + static_cast<long long>(kv * group) * g.d;
  const float scale2 = g.scale * kLog2e;
  const int tile_key0 = w.tile << kRowsLog, key0 = tile_key0 + 32 * wave, key = key0 + (lane & 31);
  const bool there = key < w.len;

  typename Op::Frag kf[L::kSteps], vf[L::kSteps];
  {
    const int left = min(w.len - key0, 32);
    const auto buffer = [&](const T* base, long long stride) {
      return row_buffer(base + key0 * stride, left > 0 ? static_cast<uint32_t>((left - 1) * stride + g.d) * static_cast<uint32_t>(sizeof(T)) : 0u);
    };
    load_row_frags<T, DP>(buffer(k, g.k_stride), static_cast<uint32_t>(lane & 31) * static_cast<uint32_t>(g.k_stride) * static_cast<uint32_t>(sizeof(T)), g.d, lane, kf);
    load_row_frags<T, DP>(buffer(v, g.v_stride), static_cast<uint32_t>(lane & 31) * static_cast<uint32_t>(g.v_stride) * static_cast<uint32_t>(sizeof(T)), g.d, lane, vf);
  }
  const int first_row = tile_key0 << g.pack, rows = w.len << g.pack;
  const int tiles = (rows - first_row + kRows - 1) / kRows, steps = tiles * subs;

  Stage<T, DP, kRows, kThreads> sq, sg;
  float next_lse = kInf, next_delta = 0.f;
  const auto load = [&](int it) {
    const int sub = it / tiles, r0 = first_row + it % tiles * kRows;
    sq.load_rows(q + static_cast<long long>(sub << g.pack) * g.d, g.q_stride, r0, w.len, g.d, g.pack);
    sg.load_rows(d_out + static_cast<long long>(sub << g.pack) * g.d, g.out_stride, r0, w.len, g.d, g.pack);
    if (threadIdx.x < kRows) {
      const int r = r0 + threadIdx.x;
      next_lse = kInf;  // (rows behind the last: probabilities of zero)
      next_delta = 0.f;
      if (r < rows) {
        const long long stat = static_cast<long long>(kv * group + (sub << g.pack) + (r & (heads - 1))) * g.tokens + w.start + (r >> g.pack);
        next_lse = offset2(g.lse[stat]);
        next_delta = g.delta[stat];
      }
    }
  };

  floatx16_t dk[DP / 32], dv[DP / 32];
  bool spoilt = false;
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dk[b] = dv[b] = floatx16_t{};
    load(0);
    for (int it = 0; it < steps; ++it) {
      T* const qt = lds + (it & 1) * 2 * kTileElems;
      T* const gt = qt + kTileElems;
      float* const lse_t = stats + (it & 1) * 2 * kRows;
      float* const delta_t = lse_t + kRows;
      if (clean) {
        sq.template store<true>(qt);
        sg.template store<true>(gt);
      } else {
        sq.template store<false>(qt);
        sg.template store<false>(gt);
      }
      if (threadIdx.x < kRows) {
        lse_t[threadIdx.x] = next_lse;
        delta_t[threadIdx.x] = next_delta;
      }
      const int sub = it / tiles, r0 = first_row + it % tiles * kRows;
      if (BIAS && it % tiles == 0) {
        __syncthreads();  // (the last tile of the heads before is done with their bias)
        fill_bias<T, kThreads>(g, kv * group + (sub << g.pack), bias);
      }
      __syncthreads();
      if (it + 1 < steps) load(it + 1);
#pragma unroll
      for (int b = 0; b < kRows / 32; ++b) {
        const int b0 = r0 + 32 * b, first_tok = b0 >> g.pack, last_tok = (b0 + 31) >> g.pack;
        if (last_tok < key0) continue;
        floatx16_t s{}, dp{};
#pragma unroll
        for (int c = 0; c < L::kSteps; ++c) Op::mma(s, L::row_frag(qt, 32 * b, c, lane), kf[c]);
#pragma unroll
        for (int c = 0; c < L::kSteps; ++c) Op::mma(dp, L::row_frag(gt, 32 * b, c, lane), vf[c]);
        // register i: token first_tok + (i's part, the same for all lanes) + (4 half >> pack), head likewise
        const int apart = first_tok + ((4 * half) >> g.pack) - key;
        const int stride = BIAS ? table_stride(g) : 0;
        const float* const my_bias = BIAS ? bias + kPad + (g.pack == 3 ? 4 * half * stride : 0) : nullptr;
        const bool near = BIAS && first_tok - (key0 + 31) < g.far, edge = key0 + 31 > first_tok;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float4 lse4 = *reinterpret_cast<const float4*>(lse_t + 32 * b + 8 * a + 4 * half);
          const float4 delta4 = *reinterpret_cast<const float4*>(delta_t + 32 * b + 8 * a + 4 * half);
          const float lse[4] = {lse4.x, lse4.y, lse4.z, lse4.w}, delta[4] = {delta4.x, delta4.y, delta4.z, delta4.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = 4 * a + j, ahead = (8 * a + j) >> g.pack;
            float offset = -lse[j];
            if (BIAS) offset += my_bias[(j & (heads - 1)) * stride + (near ? apart + ahead : g.far)];
            const float p = exp2_fast(__builtin_fmaf(s[i], scale2, offset));
            const bool hidden = edge && apart + ahead < 0;
            s[i] = hidden ? 0.f : p;
            dp[i] = hidden ? 0.f : p * (dp[i] - delta[j]);
          }
        }
#pragma unroll
        for (int c = 0; c < L::kGroups; ++c) {
          const typename Op::Frag p = Op::from_acc(s, c), ds = Op::from_acc(dp, c);
#pragma unroll
          for (int e = 0; e < DP / 32; ++e) {
            Op::mma(dv[e], L::col_frag(gt, 32 * b, c, 32 * e, lane), p);
            Op::mma(dk[e], L::col_frag(qt, 32 * b, c, 32 * e, lane), ds);
          }
        }
      }
    }
    if (clean) break;
    float check = 0.f;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) check = __builtin_fmaf(dk[b][i], 0.f, __builtin_fmaf(dv[b][i], 0.f, check));
    check += other_half(check);
    spoilt = there && check != 0.f;
    if (!__syncthreads_or(spoilt)) break;
  }
  T* const dk_rows = static_cast<T*>(g.dk) + w.start * g.dk_stride + static_cast<long long>(kv) * g.d;
  T* const dv_rows = static_cast<T*>(g.dv) + w.start * g.dv_stride + static_cast<long long>(kv) * g.d;
  if (there) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = 32 * b + acc_row(i, half);
        if (col >= g.d) continue;
        store4(dk_rows + key * g.dk_stride + col, dk[b][i] * g.scale, dk[b][i + 1] * g.scale, dk[b][i + 2] * g.scale, dk[b][i + 3] * g.scale);
        store4(dv_rows + key * g.dv_stride + col, dv[b][i], dv[b][i + 1], dv[b][i + 2], dv[b][i + 3]);
      }
  }
  if (__any(spoilt)) __threadfence();
  for (uint32_t keys = static_cast<uint32_t>(__ballot(spoilt)); keys != 0; keys &= keys - 1) {
    const int j = key0 + __builtin_ctz(keys);
    sum_key(g, w, kv, j, BIAS ? bias : nullptr, dk_rows + j * g.dk_stride, dv_rows + j * g.dv_stride);
  }
}

// d_table[b, h] = the sum over row tiles of their shares, in one order: 16 interleaved sums, then those in turn.
constexpr int kTableWaves = 16;
template <typename T>
__global__ __launch_bounds__(kTableWaves * kWave) void attn_packed_table_kernel(const float* partials, T* d_table, int slots, int heads, int buckets) {
  __shared__ float sums[kTableWaves][kWave];
  const int h = blockIdx.x, b = threadIdx.x & (kWave - 1), y = threadIdx.x / kWave;
  float sum = 0.f;
  if (b < buckets)
    for (int s = y; s < slots; s += kTableWaves) sum += partials[(static_cast<long long>(s) * heads + h) * buckets + b];
  sums[y][b] = sum;
  __syncthreads();
  if (y != 0 || b >= buckets) return;
  for (int i = 1; i < kTableWaves; ++i) sum += sums[i][b];
  store1(d_table + static_cast<long long>(b) * heads + h, sum);
}

template <typename Kernel>
hipError_t launch(Kernel kern, size_t groups, size_t lds, const PackedAttn& g, hipStream_t st) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(groups)), dim3(kThreads), lds, st, g);
  return hipGetLastError();
}
template <typename T, int DP, bool BIAS>
hipError_t launch_bwd(const PackedAttn& g, hipStream_t st) {
  const size_t slots = attn_packed_row_slots(g), table = BIAS ? static_cast<size_t>(table_floats(g)) * sizeof(float) : 0;
  const size_t by_row = BIAS ? g.buckets * kHistStride * sizeof(float) + table_stride(g) : 0;
  hipError_t e = launch(attn_packed_rows_kernel<T, DP, BIAS>, slots * (g.heads >> g.pack), Rows<T, DP, BIAS>::kLds + table + by_row, g, st);
  if (e != hipSuccess) return e;
  const size_t key_slots = (static_cast<size_t>(g.tokens) >> kRowsLog) + g.sequences;
  e = launch(attn_packed_keys_kernel<T, DP, BIAS>, key_slots * g.kv_heads, Keys<T, DP>::kLds + table, g, st);
  if (e != hipSuccess || !BIAS) return e;
  hipLaunchKernelGGL((attn_packed_table_kernel<T>), dim3(g.heads), dim3(kTableWaves * kWave), 0, st, g.partials, static_cast<T*>(g.d_table),
                     static_cast<int>(slots), g.heads, g.buckets);
  return hipGetLastError();
}
template <typename T, int DP>
hipError_t launch_bwd(const PackedAttn& g, hipStream_t st) {
  return g.table != nullptr ? launch_bwd<T, DP, true>(g, st) : launch_bwd<T, DP, false>(g, st);
}
template <typename T>
hipError_t launch_bwd(const PackedAttn& g, hipStream_t st) {
  return g.d <= 64 ? launch_bwd<T, 64>(g, st) : launch_bwd<T, 128>(g, st);
}

}  // namespace

hipError_t attn_packed_bwd(int dtype, const PackedAttn& g, hipStream_t st) {
  return dtype == 1 ? launch_bwd<bf16_t>(g, st) : launch_bwd<float>(g, st);
}

}  // namespace lynx
