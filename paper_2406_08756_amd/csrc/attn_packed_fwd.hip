// Causal attention over packed sequences with grouped heads, forward: out = softmax(scale Q K^T + bias) V, one pass over the
// keys with a running maximum and sum; no seq x seq tensor.
#include "attn_packed.h"

namespace lynx {
namespace {

template <typename T, int DP, bool SPLIT> struct Fwd {
  static constexpr int kKeys = sizeof(T) == 2 && !SPLIT ? 64 : 32;  // keys per tile
  static constexpr int kTileElems = kKeys * DP;
  // K and V, two of each, or one of each wavefront
  static constexpr size_t kTiles = (SPLIT ? 2 * kWaves : 4) * static_cast<size_t>(kTileElems) * sizeof(T);
  static constexpr size_t kLds = kTiles + (SPLIT ? 2 * kWaves * 32 * sizeof(float) : 0);
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

template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ __launch_bounds__(kThreads, SPLIT && sizeof(T) * DP == 512 ? 1 : 2) void attn_packed_fwd_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Fwd<T, DP, SPLIT> S;
  constexpr int kKeys = S::kKeys, kBlocks = kKeys / 32, kTileElems = S::kTileElems, kRowsLog = rows_log(SPLIT);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  float* const tops = reinterpret_cast<float*>(smem_raw + S::kTiles);  // SPLIT: each wavefront's maxima and sums
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

  const int row0 = (w.tile << kRowsLog) + (SPLIT ? 0 : 32 * wave);  // this wavefront's
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
  const float* const my_bias = BIAS ? bias + hp * table_stride(g) + kPad : nullptr;
  if (SPLIT && BIAS) __syncthreads();

  constexpr int kTogether = SPLIT ? kWave : kThreads;
  typedef Stage<T, DP, kKeys, kTogether> Load;
  const int part = SPLIT ? 0 : wave;  // of a tile's load
  floatx16_t o[DP / 32];
  float m, total;
  const auto load_k = [&](T* tile, int t) { Load::keys(tile, k, g.k_stride, t * kKeys, w.len, g.d, part, lane); };
  const auto load_v = [&](T* tile, int t) { Load::keys(tile, v, g.v_stride, t * kKeys, w.len, g.d, part, lane); };
  const uint32_t row_base = L::row_base(lane), col_base = L::col_base(lane);
  // The keys from key0 on, at kt and vt, for this wavefront's rows.  k_read() is called when K's tile has been read, v_there()
  // before V's is.
  const auto attend = [&](const T* kt, const T* vt, int key0, auto&& k_read, auto&& v_there) {
    typename Op::Frag rows[2][L::kSteps];
    const auto read_rows = [&](int b) {
#pragma unroll
      for (int c = 0; c < L::kSteps; ++c) rows[b & 1][c] = L::row_frag(kt, row_base, 32 * b, c);
    };
    floatx16_t s[kBlocks];
    read_rows(0);
    requested();
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      if (b + 1 < kBlocks) read_rows(b + 1);
      s[b] = floatx16_t{};
#pragma unroll
      for (int c = 0; c < L::kSteps; ++c) Op::mma(s[b], rows[b & 1][c], qf[c]);
    }
    // V's fragments are requested ahead of the arithmetic that its products wait for, as many as registers are free
    constexpr int kAhead = sizeof(T) == 2 ? L::kGroups : 1;
    typename Op::Frag vf[kAhead][DP / 32];
    const auto read_values = [&](int b, int c0) {
#pragma unroll
      for (int c = 0; c < kAhead; ++c)
#pragma unroll
        for (int e = 0; e < DP / 32; ++e) vf[c][e] = L::col_frag(vt, col_base, 32 * b, c0 + c, e);
    };
    k_read();
    v_there();
    read_values(0, 0);
    requested();
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
    top = max_of_halves(top);
    // The reference follows the maximum only where that has left it 2^8 behind: probabilities up to 256 lose nothing in
    // fp32 sums or by a rounding to the storage type, and the accumulators are hardly ever scaled.  A row decides for itself:
    // for the others of the wavefront the factor is 1.
    if (__any(top > m + 8.f)) {
      const float now = top > m + 8.f ? top : m;
      const float shrink = now == m ? 1.f : exp2_fast(m - now);
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
        if (c % kAhead == 0 && (b != 0 || c != 0)) read_values(b, c);
        const typename Op::Frag p = Op::from_acc(s[b], c);
#pragma unroll
        for (int e = 0; e < DP / 32; ++e) Op::mma(o[e], vf[c % kAhead][e], p);
      }
    }
  };

  bool spoilt = false;
  float joined[DP / 8];  // SPLIT: this lane's columns of its row
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) o[b] = floatx16_t{};
    m = -kInf;       // maximum of the logits so far, times log2 e
    total = 0.f;     // this half's share of the sum
    if constexpr (SPLIT) {
      // one tile of each: K's next one is requested when the scores are there, V's at the end
      T* const kt = lds + wave * 2 * kTileElems;
      T* const vt = kt + kTileElems;
      const int tiles = last_tok / kKeys + 1;
      if (wave < tiles) {
        load_k(kt, wave);
        load_v(vt, wave);
      }
      for (int t = wave; t < tiles; t += kWaves) {
        const bool more = t + kWaves < tiles;
        landed<Load::kLoads>();
        attend(kt, vt, t * kKeys,
               [&] {
                 lds_done();
                 if (more) load_k(kt, t + kWaves);
               },
               [&] {
                 if (more) landed<Load::kLoads>();
                 else landed<0>();
                 if (clean) Load::clean(vt, 0, lane);
               });
        lds_done();
        if (more) load_v(vt, t + kWaves);
      }
    } else {
      const int end_tok = min(((w.tile + 1) << kRowsLog) >> g.pack, w.len);  // of the workgroup: the keys it sees
      const int tiles = (end_tok + kKeys - 1) / kKeys;
      load_k(lds, 0);
      load_v(lds + kTileElems, 0);
      for (int t = 0; t < tiles; ++t) {
        T* const tile = lds + (t & 1) * 2 * kTileElems;
        landed<0>();
        if (clean) Load::clean(tile + kTileElems, part, lane);
        __syncthreads();
        if (t + 1 < tiles) {
          T* const next = lds + (~t & 1) * 2 * kTileElems;
          load_k(next, t + 1);
          load_v(next + kTileElems, t + 1);
        }
        if (t * kKeys <= last_tok) attend(tile, tile + kTileElems, t * kKeys, [] {}, [] {});
      }
    }
    total = sum_of_halves(total);
    if constexpr (SPLIT) {
      if (half == 0) {
        tops[wave * 32 + lane] = m;
        tops[(kWaves + wave) * 32 + lane] = total;
      }
      __syncthreads();
      float top = -kInf, own = m;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) top = fmaxf(top, tops[i * 32 + (lane & 31)]);
      total = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float of = tops[i * 32 + (lane & 31)];
        // (a wavefront whose keys this row does not see has an empty part)
        total += of == -kInf ? tops[(kWaves + i) * 32 + (lane & 31)] : tops[(kWaves + i) * 32 + (lane & 31)] * exp2_fast(of - top);
      }
      m = top;
      constexpr size_t kPartFloats = static_cast<size_t>(DP) * 32;
      float* const parts = reinterpret_cast<float*>(smem_raw);
      static_assert(kWaves * kPartFloats * sizeof(float) <= S::kTiles, "the parts take the tiles' place");
      write_part<DP>(parts + wave * (2 * kTileElems * sizeof(T) / sizeof(float)), o, own == -kInf ? 1.f : exp2_fast(own - top), lane);
      __syncthreads();
      join_parts<DP>(parts, 2 * kTileElems * sizeof(T) / sizeof(float), wave, lane, joined);
    }
    if (clean) break;
    float check = total * 0.f;
    if constexpr (SPLIT) {
#pragma unroll
      for (int c = 0; c < DP / 8; ++c) check = __builtin_fmaf(joined[c], 0.f, check);
    } else {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) check = __builtin_fmaf(o[b][i], 0.f, check);
    }
    check = sum_of_halves(check);
    spoilt = there && check != 0.f;
    if (!__syncthreads_or(spoilt)) break;
  }
  const float inverse = total == 0.f ? 0.f : 1.f / total;
  T* const mine = out + tok * g.out_stride + hp * g.d;
  if (SPLIT && there) store_joined<T, DP>(mine, join_column<DP>(wave, lane), g.d, joined, inverse);
  if (there) {
    if (half == 0 && (!SPLIT || wave == 0)) g.lse[static_cast<long long>(head0 + hp) * g.tokens + w.start + tok] = (m + __builtin_log2f(total)) * kLn2;
#pragma unroll
    for (int b = 0; b < (SPLIT ? 0 : DP / 32); ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = 32 * b + acc_row(i, half);
        if (col < g.d) store4(mine + col, o[b][i] * inverse, o[b][i + 1] * inverse, o[b][i + 2] * inverse, o[b][i + 3] * inverse);
      }
  }
  uint32_t rows = static_cast<uint32_t>(__ballot(spoilt));
  if constexpr (SPLIT) rows = share_rows(rows, reinterpret_cast<uint32_t*>(tops), wave);
  if (rows != 0) __threadfence();
  for (; rows != 0; rows &= rows - 1) {
    const int r = __builtin_ctz(rows), t = (row0 + r) >> g.pack, h = (row0 + r) & (heads - 1);
    sum_row_forward(g, q + t * g.q_stride + h * g.d, k, v, t, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), r)),
                    __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(total), r)), scale2,
                    BIAS ? bias + h * table_stride(g) : nullptr, out + t * g.out_stride + h * g.d);
  }
}

template <typename T, int DP, bool BIAS>
hipError_t launch_fwd(const PackedAttn& g, hipStream_t st) {
  const size_t table = BIAS ? static_cast<size_t>(table_floats(g)) * sizeof(float) : 0;
  const size_t groups = attn_packed_row_slots(g, g.split_fwd) * (g.heads >> g.pack);
  return g.split_fwd ? launch_packed<attn_packed_fwd_kernel<T, DP, BIAS, true>>(groups, Fwd<T, DP, true>::kLds + table, g, st)
                      : launch_packed<attn_packed_fwd_kernel<T, DP, BIAS, false>>(groups, Fwd<T, DP, false>::kLds + table, g, st);
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

// Fewer workgroups of 128 rows or keys than this, and 32 each go faster.
constexpr size_t kSplitBelow = 512;
// As many heads of a group as are a power of two, up to 8; fewer where their biases by distance would take more than 10 KB of
// LDS, so that with four times that for the gradient's sums and the tiles of fp32 a workgroup has what it needs.
void attn_packed_choose(int dtype, PackedAttn* g) {
  const int group = g->heads / g->kv_heads;
  g->pack = 0;
  while (g->pack < 3 && (group >> g->pack) % 2 == 0 && (g->buckets == 0 || table_stride(*g) << (g->pack + 1) <= 2560)) ++g->pack;
  g->split_fwd = attn_packed_row_slots(*g, false) * (g->heads >> g->pack) < kSplitBelow;
  g->split_rows = g->split_fwd && attn_packed_split_rows_fit(dtype, *g);
  g->split_keys = 0;
  g->split_keys = attn_packed_key_slots(*g) * g->kv_heads < kSplitBelow;
}
bool attn_packed_fits(const PackedAttn& g) {
  const long long slots = static_cast<long long>(attn_packed_row_slots(g, g.split_fwd));
  return fits_grid(slots * (g.heads >> g.pack), kThreads) && slots < (1ll << 31);
}
size_t attn_packed_row_slots(const PackedAttn& g, bool split) {
  return ((static_cast<size_t>(g.tokens) << g.pack) >> rows_log(split)) + static_cast<size_t>(g.sequences);
}
size_t attn_packed_key_slots(const PackedAttn& g) {
  return (static_cast<size_t>(g.tokens) >> rows_log(g.split_keys)) + static_cast<size_t>(g.sequences);
}
hipError_t attn_packed_fwd(int dtype, const PackedAttn& g, hipStream_t st) {
  return dtype == 1 ? launch_fwd<bf16_t>(g, st) : launch_fwd<float>(g, st);
}

}  // namespace lynx
