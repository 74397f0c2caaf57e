// Causal attention over packed sequences with grouped heads, backward: probabilities are formed again from the row statistic
// of the forward pass, p = exp(z - lse).
//   rows:  ds = p (d_out V^T - delta), dQ = scale ds K, and the gradient of the position bias, sums of ds by bucket
//   keys:  dV = P^T d_out and dK = scale dS^T Q, over all rows of all heads of the group that see the key
// Each result is summed by one workgroup in one order: no atomics between workgroups, the same bits every time.  The price is
// that both kernels form the scores and d_out V^T: seven products instead of five.
#include <type_traits>

#include "attn_packed.h"

namespace lynx {
namespace {

// The gradient of the position bias.  ds by distance, for each head of the tile and each wavefront apart: `far` distances and
// what a 32 x 32 block that holds one of them reaches beyond.  A near block is laid down in LDS by diagonals, 16 rows at a time
// (47 diagonals; which places of a diagonal exist depends on the row alone, the others stay zero), and a lane adds up one of
// them, so that each sum has one owner and one order.  Blocks whose keys are all far are summed in a register.
constexpr int kDiagonalStride = 20, kBlockFloats = 47 * kDiagonalStride + 20;
__host__ __device__ __forceinline__ int distances(const PackedAttn& g) { return (g.far + 64 + 3) & ~3; }
__host__ __device__ __forceinline__ int by_distance_floats(const PackedAttn& g) { return (distances(g) << g.pack) + kBlockFloats; }  // of a wavefront

// K and V in tiles of 32 keys: four of each, which leaves a tile the time of two to arrive, or three and two where the sums of
// the bias's gradient or fp32 leave no room for more beside another workgroup; or one of each wavefront.
template <typename T, int DP, bool BIAS, bool SPLIT> struct Rows {
  static constexpr int kTileElems = 32 * DP;
  static constexpr bool kFew = BIAS || sizeof(T) * DP == 512;
  static constexpr int kTileCount = SPLIT ? 2 * kWaves : kFew ? 5 : 8;
  static constexpr size_t kTiles = kTileCount * static_cast<size_t>(kTileElems) * sizeof(T);
  static constexpr size_t kLds = kTiles + (SPLIT ? kWaves * sizeof(uint32_t) : 0);
};
template <typename T, int DP, bool SPLIT> struct Keys {
  // of a wavefront (SPLIT): the tile at work and the next one on its way, where there is room
  static constexpr int kPlaces = sizeof(T) * DP == 512 ? 1 : 2;
  static constexpr int kTileElems = 32 * DP, kCopies = SPLIT ? kPlaces * kWaves : sizeof(T) * DP == 512 ? 3 : 4;
  static constexpr size_t kTiles = 2 * kCopies * static_cast<size_t>(kTileElems) * sizeof(T);
  static constexpr int kStat = 2 * kWave;  // floats of a tile's statistics: offset, delta, each as a wavefront loads them
  static constexpr size_t kLds = kTiles + kCopies * kStat * sizeof(float) + (SPLIT ? kWaves * sizeof(uint32_t) : 0);
};

// What the exponents are less by; a row that sees nothing but minus infinity has probabilities of zero.
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

// dQ of a tile of rows: p = 2^(s - lse log2 e), ds = p (d_out.v - delta), dQ += ds k over the tiles of 32 keys, with
// delta = sum of d_out out; the bias's gradient is summed on the way.  Rounded to the storage type: ds ahead of its product, dQ.
// Bound by the issue of instructions as the forward pass, with three products to share it: 8192 tokens in four sequences, 16
// heads of 128, bf16: 131 us, 790 TFLOP/s; with a bias, one sequence of 16384, 6 heads of 128: 720 us, 860.
// Two workgroups per CU go faster than one, a spilled register or not (that sequence: 740 us, 1260 at one); but not where each
// wavefront has tiles of its own and heads of 128 a bias (2048 tokens of 5 heads: 74 us, 43 at one; of 64: 54, 85 at one).
template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 4 && (SPLIT || DP == 128)) || (SPLIT && BIAS && DP == 128) ? 1 : 2) void attn_packed_rows_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Rows<T, DP, BIAS, SPLIT> S;
  constexpr int kTileElems = S::kTileElems, kRowsLog = rows_log(SPLIT);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  float* const bias = reinterpret_cast<float*>(smem_raw + S::kLds);
  float* const sums = bias + (BIAS ? table_floats(g) : 0);  // of the table's gradient: by_distance_floats per wavefront

  const int subs = g.heads >> g.pack, slot = static_cast<int>(blockIdx.x) / subs;
  const int head0 = (static_cast<int>(blockIdx.x) % subs) << g.pack;
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = 1 << g.pack;
  SeqTile w;
  if (!(SPLIT ? find_tile</*LAST_FIRST=*/true>(g, slot, kRowsLog, g.pack, &w) : find_ranked_tile(g, slot, kRowsLog, g.pack, &w))) {
    if (BIAS)
      for (int x = threadIdx.x; x < heads * g.buckets; x += kThreads)
        g.partials[(static_cast<long long>(slot) * g.heads + head0) * g.buckets + x] = 0.f;
    return;
  }
  const int kv = head0 / (g.heads / g.kv_heads);
  const T* const q = static_cast<const T*>(g.q) + w.start * g.q_stride + static_cast<long long>(head0) * g.d;
  const T* const k = static_cast<const T*>(g.k) + w.start * g.k_stride + static_cast<long long>(kv) * g.d;
  const T* const v = static_cast<const T*>(g.v) + w.start * g.v_stride + static_cast<long long>(kv) * g.d;
  const T* const out = static_cast<const T*>(g.out) + w.start * g.out_stride + static_cast<long long>(head0) * g.d;
  const T* const d_out = static_cast<const T*>(g.d_out) + w.start * g.out_stride + static_cast<long long>(head0) * g.d;
  T* const dq = static_cast<T*>(g.dq) + w.start * g.dq_stride + static_cast<long long>(head0) * g.d;

  const int row0 = (w.tile << kRowsLog) + (SPLIT ? 0 : 32 * wave);
  const int row = row0 + (lane & 31), tok = row >> g.pack, hp = row & (heads - 1);
  const int first_tok = row0 >> g.pack, last_tok = first_tok < w.len ? min((row0 + 31) >> g.pack, w.len - 1) : -1;
  const bool there = tok < w.len;
  const float scale2 = g.scale * kLog2e;

  constexpr int kTogether = SPLIT ? kWave : kThreads;
  typedef Stream<T, DP, kTogether> Load;
  const int part = SPLIT ? 0 : wave;  // of a tile's load
  const uint32_t lds_at = lds_address(smem_raw);
  // SPLIT: the wavefronts deal the tiles up to the last one that the rows see; else the workgroup's rows see these
  const int end_tok = SPLIT ? last_tok + 1 : min(((w.tile + 1) << kRowsLog) >> g.pack, w.len);
  const int tiles = (end_tok + 31) / 32;
  const int first_tile = SPLIT ? wave : 0, every = SPLIT ? kWaves : 1;
  constexpr int kKs = SPLIT ? 1 : S::kFew ? 3 : 4, kVs = SPLIT ? 1 : S::kFew ? 2 : 4;
  const auto k_slot = [&](int t) { return (SPLIT ? 2 * wave : t % kKs) * kTileElems; };
  const auto v_slot = [&](int t) { return (SPLIT ? 2 * wave + 1 : kKs + t % kVs) * kTileElems; };
  Load k_tiles(k, g.k_stride, 32 * first_tile, w.len, g.d, 0, part, lane), v_tiles(v, g.v_stride, 32 * first_tile, w.len, g.d, 0, part, lane);
  const auto load = [&](int kt, int vt) {  // (each in turn)
    if (kt < tiles) k_tiles.load(lds_at + k_slot(kt) * sizeof(T), part, every);
    if (vt < tiles) v_tiles.load(lds_at + v_slot(vt) * sizeof(T), part, every);
  };
  const auto load_first = [&] {
    load(first_tile, first_tile);
    if (!SPLIT && !S::kFew) load(1, 1);
  };
  load_first();

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
    // (all loads on their way before the first is waited for)
    typename Op::Frag of[L::kSteps];
    load_row_frags<T, DP>(buffer(out, g.out_stride), at(g.out_stride), g.d, lane, of);
    load_row_frags<T, DP>(buffer(d_out, g.out_stride), at(g.out_stride), g.d, lane, gf);
    load_row_frags<T, DP>(buffer(q, g.q_stride), at(g.q_stride), g.d, lane, qf);
    float lse = -kInf;
    if (there) lse = g.lse[static_cast<long long>(head0 + hp) * g.tokens + w.start + tok];
    if (BIAS) {
      fill_bias<T, kThreads>(g, head0, bias);
      for (int x = 4 * threadIdx.x; x < kWaves * by_distance_floats(g); x += 4 * kThreads) *reinterpret_cast<float4*>(sums + x) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int s = 0; s < L::kSteps; ++s) delta += Op::dot(of[s], gf[s]);
    delta = sum_of_halves(delta);
    lse2 = offset2(lse);
  }
  const float* const my_bias = BIAS ? bias + hp * table_stride(g) + kPad : nullptr;
  float* const my_sums = BIAS ? sums + wave * by_distance_floats(g) : nullptr;
  float far_sum = 0.f;
  if (SPLIT && BIAS) __syncthreads();

  floatx16_t acc[DP / 32];
  uint32_t row_base = L::row_base(lane), col_base = L::col_base(lane);
  // A tile goes by in three passes of matrix instructions, with the arithmetic between them: d_out V^T, and the probabilities;
  // the next tile's scores, and ds; the sum over K.  The order is written out (in_order()), with fragments kRing steps ahead
  // of their use: left to itself the compiler keeps one and waits for each.
  constexpr int kRing = 4, kSumSteps = L::kGroups * (DP / 32), kFrags = 2 * L::kSteps + kSumSteps;
  typename Op::Frag ring[kRing];
  // the fragments of the three passes: of V, of the next tile's K, of K
  const auto frag = [&](const T* kt, const T* vt, const T* next_kt, int i) {
    if (i < L::kSteps) return L::row_frag(vt, row_base, 0, i);
    if (i < 2 * L::kSteps) return L::row_frag(next_kt, row_base, 0, i - L::kSteps);
    const int j = i - 2 * L::kSteps;
    return L::col_frag(kt, col_base, 0, j / (DP / 32), j % (DP / 32));
  };
  const auto first_frags = [&](const T* kt, const T* vt, const T* next_kt, int first) {
    forget(row_base);  // (the offsets of all fragments, kept, would be 16 registers)
    forget(col_base);
#pragma unroll
    for (int i = 0; i < kRing; ++i) ring[i] = frag(kt, vt, next_kt, first + i);
    in_order();
  };
  const auto form_scores = [&](const T* kt, floatx16_t& s) {
    first_frags(kt, kt, kt, L::kSteps);
    s = floatx16_t{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      Op::mma(s, ring[i % kRing], qf[i]);
      if (i + kRing < L::kSteps) ring[i % kRing] = frag(kt, kt, kt, L::kSteps + i + kRing);
      in_order();
    }
  };
  // scores to exponents, with a bias (without one the probabilities do it), of the keys from key0 on
  const auto exponents = [&](floatx16_t& s, int key0) {
    if (!BIAS) return;
    const int apart = tok - key0 - 4 * half;
    if (first_tok - (key0 + 31) < g.far) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], scale2, my_bias[apart - acc_row(e, 0)] - lse2);
    } else {
      const float offset = my_bias[g.far] - lse2;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], scale2, offset);
    }
  };
  const auto probability = [&](float s) { return exp2_fast(BIAS ? s : __builtin_fmaf(s, scale2, -lse2)); };
  // The bias's share of ds, of the keys from key0 on.
  const auto add_to_table = [&](const floatx16_t& ds, int key0) {
    if (first_tok - (key0 + 31) >= g.far) {
#pragma unroll
      for (int e = 0; e < 16; ++e) far_sum += ds[e];
      return;
    }
    float* const block = my_sums + (distances(g) << g.pack);
    const int row16 = lane & 15;
    float* const mine = block + ((row16 >> g.pack) + 4 - 4 * half) * kDiagonalStride + row16;  // (of the last key of this half)
    const float4* const diagonal = reinterpret_cast<const float4*>(block + min(lane, 46) * kDiagonalStride);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      in_order();
      wave_fence();
      if (((lane >> 4) & 1) == r) {
#pragma unroll
        for (int e = 0; e < 16; ++e) mine[(27 - acc_row(e, 0)) * kDiagonalStride] = ds[e];
      }
      wave_fence();
      float sum[8];  // of the rows whose number is 0 .. 7 modulo 8
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float4 x = diagonal[j], y = diagonal[j + 2];
        sum[4 * j] = x.x + y.x;
        sum[4 * j + 1] = x.y + y.y;
        sum[4 * j + 2] = x.z + y.z;
        sum[4 * j + 3] = x.w + y.w;
      }
      // (a head's rows are every 2^pack-th)
      if (g.pack < 3) {
#pragma unroll
        for (int h = 0; h < 4; ++h) sum[h] += sum[h + 4];
      }
      if (g.pack < 2) {
        sum[0] += sum[2];
        sum[1] += sum[3];
      }
      if (g.pack < 1) sum[0] += sum[1];
      const int distance = first_tok + ((16 * r) >> g.pack) - key0 + lane - 31;
      if (distance >= 0 && lane < 31 + (16 >> g.pack)) {
#pragma unroll
        for (int h = 0; h < 8; ++h)
          if (h < heads) my_sums[h * distances(g) + distance] += sum[h];
      }
    }
    in_order();
  };
  // s: the exponents of the tile at kt (scores without a bias); next_kt: the next tile, of which it leaves them in `next`.
  const auto attend = [&](const T* kt, const T* vt, const T* next_kt, floatx16_t& s, floatx16_t& next, int key0, bool clean, auto has_next) {
    constexpr bool NEXT = decltype(has_next)::value;
    first_frags(kt, vt, next_kt, 0);
    const auto turn = [&](int i) {  // the i-th of the fragments that are used has been: without a next tile its own are left out
      const int n = NEXT || i + kRing < L::kSteps ? i + kRing : i + kRing + L::kSteps;
      if (n < kFrags) ring[i % kRing] = frag(kt, vt, next_kt, n);
    };
    floatx16_t dp{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      Op::mma(dp, ring[i % kRing], gf[i]);
      turn(i);
#pragma unroll
      for (int e = i * 16 / L::kSteps; e < (i + 1) * 16 / L::kSteps; ++e) {
        float p = probability(s[e]);
        stay(p);
        s[e] = p;
      }
      in_order();
    }
    if (NEXT) next = floatx16_t{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      if (NEXT) {
        Op::mma(next, ring[i % kRing], qf[i]);
        turn(L::kSteps + i);
      }
#pragma unroll
      for (int e = i * 16 / L::kSteps; e < (i + 1) * 16 / L::kSteps; ++e) {
        float ds = s[e] * (dp[e] - delta);
        if (NEXT) stay(ds);
        s[e] = ds;
      }
      if (NEXT) in_order();
    }
    if (key0 + 31 > first_tok || !there) {  // (by a choice: what is masked may be NaN)
      const int apart = there ? tok - key0 - 4 * half : -1;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (apart < acc_row(e, 0)) s[e] = 0.f;
    }
    if (BIAS && !clean) add_to_table(s, key0);
    if (NEXT) exponents(next, key0 + (SPLIT ? 0 : 32));
#pragma unroll
    for (int i = 0; i < kSumSteps; ++i) {
      const typename Op::Frag ds = Op::from_acc(s, i / (DP / 32));
      Op::mma(acc[i % (DP / 32)], ring[i % kRing], ds);
      turn((NEXT ? 2 : 1) * L::kSteps + i);
      in_order();
    }
  };
  // Where all keys of these rows are in one tile, delta comes from the probabilities instead: with so few the rounding of `out`
  // is felt, and a row that sees one key has a ds of zero.
  const auto own_delta = [&](const T* vt, const floatx16_t& s) {
    first_frags(vt, vt, vt, 0);
    floatx16_t dp{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      Op::mma(dp, ring[i % kRing], gf[i]);
      if (i + kRing < L::kSteps) ring[i % kRing] = frag(vt, vt, vt, i + kRing);
    }
    const int apart = tok - 4 * half;
    float sum = 0.f, weight = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float p = probability(s[e]);
      sum += apart < acc_row(e, 0) ? 0.f : p * dp[e];
      weight += apart < acc_row(e, 0) ? 0.f : p;
    }
    sum = sum_of_halves(sum);
    weight = sum_of_halves(weight);
    delta = weight == 0.f ? 0.f : sum / weight;
  };
  const bool one_tile = last_tok >= 0 && last_tok < 32;
  const auto write_delta = [&] {
    if (there && half == 0 && (!SPLIT || wave == 0)) {
      const long long stat = static_cast<long long>(head0 + hp) * g.tokens + w.start + tok;
      g.delta[stat] = delta;
      g.offset[stat] = -lse2;
    }
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;

  bool spoilt = false;
  float joined[DP / 8];  // SPLIT: this lane's columns of its row
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) acc[b] = floatx16_t{};
    if constexpr (SPLIT) {
      T* const kt = lds + k_slot(0);
      for (int t = wave; t < tiles; t += kWaves) {
        landed<0>();
        if (clean) Load::clean(kt, 0, lane);
        floatx16_t s;
        form_scores(kt, s);
        exponents(s, 32 * t);
        if (one_tile && !clean) own_delta(kt + kTileElems, s);
        attend(kt, kt + kTileElems, kt, s, s, 32 * t, clean, no);
        lds_done();
        load(t + kWaves, t + kWaves);
      }
      if (!clean) write_delta();
      __syncthreads();
      float* const parts = reinterpret_cast<float*>(smem_raw);
      constexpr size_t kPart = 2 * kTileElems * sizeof(T) / sizeof(float);
      static_assert(32 * DP <= kPart, "the parts take the tiles' place");
      write_part<DP>(parts + wave * kPart, acc, 1.f, lane);
      __syncthreads();
      join_parts<DP>(parts, kPart, wave, lane, joined);
    } else {
      const auto k_tile = [&](int t) { return lds + k_slot(t); };
      const auto v_tile = [&](int t) { return lds + v_slot(t); };
      // K up to tile t and V up to the one before are there, for all wavefronts, and the tiles before t - 1 have been read:
      // their place takes others.
      const auto arrive = [&](int t) {
        if (!S::kFew && t + 1 < tiles) landed<2 * Load::kLoads>();
        else landed<0>();
        if (clean && t < tiles) Load::clean(k_tile(t), part, lane);
        __syncthreads();
        if (S::kFew) load(t + 1, t == 0 ? tiles : t);  // (the first V has been asked for)
        else load(t + 2, t + 2);
      };
      arrive(0);
      floatx16_t s, next;
      form_scores(k_tile(0), s);
      exponents(s, 0);
      if (!clean) {
        if (one_tile) own_delta(v_tile(0), s);
        write_delta();
      }
      int t = 0;
      for (; t + 1 < tiles; ++t) {
        arrive(t + 1);
        attend(k_tile(t), v_tile(t), k_tile(t + 1), s, next, 32 * t, clean, yes);
        s = next;
      }
      if (S::kFew && t > 0) arrive(tiles);
      attend(k_tile(t), v_tile(t), k_tile(t), s, s, 32 * t, clean, no);
    }
    if (clean) break;
    float check = 0.f;
    if constexpr (SPLIT) {
#pragma unroll
      for (int c = 0; c < DP / 8; ++c) check = __builtin_fmaf(joined[c], 0.f, check);
    } else {
#pragma unroll
      for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) check = __builtin_fmaf(acc[b][i], 0.f, check);
    }
    check = sum_of_halves(check);
    spoilt = there && check != 0.f;
    if (!__syncthreads_or(spoilt)) break;
    k_tiles.start(k, g.k_stride, 32 * first_tile, w.len, g.d, 0);
    v_tiles.start(v, g.v_stride, 32 * first_tile, w.len, g.d, 0);
    load_first();
  }
  if (there) {
    T* const mine = dq + tok * g.dq_stride + hp * g.d;
    if constexpr (SPLIT) store_joined<T, DP>(mine, join_column<DP>(wave, lane), g.d, joined, g.scale);
#pragma unroll
    for (int b = 0; b < (SPLIT ? 0 : DP / 32); ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = 32 * b + acc_row(i, half);
        if (col < g.d) store4(mine + col, acc[b][i] * g.scale, acc[b][i + 1] * g.scale, acc[b][i + 2] * g.scale, acc[b][i + 3] * g.scale);
      }
  }
  uint32_t spoilt_rows = static_cast<uint32_t>(__ballot(spoilt));
  if constexpr (SPLIT) spoilt_rows = share_rows(spoilt_rows, reinterpret_cast<uint32_t*>(smem_raw + S::kTiles), wave);
  if (spoilt_rows != 0) __threadfence();
  for (uint32_t rows = spoilt_rows; rows != 0; rows &= rows - 1) {
    const int r = __builtin_ctz(rows), t = (row0 + r) >> g.pack, h = (row0 + r) & (heads - 1);
    sum_row_dq(g, q + t * g.q_stride + h * g.d, d_out + t * g.out_stride + h * g.d, k, v, t,
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lse2), r)),
               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(delta), r)), scale2, BIAS ? bias + h * table_stride(g) : nullptr,
               dq + t * g.dq_stride + h * g.d);
  }
  if (BIAS) {
    // the far part goes to the first far distance; then the wavefronts' sums together, and those of a bucket's distances
    for (int o = 32; o >= heads; o >>= 1) far_sum += __shfl_xor(far_sum, o, kWave);
    if (lane < heads) my_sums[lane * distances(g) + g.far] += far_sum;
    __syncthreads();
    for (int x = threadIdx.x; x < heads * distances(g); x += kThreads)
#pragma unroll
      for (int i = 1; i < kWaves; ++i) sums[x] += sums[i * by_distance_floats(g) + x];
    __syncthreads();
    for (int x = threadIdx.x / 8; x < heads * g.buckets; x += kThreads / 8) {
      const int h = x / g.buckets, b = x % g.buckets;
      const int end = b + 1 < g.buckets ? min(g.starts[b + 1], distances(g)) : distances(g);
      float sum = 0.f;
      for (int at = g.starts[b] + (threadIdx.x & 7); at < end; at += 8) sum += sums[h * distances(g) + at];
      sum = group8_sum(sum);
      if ((threadIdx.x & 7) == 0) g.partials[(static_cast<long long>(slot) * g.heads + head0 + h) * g.buckets + b] = sum;
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

// d_table[b, h] = the sum over row tiles of their shares, for one head, in one order: interleaved sums, then those in turn.
template <typename T>
__device__ void sum_table(const PackedAttn& g, int h, float* sums, T* d_table) {
  int width = 1;
  while (width < g.buckets) width *= 2;
  const int b = static_cast<int>(threadIdx.x) & (width - 1), y = static_cast<int>(threadIdx.x) / width, together = kThreads / width;
  const float* const at = g.partials + static_cast<long long>(h) * g.buckets + b;
  const long long step = static_cast<long long>(g.heads) * g.buckets;
  float sum = 0.f;
  if (b < g.buckets) {
#pragma unroll 8
    for (int s = y; s < g.row_slots; s += together) sum += at[s * step];
  }
  sums[threadIdx.x] = sum;
  __syncthreads();
  if (y != 0 || b >= g.buckets) return;
  for (int i = 1; i < together; ++i) sum += sums[i * width + b];
  store1(d_table + static_cast<long long>(b) * g.heads + h, sum);
}

// dK and dV of a tile of keys, whose K and V stay in registers: for each tile of 32 rows that see them dV += p d_out and
// dK += ds q, the heads of the group one after another.  Rounded to the storage type: p and ds ahead of their products, dK, dV.
// With heads of 128 the sums, K and V are 192 registers: one wavefront per SIMD, bound by what it cannot issue while it waits
// for its own results (28% of the time is matrix instructions', half of it an instruction is issued).  8192 tokens in four
// sequences, 16 heads of 128, bf16: 232 us, 590 TFLOP/s; one of 16384, 6 heads of 128 with a bias: 1530 us, 540.  fp32: one
// workgroup per CU too, for the registers (1024 tokens of 8 heads on 4 of 64: 60 us, 79 with spills at two).
template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && DP == 64 ? 2 : 1) void attn_packed_keys_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Keys<T, DP, SPLIT> S;
  constexpr int kTileElems = S::kTileElems, kKeysLog = rows_log(SPLIT);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  float* const stats = reinterpret_cast<float*>(smem_raw + S::kTiles);  // offsets and deltas, like the tiles
  float* const bias = reinterpret_cast<float*>(smem_raw + S::kLds);

  const int kv = static_cast<int>(blockIdx.x) % g.kv_heads, slot = static_cast<int>(blockIdx.x) / g.kv_heads;
  if (BIAS && slot >= g.key_slots) {
    sum_table(g, static_cast<int>(blockIdx.x) - g.key_slots * g.kv_heads, reinterpret_cast<float*>(smem_raw), static_cast<T*>(g.d_table));
    return;
  }
  SeqTile w;
  if (SPLIT || g.sequences > kRankedSequences) {
    if (!find_tile</*LAST_FIRST=*/false>(g, slot, kKeysLog, 0, &w)) return;
  } else {
    if (!find_ranked_tile(g, slot, kKeysLog, 0, &w)) return;
    w.tile = ((w.len + (1 << kKeysLog) - 1) >> kKeysLog) - 1 - w.tile;  // (the first keys are seen by the most rows)
  }

  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int heads = 1 << g.pack, group = g.heads / g.kv_heads, subs = group >> g.pack;
  const T* const k = static_cast<const T*>(g.k) + w.start * g.k_stride + static_cast<long long>(kv) * g.d;
  const T* const v = static_cast<const T*>(g.v) + w.start * g.v_stride + static_cast<long long>(kv) * g.d;
  const T* const q = static_cast<const T*>(g.q) + w.start * g.q_stride + static_cast<long long>(kv * group) * g.d;
  const T* const d_out = static_cast<const T*>(g.d_out) + w.start * g.out_stride + static_cast<long long>(kv * group) * g.d;
  const float scale2 = g.scale * kLog2e;
  const int tile_key0 = w.tile << kKeysLog, key0 = tile_key0 + (SPLIT ? 0 : 32 * wave), key = key0 + (lane & 31);
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
  const int tiles = (rows - first_row + 31) / 32, steps = tiles * subs;

  constexpr int kTogether = SPLIT ? kWave : kThreads;
  typedef Stream<T, DP, kTogether> Load;
  const int part = SPLIT ? 0 : wave;  // of a tile's load
  const uint32_t lds_at = lds_address(smem_raw), stats_at = lds_address(stats);
  constexpr uint32_t kTileBytes = kTileElems * sizeof(T), kStatBytes = S::kStat * sizeof(float);
  // The rows of Q and d_out with their statistics, 32 at a time, `tiles` of each of the group's `subs` tiles of heads; a
  // wavefront of a SPLIT workgroup takes every fourth of one of these.  What is not there becomes zeros, which add nothing.
  struct Rows {
    Load q, d_out;
    const float *offset, *delta;  // of the next tile's first token
    uint32_t at;                  // this lane's row
    int row, sub, left;           // row: this lane's; left: tiles of this sub
  };
  const int every = SPLIT ? kWaves : 1;
  const auto begin = [&](Rows& r, int sub, int first_tile) {
    const long long head = kv * group + (sub << g.pack);
    const int first = first_row + 32 * first_tile;
    r.q.start(q + static_cast<long long>(sub << g.pack) * g.d, g.q_stride, first, w.len, g.d, g.pack);
    r.d_out.start(d_out + static_cast<long long>(sub << g.pack) * g.d, g.out_stride, first, w.len, g.d, g.pack);
    const long long stat = head * g.tokens + w.start + (first >> g.pack);
    r.offset = g.offset + stat;
    r.delta = g.delta + stat;
    r.row = lane < 32 ? first + lane : rows;
    r.sub = sub;
    r.left = tiles - first_tile;
  };
  Rows stream{{q, g.q_stride, first_row, w.len, g.d, g.pack, part, lane}, {d_out, g.out_stride, first_row, w.len, g.d, g.pack, part, lane},
              nullptr, nullptr, (static_cast<uint32_t>(lane & (heads - 1)) * static_cast<uint32_t>(g.tokens) + ((lane & 31) >> g.pack)) * 4u, 0, 0, 0};
  const auto load = [&](Rows& r, uint32_t tile, uint32_t stat) {
    if (!SPLIT && r.left <= 0) begin(r, r.sub + 1, 0);
    r.q.load(tile, part, every);
    r.d_out.load(tile + kTileBytes, part, every);
    if (part == 0) {
      const uint32_t off = r.row < rows ? r.at : kOutside;
      load_word_to_lds(row_buffer(r.offset, kOutside), off, stat);
      load_word_to_lds(row_buffer(r.delta, kOutside), off, stat + kWave * sizeof(float));
    }
    r.offset += every * (32 >> g.pack);
    r.delta += every * (32 >> g.pack);
    r.row += every * 32;
    r.left -= every;
  };

  floatx16_t dk[DP / 32], dv[DP / 32];
  uint32_t row_base = L::row_base(lane), col_base = L::col_base(lane);
  // A tile of 32 rows goes by in three passes of matrix instructions, with the arithmetic between them: d_out V^T, and the
  // probabilities; the next tile's scores, and ds; dV += P^T d_out and dK += dS^T Q, and the next tile's exponents' offsets.
  // The order is written out as in the kernel above.
  constexpr int kRing = sizeof(T) == 2 && DP == 128 ? 8 : 4;
  constexpr int kCols = 2 * L::kGroups * (DP / 32), kFrags = 2 * L::kSteps + kCols;
  typename Op::Frag ring[kRing];
  // the fragments of the three passes: of d_out, of the next tile's Q, of d_out and Q in turn
  const auto frag = [&](const T* tile, const T* next_tile, int i) {
    if (i < L::kSteps) return L::row_frag(tile + kTileElems, row_base, 0, i);
    if (i < 2 * L::kSteps) return L::row_frag(next_tile, row_base, 0, i - L::kSteps);
    const int j = i - 2 * L::kSteps;
    return L::col_frag(j % 2 == 0 ? tile + kTileElems : tile, col_base, 0, j / 2 / (DP / 32), j / 2 % (DP / 32));
  };
  const auto first_frags = [&](const T* tile, const T* next_tile, int first) {
    forget(row_base);
    forget(col_base);
#pragma unroll
    for (int i = 0; i < kRing; ++i) ring[i] = frag(tile, next_tile, first + i);
    in_order();
  };
  const auto form_scores = [&](const T* tile, floatx16_t& s) {
    first_frags(tile, tile, L::kSteps);
    s = floatx16_t{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      Op::mma(s, ring[i % kRing], kf[i]);
      if (i + kRing < L::kSteps) ring[i % kRing] = frag(tile, tile, L::kSteps + i + kRing);
      in_order();
    }
  };
  // register i of a tile from row r0 on: token r0 >> pack + (i's part, the same for all lanes) + (4 half >> pack), head likewise
  const int lane_tok = ((4 * half) >> g.pack) - key, stride = BIAS ? table_stride(g) : 0;
  const float* const my_bias = BIAS ? bias + kPad + (g.pack == 3 ? 4 * half * stride : 0) : nullptr;
  // what a tile's registers need of its rows: the exponents' offsets without the bias (at 0) or delta (at kWave)
  const auto per_row = [&](const float* stat, floatx16_t& x) {
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const float4 v = *reinterpret_cast<const float4*>(stat + 8 * a + 4 * half);
      x[4 * a] = v.x;
      x[4 * a + 1] = v.y;
      x[4 * a + 2] = v.z;
      x[4 * a + 3] = v.w;
    }
  };
  // registers first.. of the bias of the tile from row r0 on
  const auto read_bias = [&](int r0, int first, int end, floatx16_t& x) {
    const int apart = (r0 >> g.pack) + lane_tok;
#pragma unroll
    for (int i = first; i < end; ++i) x[i] = my_bias[(i & 3 & (heads - 1)) * stride + min(apart + (acc_row(i, 0) >> g.pack), g.far)];
  };
  const auto offsets = [&](const float* stat, int r0, floatx16_t& offset) {
    per_row(stat, offset);
    if (BIAS) {
      floatx16_t x;
      read_bias(r0, 0, 16, x);
#pragma unroll
      for (int i = 0; i < 16; ++i) offset[i] += x[i];
    }
  };
  // s: the scores of the tile from row r0 on, `offset` their offsets; leaves those of the next one in `next` and `offset`, and
  // its first fragments (as first_frags() does) in the ring.  between() comes in the third pass.  What a pass leaves is used
  // some steps into the next, whose matrix instructions do not need it: by then it is there.
  const auto attend = [&](const T* tile, const float* stat, int r0, const T* next_tile, const float* next_stat, int next_r0, floatx16_t& s,
                          floatx16_t& next, floatx16_t& offset, auto has_next, auto between) {
    constexpr bool NEXT = decltype(has_next)::value;
    constexpr int kGroup = 16 / L::kGroups, kLag = L::kSteps >= 8 ? 2 : 1;
    constexpr bool kSummed = sizeof(T) * DP > 128;  // (a wavefront has more than 256 registers)
    forget(row_base);
    forget(col_base);
    const auto turn = [&](int i) {  // the i-th of the fragments that are used has been: without a next tile its own are left out
      const int n = NEXT || i + kRing < L::kSteps ? i + kRing : i + kRing + L::kSteps;
      if (n < kFrags) ring[i % kRing] = frag(tile, next_tile, n);
      else if (NEXT) ring[i % kRing] = frag(next_tile, next_tile, n - kFrags);
    };
    floatx16_t dp{}, delta, next_bias;  // (read ahead of their use, as the fragments are)
    per_row(stat + kWave, delta);
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      Op::mma(dp, ring[i % kRing], vf[i]);
      turn(i);
#pragma unroll
      for (int e = i * 16 / L::kSteps; e < (i + 1) * 16 / L::kSteps; ++e) {
        float p = exp2_fast(__builtin_fmaf(s[e], scale2, offset[e]));
        stay(p);
        s[e] = p;
      }
      in_order();
    }
    const int apart = (r0 >> g.pack) + lane_tok;
    const bool edge = key0 + 31 > r0 >> g.pack;
    if (edge) {  // (by a choice: what is masked may be NaN)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (apart + (acc_row(e, 0) >> g.pack) < 0) s[e] = 0.f;
    }
    typename Op::Frag p[L::kGroups], ds[L::kGroups];
    if (NEXT) next = floatx16_t{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      if (NEXT) {
        Op::mma(next, ring[i % kRing], kf[i]);
        turn(L::kSteps + i);
      }
      if (kSummed && NEXT && i == kLag) stay_summed(dp);
      if (i < kLag) {
#pragma unroll
        for (int c = i * L::kGroups / kLag; c < (i + 1) * L::kGroups / kLag; ++c) {
          p[c] = Op::from_acc(s, c);
          if (NEXT) stay(p[c]);
        }
      } else {
#pragma unroll
        for (int e = (i - kLag) * 16 / (L::kSteps - kLag); e < (i + 1 - kLag) * 16 / (L::kSteps - kLag); ++e) {
          float x = s[e] * (dp[e] - delta[e]);
          if (NEXT) stay(x);
          dp[e] = x;
          if (e % kGroup == kGroup - 1) {
            ds[e / kGroup] = Op::from_acc(dp, e / kGroup);
            if (NEXT) stay(ds[e / kGroup]);
          }
        }
      }
      if (NEXT && BIAS) read_bias(next_r0, i * 16 / L::kSteps, (i + 1) * 16 / L::kSteps, next_bias);
      if (NEXT) in_order();
    }
    if (edge) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (apart + (acc_row(e, 0) >> g.pack) < 0) dp[e] = 0.f;
#pragma unroll
      for (int c = 0; c < L::kGroups; ++c) ds[c] = Op::from_acc(dp, c);
    }
    if (NEXT) per_row(next_stat, offset);
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const int c = i / 2 / (DP / 32), e = i / 2 % (DP / 32);
      if (i % 2 == 0) Op::mma(dv[e], ring[i % kRing], p[c]);
      else Op::mma(dk[e], ring[i % kRing], ds[c]);
      turn((NEXT ? 2 : 1) * L::kSteps + i);
      if (NEXT && BIAS) {
#pragma unroll
        for (int n = i * 16 / kCols; n < (i + 1) * 16 / kCols; ++n) offset[n] += next_bias[n];
      }
      in_order();
      if (i == kCols / 4) between();
    }
  };
  const auto nothing = [] {};
  // (waited for here, or the compiler waits in every turn of the loop that uses them first, for the tiles on their way too)
  const auto have_values = [&] {
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) stay(vf[i]);
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;

  bool spoilt = false;
  float joined_k[DP / 8], joined_v[DP / 8];  // SPLIT: this lane's columns of its key
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dk[b] = dv[b] = floatx16_t{};
    if constexpr (SPLIT) {
      const auto place = [&](int n) { return wave * S::kPlaces + n % S::kPlaces; };
      const auto load_next = [&](int n) { load(stream, lds_at + place(n) * 2 * kTileBytes, stats_at + place(n) * kStatBytes); };
      const auto of_heads = [&] {
        have_values();
        for (int t = wave, n = 0; t < tiles; t += kWaves, ++n) {
          T* const mine = lds + place(n) * 2 * kTileElems;
          const float* const stat = stats + place(n) * S::kStat;
          if (S::kPlaces == 2 && t + kWaves < tiles) {
            load_next(n + 1);
            landed<2 * Load::kLoads + 2>();
          } else {
            landed<0>();
          }
          if (clean) {
            Load::clean(mine, 0, lane);
            Load::clean(mine + kTileElems, 0, lane);
          }
          const int r0 = first_row + 32 * t;
          floatx16_t s, offset;
          form_scores(mine, s);
          offsets(stat, r0, offset);
          first_frags(mine, mine, 0);
          attend(mine, stat, r0, mine, stat, r0, s, s, offset, no, nothing);
          lds_done();
          if (S::kPlaces == 1 && t + kWaves < tiles) load_next(n + 1);
        }
      };
      for (int sub = 0; sub < subs; ++sub) {
        begin(stream, sub, wave);
        if (wave < tiles) load_next(0);
        if (BIAS) {
          __syncthreads();  // (the heads before are done with their bias)
          fill_bias<T, kThreads>(g, kv * group + (sub << g.pack), bias);
          __syncthreads();
        }
        of_heads();
      }
      float* const parts = reinterpret_cast<float*>(smem_raw);
      constexpr size_t kPart = 2 * kTileElems * sizeof(T) / sizeof(float);
      static_assert(32 * DP <= kPart, "the parts take the tiles' place");
      __syncthreads();
      write_part<DP>(parts + wave * kPart, dv, 1.f, lane);
      __syncthreads();
      join_parts<DP>(parts, kPart, wave, lane, joined_v);
      __syncthreads();
      write_part<DP>(parts + wave * kPart, dk, 1.f, lane);
      __syncthreads();
      join_parts<DP>(parts, kPart, wave, lane, joined_k);
    } else {
      const auto slot = [&](int it) { return it % S::kCopies; };
      const auto tile = [&](int it) { return lds + slot(it) * 2 * kTileElems; };
      const auto stat = [&](int it) { return stats + slot(it) * S::kStat; };
      const auto load_next = [&](int it) { load(stream, lds_at + slot(it) * 2 * kTileBytes, stats_at + slot(it) * kStatBytes); };
      // With four places two tiles are in use, another there or on its way, and the last one's place takes the one after: asked
      // for a tile's time before the wait for it, in the third pass of the tile two before it.  With three it is the tile before.
      constexpr bool kBetween = S::kCopies == 4;
      // Tile `it` is there, for all wavefronts, and those before it - 2 (it - 1) have been read.
      const auto clean_tile = [&](int it) {
        Load::clean(tile(it), part, lane);
        Load::clean(tile(it) + kTileElems, part, lane);
      };
      const auto arrive = [&](int it) {
        landed<0>();
        if (clean) clean_tile(it);
        __syncthreads();
        if (it + 1 < steps) load_next(it + 1);
      };
      const auto heads_bias = [&](int sub) {
        __syncthreads();  // (the offsets of the heads before are done)
        fill_bias<T, kThreads>(g, kv * group + (sub << g.pack), bias);
        __syncthreads();
      };
      begin(stream, 0, 0);
      load_next(0);
      const int first = kBetween && steps > 1 ? 1 : 0;
      if (first == 1) {
        load_next(1);
        landed<0>();
        if (clean) clean_tile(0);
      }
      arrive(first);
      if (BIAS) heads_bias(0);
      have_values();
      floatx16_t s, next, offset;
      form_scores(tile(0), s);
      offsets(stat(0), first_row, offset);
      first_frags(tile(0), tile(0), 0);
      int it = 0, r0 = first_row, ahead = 0, sub = 0;  // ahead: tile it + 1's number among those of its heads, which `sub` are
      for (; it + 1 < steps; ++it) {
        if (++ahead == tiles) {
          ahead = 0;
          ++sub;
          if (BIAS) heads_bias(sub);
        }
        const int next_r0 = first_row + 32 * ahead;
        if (!kBetween) arrive(it + 1);
        attend(tile(it), stat(it), r0, tile(it + 1), stat(it + 1), next_r0, s, next, offset, yes, [&] {
          if (kBetween && it + 2 < steps) arrive(it + 2);
        });
        s = next;
        r0 = next_r0;
      }
      attend(tile(it), stat(it), r0, tile(it), stat(it), r0, s, s, offset, no, nothing);
    }
    if (clean) break;
    float check = 0.f;
    if constexpr (SPLIT) {
#pragma unroll
      for (int c = 0; c < DP / 8; ++c) check = __builtin_fmaf(joined_k[c], 0.f, __builtin_fmaf(joined_v[c], 0.f, check));
    } else {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) check = __builtin_fmaf(dk[b][i], 0.f, __builtin_fmaf(dv[b][i], 0.f, check));
    }
    check = sum_of_halves(check);
    spoilt = there && check != 0.f;
    if (!__syncthreads_or(spoilt)) break;
  }
  T* const dk_rows = static_cast<T*>(g.dk) + w.start * g.dk_stride + static_cast<long long>(kv) * g.d;
  T* const dv_rows = static_cast<T*>(g.dv) + w.start * g.dv_stride + static_cast<long long>(kv) * g.d;
  if (there) {
    if constexpr (SPLIT) {
      store_joined<T, DP>(dk_rows + key * g.dk_stride, join_column<DP>(wave, lane), g.d, joined_k, g.scale);
      store_joined<T, DP>(dv_rows + key * g.dv_stride, join_column<DP>(wave, lane), g.d, joined_v, 1.f);
    }
#pragma unroll
    for (int b = 0; b < (SPLIT ? 0 : DP / 32); ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = 32 * b + acc_row(i, half);
        if (col >= g.d) continue;
        store4(dk_rows + key * g.dk_stride + col, dk[b][i] * g.scale, dk[b][i + 1] * g.scale, dk[b][i + 2] * g.scale, dk[b][i + 3] * g.scale);
        store4(dv_rows + key * g.dv_stride + col, dv[b][i], dv[b][i + 1], dv[b][i + 2], dv[b][i + 3]);
      }
  }
  uint32_t spoilt_keys = static_cast<uint32_t>(__ballot(spoilt));
  if constexpr (SPLIT) spoilt_keys = share_rows(spoilt_keys, reinterpret_cast<uint32_t*>(stats + S::kCopies * S::kStat), wave);
  if (spoilt_keys != 0) __threadfence();
  for (uint32_t keys = spoilt_keys; keys != 0; keys &= keys - 1) {
    const int j = key0 + __builtin_ctz(keys);
    sum_key(g, w, kv, j, BIAS ? bias : nullptr, dk_rows + j * g.dk_stride, dv_rows + j * g.dv_stride);
  }
}

template <typename T, int DP, bool BIAS>
hipError_t launch_bwd(const PackedAttn& g, hipStream_t st) {
  PackedAttn rows = g;
  rows.pack = g.pack_rows;
  const size_t table = BIAS ? static_cast<size_t>(table_floats(g)) * sizeof(float) : 0;
  const size_t by_row = BIAS ? (table_floats(rows) + kWaves * by_distance_floats(rows)) * sizeof(float) : 0;
  const size_t row_groups = static_cast<size_t>(g.row_slots) * (g.heads >> rows.pack), key_groups = static_cast<size_t>(g.key_slots) * g.kv_heads;
  hipError_t e = g.split_rows ? launch_packed<attn_packed_rows_kernel<T, DP, BIAS, true>>(row_groups, Rows<T, DP, BIAS, true>::kLds + by_row, rows, st)
                              : launch_packed<attn_packed_rows_kernel<T, DP, BIAS, false>>(row_groups, Rows<T, DP, BIAS, false>::kLds + by_row, rows, st);
  if (e != hipSuccess) return e;
  // (behind the key tiles a workgroup per head joins the table's gradient: a launch of its own was 4 us)
  const size_t groups = key_groups + (BIAS ? g.heads : 0);
  return g.split_keys ? launch_packed<attn_packed_keys_kernel<T, DP, BIAS, true>>(groups, Keys<T, DP, true>::kLds + table, g, st)
                      : launch_packed<attn_packed_keys_kernel<T, DP, BIAS, false>>(groups, Keys<T, DP, false>::kLds + table, g, st);
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

bool attn_packed_split_rows_fit(int dtype, const PackedAttn& g) {
  const size_t tiles = dtype == 1 ? (g.d <= 64 ? Rows<bf16_t, 64, true, true>::kLds : Rows<bf16_t, 128, true, true>::kLds)
                                  : (g.d <= 64 ? Rows<float, 64, true, true>::kLds : Rows<float, 128, true, true>::kLds);
  return g.buckets == 0 || tiles + (table_floats(g) + kWaves * by_distance_floats(g)) * sizeof(float) <= kMostLds;
}
hipError_t attn_packed_bwd(int dtype, const PackedAttn& g, hipStream_t st) {
  return dtype == 1 ? launch_bwd<bf16_t>(g, st) : launch_bwd<float>(g, st);
}

}  // namespace lynx
