// Causal attention over packed sequences with grouped heads, forward: out = softmax(scale Q K^T + bias) V, one pass over the
// keys with a running maximum and sum; no seq x seq tensor.
#include <type_traits>

#include "attn_packed.h"

namespace lynx {
namespace {

// K and V in tiles of 32 keys, kCopies of each; or one of each wavefront.
template <typename T, int DP, bool SPLIT> struct Fwd {
  static constexpr int kTileElems = 32 * DP, kCopies = SPLIT ? kWaves : sizeof(T) * DP == 512 ? 3 : 4;
  static constexpr size_t kTiles = 2 * kCopies * static_cast<size_t>(kTileElems) * sizeof(T);
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

// Tile by tile of 32 keys: s = scale2 q.k + bias, m' = max(m, s), p = 2^(s - m'), o = 2^(m - m') o + p v, and so the sum of p;
// out = o / sum, lse = (m + log2 sum) ln 2.  Rounded to the storage type: p ahead of its product, out.
// Bound by the issue of instructions: a 32 x 32 block at 128 columns is 16 matrix instructions (512 cycles) and about 240
// others, which two wavefronts of a SIMD issue between each other's.  A tile of K and V is read once for the 128 rows of a
// workgroup.  8192 tokens in four sequences, 16 heads of 128, bf16: 102 us, 670 TFLOP/s; one of 16384, 6 heads of 128 with a
// bias: 500 us, 820; of a few tokens 6 us, the time of a launch and of three loads that wait for each other.
template <typename T, int DP, bool BIAS, bool SPLIT>
__global__ __launch_bounds__(kThreads, SPLIT && sizeof(T) * DP == 512 ? 1 : 2) void attn_packed_fwd_kernel(PackedAttn g) {
  typedef Tile<T, DP> L;
  typedef Operand<T> Op;
  typedef Fwd<T, DP, SPLIT> S;
  constexpr int kTileElems = S::kTileElems, kRowsLog = rows_log(SPLIT);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  T* const lds = reinterpret_cast<T*>(smem_raw);
  float* const tops = reinterpret_cast<float*>(smem_raw + S::kTiles);  // SPLIT: each wavefront's maxima, then sums
  float* const bias = reinterpret_cast<float*>(smem_raw + S::kLds);

  const int subs = g.heads >> g.pack;
  const int head0 = (static_cast<int>(blockIdx.x) % subs) << g.pack;
  SeqTile w;
  const int slot = static_cast<int>(blockIdx.x) / subs;
  if (!(SPLIT ? find_tile</*LAST_FIRST=*/true>(g, slot, kRowsLog, g.pack, &w) : find_ranked_tile(g, slot, kRowsLog, g.pack, &w))) return;

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
  constexpr int kTogether = SPLIT ? kWave : kThreads;
  typedef Stream<T, DP, kTogether> Load;
  const int part = SPLIT ? 0 : wave;  // of a tile's load
  const uint32_t lds_at = lds_address(smem_raw);
  constexpr uint32_t kTileBytes = kTileElems * sizeof(T);
  // SPLIT: the wavefronts deal the tiles up to the last one that the rows see; else the workgroup's rows see these
  const int end_tok = SPLIT ? last_tok + 1 : min(((w.tile + 1) << kRowsLog) >> g.pack, w.len);
  const int tiles = (end_tok + 31) / 32;  // (a wavefront's last ones may be all masked: leaving them out would save nothing)
  const int first_tile = SPLIT ? wave : 0, every = SPLIT ? kWaves : 1;
  Load k_tiles(k, g.k_stride, 32 * first_tile, w.len, g.d, 0, part, lane), v_tiles(v, g.v_stride, 32 * first_tile, w.len, g.d, 0, part, lane);
  const auto slot_of = [&](int t) { return (SPLIT ? wave : t % S::kCopies) * 2 * kTileElems; };
  const auto load_k = [&](int t) { k_tiles.load(lds_at + slot_of(t) * sizeof(T), part, every); };
  const auto load_v = [&](int t) { v_tiles.load(lds_at + slot_of(t) * sizeof(T) + kTileBytes, part, every); };
  const auto load_first = [&] {
#pragma unroll
    for (int t = 0; t < (SPLIT || S::kCopies < 4 ? 1 : 2); ++t)
      if (first_tile + t < tiles) {
        load_k(t);
        load_v(t);
      }
  };
  load_first();  // (ahead of what the bias waits for)
  const float* const my_bias = BIAS ? bias + hp * table_stride(g) + kPad : nullptr;
  if (BIAS) fill_bias<T, kThreads>(g, head0, bias);
  if (SPLIT && BIAS) __syncthreads();

  floatx16_t o[DP / 32];
  float m, total;
  uint32_t row_base = L::row_base(lane), col_base = L::col_base(lane);
  // A tile goes by in two passes of matrix instructions, with the arithmetic between them: the scores of tile t + 1, and the
  // probabilities of tile t; the sum of tile t over V, and the maxima of tile t + 1.  The order is written out (in_order()), with
  // fragments kRing steps ahead of their use: left to itself the compiler keeps one and waits for each.
  constexpr int kRing = 4, kValueSteps = L::kGroups * (DP / 32);
  typename Op::Frag ring[kRing];
  // the fragments of a tile's two passes: of K (kt), then of V (vt)
  const auto frag = [&](const T* kt, const T* vt, int i) {
    if (i < L::kSteps) return L::row_frag(kt, row_base, 0, i);
    const int j = i - L::kSteps;
    return L::col_frag(vt, col_base, 0, j / (DP / 32), j % (DP / 32));
  };
  const auto first_frags = [&](const T* kt, const T* vt, int first) {
    forget(row_base);  // (the offsets of all fragments, kept, would be 16 registers)
    forget(col_base);
#pragma unroll
    for (int i = 0; i < kRing; ++i) ring[i] = frag(kt, vt, first + i);
    in_order();
  };
  // scores to logits (without a bias unscaled: the probabilities scale them) of the keys from key0 on
  const auto logits = [&](floatx16_t& s, int key0) {
    const int apart = tok - key0 - 4 * half;
    if (BIAS && first_tok - (key0 + 31) < g.far) {
      const float* const at = my_bias + apart;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], scale2, at[-acc_row(e, 0)]);
    } else if (BIAS) {
      const float far = my_bias[g.far];
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], scale2, far);
    }
    if (key0 + 31 > first_tok) {  // (by a choice, not a sum: a masked score may be NaN)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (apart < acc_row(e, 0)) s[e] = -kInf;
    }
  };
  // The reference follows the maximum only where that has left it 2^8 behind: probabilities up to 256 lose nothing in fp32
  // sums or by a rounding to the storage type, and the accumulators are hardly ever scaled.  A row decides for itself: for the
  // others of the wavefront the factor is 1.  Returns what the exponents are taken from.
  const auto follow = [&](float top) {
    top = max_of_halves(BIAS ? top : top * scale2);
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
    return m == -kInf ? 0.f : m;  // (a row that has seen nothing yet: every probability 0)
  };
  const auto largest = [&](const floatx16_t& s) {
    float top = -kInf;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
    return top;
  };
  const auto form_scores = [&](const T* kt, const T* vt, floatx16_t& s) {
    first_frags(kt, vt, 0);
    s = floatx16_t{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      Op::mma(s, ring[i % kRing], qf[i]);
      if (i + kRing < L::kSteps) ring[i % kRing] = frag(kt, vt, i + kRing);
      in_order();
    }
  };
  // s: the tile's logits, with `top` their largest; kt: the next tile's keys, of which it leaves the logits in `next`.
  const auto attend = [&](const T* kt, const T* vt, floatx16_t& s, floatx16_t& next, int next_key0, float& top, auto has_next) {
    constexpr bool NEXT = decltype(has_next)::value;
    first_frags(kt, vt, NEXT ? 0 : L::kSteps);
    const float base = follow(top);
    typename Op::Frag p[L::kGroups];
    if (NEXT) next = floatx16_t{};
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i) {
      if (NEXT) {
        Op::mma(next, ring[i % kRing], qf[i]);
        ring[i % kRing] = frag(kt, vt, i + kRing);
      }
#pragma unroll
      for (int e = i * 16 / L::kSteps; e < (i + 1) * 16 / L::kSteps; ++e) {
        s[e] = exp2_fast(BIAS ? s[e] - base : __builtin_fmaf(s[e], scale2, -base));
        total += s[e];
        constexpr int kGroup = 16 / L::kGroups;
        if (e % kGroup == kGroup - 1) p[e / kGroup] = Op::from_acc(s, e / kGroup);
      }
      if (NEXT) {
        if (i % 2 == 1) stay(total);
        in_order();
      }
    }
    if (NEXT) {
#pragma unroll
      for (int c = 0; c < L::kGroups; ++c) stay(p[c]);
      logits(next, next_key0);
      top = -kInf;
    }
#pragma unroll
    for (int i = 0; i < kValueSteps; ++i) {
      Op::mma(o[i % (DP / 32)], ring[i % kRing], p[i / (DP / 32)]);
      if (i + kRing < kValueSteps) ring[i % kRing] = frag(kt, vt, L::kSteps + i + kRing);
      if (NEXT) {
#pragma unroll
        for (int e = i * 16 / kValueSteps; e < (i + 1) * 16 / kValueSteps; ++e) top = fmaxf(top, next[e]);
      }
      in_order();
    }
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;

  bool spoilt = false;
  float joined[DP / 8];  // SPLIT: this lane's columns of its row
  for (bool clean = false;; clean = true) {
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) o[b] = floatx16_t{};
    m = -kInf;       // maximum of the logits so far, times log2 e
    total = 0.f;     // this half's share of the sum
    if constexpr (SPLIT) {
      // one tile of each: K's next one is requested when the scores are there, V's at the end
      const T* const kt = lds + slot_of(0);
      T* const vt = lds + slot_of(0) + kTileElems;
      // (waited for here, or the compiler waits in every turn of the loop, for the tiles on their way too)
#pragma unroll
      for (int i = 0; i < L::kSteps; ++i) stay(qf[i]);
      for (int t = wave; t < tiles; t += kWaves) {
        const bool more = t + kWaves < tiles;
        landed<Load::kLoads>();
        floatx16_t s;
        form_scores(kt, vt, s);
        lds_done();
        if (more) {
          load_k(t);
          landed<Load::kLoads>();
        } else {
          landed<0>();
        }
        if (clean) Load::clean(vt, 0, lane);
        logits(s, 32 * t);
        float top = largest(s);
        attend(kt, vt, s, s, 0, top, no);
        lds_done();
        if (more) load_v(t);
      }
    } else {
      // Tiles up to t are there, for all wavefronts, and those before t - 1 have been read: their place takes another.
      const auto arrive = [&](int t) {
        if (S::kCopies == 4 && t + 1 < tiles) landed<2 * Load::kLoads>();
        else landed<0>();
        if (clean) Load::clean(lds + slot_of(t) + kTileElems, part, lane);
        __syncthreads();
        if (t + S::kCopies - 2 < tiles) {
          load_k(t + S::kCopies - 2);
          load_v(t + S::kCopies - 2);
        }
      };
      arrive(0);
      floatx16_t s, next;
      form_scores(lds, lds, s);
      logits(s, 0);
      float top = largest(s);
      int t = 0;
      for (; t + 1 < tiles; ++t) {
        arrive(t + 1);
        attend(lds + slot_of(t + 1), lds + slot_of(t) + kTileElems, s, next, 32 * (t + 1), top, yes);
        s = next;
      }
      attend(lds + slot_of(t), lds + slot_of(t) + kTileElems, s, s, 0, top, no);
    }
    total = sum_of_halves(total);
    if constexpr (SPLIT) {
      if (half == 0) {
        tops[wave * 32 + lane] = m;
        tops[(kWaves + wave) * 32 + lane] = total;
      }
      __syncthreads();
      float top = -kInf;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) top = fmaxf(top, tops[i * 32 + (lane & 31)]);
      total = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float of = tops[i * 32 + (lane & 31)], sum = tops[(kWaves + i) * 32 + (lane & 31)];
        total += of == -kInf ? sum : sum * exp2_fast(of - top);  // (one whose keys this row does not see has an empty part)
      }
      float* const parts = reinterpret_cast<float*>(smem_raw);
      constexpr size_t kPart = 2 * kTileElems * sizeof(T) / sizeof(float);
      static_assert(32 * DP <= kPart, "the parts take the tiles' place");
      write_part<DP>(parts + wave * kPart, o, m == -kInf ? 1.f : exp2_fast(m - top), lane);
      m = top;
      __syncthreads();
      join_parts<DP>(parts, kPart, wave, lane, joined);
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
    k_tiles.start(k, g.k_stride, 32 * first_tile, w.len, g.d, 0);
    v_tiles.start(v, g.v_stride, 32 * first_tile, w.len, g.d, 0);
    load_first();
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

// Rows outside [offsets[0], offsets[sequences]); where there are none the workgroups only look.
__global__ void attn_packed_clear_kernel(unsigned char* x, int row_bytes, int tokens, const int32_t* offsets, int sequences) {
  const int first = min(max(offsets[0], 0), tokens), end = min(max(offsets[sequences], first), tokens), outside = tokens - (end - first);
  for (int r = blockIdx.x; r < outside; r += gridDim.x) {
    unsigned char* const row = x + static_cast<long long>(r < first ? r : r - first + end) * row_bytes;
    for (int c = threadIdx.x * 16; c < row_bytes; c += kThreads * 16) *reinterpret_cast<uint4*>(row + c) = make_uint4(0, 0, 0, 0);
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

// So many workgroups of 128 rows keep the card busy; with fewer, 32 rows each go faster, although each reads K and V for itself
// (forward, 5 heads of 128, 85: 25 us against 62, 245: 42 and 54; 445: 57 and 48; 8 heads of 64, 392: 32 and 43, 5, 445: 33 and
// 35, 490: 22 and 19).  dQ with a bias changes earlier for heads of 128, whose 32 rows have a CU to themselves (245: 112 and
// 94, 376: 227 and 141, 445: 161 and 84, but 170, one sequence of 3000 among them: 83 and 125).
constexpr size_t kRowGroups = 400, kWideBiasRowGroups = 208;
// Workgroups of 128 keys are enough at 512 for heads of up to 64, at half of that for wider ones.  They differ more in size,
// and it takes two rounds of them to even that out (heads of 64, 576 of them: 361 us, with 32 keys each 194; 1088: 113 and
// 126; heads of 128, 695: 170 and 215).  And sequences that are shorter than a tile leave most of one empty (256 of 32 tokens on average: 43 us and 31).
constexpr size_t key_groups(int d) { return d <= 64 ? 512 : 256; }
constexpr int kShort = 96;
// As many heads of a group as are a power of two, up to 8; fewer where their biases by distance would take more than `floats`
// of LDS.  10 KB leave a workgroup what it needs.  The sums of the bias's gradient take four times that: where heads are wider
// than 64, half of it for dQ, so that two workgroups share a CU (seven sequences of 1500, 16 heads on 2 of 128: 288 us with 8
// heads to a tile and 185 with 4, but forward 111 and 116, dK and dV 352 and 377).
static int heads_together(const PackedAttn& g, int floats) {
  const int group = g.heads / g.kv_heads;
  int pack = 0;
  while (pack < 3 && (group >> pack) % 2 == 0 && (g.buckets == 0 || table_stride(g) << (pack + 1) <= floats)) ++pack;
  return pack;
}
void attn_packed_choose(int dtype, PackedAttn* g) {
  const auto row_groups = [&](const PackedAttn& x) { return attn_packed_row_slots(x, false) * (x.heads >> x.pack); };
  g->pack = heads_together(*g, 2560);
  g->pack_rows = heads_together(*g, g->d > 64 ? 1280 : 2560);
  g->split_fwd = row_groups(*g) < kRowGroups;
  PackedAttn rows = *g;
  rows.pack = g->pack_rows;
  g->split_rows = row_groups(rows) < (g->buckets > 0 && g->d > 64 ? kWideBiasRowGroups : kRowGroups) && attn_packed_split_rows_fit(dtype, rows);
  g->row_slots = static_cast<int>(attn_packed_row_slots(rows, g->split_rows));
  g->split_keys = 0;
  g->split_keys = attn_packed_key_slots(*g) * g->kv_heads < 2 * key_groups(g->d) || g->tokens / g->sequences < kShort;
  g->key_slots = static_cast<int>(attn_packed_key_slots(*g));
}
bool attn_packed_fits(const PackedAttn& g) {
  const long long fwd = static_cast<long long>(attn_packed_row_slots(g, g.split_fwd)) * (g.heads >> g.pack);
  const long long rows = static_cast<long long>(g.row_slots) * (g.heads >> g.pack_rows), keys = static_cast<long long>(g.key_slots) * g.kv_heads + g.heads;
  return fits_grid(fwd, kThreads) && fits_grid(rows, kThreads) && fits_grid(keys, kThreads);
}
size_t attn_packed_row_slots(const PackedAttn& g, bool split) {
  return ((static_cast<size_t>(g.tokens) << g.pack) >> rows_log(split)) + static_cast<size_t>(g.sequences);
}
size_t attn_packed_key_slots(const PackedAttn& g) {
  return (static_cast<size_t>(g.tokens) >> rows_log(g.split_keys)) + static_cast<size_t>(g.sequences);
}
hipError_t attn_packed_clear(int dtype, void* x, int cols, int tokens, const int32_t* offsets, int sequences, hipStream_t st) {
  hipLaunchKernelGGL(attn_packed_clear_kernel, dim3(tokens < 256 ? tokens : 256), dim3(kThreads), 0, st, static_cast<unsigned char*>(x),
                     cols * (dtype == 1 ? 2 : 4), tokens, offsets, sequences);
  return hipGetLastError();
}
hipError_t attn_packed_fwd(int dtype, const PackedAttn& g, hipStream_t st) {
  return dtype == 1 ? launch_fwd<bf16_t>(g, st) : launch_fwd<float>(g, st);
}

}  // namespace lynx
