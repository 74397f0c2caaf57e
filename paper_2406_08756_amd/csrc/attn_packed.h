// Building blocks of the attention kernels over packed sequences (attn_packed_fwd.hip, attn_packed_bwd.hip).
//
// A row is a (token, query head) pair.  The 2^pack query heads of a group that stand next to each other and read the same
// key head share a tile: row r of a sequence is token r >> pack, head r & (2^pack - 1), so that short sequences fill tiles
// and a tile of K and V serves them all.  A sequence of n tokens has n << pack rows and n keys; row r sees the keys up to
// its own token.
//
// All products are 32 x 32 blocks of the matrix instructions, D[m][n] += sum_k A[m][k] B[k][n].  Lane l holds A's row and
// B's column l % 32, and of D's column l % 32 the rows acc_row(i, l / 32).  Formed as D = S^T (keys down, rows across), a
// lane has the scores of one row: its maximum and sum are sums in a lane and one exchange with the other half.  The order
// in which k is dealt to lanes and registers is free as long as A and B agree, and it is chosen so that the registers of D
// are, rounded, the B operand of the next product, O^T += V^T P^T: no probability moves between lanes.
#pragma once
#include <atomic>

#include "kernels.h"
#include "mfma_common.h"

namespace lynx {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();
typedef float floatx4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ constexpr int acc_row(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }
// A value of this lane's and the one of the other half's lane, in the order of the halves.
__device__ __forceinline__ float2 of_both_halves(float v) {
  const uint32_t w = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const float2 b = of_both_halves(v);
  return b.x + b.y;
}
__device__ __forceinline__ float max_of_halves(float v) {
  const float2 b = of_both_halves(v);
  return fmaxf(b.x, b.y);
}
// What the compiler has derived from x is derived again.
__device__ __forceinline__ void forget(uint32_t& x) { asm volatile("" : "+v"(x)); }
// x is computed before this point, not where it is used.
template <typename X> __device__ __forceinline__ void stay(X& x) { asm volatile("" : "+v"(x)); }
// Likewise sums of matrix instructions, in the accumulation registers: they are not copied from there before this point.
__device__ __forceinline__ void stay_summed(floatx16_t& x) { asm volatile("" : "+a"(x)); }
// What stands above is issued before anything below.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < kInf; }

// A wavefront has 32 rows (or keys).  A workgroup has 128, whose wavefronts share the tiles that they go through; or, where
// there are too few of those to fill the card (SPLIT), 32, whose wavefronts deal the 32-key tiles among themselves, each on
// its own without a barrier, and join their parts at the end.
constexpr int rows_log(bool split) { return split ? 5 : 7; }
__device__ __forceinline__ void wave_fence() {  // the wavefront's LDS accesses stay in program order
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- which tile of which sequence ------------------------------------------
struct SeqTile {
  int start, len, tile;
};
__device__ __forceinline__ int2 sequence_span(const PackedAttn& g, int s) {
  // (whatever the offsets hold, no row outside the tensors is named)
  const int a = min(max(g.offsets[s], 0), g.tokens);
  return make_int2(a, min(max(g.offsets[s + 1], a), g.tokens) - a);
}
// Tile number `slot`; with LAST_FIRST counted from the last, so that the tiles at the end of a long sequence, whose rows see
// the most keys, start first (of key tiles, the first ones are seen by the most rows).
// Every wavefront looks for itself; each lane sums the tiles of its share of the sequences, a prefix sum finds the share,
// and the search goes on within it.  False if there are not that many tiles.
constexpr int kMostTiles = 1 << 29;
template <bool LAST_FIRST>
__device__ __forceinline__ bool find_tile(const PackedAttn& g, int slot, int tile_log, int pack, SeqTile* out) {
  const int lane = threadIdx.x & (kWave - 1);
  int first = 0, count = g.sequences, target = slot;
  bool top = true;
  while (true) {
    const int per = (count + kWave - 1) / kWave;
    int sum = 0;
    int2 span = make_int2(0, 0);
    for (int i = 0; i < per; ++i) {
      const int s = lane * per + i;
      if (s >= count) continue;
      span = sequence_span(g, first + s);
      // (the limit: offsets that fall name rows many times, and their sum must not pass 32 bits)
      sum = min(sum + (((span.y << pack) + (1 << tile_log) - 1) >> tile_log), kMostTiles);
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int v = __shfl_up(upto, o, kWave);
      if (lane >= o) upto = min(upto + v, kMostTiles);
    }
    if (top) {
      const int total = __builtin_amdgcn_readlane(upto, kWave - 1);
      if (slot >= total) return false;
      if (LAST_FIRST) target = total - 1 - slot;
      top = false;
    }
    const int at = __builtin_ctzll(__ballot(upto > target));
    target -= __builtin_amdgcn_readlane(upto - sum, at);
    if (per == 1) {
      out->start = __builtin_amdgcn_readlane(span.x, at);
      out->len = __builtin_amdgcn_readlane(span.y, at);
      out->tile = __builtin_amdgcn_readfirstlane(target);
      return true;
    }
    first += at * per;
    count = min(per, count - at * per);
  }
}

// The same, the tiles with the most to see first over all sequences: a tile's size is its number, counted from the end that
// sees least (rows: the start, keys: the end), and slot 0 is one of the largest.  The card waits for the last workgroup, and in
// the order of the sequences that may be a large one (four sequences of 2048 tokens: 1.4 times the work's share).  For up to
// 128 sequences; with more there are many tiles of every size and the plain order serves.
constexpr int kRankedSequences = 128;
__device__ __forceinline__ bool find_ranked_tile(const PackedAttn& g, int slot, int tile_log, int pack, SeqTile* out) {
  if (g.sequences > kRankedSequences) return find_tile<true>(g, slot, tile_log, pack, out);
  const int lane = threadIdx.x & (kWave - 1);
  int tiles[2];
  int2 span[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = k * kWave + lane;
    span[k] = s < g.sequences ? sequence_span(g, s) : make_int2(0, 0);
    tiles[k] = ((span[k].y << pack) + (1 << tile_log) - 1) >> tile_log;
  }
  // how many tiles have a number of `from` or more: falls with `from`; each lane counts for one number
  const auto count = [&](int from) {
    int sum = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      for (int i = 0; i < min(g.sequences - k * kWave, kWave); ++i) sum += max(__builtin_amdgcn_readlane(tiles[k], i) - from, 0);
    return sum;
  };
  // the largest number of which, with those above it, there are more than `slot`: in [lo, lo + range)
  int lo = 0, range = (g.tokens << pack >> tile_log) + 1, above = 0;
  while (true) {
    const int step = (range + kWave - 1) / kWave, from = lo + lane * step;
    const int n = count(from);
    const unsigned long long more = __ballot(n > slot);
    if (more == 0) return false;
    const int last = 63 - __builtin_clzll(more);
    if (step == 1) {
      above = last < kWave - 1 ? __builtin_amdgcn_readlane(n, last + 1) : __builtin_amdgcn_readfirstlane(count(lo + kWave));
      lo += last;
      break;
    }
    lo += last * step;
    range = step;
  }
  int rank = slot - above;  // among the sequences that have a tile of that number
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    unsigned long long has = __ballot(tiles[k] > lo);
    const int n = __builtin_popcountll(has);
    if (rank >= 0 && rank < n) {
      for (int i = 0; i < rank; ++i) has &= has - 1;
      const int at = __builtin_ctzll(has);
      out->start = __builtin_amdgcn_readlane(span[k].x, at);
      out->len = __builtin_amdgcn_readlane(span[k].y, at);
    }
    rank -= n;
  }
  out->tile = lo;
  return true;
}

// ---- operands ---------------------------------------------------------------
template <typename T> struct Operand;
template <> struct Operand<bf16_t> {
  typedef bf16x8_t Frag;
  static constexpr int kGroup = 16;  // rows of a column fragment pair
  __device__ static __forceinline__ void mma(floatx16_t& acc, Frag a, Frag b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
  }
  // registers kGroup / 2 c .. of an accumulator block as a B operand (one rounding to the storage type: the matrix
  // instructions take nothing wider, and the error averages out over the sum)
  __device__ static __forceinline__ Frag from_acc(const floatx16_t& v, int c) {
    uintx4_t w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_bf16(v[8 * c + 2 * j], v[8 * c + 2 * j + 1]);
    return __builtin_bit_cast(Frag, w);
  }
  __device__ static __forceinline__ Frag from_raw(uintx4_t w) { return __builtin_bit_cast(Frag, w); }
  __device__ static __forceinline__ float dot(Frag a, Frag b) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __builtin_fmaf(static_cast<float>(a[j]), static_cast<float>(b[j]), s);
    return s;
  }
};
template <> struct Operand<float> {
  typedef floatx4_t Frag;
  static constexpr int kGroup = 8;
  __device__ static __forceinline__ void mma(floatx16_t& acc, Frag a, Frag b) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
  }
  __device__ static __forceinline__ Frag from_acc(const floatx16_t& v, int c) {
    return Frag{v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]};
  }
  __device__ static __forceinline__ Frag from_raw(uintx4_t w) { return __builtin_bit_cast(Frag, w); }
  __device__ static __forceinline__ float dot(Frag a, Frag b) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_fmaf(a[j], b[j], s);
    return s;
  }
};

// acc += A B in an accumulation register.  A kernel of one wavefront per SIMD has 256 of them beside 256 ordinary ones, and
// sums that live through its branches were copied back and forth between the two kinds (272 moves per block of 32 rows)
// until their kind was named.  What the compiler does for its own instructions stands here: two wait states behind a vector
// instruction that wrote A or B, and settled() before the sums are read.
__device__ __forceinline__ void mma_aside(floatx16_t& acc, bf16x8_t a, bf16x8_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
#endif
}
__device__ __forceinline__ void mma_aside(floatx16_t& acc, floatx4_t a, floatx4_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int j = 0; j < 4; ++j) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x2_f32 %0, %1, %2, %0" : "+a"(acc) : "v"(a[j]), "v"(b[j]));
#endif
}
__device__ __forceinline__ void settled(floatx16_t& acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc));
#endif
}

// 16 bytes with every infinity and NaN replaced by zero.
__device__ __forceinline__ uintx4_t without_nonfinite(uintx4_t w, const bf16_t*) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if ((w[j] & 0x7F80u) == 0x7F80u) w[j] &= 0xFFFF0000u;
    if ((w[j] & 0x7F800000u) == 0x7F800000u) w[j] &= 0xFFFFu;
  }
  return w;
}
__device__ __forceinline__ uintx4_t without_nonfinite(uintx4_t w, const float*) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if ((w[j] & 0x7F800000u) == 0x7F800000u) w[j] = 0;
  return w;
}

// A tile in LDS: rows of DP elements, whose 16-byte chunks are permuted within the row so that both reads below meet all
// 64 banks: 16 lanes of a row fragment read one chunk of 16 consecutive rows, and a transposing read takes 32 bytes of
// each of four consecutive rows per 16 lanes (fp32: whole rows r and r + 4).
template <typename T, int DP> struct Tile {
  static constexpr int kChunk = 16 / static_cast<int>(sizeof(T));
  static constexpr int kChunks = DP / kChunk;
  static constexpr int kSteps = DP / (2 * kChunk);       // row fragments of a row
  static constexpr int kGroups = 32 / Operand<T>::kGroup;  // column fragments of 32 rows
  typedef typename Operand<T>::Frag Frag;

  __device__ static __forceinline__ int swizzle(int row) {
    if constexpr (sizeof(T) == 4) return (((row >> 2) & 1) << 3) | (((row >> 3) & 1) << 2) | (row & 3);
    else if constexpr (kChunks >= 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    else return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  }
  __device__ static __forceinline__ int at(int row, int chunk) { return row * DP + (chunk ^ swizzle(row)) * kChunk; }
  // Fragments are read at a lane's own offset (bytes, of the first fragment), whose swizzled bits the step, column block and
  // row group change by exclusive ors alone: one register serves all of them.  r0 is a multiple of 32.
  // Row r0 + lane % 32, elements 2 kChunk step + kChunk (lane / 32) ..:
  __device__ static __forceinline__ uint32_t row_base(int lane) { return at(lane & 31, lane >> 5) * static_cast<int>(sizeof(T)); }
  __device__ static __forceinline__ Frag row_frag(const T* tile, uint32_t base, int r0, int step) {
    return *reinterpret_cast<const Frag*>(bytes(tile, base ^ (step << 5)) + r0 * kRowBytes);
  }
  // Column 32 e + lane % 32 of the rows r0 + acc_row(.., lane / 32) that registers from_acc(.., c) hold.  bf16, 16 lanes: lane i
  // points at row i / 4, columns 4 (i % 4).., and receives column i of the four rows.
  __device__ static __forceinline__ uint32_t col_base(int lane) {
    const int b = lane >> 4, i = lane & 15;
    const int row = sizeof(T) == 4 ? 4 * (lane >> 5) : 4 * (b >> 1) + (i >> 2), col = sizeof(T) == 4 ? lane & 31 : 16 * (b & 1) + 4 * (i & 3);
    return (at(row, col / kChunk) + col % kChunk) * static_cast<int>(sizeof(T));
  }
  __device__ static __forceinline__ Frag col_frag(const T* tile, uint32_t base, int r0, int c, int e) {
    if constexpr (sizeof(T) == 4) {
      Frag f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = *reinterpret_cast<const float*>(bytes(tile, base ^ (e << 7) ^ ((c & 1) << 6) ^ (j << 4)) + (r0 + 8 * c + j) * kRowBytes);
      return f;
    } else {
      typedef __attribute__((address_space(3))) short4_t* lds_short4;
      const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)(bytes(tile, base ^ (e << 6)) + (r0 + 16 * c) * kRowBytes));
      const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)(bytes(tile, base ^ (e << 6) ^ 32) + (r0 + 16 * c + 8) * kRowBytes));
      const short8_t v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(Frag, v);
    }
  }

 private:
  static constexpr int kRowBytes = DP * static_cast<int>(sizeof(T));
  __device__ static __forceinline__ const unsigned char* bytes(const T* tile, uint32_t offset) {
    return reinterpret_cast<const unsigned char*>(tile) + offset;
  }
};

// Byte offset that every row buffer reads as zero.
constexpr uint32_t kOutside = 0x80000000u;

// One 16-byte load per lane straight into LDS, at the address `to` (uniform) + 16 lane; outside the buffer it stores zeros.
// Written out because the compiler takes every LDS read behind such a load, as a builtin, to wait for it: here a tile is read
// while the next one is on its way.  The load has no result register; landed() is the wait, and other wavefronts need a
// barrier after it.  (Loads that the compiler counts are only waited for the longer.  Nothing else in these kernels uses M0,
// which the load takes its place from.)
__device__ __forceinline__ void load_to_lds(const RowBuffer& b, uint32_t offset, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(b.rsrc) : "memory");
#endif
}
// ... of 4 bytes per lane, at `to` + 4 lane
__device__ __forceinline__ void load_word_to_lds(const RowBuffer& b, uint32_t offset, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(b.rsrc) : "memory");
#endif
}
// The address that the loads above take.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  typedef const __attribute__((address_space(3))) void* lds_ptr_t;
  return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_ptr_t)(p))));
}
// Waits until at most N of this wavefront's loads are in flight; with LDS, until its LDS accesses are done too.
template <int N>
__device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Tiles of 32 rows, one after another, by THREADS threads (`wave`: which wavefront of them).  What a tile's loads need is kept
// and moved along: 64-bit multiplications and divisions per tile were a third of a wavefront's instructions.
template <typename T, int DP, int THREADS> struct Stream {
  typedef Tile<T, DP> L;
  static constexpr int kLoads = 32 * L::kChunks / THREADS;
  static_assert(32 * L::kChunks % THREADS == 0 && THREADS % kWave == 0, "a tile splits over the wavefronts");
  const unsigned char* at;  // the next tile's first row
  long long left;           // bytes from there to the end of the last row
  uint32_t step;
  uint32_t offset[kLoads];  // this lane's
  // Rows are (token, head) pairs, 1 << pack heads of a token (keys: pack = 0); `base`: token 0 of `tokens`, `first`: the row that
  // the first tile starts at, a whole token's.  Zeros come behind the last token and behind column d.
  __device__ __forceinline__ Stream(const T* base, long long stride, int first, int tokens, int d, int pack, int wave, int lane) {
    const int heads = 1 << pack;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int e = wave * kWave + lane + THREADS * j, row = e / L::kChunks, col = (e % L::kChunks ^ L::swizzle(row)) * L::kChunk;
      const uint32_t off = (static_cast<uint32_t>(row >> pack) * static_cast<uint32_t>(stride) + (row & (heads - 1)) * d + col) * static_cast<uint32_t>(sizeof(T));
      offset[j] = col < d ? off : kOutside;
    }
    step = static_cast<uint32_t>(32 >> pack) * static_cast<uint32_t>(stride) * static_cast<uint32_t>(sizeof(T));
    start(base, stride, first, tokens, d, pack);
  }
  __device__ __forceinline__ void start(const T* base, long long stride, int first, int tokens, int d, int pack) {
    at = reinterpret_cast<const unsigned char*>(base + (first >> pack) * stride);
    left = ((tokens - 1 - (first >> pack)) * stride + (d << pack)) * static_cast<long long>(sizeof(T));
  }
  // the next tile to `tile` (uniform), and on by `tiles`
  __device__ __forceinline__ void load(uint32_t tile, int wave, int tiles = 1) {
    const RowBuffer b = row_buffer(at, left <= 0 ? 0u : left < static_cast<long long>(kOutside) ? static_cast<uint32_t>(left) : kOutside);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load_to_lds(b, offset[j], tile + (wave * kWave + THREADS * j) * 16);
    at += static_cast<unsigned long long>(step) * tiles;
    left -= static_cast<long long>(step) * tiles;
  }
  // what this lane has loaded, without infinities and NaN
  __device__ static __forceinline__ void clean(T* tile, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      uintx4_t* const p = reinterpret_cast<uintx4_t*>(tile + (wave * kWave + lane + THREADS * j) * L::kChunk);
      *p = without_nonfinite(*p, static_cast<const T*>(nullptr));
    }
  }
};

// A wavefront's 32 rows as row fragments in registers, straight from memory.
template <typename T, int DP>
__device__ __forceinline__ void load_row_frags(const RowBuffer& b, uint32_t row_offset, int d, int lane, typename Operand<T>::Frag (&f)[Tile<T, DP>::kSteps]) {
  typedef Tile<T, DP> L;
#pragma unroll
  for (int s = 0; s < L::kSteps; ++s) {
    const int col = (2 * s + (lane >> 5)) * L::kChunk;
    f[s] = Operand<T>::from_raw(row_buffer_load(b, col < d ? row_offset + col * static_cast<uint32_t>(sizeof(T)) : kOutside));
  }
}

__device__ __forceinline__ void store4(bf16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }

// ---- position bias -----------------------------------------------------------
// Bias by distance, times log2 e: `far` distances, and kPad more on both sides so that the reads of a 32-row strip against
// 64 keys that holds one near or masked pair need no limits.
constexpr int kPad = 96;
__host__ __device__ __forceinline__ int table_stride(const PackedAttn& g) { return (g.far + 2 * kPad + 3) & ~3; }  // (what follows is read 16 bytes at a time)
__host__ __device__ __forceinline__ int table_floats(const PackedAttn& g) { return table_stride(g) << g.pack; }
__device__ __forceinline__ int bucket_of(const PackedAttn& g, int distance) {
  // (all kMaxBuckets starts, those behind the last bucket at the largest number: a loop to the last would wait for each)
  int b = 0;
#pragma unroll
  for (int i = 1; i < kMaxBuckets; ++i) b += distance >= g.starts[i] ? 1 : 0;
  return b;
}
template <typename T, int THREADS>
__device__ __forceinline__ void fill_bias(const PackedAttn& g, int head0, float* by_distance) {
  const int n = table_stride(g);
  for (int x = threadIdx.x; x < n; x += THREADS) {
    const int distance = x - kPad, b = bucket_of(g, distance);
    for (int h = 0; h < (1 << g.pack); ++h)
      by_distance[h * n + x] = load1(static_cast<const T*>(g.table) + static_cast<long long>(b) * g.heads + head0 + h) * kLog2e;
  }
}

constexpr int kMostLds = 159 << 10;  // (the barrier that joins a truth value has 1 KB of its own)
template <auto KERNEL>
hipError_t launch_packed(size_t groups, size_t lds, const PackedAttn& g, hipStream_t st) {
  static std::atomic<uint64_t> allowed{0};  // a bit per device (the first 64; for others every time)
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? uint64_t{1} << device : 0;
  if ((allowed.load(std::memory_order_relaxed) & bit) == 0) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, kMostLds);
    if (e != hipSuccess) return e;
    allowed.fetch_or(bit, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL(KERNEL, dim3(static_cast<unsigned>(groups)), dim3(kThreads), lds, st, g);
  return hipGetLastError();
}

// ---- joining the parts of a SPLIT workgroup's wavefronts ----------------------
// A part: [DP columns][32 rows] floats, as the accumulator blocks hold them; it takes the wavefront's two tiles' place.
template <int DP>
__device__ __forceinline__ void write_part(float* part, const floatx16_t (&acc)[DP / 32], float factor, int lane) {
#pragma unroll
  for (int b = 0; b < DP / 32; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) part[(32 * b + acc_row(i, lane >> 5)) * 32 + (lane & 31)] = acc[b][i] * factor;
}
// The sum of the parts, in the order of the wavefronts: DP / 8 columns from join_column of row lane % 32.
template <int DP> __device__ __forceinline__ int join_column(int wave, int lane) { return wave * (DP / 4) + (lane >> 5) * (DP / 8); }
template <int DP>
__device__ __forceinline__ void join_parts(const float* parts, size_t part_floats, int wave, int lane, float (&sum)[DP / 8]) {
  const int at = join_column<DP>(wave, lane) * 32 + (lane & 31);
#pragma unroll
  for (int c = 0; c < DP / 8; ++c) {
    sum[c] = parts[at + 32 * c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum[c] += parts[w * part_floats + at + 32 * c];
  }
}
template <typename T, int DP>
__device__ __forceinline__ void store_joined(T* row, int column, int d, const float (&sum)[DP / 8], float factor) {
#pragma unroll
  for (int c = 0; c < DP / 8; c += 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = sum[c + j] * factor;
    if (column + c < d) store8(row + column + c, v);
  }
}

// Every wavefront's bits together, dealt out again: this one has those whose number is its own modulo the wavefronts.
__device__ __forceinline__ uint32_t share_rows(uint32_t rows, uint32_t* all, int wave) {
  __syncthreads();
  all[wave] = rows;
  __syncthreads();
  uint32_t any = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) any |= all[w];
  return any & (0x11111111u << wave);
}

// ---- rows and keys that meet infinities or NaN ---------------------------------
// A masked pair has probability 0, but 0 times infinity is NaN, and a matrix instruction multiplies every pair of its block.
// Results that come out infinite or NaN are therefore looked at again: the tile is done once more with such elements as
// zeros, which gives the rows that see none of them the bits that they have without them, and each row that does see some
// is summed pair by pair, over the pairs it sees.  Nothing of this runs where all results are finite.
template <typename T>
__device__ __forceinline__ float row_dot(const T* x, const T* y, int d) {
  float s = 0.f;
  for (int c = 0; c < d; c += 8) {
    float a[8], b[8];
    load8(x + c, a);
    load8(y + c, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __builtin_fmaf(a[j], b[j], s);
  }
  return s;
}
template <typename T>
__device__ __forceinline__ bool row_finite(const T* x, int d) {
  bool ok = true;
  for (int c = 0; c < d; c += 8) {
    float a[8];
    load8(x + c, a);
#pragma unroll
    for (int j = 0; j < 8; ++j) ok = ok && finite(a[j]);
  }
  return ok;
}

}  // namespace
}  // namespace lynx
