// The weight gradient of a linear layer from its input's 8-bit checkpoint:
//   dw[o][i] (+)= sum over tokens t of dy[t][o] x[t][i],   db[o] (+)= sum over t of dy[t][o].
//
// A matrix product on the matrix cores with the sum along both operands' slow axis.  A checkpoint's values are bf16 numbers (4
// significant bits, a normal exponent), so they go to the matrix cores as they are; so does a bf16 dy; a binary32 dy is cut into
// three bf16 numbers whose sum it is (8 of its 24 significant bits each, cut off, not rounded: no part overflows), and there are
// three products.  Sums are binary32, in the matrix cores' accumulators.
//
// The operands lie in LDS as in memory, tokens by rows, and go to the matrix cores through transposing reads (ds_read_b64_tr_b16):
// a group of 16 lanes reads 4 tokens by 16 columns, and each lane gets one column's 4 tokens.  Which 8 of a product's 16 tokens a lane
// holds is the same for both operands, so their order does not matter.  A row of LDS is 64 bytes more than a multiple of 256: the
// four rows of a read then start a quarter of the banks apart.
#include "act_rows.h"

namespace dq {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct WGrad {
  Rows dy;
  CkptIn x;
  uint64_t rows, outs, cols, pitch;
  void *dw, *db;
  uint64_t ld;
  float *part;                // [splits][tiles][a tile's sums in the accumulators' order], then [splits][outs]: null without a split
  uint64_t tiles;
  uint32_t tiles_out, tiles_in, splits, accumulate;
  uint64_t split_rows;        // tokens of a split, a multiple of the step
};

constexpr uint32_t kJoinThreads = 256;

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) a32x4 lds_a32x4;
typedef __attribute__((address_space(3))) float lds_float;

// A lane's part of the address of 16 tokens of 32 columns.
__device__ __forceinline__ uint32_t read_at(uint32_t stride) {
  const uint32_t l = threadIdx.x & 63u;
  return ((l >> 5) * 8 + (l & 15u) / 4) * stride + ((l >> 4) & 1u) * 32 + (l & 3u) * 8;
}
__device__ __forceinline__ bf16x8 read16(uint32_t at, uint32_t stride) {
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>(at));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>(at + 4 * stride));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// Waits for this wave's LDS accesses only, then for the block's other waves: loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <typename O>
__device__ __forceinline__ void put(void *out, uint64_t at, float v, uint32_t accumulate) {
  if constexpr (__is_same(O, F32)) {
    float *p = static_cast<float *>(out) + at;
    a_st<float>(p, accumulate ? a_ld<float>(p) + v : v);
  } else {
    uint16_t *p = static_cast<uint16_t *>(out) + at;
    if (accumulate) v += a_float((uint32_t)a_ld<uint16_t>(p) << 16);
    a_st<uint16_t>(p, (uint16_t)to_bf16x2(v, v));
  }
}
// 16 bytes of sums, at `row` from column i on; cols: the row's length.
template <typename O>
constexpr uint32_t kPut = 16 / kEntry<O>;
template <typename O>
__device__ __forceinline__ void put16(void *row, uint64_t i, uint64_t cols, uint32_t accumulate, float (&v)[kPut<O>]) {
  if (accumulate) {
    float old[kPut<O>];
    load_entries<O, kPut<O>>(row, i, cols, old);
#pragma unroll
    for (uint32_t k = 0; k < kPut<O>; ++k) v[k] += old[k];
  }
  store_entries<O, kPut<O>>(row, i, cols, v);
}

// A block's tile: kOut x kIn sums, kTok tokens a step; its waves, 2 by WAVES_IN, have kWaveOut x kWaveIn each.
template <typename T, uint32_t OUT, uint32_t IN, uint32_t TOK, uint32_t WAVES_IN>
struct Tile {
  static constexpr uint32_t kOut = OUT, kIn = IN, kTok = TOK;
  static constexpr uint32_t kThreads = 128 * WAVES_IN, kWaveOut = OUT / 2, kWaveIn = IN / WAVES_IN;
  static constexpr uint32_t kPlanes = __is_same(T, F32) ? 3 : 1;
  static constexpr uint32_t kOutStride = OUT * 2 + 64, kInStride = IN * 2 + 64;        // bytes of an LDS row
  static constexpr uint32_t kX = kPlanes * TOK * kOutStride;                           // where x's rows begin
  static constexpr uint32_t kBuffer = kX + TOK * kInStride;
  static constexpr uint32_t kOutLanes = OUT / 8, kOutRows = kThreads / kOutLanes, kOutLoads = TOK / kOutRows;   // 8 entries of dy a lane
  static constexpr uint32_t kCodes = TOK * IN >= 16 * kThreads ? 16 : 8;                                        // a lane's, of a row
  static constexpr uint32_t kInLanes = IN / kCodes, kInRows = kThreads / kInLanes, kInLoads = TOK / kInRows;
  static constexpr uint32_t kPieces = kOutLoads + kInLoads, kSlices = TOK / 16 * kPlanes;
  static constexpr uint32_t kM = kWaveOut / 32, kN = kWaveIn / 32;                               // products of 32 x 32 of a wave
  static_assert(kOutStride % 256 % 128 == 64 && kInStride % 256 % 128 == 64 && kOutRows * kOutLoads == TOK && kInRows * kInLoads == TOK && kSlices % 2 == 0 && TOK / 16 % 2 == 0, "");
};

// Tiles are numbered in strips of up to 8 along x, row by row of a strip: neighbours in number share columns of dy or of x.
__device__ __forceinline__ uint64_t tile_strip(const WGrad &g, uint64_t tile) { return tile / (8 * (uint64_t)g.tiles_out) * 8; }
__device__ __forceinline__ uint64_t strip_width(const WGrad &g, uint64_t strip) { return g.tiles_in - strip < 8 ? g.tiles_in - strip : 8; }
__device__ __forceinline__ uint64_t tile_out(const WGrad &g, uint64_t tile) {
  const uint64_t s = tile_strip(g, tile);
  return (tile - s * g.tiles_out) / strip_width(g, s);
}
__device__ __forceinline__ uint64_t tile_in(const WGrad &g, uint64_t tile) {
  const uint64_t s = tile_strip(g, tile);
  return s + (tile - s * g.tiles_out) % strip_width(g, s);
}
// Which of a tile's columns of dy, of which `outs` exist, its column c holds (see begin()); outs or more: none, or one that another
// column holds too.
template <bool SMALL>
__device__ __forceinline__ uint32_t column(uint32_t outs, uint32_t c) {
  const uint32_t chunk = c & ~7u;
  if (SMALL || chunk >= outs || chunk + 8 <= outs) return c;
  const uint32_t shift = chunk + 8 - outs;
  return (c & 7u) < shift ? outs : c - shift;
}
template <typename S>
__device__ __forceinline__ uint32_t tile_outs(const WGrad &g, uint64_t o0) { return g.outs - o0 < S::kOut ? (uint32_t)(g.outs - o0) : S::kOut; }
// What a lane has on its way from memory: its part of a step.
template <typename T, typename S>
struct Stage {
  a32x4 dy[S::kOutLoads * (__is_same(T, F32) ? 2 : 1)], x[S::kInLoads];  // (8 codes: the first half)
  uint32_t scale[S::kInLoads];
};

// A block's walk over the tokens, one tile at a time.  Steps go through two buffers in LDS: while the matrix cores read one, the next
// step's operands go to the other, from registers.  SMALL: fewer than 8 outs, loaded entry by entry.
//
// Tiles of 256 x 256 by 8 waves: bf16 16384 x 8192 x 2048 in 434 to 486 us by the card (1.13 to 1.27 PFLOP/s; the library's best large
// product, 1.34), the matrix cores busy 68 % of the cycles at a clock of 1.74 GHz: power bounds it.  Four waves of 128 x 128 took 514
// us; x written to LDS without bank conflicts, by lanes that swap their halves, 4 % more (the selections cost more than the conflicts);
// waves of raised priority around the products 3 % more.  fp32 4096 x 8192 x 8192: 1,220 us, three products each (1.35 PFLOP/s).
template <typename T, typename O, typename S, bool SMALL>
struct Walker {
  const WGrad &g;
  const uint32_t base, wave, out_row, out_col, in_row, in_col;
  uint64_t o0, i0, first, end;
  const uint8_t *dy, *codes, *scales;  // this lane's first row of the step that is loaded next
  uint64_t dy_row;                     // bytes from a row to the next
  uint32_t put_dy, put_x, get_dy, get_x;  // LDS addresses in the first buffer
  bool bias;
  Stage<T, S> st;
  float sums[8];
  bf16x8 a[2][S::kM], b[2][S::kN];
  f32x16 acc[S::kM][S::kN];

  __device__ __forceinline__ Walker(const WGrad &g_, uint32_t lds)
      : g(g_), base(lds), wave(threadIdx.x >> 6), out_row(threadIdx.x / S::kOutLanes), out_col(threadIdx.x % S::kOutLanes * 8),
        in_row(threadIdx.x / S::kInLanes), in_col(threadIdx.x % S::kInLanes * S::kCodes) {
    put_dy = base + out_row * S::kOutStride + out_col * 2;
    put_x = base + S::kX + in_row * S::kInStride + in_col * 2;
    get_dy = base + (wave & 1u) * (S::kWaveOut * 2) + read_at(S::kOutStride);
    get_x = base + S::kX + (wave >> 1) * (S::kWaveIn * 2) + read_at(S::kInStride);
    // kept as they are: what is added to them below fits the instructions' offsets
    asm volatile("" : "+v"(put_dy), "+v"(put_x), "+v"(get_dy), "+v"(get_x));
  }

  __device__ __forceinline__ void begin(uint64_t tile, uint64_t from, uint64_t to) {
    o0 = tile_out(g, tile) * S::kOut;
    i0 = tile_in(g, tile) * S::kIn;
    first = from;
    end = to;
    bias = g.db && i0 == 0;
    // A lane's 8 entries of dy that would pass the row's end are taken up to it: they hold earlier columns then (see column()).
    // Columns beyond the matrices are read as their first ones and not stored.
    const uint64_t o = o0 + out_col;
    const uint64_t from_o = SMALL ? 0 : o >= g.outs ? 0 : o + 8 > g.outs ? g.outs - 8 : o, from_i = i0 + in_col < g.pitch ? i0 + in_col : 0;
    dy_row = g.dy.ld * kEntry<T>;
    dy = static_cast<const uint8_t *>(g.dy.data) + (first + out_row) * dy_row + from_o * kEntry<T>;
    codes = g.x.codes + (first + in_row) * g.pitch + from_i;
    scales = g.x.scales + ((first + in_row) * g.pitch + from_i) / kCkptBlock;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[i] = 0.0f;
#pragma unroll
    for (uint32_t m = 0; m < S::kM; ++m)
#pragma unroll
      for (uint32_t n = 0; n < S::kN; ++n) acc[m][n] = f32x16{};
  }

  // A lane's share of a step is kPieces loads: first of dy, then of the checkpoint.
  // LAST: the step may end behind the last token; tokens there are read as the last one.
  template <bool LAST>
  __device__ __forceinline__ void load(uint32_t step, uint32_t piece) {
    if (piece < S::kOutLoads) {
      const uint32_t j = piece;
      uint64_t ahead = j * S::kOutRows;
      const uint64_t t = first + (uint64_t)step * S::kTok + out_row;
      if (LAST && t + ahead >= end) ahead = end - 1 - t;  // (modulo 2^64)
      const uint8_t *p = dy + ahead * dy_row;
      if constexpr (SMALL) {
        float v[8];
        load8<T>(p, o0 + out_col, g.outs, v);
        if constexpr (__is_same(T, F32)) {
          st.dy[2 * j] = a32x4{a_bits(v[0]), a_bits(v[1]), a_bits(v[2]), a_bits(v[3])};
          st.dy[2 * j + 1] = a32x4{a_bits(v[4]), a_bits(v[5]), a_bits(v[6]), a_bits(v[7])};
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) st.dy[j][i] = high_halves(a_bits(v[2 * i]), a_bits(v[2 * i + 1]));
        }
      } else if constexpr (__is_same(T, F32)) {
        st.dy[2 * j] = a_ld<a32x4_any>(p);
        st.dy[2 * j + 1] = a_ld<a32x4_any>(p + 16);
      } else {
        st.dy[j] = a_ld<a32x4_any>(p);
      }
    } else {
      const uint32_t j = piece - S::kOutLoads;
      uint64_t ahead = j * S::kInRows;
      const uint64_t t = first + (uint64_t)step * S::kTok + in_row;
      if (LAST && t + ahead >= end) ahead = end - 1 - t;
      if constexpr (S::kCodes == 16) {
        st.x[j] = a_ld<a32x4>(codes + ahead * g.pitch);
      } else {
        const a32x2 c = a_ld<a32x2>(codes + ahead * g.pitch);
        st.x[j] = a32x4{c.x, c.y, 0u, 0u};
      }
      st.scale[j] = a_ld<uint8_t>(scales + ahead * (g.pitch / kCkptBlock));
    }
  }
  __device__ __forceinline__ void loaded() {
    dy += S::kTok * dy_row;
    codes += S::kTok * g.pitch;
    scales += S::kTok * (g.pitch / kCkptBlock);
  }
  // To LDS.  LAST: the last step's tokens behind the end count nothing.
  template <bool BIAS, bool LAST>
  __device__ __forceinline__ void store(uint32_t step, uint32_t piece) {
    const uint32_t buffer = (step & 1u) * S::kBuffer;
    if (piece < S::kOutLoads) {
      const uint32_t j = piece, at = put_dy + buffer + j * S::kOutRows * S::kOutStride;
      constexpr uint32_t n = __is_same(T, F32) ? 2 : 1;
      if (LAST) {
        const bool none = first + (uint64_t)step * S::kTok + j * S::kOutRows + out_row >= end;
#pragma unroll
        for (uint32_t h = 0; h < n; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) st.dy[n * j + h][i] = none ? 0u : st.dy[n * j + h][i];
      }
      if constexpr (__is_same(T, F32)) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a_float(st.dy[2 * j][i]); v[4 + i] = a_float(st.dy[2 * j + 1][i]); }
        if constexpr (BIAS) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sums[i] += v[i];
        }
#pragma unroll
        for (uint32_t p = 0; p < S::kPlanes; ++p) {
          a32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = high_halves(a_bits(v[2 * i]), a_bits(v[2 * i + 1]));
          *reinterpret_cast<lds_a32x4 *>(at + p * S::kTok * S::kOutStride) = w;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] -= a_float(a_bits(v[i]) & 0xFFFF0000u);
        }
      } else {
        *reinterpret_cast<lds_a32x4 *>(at) = st.dy[j];
        if constexpr (BIAS) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sums[2 * i] += a_float(st.dy[j][i] << 16);
            sums[2 * i + 1] += a_float(st.dy[j][i] & 0xFFFF0000u);
          }
        }
      }
    } else {
      const uint32_t j = piece - S::kOutLoads, at = put_x + buffer + j * S::kInRows * S::kInStride;
      const float X = a_float(st.scale[j] << 23);
      a32x4 w[2];
#pragma unroll
      for (int i = 0; i < (int)S::kCodes / 4; ++i) {
        w[i / 2][i % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(st.x[j][i], X, false));
        w[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(st.x[j][i], X, true));
      }
      *reinterpret_cast<lds_a32x4 *>(at) = w[0];
      if constexpr (S::kCodes == 16) *reinterpret_cast<lds_a32x4 *>(at + 16) = w[1];
    }
  }
  // A step is kSlices rounds of kM x kN products: 16 tokens, and of a binary32 dy one of its three parts.
  __device__ __forceinline__ void read(uint32_t step, uint32_t slice) {
    const uint32_t buffer = (step & 1u) * S::kBuffer, k = slice / S::kPlanes * 16, p = slice % S::kPlanes;
    if (p == 0) {
#pragma unroll
      for (uint32_t n = 0; n < S::kN; ++n) b[slice / S::kPlanes % 2][n] = read16(get_x + buffer + k * S::kInStride + n * 64, S::kInStride);
    }
#pragma unroll
    for (uint32_t m = 0; m < S::kM; ++m) a[slice % 2][m] = read16(get_dy + buffer + (p * S::kTok + k) * S::kOutStride + m * 64, S::kOutStride);
  }
  __device__ __forceinline__ void multiply(uint32_t slice) {
#pragma unroll
    for (uint32_t m = 0; m < S::kM; ++m)
#pragma unroll
      for (uint32_t n = 0; n < S::kN; ++n)
        acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[slice % 2][m], b[slice / S::kPlanes % 2][n], acc[m][n], 0, 0, 0);
  }
  // One step.  Its first slice's operands are in registers already; each slice reads the next one's while the matrix cores work, and
  // moves its share of the next step's pieces to LDS, each followed by its load for the step after that, which has a whole step to
  // arrive.  The barrier stands in front of the last slice: by then this step has been read and the next one written, and the next
  // step's first operands are read behind it, in the last slice's time.
  // STEADY: neither of the two steps that follow is the last.
  template <bool BIAS, bool STEADY>
  __device__ __forceinline__ void advance(uint32_t step, uint32_t last) {
#pragma unroll
    for (uint32_t s = 0; s < S::kSlices; ++s) {
      if (s + 1 < S::kSlices) {
        read(step, s + 1);
      } else {
        lds_barrier();
        if (STEADY || step < last) read(step + 1, 0);
      }
      multiply(s);
      const uint32_t from = s * S::kPieces / (S::kSlices - 1), to = s + 1 < S::kSlices ? (s + 1) * S::kPieces / (S::kSlices - 1) : from;
#pragma unroll
      for (uint32_t i = from; i < to; ++i) {
        if constexpr (STEADY) {
          store<BIAS, false>(step + 1, i);
          load<false>(step + 2, i);
        } else {
          if (step + 1 <= last) store<BIAS, true>(step + 1, i);
          if (step + 2 <= last) load<true>(step + 2, i);
        }
      }
      if (s + 2 == S::kSlices) loaded();
      if constexpr (STEADY) mix();
    }
  }
  // A slice's instructions in turn: the matrix cores are given the next product before the rest.
  __device__ __forceinline__ void mix() {
#pragma unroll
    for (uint32_t i = 0; i < S::kM * S::kN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);  // vector arithmetic
      __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);  // LDS writes
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // loads
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  template <bool BIAS>
  __device__ __forceinline__ void walk() {
    const uint32_t steps = end > first ? (uint32_t)((end - first + S::kTok - 1) / S::kTok) : 0u;
    if (steps == 0) return;
    const uint32_t last = steps - 1;
#pragma unroll
    for (uint32_t i = 0; i < S::kPieces; ++i) load<true>(0, i);
    loaded();
#pragma unroll
    for (uint32_t i = 0; i < S::kPieces; ++i) store<BIAS, true>(0, i);
    if (last > 0) {
#pragma unroll
      for (uint32_t i = 0; i < S::kPieces; ++i) load<true>(1, i);
    }
    loaded();
    lds_barrier();
    read(0, 0);
    uint32_t step = 0;
    for (; step + 2 < last; ++step) advance<BIAS, true>(step, last);
    for (; step <= last; ++step) advance<BIAS, false>(step, last);
  }
  // A product's 32 x 32 sums go through a patch of LDS of the wave's own, so that the lanes of a row have 16 bytes each, side by side
  // (with half a row to a lane, stores covered lines in parts: one token, 8192 x 8192, fp32 54 us and 91, bf16 40 and 44).
  __device__ __forceinline__ void put_tile() {
    constexpr uint32_t kRow = 144, kLanes = 32 / kPut<O>, kRows = 64 / kLanes;  // lanes to a row, rows at once
    uint32_t l = threadIdx.x & 63u;
    asm volatile("" : "+v"(l));  // what follows from it is worked out here, not kept in registers through the steps
    const uint32_t patch = base + wave * (32 * kRow), to = patch + 4 * (l >> 5) * kRow + (l & 31u) * 4, from = patch + l / kLanes * kRow + l % kLanes * (kPut<O> * 4);
    const uint32_t c = (wave & 1u) * S::kWaveOut + l / kLanes, outs = tile_outs<S>(g, o0);
    const uint64_t i = i0 + (wave >> 1) * S::kWaveIn + l % kLanes * kPut<O>, row_bytes = g.ld * kEntry<O>;
    uint8_t *const dw = static_cast<uint8_t *>(g.dw) + o0 * row_bytes;
#pragma unroll
    for (uint32_t m = 0; m < S::kM; ++m)
#pragma unroll
      for (uint32_t n = 0; n < S::kN; ++n) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) *reinterpret_cast<lds_float *>(to + (8 * (r / 4) + r % 4) * kRow) = acc[m][n][r];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        float v[32 / kRows][kPut<O>];
#pragma unroll
        for (uint32_t h = 0; h < 32 / kRows; ++h)
#pragma unroll
          for (uint32_t q = 0; q < kPut<O> / 4; ++q) {
            const a32x4 w = *reinterpret_cast<lds_a32x4 *>(from + h * kRows * kRow + q * 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h][q * 4 + k] = a_float(w[k]);
          }
        __builtin_amdgcn_wave_barrier();
        if (i + n * 32 < g.cols) {
          uint32_t first_row = c + m * 32;
          asm volatile("" : "+v"(first_row));  // (nor these rows' addresses for all products)
#pragma unroll
          for (uint32_t h = 0; h < 32 / kRows; ++h) {
            const uint32_t o = column<SMALL>(outs, first_row + h * kRows);
            if (o < outs) put16<O>(dw + o * row_bytes, i + n * 32, g.cols, g.accumulate, v[h]);
          }
        }
      }
  }
  __device__ __forceinline__ void put_part(uint64_t unit) {
    const uint64_t o = o0 + (wave & 1u) * S::kWaveOut, i = i0 + (wave >> 1) * S::kWaveIn;
    float *p = g.part + (unit * (S::kThreads / 64) + wave) * (uint64_t)(S::kM * S::kN * 1024) + (threadIdx.x & 63u) * 4;
#pragma unroll
    for (uint32_t m = 0; m < S::kM; ++m)
#pragma unroll
      for (uint32_t n = 0; n < S::kN; ++n) {
        if (o + m * 32 >= g.outs || i + n * 32 >= g.cols) continue;  // nobody reads them
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
          a_st<af32x4>(p + ((m * S::kN + n) * 4 + q) * 256, af32x4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]});
      }
  }
  // The lanes of a column, through LDS.
  __device__ __forceinline__ void put_bias(uint64_t units, uint32_t split) {
    const uint32_t to = base + (out_row * S::kOut + out_col) * 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<lds_float *>(to + 4 * i) = sums[i];
    lds_barrier();
    const uint32_t outs = tile_outs<S>(g, o0);
    for (uint32_t c = threadIdx.x; c < S::kOut; c += S::kThreads) {
      float v = 0.0f;
      for (uint32_t r = 0; r < S::kOutRows; ++r) v += *reinterpret_cast<lds_float *>(base + (r * S::kOut + c) * 4);
      const uint32_t o = column<SMALL>(outs, c);
      if (o >= outs) continue;
      if (g.splits > 1) a_st<float>(g.part + units * (S::kOut * S::kIn) + split * g.outs + o0 + o, v);
      else put<O>(g.db, o0 + o, v, g.accumulate);
    }
  }
};

template <typename T, typename O, typename S, bool SMALL>
__global__ __launch_bounds__(S::kThreads, S::kOut > 64 ? 2 : 3) void k_wgrad(WGrad g) {  // waves to a SIMD, as many as LDS lets in
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * S::kBuffer];
  Walker<T, O, S, SMALL> w(g, (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds);
  const uint64_t units = g.tiles * g.splits;
  for (uint64_t turn = blockIdx.x; turn < units; turn += gridDim.x) {
    // blocks go to the 8 XCDs in turn: each gets units that follow each other, whose operands its L2 then holds
    const uint64_t xcd = turn % 8, each = units / 8, over = units % 8, unit = xcd * each + (xcd < over ? xcd : over) + turn / 8;
    const uint32_t split = (uint32_t)(unit / g.tiles);
    const uint64_t first = split * g.split_rows;
    w.begin(unit % g.tiles, first, first + g.split_rows < g.rows ? first + g.split_rows : g.rows);
    if (w.bias) w.template walk<true>();
    else w.template walk<false>();
    lds_barrier();
    if (g.splits > 1) w.put_part(unit);
    else w.put_tile();
    if (w.bias) {
      lds_barrier();
      w.put_bias(units, split);
    }
    lds_barrier();  // the next tile's steps go where this one's sums went
  }
}

// The splits' sums.  A thread has four of a tile, as a lane of the kernel above had them; where splits are many, WAYS threads share them,
// each every WAYS-th, and their sums are added in order.
template <typename O, typename S, bool SMALL, uint32_t WAYS>
__global__ __launch_bounds__(kJoinThreads) void k_wgrad_join(WGrad g) {
  constexpr uint64_t kQuads = S::kOut * S::kIn / 4;
  constexpr uint32_t kEach = kJoinThreads / WAYS;
  __shared__ af32x4 lds[WAYS > 1 ? kJoinThreads : 1];
  const uint32_t way = threadIdx.x / kEach;
  const uint64_t quads = g.tiles * kQuads, all = quads + (g.db ? g.outs : 0);
  for (uint64_t first = (uint64_t)blockIdx.x * kEach; first < all; first += (uint64_t)gridDim.x * kEach) {
    const uint64_t i = first + threadIdx.x % kEach;
    af32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    uint64_t o0 = 0, at = 0;
    uint32_t row = 0;
    bool here = i < all;
    if (i < quads) {
      const uint64_t tile = i / kQuads;
      const uint32_t k = (uint32_t)(i % kQuads), l = k & 63u, q = (k >> 6) & 3u, mn = (k >> 8) % (S::kM * S::kN), wave = (k >> 8) / (S::kM * S::kN);
      const uint32_t patch = (wave & 1u) * S::kWaveOut + mn / S::kN * 32;
      o0 = tile_out(g, tile) * S::kOut;
      row = patch + 8 * q + 4 * (l >> 5);
      at = tile_in(g, tile) * S::kIn + (wave >> 1) * S::kWaveIn + mn % S::kN * 32 + (l & 31u);
      here = o0 + patch < g.outs && at < g.cols;
      if (here) {
#pragma unroll 4
        for (uint32_t s = way; s < g.splits; s += WAYS) v += a_ld<af32x4>(g.part + (s * quads + i) * 4);
      }
    } else if (here) {
      const float *p = g.part + g.splits * quads * 4 + (i - quads);
#pragma unroll 4
      for (uint32_t s = way; s < g.splits; s += WAYS) v[0] += a_ld<float>(p + s * g.outs);
    }
    if constexpr (WAYS > 1) {
      __syncthreads();  // the last sums have been read
      lds[threadIdx.x] = v;
      __syncthreads();
      if (way) continue;
#pragma unroll
      for (uint32_t w = 1; w < WAYS; ++w) v += lds[w * kEach + threadIdx.x];
    }
    if (!here) continue;
    if (i < quads) {
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) {
        const uint32_t outs = tile_outs<S>(g, o0), o = column<SMALL>(outs, row + r);
        if (o < outs) put<O>(g.dw, (o0 + o) * g.ld + at, v[r], g.accumulate);
      }
    } else {
      put<O>(g.db, i - quads, v[0], g.accumulate);
    }
  }
}

// How a product is cut: the tile, and the tokens into splits.
struct Cut {
  uint32_t size;     // 0: 64 x 64, 1: 128 x 128, 2: 256 x 256
  uint32_t splits;
  uint64_t tiles_out, tiles_in, split_rows;
};
constexpr uint32_t kEdges[3] = {64, 128, 256}, kToks[2][3] = {{32, 32, 32}, {64, 64, 64}};  // [bf16][size]
constexpr uint32_t kManySplits = 16;  // of which several threads join one sum (30000 x 64 x 64, a hundred splits: 10 us; 40 by one thread a sum)

// The cut that costs least, by what was measured (MI355X, microseconds): a step of a block alone on its CU and of one among as many as
// fit, the launch, the tiles' way to memory, and what splits add, a launch and their sums' way to memory and back at 5 TB/s.  Large tiles
// read and move least for what they multiply; small ones and splits give every CU a part where sums are few.  Over 16 sizes in each type
// the choice is within 10 % of the best tile and split, but for fp32 65537 x 200 x 136 (34 to 39 us, 33 with 128 x 128).  256 CUs whatever the
// device has: the order of sums and the scratch memory follow from sizes and types alone.
Cut cut_of(dq_dtype dtype, uint64_t rows, uint64_t outs, uint64_t cols) {
  constexpr uint64_t kCus = 256;
  struct Cost { uint32_t fit; double alone, among, tile; };  // blocks on a CU, a step's time, their tiles' way to memory
  static constexpr Cost kCosts[2][3] = {{{3, 0.33, 0.77, 4.2}, {2, 0.74, 1.37, 9.6}, {1, 2.25, 2.25, 21}}, {{3, 0.33, 0.78, 2.2}, {2, 0.65, 1.11, 4.1}, {1, 1.72, 1.72, 10}}};
  Cut best = {};
  double least = 0;
  for (uint32_t size = 0; size < (outs < 8 ? 1u : 3u); ++size) {
    const Cost &cost = kCosts[dtype == DQ_BF16][size];
    const uint64_t e = kEdges[size], tok = kToks[dtype == DQ_BF16][size], steps = (rows + tok - 1) / tok;
    Cut c = {size, 1, (outs + e - 1) / e, (cols + e - 1) / e, steps * tok};
    const uint64_t tiles = c.tiles_out * c.tiles_in;
    for (uint64_t k = 0; k <= 2 * cost.fit; ++k) {  // one split, or as many as make up to k units for every CU
      uint64_t splits = 1;
      if (k) {
        splits = k * kCus / tiles < steps / 4 ? k * kCus / tiles : steps / 4;
        if (splits <= 1) continue;
      }
      const uint64_t each = steps ? (steps + splits - 1) / splits : 1;
      if (steps) splits = (steps + each - 1) / each;
      const uint64_t on_cu = (tiles * splits + kCus - 1) / kCus, rest = on_cu % cost.fit;
      double us = 3 + (double)each * ((double)(on_cu / cost.fit) * cost.among +
                                      (rest ? cost.alone + (cost.among - cost.alone) * (double)(rest - 1) / (cost.fit > 1 ? cost.fit - 1 : 1) : 0.0));
      if (splits > 1) us += 3 + (double)(splits * tiles * e * e) * 8 / 5.0e6;
      else us += cost.tile * (double)on_cu / cost.fit;
      if ((size == 0 && k == 0) || us < least) {
        least = us;
        best = c;
        best.splits = (uint32_t)splits;
        best.split_rows = each * tok;
      }
    }
  }
  return best;
}

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename T, typename O, typename S, bool SMALL>
hipError_t run(const WGrad &g, hipStream_t s) {
  const uint64_t units = g.tiles * g.splits;
  hipLaunchKernelGGL((k_wgrad<T, O, S, SMALL>), dim3((uint32_t)(units < 65536 ? units : 65536)), dim3(S::kThreads), 0, s, g);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.splits == 1) return e;
  const uint64_t all = g.tiles * (S::kOut * S::kIn / 4) + (g.db ? g.outs : 0);
  constexpr uint32_t kWays = 8;
  const uint64_t per_block = g.splits < kManySplits ? kJoinThreads : kJoinThreads / kWays, blocks = (all + per_block - 1) / per_block;
  const dim3 grid((uint32_t)(blocks < 65536 ? blocks : 65536));
  if (g.splits < kManySplits) hipLaunchKernelGGL((k_wgrad_join<O, S, SMALL, 1>), grid, dim3(kJoinThreads), 0, s, g);
  else hipLaunchKernelGGL((k_wgrad_join<O, S, SMALL, kWays>), grid, dim3(kJoinThreads), 0, s, g);
  return hipGetLastError();
}
template <typename T, typename O>
hipError_t run_cut(const Cut &c, const WGrad &g, hipStream_t s) {
  constexpr int b = __is_same(T, Bf16);
  if (g.outs < 8) return run<T, O, Tile<T, 64, 64, kToks[b][0], 2>, true>(g, s);
  if (c.size == 0) return run<T, O, Tile<T, 64, 64, kToks[b][0], 2>, false>(g, s);
  if (c.size == 1) return run<T, O, Tile<T, 128, 128, kToks[b][1], 2>, false>(g, s);
  return run<T, O, Tile<T, 256, 256, kToks[b][2], 4>, false>(g, s);
}

}  // namespace
}  // namespace dq

using namespace dq;

#define DQ_TRY(x)                 \
  do {                            \
    const dq_status st_ = (x);    \
    if (st_ != DQ_OK) return st_; \
  } while (0)

extern "C" {

size_t dq_ckpt_weight_grad_scratch_bytes(dq_dtype dtype, uint64_t rows, uint64_t outs, uint64_t cols) {
  if (rows == 0 || outs == 0 || cols == 0 || (rows | outs | cols) >> 31) return 0;
  const Cut c = cut_of(dtype, rows, outs, cols);
  if (c.splits == 1) return 0;
  return (size_t)(c.splits * (c.tiles_out * c.tiles_in * kEdges[c.size] * kEdges[c.size] + outs) * 4);
}

dq_status dq_ckpt_weight_grad(const dq_matrix *dy, const void *ckpt, uint64_t rows, uint64_t outs, uint64_t cols, const dq_matrix *dw, void *db,
                              int accumulate, void *scratch, size_t scratch_bytes, void *hip_stream) {
  DQ_TRY(check_matrix(dy, rows, outs));
  DQ_TRY(check_matrix(dw, outs, cols));
  if (outs == 0 || cols == 0) return db && outs ? DQ_EINVAL : DQ_OK;
  const uint64_t ob = entry_bytes(dw->dtype);
  if (outs >> 31 || cols >> 31 || rows >> 31) return DQ_EUNSUPPORTED;
  if ((uintptr_t)db % ob) return DQ_EALIGN;
  const size_t bytes = rows ? dq_ckpt_bytes(rows, cols) : 0, need = dq_ckpt_weight_grad_scratch_bytes(dy->dtype, rows, outs, cols);
  if (rows) {
    if (bytes == 0) return DQ_EUNSUPPORTED;
    if (!ckpt || (need && (!scratch || scratch_bytes < need))) return DQ_EINVAL;
    if (!al16(ckpt) || (need && !al16(scratch))) return DQ_EALIGN;
  }
  const Region r[] = {region(dy, rows, outs, false), region(rows ? ckpt : nullptr, bytes, false), region(dw, outs, cols, true),
                      region(db, outs * ob, true), region(need ? scratch : nullptr, need, true)};
  if (regions_meet(r, 5)) return DQ_EINVAL;
  if (rows == 0 && accumulate) return DQ_OK;
  const Cut c = cut_of(dy->dtype, rows, outs, cols);
  WGrad g = {};
  g.dy = {dy->data, dy->ld};
  g.x = ckpt_in(ckpt, rows, cols);
  g.rows = rows;
  g.outs = outs;
  g.cols = cols;
  g.pitch = ckpt_pitch(cols);
  g.dw = dw->data;
  g.db = db;
  g.ld = dw->ld;
  g.part = static_cast<float *>(scratch);
  g.tiles = c.tiles_out * c.tiles_in;
  g.tiles_out = (uint32_t)c.tiles_out;
  g.tiles_in = (uint32_t)c.tiles_in;
  g.splits = c.splits;
  g.split_rows = c.split_rows;
  g.accumulate = accumulate != 0;
  hipStream_t s = (hipStream_t)hip_stream;
  if (dy->dtype == DQ_F32) return hip_status(dw->dtype == DQ_F32 ? run_cut<F32, F32>(c, g, s) : run_cut<F32, Bf16>(c, g, s));
  return hip_status(dw->dtype == DQ_F32 ? run_cut<Bf16, F32>(c, g, s) : run_cut<Bf16, Bf16>(c, g, s));
}

}  // extern "C"
