// Rows of activations as the checkpoint, layer norm, gate and weight-gradient kernels read and write them, and the checkpoint's
// 8-bit blocks.
//
// A row is cut into chunks, one lane's share; the neighbouring lanes of a block of 32 hold it together.  Rows start at any multiple
// of the entry size: gfx950 loads and stores 16 bytes from any address, at full rate where they do not cross a cache line, so
// there is one path for every stride, and only a row's last chunk may have to go entry by entry.
#pragma once
#include <type_traits>

#include "dq_device.h"

namespace dq {

typedef uint32_t a32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t a32x4 __attribute__((ext_vector_type(4)));
typedef float af32x4 __attribute__((ext_vector_type(4)));
typedef float af32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef a32x4 a32x4_any __attribute__((aligned(2)));   // 16 bytes from any bf16's address

// rows x cols entries, row r from data + r * ld entries on
struct Rows {
  void *data;
  uint64_t ld;
};
inline uint32_t entry_bytes(dq_dtype t) { return t == DQ_F32 ? 4u : 2u; }

constexpr uint32_t kCkptBlock = 32;
// Scale bytes: 10 is the least (8-bit values are then normal bf16 numbers or zero, whatever reads them), 246 is that of the
// largest binary32; 255 marks a block with an infinity or NaN, all of whose codes are NaN.
constexpr uint32_t kCkptLeast = 10;
inline __host__ __device__ uint64_t ckpt_pitch(uint64_t cols) { return (cols + kCkptBlock - 1) / kCkptBlock * kCkptBlock; }

template <typename T>
__device__ __forceinline__ T a_ld(const void *p) {
  return *(const __attribute__((address_space(1))) T *)p;
}
template <typename T>
__device__ __forceinline__ void a_st(void *p, T v) {
  *(__attribute__((address_space(1))) T *)p = v;
}
__device__ __forceinline__ float a_float(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t a_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

struct F32 {};
struct Bf16 {};
template <typename T>
constexpr uint32_t kEntry = __is_same(T, F32) ? 4 : 2;

// Two binary32 numbers as bf16, rounded to nearest even.
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(af32x2{a, b}, bf16x2));
}
// N entries of a row, 16 bytes or 32, as they lie in memory.
template <typename T, uint32_t N>
struct Raw {
  a32x4 w[N * kEntry<T> / 16];
};
// Entries col .. col + N - 1 of the row at `row`, of which `cols` exist; the others are zero.  PAST: past the caches, for rows on
// 16-byte borders.
template <typename T, uint32_t N, bool PAST = false>
__device__ __forceinline__ Raw<T, N> load_raw(const void *row, uint64_t col, uint64_t cols) {
  const uint8_t *p = static_cast<const uint8_t *>(row) + col * kEntry<T>;
  Raw<T, N> r;
  if (col + N <= cols) {
#pragma unroll
    for (uint32_t q = 0; q < N * kEntry<T> / 16; ++q) {
      if constexpr (PAST) r.w[q] = __builtin_nontemporal_load((const __attribute__((address_space(1))) a32x4 *)(p + 16 * q));
      else r.w[q] = a_ld<a32x4_any>(p + 16 * q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < (int)(N * kEntry<T> / 4); ++i) {
      uint32_t v = 0;
      if constexpr (__is_same(T, F32)) {
        if (col + i < cols) v = a_ld<uint32_t>(p + 4 * i);
      } else {
        if (col + 2 * i < cols) v = a_ld<uint16_t>(p + 4 * i);
        if (col + 2 * i + 1 < cols) v |= (uint32_t)a_ld<uint16_t>(p + 4 * i + 2) << 16;
      }
      r.w[i / 4][i % 4] = v;
    }
  }
  return r;
}
template <typename T, uint32_t N>
__device__ __forceinline__ void widen(const Raw<T, N> &r, float (&v)[N]) {
#pragma unroll
  for (uint32_t i = 0; i < N * kEntry<T> / 4; ++i) {
    const uint32_t w = r.w[i / 4][i % 4];
    if constexpr (__is_same(T, F32)) {
      v[i] = a_float(w);
    } else {
      v[2 * i] = a_float(w << 16);
      v[2 * i + 1] = a_float(w & 0xFFFF0000u);
    }
  }
}
template <typename T, uint32_t N>
__device__ __forceinline__ void load_entries(const void *row, uint64_t col, uint64_t cols, float (&v)[N]) {
  if constexpr (N * kEntry<T> >= 16) {
    widen(load_raw<T, N>(row, col, cols), v);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) v[i] = col + i < cols ? a_float((uint32_t)a_ld<uint16_t>(static_cast<const uint8_t *>(row) + (col + i) * 2) << 16) : 0.0f;
  }
}
template <typename T, uint32_t N, bool PAST = false>
__device__ __forceinline__ void store_entries(void *row, uint64_t col, uint64_t cols, const float (&v)[N]) {
  uint8_t *p = static_cast<uint8_t *>(row) + col * kEntry<T>;
  Raw<T, N> r;
#pragma unroll
  for (uint32_t i = 0; i < N * kEntry<T> / 4; ++i) {
    if constexpr (__is_same(T, F32)) r.w[i / 4][i % 4] = a_bits(v[i]);
    else r.w[i / 4][i % 4] = to_bf16x2(v[2 * i], v[2 * i + 1]);
  }
  if (col + N <= cols) {
#pragma unroll
    for (uint32_t q = 0; q < N * kEntry<T> / 16; ++q) {
      if constexpr (PAST) __builtin_nontemporal_store(r.w[q], (__attribute__((address_space(1))) a32x4 *)(p + 16 * q));
      else a_st<a32x4_any>(p + 16 * q, r.w[q]);
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
      if (col + i < cols) {
        if constexpr (__is_same(T, F32)) a_st<uint32_t>(p + 4 * i, r.w[i / 4][i % 4]);
        else a_st<uint16_t>(p + 2 * i, (uint16_t)(r.w[i / 8][i / 2 % 4] >> (16 * (i % 2))));
      }
  }
}
template <typename T>
__device__ __forceinline__ void load8(const void *row, uint64_t col, uint64_t cols, float (&v)[8]) {
  load_entries<T, 8>(row, col, cols, v);
}
template <typename T>
__device__ __forceinline__ void store8(void *row, uint64_t col, uint64_t cols, const float (&v)[8]) {
  store_entries<T, 8>(row, col, cols, v);
}

// The largest of the four lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}
// Four codes of a block whose largest magnitude has the exponent field `top`, and the block's scale byte.  The scaled conversions take
// the scale's exponent field; the narrowing one makes NaN of what is too large, so values are clamped first (448 is the largest).
__device__ __forceinline__ uint32_t ckpt_codes(float a, float b, float c, float d, uint32_t top, uint32_t *scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  const uint32_t e = max(top, kCkptLeast + 8) - 8;
  const float X = a_float(e << 23), most = 448.0f * X;
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __builtin_amdgcn_fmed3f(a, -most, most), __builtin_amdgcn_fmed3f(b, -most, most), X, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __builtin_amdgcn_fmed3f(c, -most, most), __builtin_amdgcn_fmed3f(d, -most, most), X, true);
  *scale = top == 255 ? 255u : e;
  return top == 255 ? 0x7F7F7F7Fu : __builtin_bit_cast(uint32_t, r);
}
// A lane's 8 entries of a block as codes.  All four lanes of the block call it.
__device__ __forceinline__ a32x2 ckpt_encode(const float (&v)[8], uint32_t *scale) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, a_bits(v[i]) & 0x7FFFFFFFu);
  m = block_max(m) >> 23;
  const uint32_t lo = ckpt_codes(v[0], v[1], v[2], v[3], m, scale), hi = ckpt_codes(v[4], v[5], v[6], v[7], m, scale);
  return a32x2{lo, hi};
}
__device__ __forceinline__ void ckpt_decode(a32x2 codes, uint32_t scale, float (&v)[8]) {
  const float X = a_float(scale << 23);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const af32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[h], X, false);
    const af32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[h], X, true);
    v[4 * h] = lo.x; v[4 * h + 1] = lo.y; v[4 * h + 2] = hi.x; v[4 * h + 3] = hi.y;
  }
}
// The same with four entries of binary32 a lane, eight lanes to a block.
__device__ __forceinline__ uint32_t ckpt_encode(const float (&v)[4], uint32_t *scale) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, a_bits(v[i]) & 0x7FFFFFFFu);
  m = block_max(m);
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, true));  // mirrored within 8 lanes
  return ckpt_codes(v[0], v[1], v[2], v[3], m >> 23, scale);
}
__device__ __forceinline__ void ckpt_decode(uint32_t codes, uint32_t scale, float (&v)[4]) {
  const float X = a_float(scale << 23);
  const af32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, X, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, X, true);
  v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
}
// The codes of a chunk of N entries as they lie in memory.
template <uint32_t N>
using CkptCodes = std::conditional_t<N == 8, a32x2, uint32_t>;
struct CkptIn {
  const uint8_t *codes, *scales;
};
struct CkptOut {
  uint8_t *codes, *scales;
};
inline CkptIn ckpt_in(const void *p, uint64_t rows, uint64_t cols) {
  if (!p) return {nullptr, nullptr};
  return {static_cast<const uint8_t *>(p), static_cast<const uint8_t *>(p) + rows * ckpt_pitch(cols)};
}
inline CkptOut ckpt_out(void *p, uint64_t rows, uint64_t cols) {
  if (!p) return {nullptr, nullptr};
  return {static_cast<uint8_t *>(p), static_cast<uint8_t *>(p) + rows * ckpt_pitch(cols)};
}
// Chunk number `chunk` of a checkpoint (its rows back to back, each pitch / N chunks): its codes, and its block's scale behind all codes.
// All lanes of a block save together.
template <uint32_t N>
__device__ __forceinline__ void ckpt_load(const CkptIn &c, uint64_t chunk, float (&v)[N]) {
  ckpt_decode(a_ld<CkptCodes<N>>(c.codes + chunk * N), a_ld<uint8_t>(c.scales + chunk / (kCkptBlock / N)), v);
}
template <uint32_t N>
__device__ __forceinline__ void ckpt_store(const CkptOut &c, uint64_t chunk, const float (&v)[N]) {
  uint32_t scale;
  const CkptCodes<N> codes = ckpt_encode(v, &scale);
  a_st<CkptCodes<N>>(c.codes + chunk * N, codes);
  if (chunk % (kCkptBlock / N) == 0) a_st<uint8_t>(c.scales + chunk / (kCkptBlock / N), (uint8_t)scale);
}

// Host side: what the entry points check.
struct Region {  // rows of `bytes` bytes, `stride` bytes apart
  const void *p;
  uint64_t rows, bytes, stride;
  bool written;
};
inline Region region(const void *p, uint64_t bytes, bool written) { return {p, 1, bytes, bytes, written}; }
inline Region region(const dq_matrix *m, uint64_t rows, uint64_t cols, bool written) {
  const uint64_t e = entry_bytes(m->dtype);
  return {m->data, rows, cols * e, rows > 1 ? m->ld * e : cols * e, written};
}
// Matrices of one call that together are larger than what the caches could keep of them go past the caches, where their rows lie on
// 16-byte borders.  What counts is a call and the one that reads what it wrote: us of both, 4096 columns, through the caches and past
// them, the first call's inputs not in the caches:
//   save and load       bf16 64 MiB a matrix 39, 37; 128 MiB 74, 67; 192 MiB 125, 102       fp32 64 MiB 33, 28; 100 MiB 50, 45; 128 MiB 62, 57
//   gate, its gradient  bf16 32 MiB 48, 48; 48 MiB 67, 69; 64 MiB 99, 94; 100 MiB 166, 143  fp32 43, 42; 60, 62; 82, 81; 145, 125
//   layer norm, its backward pass past them  bf16 32 MiB 43, 42; 64 MiB 69, 67               fp32 41, 37; 63, 58; its forward pass too: 72 and 64
// With inputs that are still there, 64 MiB saved and loaded 34, 37; gates of 32 MiB 44, 48; the others are in the same order.  A single call
// that is repeated on one input of 64 to 128 MiB takes up to a quarter less through the caches, which is not what a program does.
constexpr uint64_t kPastBytes = 128ull << 20;
inline bool on_16(const dq_matrix *m, uint64_t rows) { return (uintptr_t)m->data % 16 == 0 && (rows == 1 || m->ld * entry_bytes(m->dtype) % 16 == 0); }
// Whether some written region meets another one.
bool regions_meet(const Region *r, int n);
// A matrix that a call may read or write: DQ_OK, DQ_EINVAL or DQ_EALIGN.
dq_status check_matrix(const dq_matrix *m, uint64_t rows, uint64_t cols);
uint32_t device_cu_count();

}  // namespace dq
