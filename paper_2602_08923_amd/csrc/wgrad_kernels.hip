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
  uint64_t rows, outs, cols;
  void *dw, *db;
  uint64_t ld, tiles, tiles_out;
  uint32_t accumulate;
};

constexpr uint32_t kThreads = 256;

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) a32x4 lds_a32x4;
// Tokens 0 .. 15 of 32 columns: `at` is the LDS address of the first token's first column plus the lane's part (read_at).
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

// A block's tile is 64 by 64, a wave's 32 by 32.
template <typename T, typename O>
__global__ __launch_bounds__(kThreads) void k_wgrad(WGrad g) {
  constexpr uint32_t kPlanes = __is_same(T, F32) ? 3 : 1, kTok = 32, kStride = 192;
  __shared__ __attribute__((aligned(16))) uint8_t lds[(kPlanes + 1) * kTok * kStride];
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds, xbase = base + kPlanes * kTok * kStride;
  const uint64_t pitch = ckpt_pitch(g.cols);
  const uint32_t wave = threadIdx.x >> 6, wo = (wave & 1u) * 32, wi = (wave >> 1) * 32;
  const uint32_t tok = threadIdx.x >> 3, chunk = (threadIdx.x & 7u) * 8;
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  for (uint64_t tile = blockIdx.x; tile < g.tiles; tile += gridDim.x) {
  const uint64_t o0 = tile % g.tiles_out * 64, i0 = tile / g.tiles_out * 64;
  const bool bias = g.db && i0 == 0 && wi == 0;
  f32x16 acc = {}, sums = {};
  for (uint64_t t0 = 0; t0 < g.rows; t0 += kTok) {
    const uint64_t t = t0 + tok;
    float v[8] = {};
    a32x4 x = {0u, 0u, 0u, 0u};
    if (t < g.rows) {
      load8<T>(static_cast<const uint8_t *>(g.dy.data) + t * g.dy.ld * kEntry<T>, o0 + chunk, g.outs, v);
      if (i0 + chunk < pitch) {
        float xv[8];
        ckpt_load8(g.x, (t * pitch + i0 + chunk) / 8, xv);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = high_halves(a_bits(xv[2 * i]), a_bits(xv[2 * i + 1]));
      }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t p = 0; p < kPlanes; ++p) {
      a32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = high_halves(a_bits(v[2 * i]), a_bits(v[2 * i + 1]));
      *reinterpret_cast<lds_a32x4 *>(base + (p * kTok + tok) * kStride + chunk * 2) = w;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= a_float(a_bits(v[i]) & 0xFFFF0000u);
    }
    *reinterpret_cast<lds_a32x4 *>(xbase + tok * kStride + chunk * 2) = x;
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < kTok; k += 16) {
      const bf16x8 b = read16(xbase + k * kStride + wi * 2 + read_at(kStride), kStride);
#pragma unroll
      for (uint32_t p = 0; p < kPlanes; ++p) {
        const bf16x8 a = read16(base + (p * kTok + k) * kStride + wo * 2 + read_at(kStride), kStride);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
        if (bias) sums = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, ones, sums, 0, 0, 0);
      }
    }
  }
  const uint32_t l = threadIdx.x & 63u;
  const uint64_t i = i0 + wi + (l & 31u);
#pragma unroll
  for (uint32_t r = 0; r < 16; ++r) {
    const uint64_t o = o0 + wo + 8 * (r / 4) + 4 * (l >> 5) + r % 4;
    if (o >= g.outs) continue;
    if (i < g.cols) put<O>(g.dw, o * g.ld + i, acc[r], g.accumulate);
    if (bias && (l & 31u) == 0) put<O>(g.db, o, sums[r], g.accumulate);
  }
  }
}

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

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
  (void)dtype; (void)rows; (void)outs; (void)cols;
  return 0;
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
  const WGrad g = {{dy->data, dy->ld}, ckpt_in(ckpt, rows, cols), rows, outs, cols, dw->data, db, dw->ld, (outs + 63) / 64 * ((cols + 63) / 64), (outs + 63) / 64, (uint32_t)(accumulate != 0)};
  const uint32_t blocks = (uint32_t)(g.tiles < 65536 ? g.tiles : 65536);
#define DQ_WGRAD(T, O) hipLaunchKernelGGL((k_wgrad<T, O>), dim3(blocks), dim3(kThreads), 0, (hipStream_t)hip_stream, g)
  if (dy->dtype == DQ_F32 && dw->dtype == DQ_F32) DQ_WGRAD(F32, F32);
  else if (dy->dtype == DQ_F32) DQ_WGRAD(F32, Bf16);
  else if (dw->dtype == DQ_F32) DQ_WGRAD(Bf16, F32);
  else DQ_WGRAD(Bf16, Bf16);
  return hip_status(hipGetLastError());
}

}  // extern "C"
