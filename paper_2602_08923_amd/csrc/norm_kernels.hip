// Layer norm: y = (x - mean) rstd w + b along each row, with an 8-bit checkpoint of x beside it, and the backward pass that reads
// x from the checkpoint:
//   n = (x - mean) rstd, q = dy w:  dx = rstd (q - avg(q) - n avg(q n)),  dw = sum over rows of dy n,  db = sum over rows of dy.
// mean and rstd are those of the forward pass, from x itself; sums and statistics are binary32, the variance from differences to
// the mean.
#include <math.h>

#include "act_rows.h"

namespace dq {
namespace {

constexpr uint32_t kThreads = 256;

// Sums of a and b over the block, in every thread; the order is fixed.
__device__ __forceinline__ void block_sums(float &a, float &b, float *lds) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    a += __shfl_xor(a, d);
    b += __shfl_xor(b, d);
  }
  const uint32_t wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  __syncthreads();  // the last row's sums have been read
  if ((threadIdx.x & 63u) == 0) {
    lds[2 * wave] = a;
    lds[2 * wave + 1] = b;
  }
  __syncthreads();
  a = b = 0.0f;
  for (uint32_t i = 0; i < waves; ++i) {
    a += lds[2 * i];
    b += lds[2 * i + 1];
  }
}

struct NormIn {
  Rows x;
  uint64_t rows, cols;
  const void *weight, *bias;  // or null: ones, zeros
  float eps;
};
template <typename W>
__device__ __forceinline__ void weight8(const void *w, uint64_t col, uint64_t cols, float otherwise, float (&v)[8]) {
  if (w) {
    load8<W>(w, col, cols, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = otherwise;
  }
}

// A block per row, which it reads three times (the second and third time from the cache).
template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void k_norm_wide(NormIn in, Rows y, CkptOut saved, float *mean, float *rstd) {
  __shared__ float lds[2 * kThreads / 64];
  const uint64_t chunks = ckpt_pitch(in.cols) / 8;
  const float inv = 1.0f / (float)in.cols;
  for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
    const uint8_t *x = static_cast<const uint8_t *>(in.x.data) + r * in.x.ld * kEntry<T>;
    float v[8], s = 0.0f, s2 = 0.0f;
    for (uint64_t c = threadIdx.x; c < chunks; c += kThreads) {
      load8<T>(x, c * 8, in.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    block_sums(s, s2, lds);
    const float m = s * inv;
    s = s2 = 0.0f;
    for (uint64_t c = threadIdx.x; c < chunks; c += kThreads) {
      load8<T>(x, c * 8, in.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = c * 8 + i < in.cols ? v[i] - m : 0.0f;
        s = fmaf(d, d, s);
      }
    }
    block_sums(s, s2, lds);
    const float k = 1.0f / sqrtf(fmaf(s, inv, in.eps));
    for (uint64_t c = threadIdx.x; c < chunks; c += kThreads) {
      float w[8], b[8];
      load8<T>(x, c * 8, in.cols, v);
      if (saved.codes) ckpt_store8(saved, r * chunks + c, v);
      weight8<W>(in.weight, c * 8, in.cols, 1.0f, w);
      weight8<W>(in.bias, c * 8, in.cols, 0.0f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = fmaf((v[i] - m) * k, w[i], b[i]);
      store8<T>(static_cast<uint8_t *>(y.data) + r * y.ld * kEntry<T>, c * 8, in.cols, v);
    }
    if (threadIdx.x == 0 && mean) {
      mean[r] = m;
      rstd[r] = k;
    }
  }
}

struct NormGrad {
  Rows dy, dx;
  uint64_t rows, cols;
  CkptIn x;
  const float *mean, *rstd;
  const void *weight;
};
template <typename T, typename W>
__global__ __launch_bounds__(kThreads) void k_norm_grad_wide(NormGrad in) {
  __shared__ float lds[2 * kThreads / 64];
  const uint64_t chunks = ckpt_pitch(in.cols) / 8;
  const float inv = 1.0f / (float)in.cols;
  for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
    const uint8_t *dy = static_cast<const uint8_t *>(in.dy.data) + r * in.dy.ld * kEntry<T>;
    const float m = in.mean[r], k = in.rstd[r];
    float x[8], q[8], w[8], s = 0.0f, sn = 0.0f;
    for (uint64_t c = threadIdx.x; c < chunks; c += kThreads) {
      load8<T>(dy, c * 8, in.cols, q);  // zero behind the row's end
      ckpt_load8(in.x, r * chunks + c, x);
      weight8<W>(in.weight, c * 8, in.cols, 1.0f, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        q[i] *= w[i];
        s += q[i];
        sn = fmaf(q[i], (x[i] - m) * k, sn);
      }
    }
    block_sums(s, sn, lds);
    s *= inv;
    sn *= inv;
    for (uint64_t c = threadIdx.x; c < chunks; c += kThreads) {
      load8<T>(dy, c * 8, in.cols, q);
      ckpt_load8(in.x, r * chunks + c, x);
      weight8<W>(in.weight, c * 8, in.cols, 1.0f, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = k * (fmaf(q[i], w[i], -s) - (x[i] - m) * k * sn);
      store8<T>(static_cast<uint8_t *>(in.dx.data) + r * in.dx.ld * kEntry<T>, c * 8, in.cols, q);
    }
  }
}

// The sums over rows, a slice of the rows and a thread per chunk of columns; part: [slices][2][pitch].
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_columns(NormGrad in, uint64_t slice_rows, float *part) {
  const uint64_t pitch = ckpt_pitch(in.cols), chunks = pitch / 8, c = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= chunks) return;
  const uint64_t first = blockIdx.y * slice_rows, end = first + slice_rows < in.rows ? first + slice_rows : in.rows;
  float dw[8] = {}, db[8] = {};
  for (uint64_t r = first; r < end; ++r) {
    float g[8], x[8];
    load8<T>(static_cast<const uint8_t *>(in.dy.data) + r * in.dy.ld * kEntry<T>, c * 8, in.cols, g);
    ckpt_load8(in.x, r * chunks + c, x);
    const float m = in.mean[r], k = in.rstd[r];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dw[i] = fmaf(g[i], (x[i] - m) * k, dw[i]);
      db[i] += g[i];
    }
  }
  float *p = part + (uint64_t)blockIdx.y * 2 * pitch + c * 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = dw[i];
    p[pitch + i] = db[i];
  }
}

// The parts of dw and db joined, in their order: 16 threads of a block to four columns, then the 16 sums.
constexpr uint32_t kJoinThreads = 1024, kJoinCols = 64, kJoinWays = kJoinThreads / (kJoinCols / 4);
template <typename W>
__global__ __launch_bounds__(kJoinThreads) void k_norm_join(const float *part, uint64_t pitch, uint64_t cols, uint32_t parts, void *dw, void *db,
                                                           uint32_t accumulate) {
  __shared__ af32x4 lds[kJoinWays][kJoinCols / 4];
  const uint32_t t = threadIdx.x % (kJoinCols / 4), way = threadIdx.x / (kJoinCols / 4);
  for (uint64_t first = (uint64_t)blockIdx.x * kJoinCols; first < 2 * pitch; first += (uint64_t)gridDim.x * kJoinCols) {  // dw's columns, then db's
    af32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t i = way; i < parts; i += kJoinWays) s += a_ld<af32x4>(part + (uint64_t)i * 2 * pitch + first + t * 4);
    __syncthreads();  // the last columns' sums have been read
    lds[way][t] = s;
    __syncthreads();
    const uint32_t c = threadIdx.x;
    const uint64_t k = first + c < pitch ? first + c : first + c - pitch;
    if (c >= kJoinCols || k >= cols) continue;
    float v = 0.0f;
    for (uint32_t i = 0; i < kJoinWays; ++i) v += lds[i][c / 4][c % 4];
    void *out = first + c < pitch ? dw : db;
    if constexpr (__is_same(W, F32)) {
      float *p = static_cast<float *>(out) + k;
      *p = accumulate ? *p + v : v;
    } else {
      uint16_t *p = static_cast<uint16_t *>(out) + k;
      if (accumulate) v += a_float((uint32_t)*p << 16);
      *p = (uint16_t)to_bf16x2(v, v);
    }
  }
}

constexpr uint32_t kRowBlocks = 2048;  // blocks that rows are dealt to
uint32_t row_blocks(uint64_t rows) { return (uint32_t)(rows < kRowBlocks ? rows : kRowBlocks); }
// Slices of the rows for the sums over them.
uint32_t norm_slices(uint64_t rows) { return (uint32_t)(rows < 256 * 8 ? (rows + 7) / 8 : 256); }

uint32_t join_grid(uint64_t pitch) { return (uint32_t)(2 * pitch / kJoinCols < 4096 ? 2 * pitch / kJoinCols : 4096); }

bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool al4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace
}  // namespace dq

using namespace dq;

#define DQ_TRY(x)                 \
  do {                            \
    const dq_status st_ = (x);    \
    if (st_ != DQ_OK) return st_; \
  } while (0)

extern "C" {

dq_status dq_layer_norm(const dq_matrix *x, uint64_t rows, uint64_t cols, const void *weight, const void *bias, dq_dtype weight_dtype, float eps,
                        const dq_matrix *y, void *ckpt, float *mean, float *rstd, void *hip_stream) {
  DQ_TRY(check_matrix(x, rows, cols));
  DQ_TRY(check_matrix(y, rows, cols));
  if (y->dtype != x->dtype || (weight_dtype != DQ_F32 && weight_dtype != DQ_BF16) || !isfinite(eps) || eps < 0.0f) return DQ_EINVAL;
  if (rows == 0 || cols == 0) return DQ_OK;
  const size_t bytes = dq_ckpt_bytes(rows, cols);
  if (bytes == 0 || cols >> 31) return DQ_EUNSUPPORTED;
  if (!ckpt != !mean || !ckpt != !rstd) return DQ_EINVAL;
  const uint64_t wb = entry_bytes(weight_dtype);
  if (!al16(ckpt) || !al4(mean) || !al4(rstd) || (uintptr_t)weight % wb || (uintptr_t)bias % wb) return DQ_EALIGN;
  const Region r[] = {region(x, rows, cols, false), region(weight, cols * wb, false), region(bias, cols * wb, false), region(y, rows, cols, true),
                      region(ckpt, bytes, true), region(mean, rows * 4, true), region(rstd, rows * 4, true)};
  if (regions_meet(r, 7)) return DQ_EINVAL;
  const NormIn in = {{x->data, x->ld}, rows, cols, weight, bias, eps};
  const Rows out = {y->data, y->ld};
  const CkptOut saved = ckpt_out(ckpt, rows, cols);
#define DQ_NORM(T, W) hipLaunchKernelGGL((k_norm_wide<T, W>), dim3(row_blocks(rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, in, out, saved, mean, rstd)
  if (x->dtype == DQ_F32 && weight_dtype == DQ_F32) DQ_NORM(F32, F32);
  else if (x->dtype == DQ_F32) DQ_NORM(F32, Bf16);
  else if (weight_dtype == DQ_F32) DQ_NORM(Bf16, F32);
  else DQ_NORM(Bf16, Bf16);
  return hip_status(hipGetLastError());
}

size_t dq_layer_norm_grad_scratch_bytes(uint64_t rows, uint64_t cols) {
  if (dq_ckpt_bytes(rows, cols) == 0 || cols >> 31) return 0;
  return (size_t)norm_slices(rows) * 2 * ckpt_pitch(cols) * 4;
}

dq_status dq_layer_norm_grad(const dq_matrix *dy, const void *ckpt, const float *mean, const float *rstd, uint64_t rows, uint64_t cols,
                             const void *weight, dq_dtype weight_dtype, const dq_matrix *dx, void *dweight, void *dbias, int accumulate, void *scratch,
                             size_t scratch_bytes, void *hip_stream) {
  DQ_TRY(check_matrix(dy, rows, cols));
  DQ_TRY(check_matrix(dx, rows, cols));
  if (dx->dtype != dy->dtype || (weight_dtype != DQ_F32 && weight_dtype != DQ_BF16) || !dweight != !dbias) return DQ_EINVAL;
  if (cols == 0) return DQ_OK;
  if (cols >> 31) return DQ_EUNSUPPORTED;
  const uint64_t wb = entry_bytes(weight_dtype);
  if (rows == 0) {  // nothing to sum
    if (!dweight || accumulate) return DQ_OK;
    if ((uintptr_t)dweight % wb || (uintptr_t)dbias % wb) return DQ_EALIGN;
    const Region r[] = {region(dweight, cols * wb, true), region(dbias, cols * wb, true)};
    if (regions_meet(r, 2)) return DQ_EINVAL;
  }
  const size_t bytes = rows ? dq_ckpt_bytes(rows, cols) : 0, need = dq_layer_norm_grad_scratch_bytes(rows, cols);
  const uint64_t pitch = ckpt_pitch(cols);
  const uint32_t slices = norm_slices(rows), join_blocks = join_grid(pitch);
  hipStream_t s = (hipStream_t)hip_stream;
  if (rows) {
    if (bytes == 0) return DQ_EUNSUPPORTED;
    if (!ckpt || !mean || !rstd || (dweight && (!scratch || scratch_bytes < need))) return DQ_EINVAL;
    if (!al16(ckpt) || !al4(mean) || !al4(rstd) || (uintptr_t)weight % wb || (uintptr_t)dweight % wb || (uintptr_t)dbias % wb || !al16(scratch))
      return DQ_EALIGN;
    const Region r[] = {region(dy, rows, cols, false),      region(ckpt, bytes, false),         region(mean, rows * 4, false),
                        region(rstd, rows * 4, false),      region(weight, cols * wb, false),   region(dx, rows, cols, true),
                        region(dweight, cols * wb, true),   region(dbias, cols * wb, true),     region(dweight ? scratch : nullptr, need, true)};
    if (regions_meet(r, 9)) return DQ_EINVAL;
    const NormGrad in = {{dy->data, dy->ld}, {dx->data, dx->ld}, rows, cols, ckpt_in(ckpt, rows, cols), mean, rstd, weight};
#define DQ_NORM_GRAD(T, W) hipLaunchKernelGGL((k_norm_grad_wide<T, W>), dim3(row_blocks(rows)), dim3(kThreads), 0, s, in)
    if (dy->dtype == DQ_F32 && weight_dtype == DQ_F32) DQ_NORM_GRAD(F32, F32);
    else if (dy->dtype == DQ_F32) DQ_NORM_GRAD(F32, Bf16);
    else if (weight_dtype == DQ_F32) DQ_NORM_GRAD(Bf16, F32);
    else DQ_NORM_GRAD(Bf16, Bf16);
    DQ_TRY(hip_status(hipGetLastError()));
    if (!dweight) return DQ_OK;
    const dim3 grid((uint32_t)((pitch / 8 + kThreads - 1) / kThreads), slices);
    const uint64_t slice_rows = (rows + slices - 1) / slices;
    if (dy->dtype == DQ_F32) hipLaunchKernelGGL((k_norm_columns<F32>), grid, dim3(kThreads), 0, s, in, slice_rows, (float *)scratch);
    else hipLaunchKernelGGL((k_norm_columns<Bf16>), grid, dim3(kThreads), 0, s, in, slice_rows, (float *)scratch);
    DQ_TRY(hip_status(hipGetLastError()));
  }
  if (weight_dtype == DQ_F32)
    hipLaunchKernelGGL((k_norm_join<F32>), dim3(join_blocks), dim3(kJoinThreads), 0, s, (const float *)scratch, pitch, cols, slices, dweight, dbias,
                       (uint32_t)(accumulate != 0));
  else
    hipLaunchKernelGGL((k_norm_join<Bf16>), dim3(join_blocks), dim3(kJoinThreads), 0, s, (const float *)scratch, pitch, cols, slices, dweight, dbias,
                       (uint32_t)(accumulate != 0));
  return hip_status(hipGetLastError());
}

}  // extern "C"
