// Layer norm: y = (x - mean) rstd w + b along each row, with an 8-bit checkpoint of x beside it, and the backward pass that reads
// x from the checkpoint:
//   n = (x - mean) rstd, q = dy w:  dx = rstd (q - avg(q) - n avg(q n)),  dw = sum over rows of dy n,  db = sum over rows of dy.
// mean and rstd are those of the forward pass, from x itself; sums and statistics are binary32, the variance from differences to
// the mean.
#include <math.h>

#include "act_rows.h"

namespace dq {
namespace {

constexpr uint32_t kWideThreads = 1024, kThreads = 256;

// The sum over a wave, or over each 16 or 32 of its lanes, in all of them: within rows of 16 lanes by moves that the addition makes
// itself, then over the rows and the halves.  Through LDS, as shuffles go, a sum took 100 cycles a step.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + a_float((uint32_t)__builtin_amdgcn_mov_dpp((int)a_bits(v), CTRL, 0xF, 0xF, true));
}
// A swap of a's odd rows with b's even ones (of a's upper half with b's lower one) leaves two values whose sum has a's neighbouring rows (halves)
// added up in a's places, b's in b's.
__device__ __forceinline__ float rows_sum(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a_bits(a), a_bits(b), false, false);
  return a_float(r[0]) + a_float(r[1]);
}
__device__ __forceinline__ float halves_sum(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a_bits(a), a_bits(b), false, false);
  return a_float(r[0]) + a_float(r[1]);
}
template <uint32_t LANES = 64>
__device__ __forceinline__ float lanes_sum(float v) {
  v = add_dpp<0xB1>(v);   // lanes 1 0 3 2
  v = add_dpp<0x4E>(v);   // lanes 2 3 0 1
  v = add_dpp<0x141>(v);  // mirrored within 8
  v = add_dpp<0x140>(v);  // mirrored within 16
  if constexpr (LANES > 16) v = rows_sum(v, v);
  if constexpr (LANES > 32) v = halves_sum(v, v);
  return v;
}
// Sums of a and b over the block, in every thread; the order is fixed.
__device__ __forceinline__ void block_sums(float &a, float &b, float *lds) {
  a = lanes_sum(a);
  b = lanes_sum(b);
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
  uint32_t bf16;              // whether they are bf16
  float eps;
};
template <uint32_t N>
__device__ __forceinline__ void weights_at(const void *w, uint32_t bf16, uint64_t col, uint64_t cols, float otherwise, float (&v)[N]) {
  if (w) {
    if (bf16) load_entries<Bf16, N>(w, col, cols, v);
    else load_entries<F32, N>(w, col, cols, v);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) v[i] = otherwise;
  }
}

// Memory bounds both passes: rows of up to 16,384 entries stay in registers, so that they are read once.  GROUP threads have a row,
// KEEP chunks of 8 entries each.  A row goes to one wave where that is enough (up to 2,048 entries) and there are rows for all, so that
// its sums need no barrier; a wave has two or four of the short rows (up to 256 and 128 entries).  The next row is loaded while one
// is worked on, and there are as many blocks as stay resident, so that most rows are loaded so.
// Measured (forward and backward, 5.2 TB/s being a large copy's rate): bf16 16384 x 2048 68 to 73 us (4.6 to 5.0 TB/s), 200000 x 128 53
// (4.9), 65536 x 2048 224 (6.0), 16384 x 4096 128 (5.3), 4096 x 16384 152 (4.5); fp32 16384 x 4096 208 (5.8), 8192 x 8192 216 (5.6), 4096 x
// 16384 233 (5.2), 65536 x 500 135 (4.4), 1021 x 6151 38 (3.0).
//
// PAST: rows of large calls go past the caches.  A wave's loads and stores then have to cover memory without gaps, so a chunk is 16 bytes,
// twice as many of 4 entries in fp32.  Forward and backward, through the caches and past them: bf16 65536 x 2048 265 and 228 us,
// 16384 x 4096 136 and 128, fp32 16384 x 4096 231 and 207.  Below, chunks of 8 are as good or better (fp32 1024 x 8192 41 and 43), and
// better over odd rows (fp32 3000 x 7001 96, 105 with 4).  Both add a row up in the same order (see RowSums).  The forward pass takes twice
// the size for large (see kPastBytes: 128 MiB of x and y in bf16, with the backward pass, 67 us, 72 if it went past the caches too).
//
// A block's groups take a row each, the block then the next rows; all of them come round as often as each other.
template <typename T, uint32_t GROUP, uint32_t KEEP, bool PAST>
struct Fit {
  typedef T Type;
  static constexpr uint32_t kEntries = PAST ? 16 / kEntry<T> : 8;  // of a chunk
  static constexpr uint32_t kGroup = GROUP, kEights = KEEP, kKeep = KEEP * 8 / kEntries;
  static constexpr bool kPast = PAST, kAheadBackward = GROUP <= 64 || KEEP <= 3;  // with more, the backward pass has no registers to load ahead
  static constexpr uint32_t kBlock = 512, kGroups = kBlock / GROUP;  // of the backward pass
};
// SUMS sums over a row, in an order that does not depend on where rows lie.  bf16: a thread's entries, one after the other; the group's
// threads in pairs, fours and so on up to 64; the waves.  fp32, whose chunks are 8 entries or 4: of a thread's chunks of 8 the first fours, one
// after the other, and the second ones; the two; threads and waves as above.
//
// Where a chunk is 4, the two fours of 8 are neighbouring lanes'.  Eight number l + GROUP k, thread l's chunk k where chunks are 8, is two lanes'
// chunk 2 k if l is in the lower half of the group, and 2 k + 1 if not: a thread has the first, or second, fours of two threads, and
// two waves together have those of 64.
template <typename F, uint32_t SUMS>
struct RowSums {
  static constexpr bool kFours = __is_same(typename F::Type, F32), kShared = F::kEntries == 4;
  static constexpr uint32_t kOwn = kFours ? 2 : 1, kLeft = kShared ? 2 : 1;  // a thread's sums, and those that a wave leaves
  float v[SUMS][kOwn];
  typedef float Slot[SUMS * kLeft];  // of LDS, one for each wave of the block
  __device__ __forceinline__ RowSums() {
#pragma unroll
    for (uint32_t s = 0; s < SUMS; ++s)
#pragma unroll
      for (uint32_t h = 0; h < kOwn; ++h) v[s][h] = 0.0f;
  }
  // What entry i of a thread's chunk k is added to.
  __device__ __forceinline__ float &of(uint32_t s, uint32_t k, uint32_t i) { return v[s][kShared ? k % 2 : kFours ? i / 4 : 0]; }
  // The sums, in all threads of the group.  All threads of the block come here.
  __device__ __forceinline__ void group(float (&out)[SUMS], Slot *lds) {
    constexpr uint32_t kLanes = F::kGroup < 64 ? F::kGroup : 64, kWaves = F::kGroup / 64;
    const uint32_t wave = threadIdx.x >> 6;
    if constexpr (kShared && SUMS == 2 && kWaves > 1) {
      // four sums: within rows of 16 lanes each, then a swap of rows adds up two of them at once, one of halves all four, which leaves a row each
      float w[4];
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) w[i] = lanes_sum<16>(v[i / 2][i % 2]);
      const float all = halves_sum(rows_sum(w[0], w[1]), rows_sum(w[2], w[3]));
      __syncthreads();  // the last sums have been read
      if ((threadIdx.x & 15u) == 0) lds[wave][(threadIdx.x & 63u) >> 4] = all;
    } else {
      float w[SUMS][kLeft];
#pragma unroll
      for (uint32_t s = 0; s < SUMS; ++s) {
        if constexpr (kShared) {
          w[s][0] = lanes_sum<kLanes>(v[s][0]);
          w[s][1] = lanes_sum<kLanes>(v[s][1]);
        } else {
          w[s][0] = lanes_sum<kLanes>(kFours ? v[s][0] + v[s][kOwn - 1] : v[s][0]);
        }
      }
      if constexpr (kWaves <= 1) {
#pragma unroll
        for (uint32_t s = 0; s < SUMS; ++s) out[s] = kShared ? w[s][0] + w[s][kLeft - 1] : w[s][0];
      } else {
        __syncthreads();  // the last sums have been read
        if ((threadIdx.x & 63u) == 0) {
#pragma unroll
          for (uint32_t s = 0; s < SUMS; ++s)
#pragma unroll
            for (uint32_t h = 0; h < kLeft; ++h) lds[wave][s * kLeft + h] = w[s][h];
        }
      }
    }
    if constexpr (kWaves > 1) {
      const uint32_t first = wave / kWaves * kWaves;
      __syncthreads();
#pragma unroll
      for (uint32_t s = 0; s < SUMS; ++s) {
        out[s] = 0.0f;
#pragma unroll
        for (uint32_t h = 0; h < kLeft; ++h)
#pragma unroll
          for (uint32_t i = 0; i < kWaves; i += kLeft)
            out[s] += kShared ? lds[first + i][s * kLeft + h] + lds[first + i + kLeft - 1][s * kLeft + h] : lds[first + i][s];
      }
    }
  }
};

// A weight (or a bias) as the threads of a group read it, a chunk at a time: from registers, or, where a wave has a row and many
// rows pass, from LDS, which leaves registers for the next row.
template <typename F>
struct Weight {
  typedef __attribute__((address_space(3))) af32x4 lds_quad;
  static constexpr bool kInLds = F::kGroup <= 64;
  static constexpr uint32_t N = F::kEntries, kChunks = F::kGroup * F::kKeep, kLds = kInLds ? kChunks * N : 4;  // floats
  float v[kInLds ? 1 : F::kKeep][N];
  uint32_t lds;
  __device__ __forceinline__ Weight(const void *w, uint32_t bf16, uint32_t cols, float otherwise, float *buffer)
      : lds((uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)buffer) {
    if constexpr (!kInLds) {
#pragma unroll
      for (uint32_t k = 0; k < F::kKeep; ++k) weights_at(w, bf16, (threadIdx.x % F::kGroup + k * F::kGroup) * N, cols, otherwise, v[k]);
    } else {  // the chunks' first four, then their second ones: 16 bytes a lane, side by side
      for (uint32_t c = threadIdx.x; c < kChunks; c += blockDim.x) {
        float u[N];
        weights_at(w, bf16, c * N, cols, otherwise, u);
#pragma unroll
        for (uint32_t h = 0; h < N / 4; ++h) *reinterpret_cast<lds_quad *>(lds + (h * kChunks + c) * 16) = af32x4{u[4 * h], u[4 * h + 1], u[4 * h + 2], u[4 * h + 3]};
      }
    }
  }
  __device__ __forceinline__ void get(uint32_t k, uint32_t chunk, float (&u)[N]) const {
    if constexpr (kInLds) {
#pragma unroll
      for (uint32_t h = 0; h < N / 4; ++h) {
        const af32x4 a = *reinterpret_cast<const lds_quad *>(lds + (h * kChunks + chunk) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[4 * h + i] = a[i];
      }
    } else {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) u[i] = v[k][i];
    }
  }
};

template <typename F>
__global__ __launch_bounds__(F::kGroup < 256 ? 256 : F::kGroup) void k_norm(NormIn in, Rows y, CkptOut saved, float *mean, float *rstd) {
  typedef typename F::Type T;
  typedef RowSums<F, 1> Sum;
  constexpr uint32_t N = F::kEntries, kBlock = F::kGroup < 256 ? 256 : F::kGroup, kGroups = kBlock / F::kGroup;
  __shared__ __attribute__((aligned(16))) typename Sum::Slot lds[kBlock / 64];
  __shared__ __attribute__((aligned(16))) float weights[2][Weight<F>::kLds];
  const uint32_t chunks = (uint32_t)(ckpt_pitch(in.cols) / N), me = threadIdx.x % F::kGroup, cols = (uint32_t)in.cols;
  const float inv = 1.0f / (float)in.cols;
  const Weight<F> w(in.weight, in.bf16, cols, 1.0f, weights[0]), b(in.bias, in.bf16, cols, 0.0f, weights[1]);
  if constexpr (Weight<F>::kInLds) __syncthreads();
  Raw<T, N> next[F::kKeep];
  auto load = [&](uint64_t r) {
    const uint8_t *x = static_cast<const uint8_t *>(in.x.data) + r * in.x.ld * kEntry<T>;
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      const uint32_t c = me + k * F::kGroup;
      next[k] = Raw<T, N>{};
      if (r < in.rows && c < chunks) next[k] = load_raw<T, N, F::kPast>(x, c * N, cols);
    }
  };
  const uint64_t step = (uint64_t)gridDim.x * kGroups;
  uint64_t r = (uint64_t)blockIdx.x * kGroups + threadIdx.x / F::kGroup;
  load(r);
  for (uint64_t first = (uint64_t)blockIdx.x * kGroups; first < in.rows; first += step, r += step) {
    const bool here = r < in.rows;
    float v[F::kKeep][N], s[1];
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) widen(next[k], v[k]);
    load(r + step);
    Sum sum;
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k)
#pragma unroll
      for (int i = 0; i < (int)N; ++i) sum.of(0, k, i) += v[k][i];
    sum.group(s, lds);
    const float m = s[0] * inv;
    Sum squares;
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      int left = (int)cols - (int)((me + k * F::kGroup) * N);  // of the row from this chunk on
      asm volatile("" : "+v"(left));                            // (compared here, not in front of the loop, which would take 64 masks)
      if (left >= (int)N) {
#pragma unroll
        for (int i = 0; i < (int)N; ++i) {
          const float d = v[k][i] - m;
          squares.of(0, k, i) = fmaf(d, d, squares.of(0, k, i));
        }
      } else if (left > 0) {
#pragma unroll
        for (int i = 0; i < (int)N; ++i) {
          const float d = i < left ? v[k][i] - m : 0.0f;
          squares.of(0, k, i) = fmaf(d, d, squares.of(0, k, i));
        }
      }
    }
    squares.group(s, lds);
    if (!here) continue;
    const float scale = 1.0f / sqrtf(fmaf(s[0], inv, in.eps));
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      const uint32_t c = me + k * F::kGroup;
      if (c >= chunks) continue;
      if (saved.codes) ckpt_store(saved, r * chunks + c, v[k]);
      float wk[N], bk[N];
      w.get(k, c, wk);
      b.get(k, c, bk);
#pragma unroll
      for (int i = 0; i < (int)N; ++i) v[k][i] = fmaf((v[k][i] - m) * scale, wk[i], bk[i]);
      store_entries<T, N, F::kPast>(static_cast<uint8_t *>(y.data) + r * y.ld * kEntry<T>, c * N, cols, v[k]);
    }
    if (me == 0 && mean) {
      mean[r] = m;
      rstd[r] = scale;
    }
  }
}

// Longer rows: a block per row, which it reads three times (the second and third time from the cache).
template <typename T>
__global__ __launch_bounds__(kWideThreads) void k_norm_wide(NormIn in, Rows y, CkptOut saved, float *mean, float *rstd) {
  __shared__ float lds[2 * kWideThreads / 64];
  const uint64_t chunks = ckpt_pitch(in.cols) / 8;
  const float inv = 1.0f / (float)in.cols;
  for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
    const uint8_t *x = static_cast<const uint8_t *>(in.x.data) + r * in.x.ld * kEntry<T>;
    float v[8], s = 0.0f, s2 = 0.0f;
    for (uint64_t c = threadIdx.x; c < chunks; c += kWideThreads) {
      load8<T>(x, c * 8, in.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    block_sums(s, s2, lds);
    const float m = s * inv;
    s = s2 = 0.0f;
    for (uint64_t c = threadIdx.x; c < chunks; c += kWideThreads) {
      load8<T>(x, c * 8, in.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = c * 8 + i < in.cols ? v[i] - m : 0.0f;
        s = fmaf(d, d, s);
      }
    }
    block_sums(s, s2, lds);
    const float k = 1.0f / sqrtf(fmaf(s, inv, in.eps));
    for (uint64_t c = threadIdx.x; c < chunks; c += kWideThreads) {
      float w[8], b[8];
      load8<T>(x, c * 8, in.cols, v);
      if (saved.codes) ckpt_store(saved, r * chunks + c, v);
      weights_at(in.weight, in.bf16, c * 8, in.cols, 1.0f, w);
      weights_at(in.bias, in.bf16, c * 8, in.cols, 0.0f, b);
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
  uint32_t bf16;
};

// The backward pass of rows that stay in registers, with the sums over rows beside: a thread's columns are the same in all of its
// rows, so it sums them up as they pass; at the end the block's groups add up and the block's sums go to `part`
// ([blocks][2][pitch]).  One block of 512 threads to a CU (8 waves have what it takes in flight), so that there are few.
template <typename F>
__global__ __launch_bounds__(F::kBlock) void k_norm_grad(NormGrad in, float *part) {
  typedef typename F::Type T;
  constexpr uint32_t N = F::kEntries;
  typedef RowSums<F, 2> Sums;
  constexpr bool kAhead = F::kAheadBackward;
  __shared__ __attribute__((aligned(16))) typename Sums::Slot lds[F::kBlock / 64];
  __shared__ __attribute__((aligned(16))) float weights[Weight<F>::kLds], columns[F::kGroups > 1 ? F::kGroups / 2 * F::kGroup * F::kKeep * N * 2 : 4];
  const uint32_t chunks = (uint32_t)(ckpt_pitch(in.cols) / N), me = threadIdx.x % F::kGroup, group = threadIdx.x / F::kGroup, cols = (uint32_t)in.cols;
  const float inv = 1.0f / (float)in.cols;
  const Weight<F> w(in.weight, in.bf16, cols, 1.0f, weights);
  if constexpr (Weight<F>::kInLds) __syncthreads();
  float dw[F::kKeep][N], db[F::kKeep][N];
#pragma unroll
  for (uint32_t k = 0; k < F::kKeep; ++k)
#pragma unroll
    for (int i = 0; i < (int)N; ++i) dw[k][i] = db[k][i] = 0.0f;
  Raw<T, N> next[F::kKeep];
  CkptCodes<N> codes[F::kKeep];
  uint32_t scales[F::kKeep];
  float next_m, next_scale;
  auto load = [&](uint64_t r) {
    const bool here = r < in.rows;
    next_m = next_scale = 0.0f;
    if (here) {
      next_m = a_ld<float>(in.mean + r);
      next_scale = a_ld<float>(in.rstd + r);
    }
    const uint8_t *dy = static_cast<const uint8_t *>(in.dy.data) + r * in.dy.ld * kEntry<T>;
    uint32_t at = me;
    if constexpr (Sums::kShared && !kAhead) asm volatile("" : "+v"(at));  // (the chunks' places are worked out here, not kept in registers between rows)
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      const uint32_t c = at + k * F::kGroup;
      next[k] = Raw<T, N>{};
      codes[k] = CkptCodes<N>{};
      scales[k] = kCkptLeast;
      if (here && c < chunks) {
        next[k] = load_raw<T, N, F::kPast>(dy, c * N, cols);
        codes[k] = a_ld<CkptCodes<N>>(in.x.codes + (r * chunks + c) * N);
        scales[k] = a_ld<uint8_t>(in.x.scales + (r * chunks + c) / (kCkptBlock / N));
      }
    }
  };
  const uint64_t step = (uint64_t)gridDim.x * F::kGroups;
  uint64_t r = (uint64_t)blockIdx.x * F::kGroups + group;
  if (kAhead) load(r);
  for (uint64_t first = (uint64_t)blockIdx.x * F::kGroups; first < in.rows; first += step, r += step) {
    const bool here = r < in.rows;
    if (!kAhead) load(r);
    float g[F::kKeep][N], n[F::kKeep][N], s[2];
    const float m = next_m, scale = next_scale;
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      widen(next[k], g[k]);
      ckpt_decode(codes[k], scales[k], n[k]);
    }
    if (kAhead) load(r + step);
    Sums sums;  // of q and of q n
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      float wk[N];
      w.get(k, me + k * F::kGroup, wk);
#pragma unroll
      for (int i = 0; i < (int)N; ++i) {
        n[k][i] = (n[k][i] - m) * scale;
        dw[k][i] = fmaf(g[k][i], n[k][i], dw[k][i]);
        db[k][i] += g[k][i];
        g[k][i] *= wk[i];
        sums.of(0, k, i) += g[k][i];
        sums.of(1, k, i) = fmaf(g[k][i], n[k][i], sums.of(1, k, i));
      }
    }
    sums.group(s, lds);
    if (!here) continue;
    s[0] *= inv;
    s[1] *= inv;
#pragma unroll
    for (uint32_t k = 0; k < F::kKeep; ++k) {
      const uint32_t c = me + k * F::kGroup;
      if (c >= chunks) continue;
#pragma unroll
      for (int i = 0; i < (int)N; ++i) g[k][i] = scale * ((g[k][i] - s[0]) - n[k][i] * s[1]);
      store_entries<T, N, F::kPast>(static_cast<uint8_t *>(in.dx.data) + r * in.dx.ld * kEntry<T>, c * N, cols, g[k]);
    }
  }
  if (!part) return;
  float *out = part + (uint64_t)blockIdx.x * 2 * chunks * N;
  // The upper half of the groups leaves its sums in LDS, the lower half adds them, until one group has them all.
  typedef __attribute__((address_space(3))) af32x4 lds_quad;
  constexpr uint32_t kSlot = F::kGroup * F::kKeep * N / 2;  // quads of a group's sums, dw's then db's, as the weights lie: 16 bytes a lane, side by side
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)columns + me * 16;
#pragma unroll
  for (uint32_t half = F::kGroups / 2; half; half /= 2) {
    const bool gives = group >= half && group < 2 * half, takes = group < half;
    const uint32_t slot = base + (gives ? group - half : group) * (kSlot * 16);
    if (gives) {
#pragma unroll
      for (uint32_t k = 0; k < F::kKeep; ++k)
#pragma unroll
        for (int h = 0; h < (int)N / 4; ++h) {
          lds_quad *at = reinterpret_cast<lds_quad *>(slot + (h * F::kKeep + k) * (F::kGroup * 16));
          *at = af32x4{dw[k][4 * h], dw[k][4 * h + 1], dw[k][4 * h + 2], dw[k][4 * h + 3]};
          at[kSlot / 2] = af32x4{db[k][4 * h], db[k][4 * h + 1], db[k][4 * h + 2], db[k][4 * h + 3]};
        }
    }
    __syncthreads();
    if (takes) {
#pragma unroll
      for (uint32_t k = 0; k < F::kKeep; ++k)
#pragma unroll
        for (int h = 0; h < (int)N / 4; ++h) {
          const lds_quad *at = reinterpret_cast<const lds_quad *>(slot + (h * F::kKeep + k) * (F::kGroup * 16));
          const af32x4 a = *at, b = at[kSlot / 2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dw[k][4 * h + i] += a[i];
            db[k][4 * h + i] += b[i];
          }
        }
    }
    __syncthreads();
  }
  if (group) return;
#pragma unroll
  for (uint32_t k = 0; k < F::kKeep; ++k) {
    const uint32_t c = me + k * F::kGroup;
    if (c >= chunks) continue;
#pragma unroll
    for (int h = 0; h < (int)N / 4; ++h) {
      a_st<af32x4>(out + c * N + 4 * h, af32x4{dw[k][4 * h], dw[k][4 * h + 1], dw[k][4 * h + 2], dw[k][4 * h + 3]});
      a_st<af32x4>(out + (chunks + c) * N + 4 * h, af32x4{db[k][4 * h], db[k][4 * h + 1], db[k][4 * h + 2], db[k][4 * h + 3]});
    }
  }
}

// Longer rows, in two kernels.
template <typename T>
__global__ __launch_bounds__(kWideThreads) void k_norm_grad_wide(NormGrad in) {
  __shared__ float lds[2 * kWideThreads / 64];
  const uint64_t chunks = ckpt_pitch(in.cols) / 8;
  const float inv = 1.0f / (float)in.cols;
  for (uint64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
    const uint8_t *dy = static_cast<const uint8_t *>(in.dy.data) + r * in.dy.ld * kEntry<T>;
    const float m = in.mean[r], k = in.rstd[r];
    float x[8], q[8], w[8], s = 0.0f, sn = 0.0f;
    for (uint64_t c = threadIdx.x; c < chunks; c += kWideThreads) {
      load8<T>(dy, c * 8, in.cols, q);  // zero behind the row's end
      ckpt_load(in.x, r * chunks + c, x);
      weights_at(in.weight, in.bf16, c * 8, in.cols, 1.0f, w);
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
    for (uint64_t c = threadIdx.x; c < chunks; c += kWideThreads) {
      load8<T>(dy, c * 8, in.cols, q);
      ckpt_load(in.x, r * chunks + c, x);
      weights_at(in.weight, in.bf16, c * 8, in.cols, 1.0f, w);
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
    ckpt_load(in.x, r * chunks + c, x);
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

constexpr uint32_t kRowBlocks = 512;  // blocks that longer rows are dealt to
uint32_t row_blocks(uint64_t rows) { return (uint32_t)(rows < kRowBlocks ? rows : kRowBlocks); }

// How rows are kept: threads to a row and chunks to a thread (group 0: the row is too long).  Measured, forward and backward:
// (through the caches) 16384 x 2056 in bf16 takes 89 us by groups of 128, 116 by 256; 4096 x 16384 169 us by groups of 512 that load ahead,
// 185 by 1,024 that have no registers for it; 200000 x 128 59 us by groups of 16, 150 by 64.  Few rows are shared by more threads: the two
// kernels take 6 and 11 us for 1024 x 2048 by groups of 64, 6 and 7 by 256 (256 rows: 5 and 10, 4 and 4; 3000: 10 and 15, 11 and 12; 6000: 14
// and 18, 17 and 19), for 2000 x 1024 5 and 7 by 64, 7 and 8 by 256.  Rows of 1,025 to 2,048 entries: bf16 8192 x 2048 42 us by 64, 43 by 128
// (8192 x 2047 48 and 57); fp32, whose next row takes twice the registers, 72 by 64 (the backward pass then spills), 63 by 128.  Longer rows that
// three chunks of 128 threads hold, the two calls by 128 and by 256: bf16 1000 x 3000 8 and 14, 8 and 14; 2048 rows 11 and 16, 13 and 17; 3000 13 and 18,
// 15 and 21; 8000 24 and 33, 26 and 40; fp32 1000 10 and 15, 9 and 15; 2048 14 and 19, 13 and 20; 4000 20 and 28, 21 and 29; 8000 39 and 49, 39 and 54.
struct Kept {
  uint32_t group, keep;
};
Kept kept(uint64_t rows, uint64_t cols, bool f32) {
  const uint64_t chunks = ckpt_pitch(cols) / 8;
  const uint64_t few = chunks <= 128 ? 1024 : 4096;
  uint32_t group = 512;
  if (chunks <= 64) group = chunks <= 16 ? 16 : chunks <= 32 ? 32 : 64;
  else if (chunks <= 256) group = rows < few ? 256 : f32 && chunks > 128 ? 128 : 64;
  else if (chunks <= 1024) group = chunks <= 384 && rows >= 2048 ? 128 : 256;
  uint32_t keep = group == 128 && chunks > 256 ? 3 : 1;
  while (keep < 4 && (uint64_t)group * keep < chunks) keep += group == 64 && keep == 2 ? 2 : 1;
  if ((uint64_t)group * keep < chunks) group = 0;
  return {group, keep};
}
// Parts of the sums over rows: blocks of the backward pass (Fit::kGroups rows at a time), or slices of the rows.  256, an MI355X's CUs, whatever the
// device has: the sums' order and the scratch memory follow from sizes alone.
uint32_t norm_parts(uint64_t rows, uint64_t cols) {
  const Kept k = kept(rows, cols, false);  // (fp32 differs only where there are rows enough for 256 parts either way)
  const uint64_t at_once = k.group == 0 ? 8 : k.group < 512 ? 512 / k.group : 1, parts = (rows + at_once - 1) / at_once;
  return (uint32_t)(parts < 256 ? parts : 256);
}
// As many blocks as an MI355X keeps by their registers.  One block more to a CU, and one fewer: forward pass, fp32 8192 x 8192 (two to a CU) 119
// and 147 us, 108 as it is; 16384 x 3000 (three) 94 and 88, 88; bf16 50 and 56, 49; 8192 x 6000 (three) 49 and 55, 49; 100000 x 512 (four; eight
// for more) 52 and 55, 52; 4096 x 16384 (one; two for more) 75, 75.
template <typename F>
hipError_t run_norm(const NormIn &in, const Rows &y, const CkptOut &saved, float *mean, float *rstd, hipStream_t s) {
  constexpr uint32_t kBlock = F::kGroup < 256 ? 256 : F::kGroup, kGroups = kBlock / F::kGroup;
  const uint64_t blocks = (in.rows + kGroups - 1) / kGroups, most = 256 * (kBlock > 256 ? 1 : F::kGroup == 256 && F::kEights > 2 ? 6 - F::kEights : F::kGroup == 128 ? 3 : 4);
  hipLaunchKernelGGL((k_norm<F>), dim3((uint32_t)(blocks < most ? blocks : most)), dim3(kBlock), 0, s, in, y, saved, mean, rstd);
  return hipGetLastError();
}
template <typename F>
hipError_t run_norm_grad(const NormGrad &in, float *part, uint32_t parts, hipStream_t s) {
  hipLaunchKernelGGL((k_norm_grad<F>), dim3(parts), dim3(F::kBlock), 0, s, in, part);
  return hipGetLastError();
}
#define DQ_FIT(run, group, keep, ...) \
  case group * 8 + keep: return past ? run<Fit<T, group, keep, true>>(__VA_ARGS__) : run<Fit<T, group, keep, false>>(__VA_ARGS__);
#define DQ_FITS(run, ...)                                                                                             \
  switch (k.group * 8 + k.keep) {                                                                                     \
    DQ_FIT(run, 16, 1, __VA_ARGS__) DQ_FIT(run, 32, 1, __VA_ARGS__)                                                   \
    DQ_FIT(run, 64, 1, __VA_ARGS__) DQ_FIT(run, 64, 2, __VA_ARGS__)                                                   \
    case 64 * 8 + 4:                                                                                                  \
      if constexpr (__is_same(T, Bf16)) return past ? run<Fit<T, 64, 4, true>>(__VA_ARGS__) : run<Fit<T, 64, 4, false>>(__VA_ARGS__); \
      break;                                                                                                          \
    case 128 * 8 + 2:                                                                                                 \
      if constexpr (__is_same(T, F32)) return past ? run<Fit<T, 128, 2, true>>(__VA_ARGS__) : run<Fit<T, 128, 2, false>>(__VA_ARGS__); \
      break;                                                                                                          \
    case 256 * 8 + 1: return run<Fit<T, 256, 1, false>>(__VA_ARGS__); /* few rows: never large */                     \
    DQ_FIT(run, 128, 3, __VA_ARGS__)                                                                                  \
    DQ_FIT(run, 256, 2, __VA_ARGS__) DQ_FIT(run, 256, 3, __VA_ARGS__) DQ_FIT(run, 256, 4, __VA_ARGS__) \
    DQ_FIT(run, 512, 3, __VA_ARGS__) DQ_FIT(run, 512, 4, __VA_ARGS__)                                                 \
  }
template <typename T>
hipError_t norm_forward(bool past, const NormIn &in, const Rows &y, const CkptOut &saved, float *mean, float *rstd, hipStream_t s) {
  const Kept k = kept(in.rows, in.cols, __is_same(T, F32));
  DQ_FITS(run_norm, in, y, saved, mean, rstd, s)
  hipLaunchKernelGGL((k_norm_wide<T>), dim3(row_blocks(in.rows)), dim3(kWideThreads), 0, s, in, y, saved, mean, rstd);
  return hipGetLastError();
}
// part: null if nobody wants the sums over rows.
template <typename T>
hipError_t norm_backward(bool past, const NormGrad &in, float *part, uint32_t parts, hipStream_t s) {
  const Kept k = kept(in.rows, in.cols, __is_same(T, F32));
  DQ_FITS(run_norm_grad, in, part, parts, s)
  hipLaunchKernelGGL((k_norm_grad_wide<T>), dim3(row_blocks(in.rows)), dim3(kWideThreads), 0, s, in);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  const dim3 grid((uint32_t)((ckpt_pitch(in.cols) / 8 + kThreads - 1) / kThreads), parts);
  hipLaunchKernelGGL((k_norm_columns<T>), grid, dim3(kThreads), 0, s, in, (in.rows + parts - 1) / parts, part);
  return hipGetLastError();
}

bool goes_past(const dq_matrix *a, const dq_matrix *b, uint64_t rows, uint64_t cols, uint64_t least) {
  return on_16(a, rows) && on_16(b, rows) && 2 * rows * cols * entry_bytes(a->dtype) >= least;
}
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
  const NormIn in = {{x->data, x->ld}, rows, cols, weight, bias, (uint32_t)(weight_dtype == DQ_BF16), eps};
  const Rows out = {y->data, y->ld};
  const CkptOut saved = ckpt_out(ckpt, rows, cols);
  hipStream_t s = (hipStream_t)hip_stream;
  const bool past = goes_past(x, y, rows, cols, 2 * kPastBytes);
  return hip_status(x->dtype == DQ_F32 ? norm_forward<F32>(past, in, out, saved, mean, rstd, s) : norm_forward<Bf16>(past, in, out, saved, mean, rstd, s));
}

size_t dq_layer_norm_grad_scratch_bytes(uint64_t rows, uint64_t cols) {
  if (dq_ckpt_bytes(rows, cols) == 0 || cols >> 31) return 0;
  return (size_t)norm_parts(rows, cols) * 2 * ckpt_pitch(cols) * 4;
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
  const uint32_t parts = rows ? norm_parts(rows, cols) : 0, join_blocks = join_grid(pitch);
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
    const NormGrad in = {{dy->data, dy->ld}, {dx->data, dx->ld}, rows, cols, ckpt_in(ckpt, rows, cols), mean, rstd, weight, (uint32_t)(weight_dtype == DQ_BF16)};
    float *part = dweight ? static_cast<float *>(scratch) : nullptr;
    const bool past = goes_past(dy, dx, rows, cols, kPastBytes);
    DQ_TRY(hip_status(dy->dtype == DQ_F32 ? norm_backward<F32>(past, in, part, parts, s) : norm_backward<Bf16>(past, in, part, parts, s)));
    if (!dweight) return DQ_OK;
  }
  if (weight_dtype == DQ_F32)
    hipLaunchKernelGGL((k_norm_join<F32>), dim3(join_blocks), dim3(kJoinThreads), 0, s, (const float *)scratch, pitch, cols, parts, dweight, dbias,
                       (uint32_t)(accumulate != 0));
  else
    hipLaunchKernelGGL((k_norm_join<Bf16>), dim3(join_blocks), dim3(kJoinThreads), 0, s, (const float *)scratch, pitch, cols, parts, dweight, dbias,
                       (uint32_t)(accumulate != 0));
  return hip_status(hipGetLastError());
}

}  // extern "C"
