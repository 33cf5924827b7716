// 8-bit activation checkpoints (save, load) and the activation between two linear layers, which saves its inputs as it reads them
// and whose backward pass reads them from there.
//
// All are streams: every entry is read once and written once, a few dozen operations each, so memory bounds them.  Measured: a
// checkpoint of bf16 16384 x 8192, saved and loaded, 134 us (6.1 TB/s), SiLU with a gate there, forward and backward, 351 us (6.1), GELU
// at 16384 x 4096 128 us (5.3; with a gate 177, 6.1); rows off 16-byte borders up to 40 % more.
#include <atomic>
#include <initializer_list>

#include "act_rows.h"

namespace dq {
namespace {

constexpr uint32_t kMapThreads = 256;

// Here a lane's chunk is 16 bytes of a row, so that a wave's loads and stores each cover memory without gaps: 8 entries of bf16, 4 of
// binary32 (with 8 of them, 32 bytes, half of each line a store touched came with the next one: 16384 x 4096, saved and loaded through
// the caches, took 174 us, not 146).
template <typename T>
constexpr uint32_t kChunk = 16 / kEntry<T>;
template <typename T>
struct Chunk {
  float v[kChunk<T>];
};
template <typename T, bool PAST>
__device__ __forceinline__ Chunk<T> load_chunk(const void *row, uint64_t at, uint64_t cols) {
  Chunk<T> c;
  widen(load_raw<T, kChunk<T>, PAST>(row, at * kChunk<T>, cols), c.v);
  return c;
}
template <typename T>
__device__ __forceinline__ Chunk<T> saved_chunk(const CkptIn &in, uint64_t n) {
  Chunk<T> c;
  ckpt_load(in, n, c.v);
  return c;
}

// The chunks of a matrix, in order, dealt to the threads; rows that lie back to back are one long row (the host sees to it).
struct Walk8 {
  uint64_t chunks;             // in all
  uint64_t per_row;            // of a row
  uint64_t cols;
  uint64_t step_rows, step_at; // a step of the whole grid, as rows and chunks
};
struct At {
  uint64_t row, at, chunk;
  __device__ __forceinline__ At(const Walk8 &w) {
    chunk = (uint64_t)blockIdx.x * kMapThreads + threadIdx.x;
    if (w.chunks >> 32) {
      row = chunk / w.per_row;
      at = chunk - row * w.per_row;
    } else {
      row = (uint32_t)chunk / (uint32_t)w.per_row;
      at = (uint32_t)chunk - (uint32_t)row * (uint32_t)w.per_row;
    }
  }
  __device__ __forceinline__ void next(const Walk8 &w) {
    chunk += (uint64_t)gridDim.x * kMapThreads;
    row += w.step_rows;
    at += w.step_at;
    if (at >= w.per_row) {
      at -= w.per_row;
      ++row;
    }
  }
};
template <typename T>
__device__ __forceinline__ uint8_t *row_of(const Rows &m, uint64_t row) {
  return static_cast<uint8_t *>(m.data) + row * m.ld * kEntry<T>;
}

template <typename T, bool PAST>
__global__ __launch_bounds__(kMapThreads) void k_ckpt_save(Walk8 w, Rows x, CkptOut out) {
  for (At i(w); i.chunk < w.chunks; i.next(w)) {
    ckpt_store(out, i.chunk, load_chunk<T, PAST>(row_of<T>(x, i.row), i.at, w.cols).v);
  }
}
template <typename T, bool PAST>
__global__ __launch_bounds__(kMapThreads) void k_ckpt_load(Walk8 w, CkptIn in, Rows x) {
  for (At i(w); i.chunk < w.chunks; i.next(w)) {
    store_entries<T, kChunk<T>, PAST>(row_of<T>(x, i.row), i.at * kChunk<T>, w.cols, saved_chunk<T>(in, i.chunk).v);
  }
}

// a = act(z), d = act'(z).  The exponential and the reciprocal are the hardware's: over whole octaves they were off by 1.42 and 1.53 half
// steps at most, 0.58 and 0.48 in the mean square; what would be a subnormal number they make zero.
template <typename T, int KIND>
__device__ __forceinline__ void activation(float z, float *a, float *d) {
  if constexpr (KIND == DQ_SILU) {  // z p with p = 1 / (1 + e^-z); the derivative is p + z p (1 - p)
    float p;
    if constexpr (__is_same(T, F32)) {
      // -z log2 e is x + rest, x as rounded: p(x + rest) is p + p (p - 1) rest ln 2.  Without the rest e^-z would be off by |z| half steps
      // (which a bf16 result, of 2^16 times larger steps, does not show).  Beyond +-100 p is zero or one, and rest might not be finite.
      const float c = __builtin_amdgcn_fmed3f(z, -100.0f, 100.0f), x = c * -1.44269504f;
      const float rest = fmaf(c, -1.92596299e-8f, fmaf(c, -1.44269504f, -x));
      p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x));
      p = fmaf(p * (p - 1.0f), rest * 0.693147181f, p);
    } else {
      p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
    }
    *a = z * p;
    *d = p * fmaf(z, 1.0f - p, 1.0f);
  } else {
    // z p with p the normal distribution's value at z; the derivative is p + z times its density.  Both need E = e^(-z^2 / 2): below
    // zero p = E t P(t), t = 1 / (1 + 0.3 |z| / sqrt 2), and above it 1 - that.  P is half of erfcx(|z| / sqrt 2) / t, fitted as a
    // polynomial of degree 8 with the smallest largest relative error over |z| < 17 (iteratively reweighted least squares; 4.6e-8 with
    // its coefficients in binary32).  One call each of erfcf and expf took 1.6 times as long in all as the memory did.
    // E is a square, so that it is not cut off below the least normal number; 24 added to the exponent instead, and taken off again, rounds
    // the exponent to 2^-20 and E by 11 half steps.  For -1 < z < 0 p is off by 3 half steps in the mean square; E's argument adds z^2.
    const float root = __builtin_amdgcn_exp2f(z * z * -0.36067376f), E = root * root;
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.212132037f, 1.0f));
    float P = -0.0646262318f;
    P = fmaf(P, t, 0.242149144f);
    P = fmaf(P, t, -0.254882902f);
    P = fmaf(P, t, 0.272480011f);
    P = fmaf(P, t, -0.0464108214f);
    P = fmaf(P, t, 0.107089855f);
    P = fmaf(P, t, 0.0742608309f);
    P = fmaf(P, t, 0.0853454396f);
    P = fmaf(P, t, 0.0845946819f);
    const float tail = E * t * P;
    float p = z < 0.0f ? tail : 1.0f - tail;
    if constexpr (__is_same(T, F32)) {
      // Near zero t's rounding counts 3.8 times in p, and 0.5 + z Q(z^2) is better: Q of degree 4, fitted as P was, 5.2e-8 with its
      // coefficients in binary32.  z p for -1 < z < 0 is off by 0.8 half steps in the mean square, 2.5 without.
      const float w = z * z;
      float Q = 9.4235198e-05f;
      Q = fmaf(Q, w, -0.00116935337f);
      Q = fmaf(Q, w, 0.00996719673f);
      Q = fmaf(Q, w, -0.0664895847f);
      Q = fmaf(Q, w, 0.398942262f);
      p = fabsf(z) < 1.0f ? fmaf(z, Q, 0.5f) : p;
    }
    *a = z * p;
    *d = fmaf(z * 0.39894228040143268f, E, p);
  }
}

template <typename T, int KIND, bool GATED, bool SAVE, bool PAST>
__global__ __launch_bounds__(kMapThreads) void k_gate(Walk8 w, Rows z, Rows u, Rows h, CkptOut sz, CkptOut su) {
  for (At i(w); i.chunk < w.chunks; i.next(w)) {
    Chunk<T> a = load_chunk<T, PAST>(row_of<T>(z, i.row), i.at, w.cols), b;
    if constexpr (GATED) b = load_chunk<T, PAST>(row_of<T>(u, i.row), i.at, w.cols);
    if constexpr (SAVE) ckpt_store(sz, i.chunk, a.v);
    if constexpr (SAVE && GATED) ckpt_store(su, i.chunk, b.v);
#pragma unroll
    for (uint32_t k = 0; k < kChunk<T>; ++k) {
      float d;
      activation<T, KIND>(a.v[k], &a.v[k], &d);
      if constexpr (GATED) a.v[k] *= b.v[k];
    }
    store_entries<T, kChunk<T>, PAST>(row_of<T>(h, i.row), i.at * kChunk<T>, w.cols, a.v);
  }
}
template <typename T, int KIND, bool GATED, bool PAST>
__global__ __launch_bounds__(kMapThreads) void k_gate_grad(Walk8 w, Rows dh, CkptIn sz, CkptIn su, Rows dz, Rows du) {
  for (At i(w); i.chunk < w.chunks; i.next(w)) {
    const Chunk<T> g = load_chunk<T, PAST>(row_of<T>(dh, i.row), i.at, w.cols);
    Chunk<T> a = saved_chunk<T>(sz, i.chunk), b;
    if constexpr (GATED) b = saved_chunk<T>(su, i.chunk);
#pragma unroll
    for (uint32_t k = 0; k < kChunk<T>; ++k) {
      float act, d;
      activation<T, KIND>(a.v[k], &act, &d);
      if constexpr (GATED) {
        a.v[k] = g.v[k] * d * b.v[k];  // (dh u may be infinite where act' makes nothing of it)
        b.v[k] = g.v[k] * act;
      } else {
        a.v[k] = g.v[k] * d;
      }
    }
    store_entries<T, kChunk<T>, PAST>(row_of<T>(dz, i.row), i.at * kChunk<T>, w.cols, a.v);
    if constexpr (GATED) store_entries<T, kChunk<T>, PAST>(row_of<T>(du, i.row), i.at * kChunk<T>, w.cols, b.v);
  }
}

struct Map {
  Walk8 walk;
  uint32_t blocks;
  bool past;
};
// Rows back to back without padding in any operand are walked as one long row.
//
// Large matrices go past the caches: bf16 16384 x 8192, a checkpoint there and back 160 -> 134 us, SiLU with a gate and its gradient 431 -> 351; fp32 8192 x 4096, 62 -> 57.
// Below, and over odd rows, where lanes share lines, the caches help:
// fp32 4099 x 2051, 16.6 us, takes 18.0 past them.  A feed-forward block of 16384 tokens, its products included, gains 1 % forward and loses nothing.
Map plan_map(uint64_t rows, uint64_t cols, std::initializer_list<const dq_matrix *> m) {
  bool flat = cols % kCkptBlock == 0, even = true;
  for (const dq_matrix *x : m) {
    flat = flat && (rows == 1 || x->ld == cols);
    even = even && on_16(x, rows);
  }
  Map p;
  p.past = even && m.size() * rows * cols * entry_bytes((*m.begin())->dtype) >= kPastBytes;
  if (flat) {
    cols *= rows;
    rows = 1;
  }
  p.walk.per_row = ckpt_pitch(cols) * entry_bytes((*m.begin())->dtype) / 16;
  p.walk.chunks = rows * p.walk.per_row;
  p.walk.cols = cols;
  const uint64_t want = (p.walk.chunks + kMapThreads - 1) / kMapThreads, most = (uint64_t)device_cu_count() * 8;
  p.blocks = (uint32_t)(want < most ? want : most);
  const uint64_t step = (uint64_t)p.blocks * kMapThreads;
  p.walk.step_rows = step / p.walk.per_row;
  p.walk.step_at = step % p.walk.per_row;
  return p;
}
Rows rows_of(const dq_matrix *m) { return m ? Rows{m->data, m->ld} : Rows{nullptr, 0}; }

bool good_kind(dq_activation k) { return k == DQ_SILU || k == DQ_GELU; }
bool al16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

bool regions_meet(const Region *r, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j) {
      const Region &a = r[i], &b = r[j];
      if (!a.p || !b.p || (!a.written && !b.written) || !a.rows || !b.rows || !a.bytes || !b.bytes) continue;
      const uint64_t pa = (uint64_t)(uintptr_t)a.p, pb = (uint64_t)(uintptr_t)b.p;
      if (pa + (a.rows - 1) * a.stride + a.bytes <= pb || pb + (b.rows - 1) * b.stride + b.bytes <= pa) continue;
      if (a.rows > 1 && b.rows > 1 && a.stride == b.stride) {  // side by side in one wider matrix
        const uint64_t off = pb >= pa ? (pb - pa) % a.stride : (a.stride - (pa - pb) % a.stride) % a.stride;
        if (off >= a.bytes && off + b.bytes <= a.stride) continue;
      }
      return true;
    }
  return false;
}

dq_status check_matrix(const dq_matrix *m, uint64_t rows, uint64_t cols) {
  if (!m || (m->dtype != DQ_F32 && m->dtype != DQ_BF16)) return DQ_EINVAL;
  if (rows == 0 || cols == 0) return DQ_OK;
  if (!m->data || (rows > 1 && m->ld < cols)) return DQ_EINVAL;
  if ((uintptr_t)m->data % entry_bytes(m->dtype)) return DQ_EALIGN;
  const uint64_t most = 1ull << 46;  // entries from the first to the last
  if (cols > most || (rows > 1 && (m->ld > most || (rows - 1) > (most - cols) / m->ld))) return DQ_EUNSUPPORTED;
  return DQ_OK;
}

// Asked once per device and kept (the number of CUs does not change).
uint32_t device_cu_count() {
  static std::atomic<uint32_t> known[64];
  int device = 0;
  if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64) return 256;
  uint32_t n = known[device].load(std::memory_order_relaxed);
  if (n == 0) {
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || cus <= 0) return 256;
    known[device].store(n = (uint32_t)cus, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace dq

using namespace dq;

#define DQ_TRY(x)                     \
  do {                                \
    const dq_status st_ = (x);        \
    if (st_ != DQ_OK) return st_;     \
  } while (0)
// The kernel with its template arguments `of` (in parentheses), past the caches or not.
#define DQ_LIST(...) __VA_ARGS__
#define DQ_RUN(kernel, of, p, ...)                                                                                                                  \
  do {                                                                                                                                              \
    if ((p).past) hipLaunchKernelGGL((kernel<DQ_LIST of, true>), dim3((p).blocks), dim3(kMapThreads), 0, (hipStream_t)hip_stream, (p).walk, __VA_ARGS__); \
    else hipLaunchKernelGGL((kernel<DQ_LIST of, false>), dim3((p).blocks), dim3(kMapThreads), 0, (hipStream_t)hip_stream, (p).walk, __VA_ARGS__);    \
  } while (0)

extern "C" {

size_t dq_ckpt_bytes(uint64_t rows, uint64_t cols) {
  if (rows == 0 || cols == 0 || cols > (1ull << 46) || rows > (1ull << 46) / ckpt_pitch(cols)) return 0;
  const uint64_t codes = rows * ckpt_pitch(cols);
  return (size_t)(codes + codes / kCkptBlock);
}

dq_status dq_ckpt_save(const dq_matrix *x, uint64_t rows, uint64_t cols, void *ckpt, void *hip_stream) {
  DQ_TRY(check_matrix(x, rows, cols));
  if (rows == 0 || cols == 0) return DQ_OK;
  const size_t bytes = dq_ckpt_bytes(rows, cols);
  if (bytes == 0) return DQ_EUNSUPPORTED;
  if (!ckpt) return DQ_EINVAL;
  if (!al16(ckpt)) return DQ_EALIGN;
  const Region r[] = {region(x, rows, cols, false), region(ckpt, bytes, true)};
  if (regions_meet(r, 2)) return DQ_EINVAL;
  const Map p = plan_map(rows, cols, {x});
  if (x->dtype == DQ_F32) DQ_RUN(k_ckpt_save, (F32), p, rows_of(x), ckpt_out(ckpt, rows, cols));
  else DQ_RUN(k_ckpt_save, (Bf16), p, rows_of(x), ckpt_out(ckpt, rows, cols));
  return hip_status(hipGetLastError());
}

dq_status dq_ckpt_load(const void *ckpt, uint64_t rows, uint64_t cols, const dq_matrix *out, void *hip_stream) {
  DQ_TRY(check_matrix(out, rows, cols));
  if (rows == 0 || cols == 0) return DQ_OK;
  const size_t bytes = dq_ckpt_bytes(rows, cols);
  if (bytes == 0) return DQ_EUNSUPPORTED;
  if (!ckpt) return DQ_EINVAL;
  if (!al16(ckpt)) return DQ_EALIGN;
  const Region r[] = {region(ckpt, bytes, false), region(out, rows, cols, true)};
  if (regions_meet(r, 2)) return DQ_EINVAL;
  const Map p = plan_map(rows, cols, {out});
  if (out->dtype == DQ_F32) DQ_RUN(k_ckpt_load, (F32), p, ckpt_in(ckpt, rows, cols), rows_of(out));
  else DQ_RUN(k_ckpt_load, (Bf16), p, ckpt_in(ckpt, rows, cols), rows_of(out));
  return hip_status(hipGetLastError());
}

dq_status dq_gate(dq_activation kind, const dq_matrix *z, const dq_matrix *u, uint64_t rows, uint64_t cols, const dq_matrix *h, void *ckpt_z,
                  void *ckpt_u, void *hip_stream) {
  if (!good_kind(kind)) return DQ_EINVAL;
  DQ_TRY(check_matrix(z, rows, cols));
  DQ_TRY(check_matrix(h, rows, cols));
  if (u) DQ_TRY(check_matrix(u, rows, cols));
  if (h->dtype != z->dtype || (u && u->dtype != z->dtype) || (u ? !ckpt_z != !ckpt_u : ckpt_u != nullptr)) return DQ_EINVAL;
  if (rows == 0 || cols == 0) return DQ_OK;
  const size_t bytes = dq_ckpt_bytes(rows, cols);
  if (bytes == 0) return DQ_EUNSUPPORTED;
  if (!al16(ckpt_z) || !al16(ckpt_u)) return DQ_EALIGN;
  const Region r[] = {region(z, rows, cols, false), region(u ? u : z, rows, cols, false), region(h, rows, cols, true), region(ckpt_z, bytes, true),
                      region(ckpt_u, bytes, true)};
  if (regions_meet(r, 5)) return DQ_EINVAL;
  const Map p = u ? plan_map(rows, cols, {z, u, h}) : plan_map(rows, cols, {z, h});
  const Rows rz = rows_of(z), ru = rows_of(u), rh = rows_of(h);
  const CkptOut sz = ckpt_out(ckpt_z, rows, cols), su = ckpt_out(ckpt_u, rows, cols);
#define DQ_GATE(T, K)                                                                   \
  do {                                                                                  \
    if (u && ckpt_z) DQ_RUN(k_gate, (T, K, true, true), p, rz, ru, rh, sz, su);         \
    else if (u) DQ_RUN(k_gate, (T, K, true, false), p, rz, ru, rh, sz, su);             \
    else if (ckpt_z) DQ_RUN(k_gate, (T, K, false, true), p, rz, ru, rh, sz, su);        \
    else DQ_RUN(k_gate, (T, K, false, false), p, rz, ru, rh, sz, su);                   \
  } while (0)
  if (z->dtype == DQ_F32) {
    if (kind == DQ_SILU) DQ_GATE(F32, DQ_SILU);
    else DQ_GATE(F32, DQ_GELU);
  } else {
    if (kind == DQ_SILU) DQ_GATE(Bf16, DQ_SILU);
    else DQ_GATE(Bf16, DQ_GELU);
  }
  return hip_status(hipGetLastError());
}

dq_status dq_gate_grad(dq_activation kind, const dq_matrix *dh, const void *ckpt_z, const void *ckpt_u, uint64_t rows, uint64_t cols,
                       const dq_matrix *dz, const dq_matrix *du, void *hip_stream) {
  if (!good_kind(kind)) return DQ_EINVAL;
  DQ_TRY(check_matrix(dh, rows, cols));
  DQ_TRY(check_matrix(dz, rows, cols));
  if (du) DQ_TRY(check_matrix(du, rows, cols));
  if (dz->dtype != dh->dtype || (du && du->dtype != dh->dtype)) return DQ_EINVAL;
  if (rows == 0 || cols == 0) return DQ_OK;
  const size_t bytes = dq_ckpt_bytes(rows, cols);
  if (bytes == 0) return DQ_EUNSUPPORTED;
  if (!ckpt_z || !ckpt_u != !du) return DQ_EINVAL;
  if (!al16(ckpt_z) || !al16(ckpt_u)) return DQ_EALIGN;
  const Region r[] = {region(dh, rows, cols, false), region(ckpt_z, bytes, false), region(ckpt_u, bytes, false), region(dz, rows, cols, true),
                      du ? region(du, rows, cols, true) : region(nullptr, 0, true)};
  if (regions_meet(r, 5)) return DQ_EINVAL;
  const Map p = du ? plan_map(rows, cols, {dh, dz, du}) : plan_map(rows, cols, {dh, dz});
  const Rows rg = rows_of(dh), rz = rows_of(dz), ru = rows_of(du);
  const CkptIn sz = ckpt_in(ckpt_z, rows, cols), su = ckpt_in(ckpt_u, rows, cols);
#define DQ_GATE_GRAD(T, K)                                                        \
  do {                                                                            \
    if (du) DQ_RUN(k_gate_grad, (T, K, true), p, rg, sz, su, rz, ru);             \
    else DQ_RUN(k_gate_grad, (T, K, false), p, rg, sz, su, rz, ru);               \
  } while (0)
  if (dh->dtype == DQ_F32) {
    if (kind == DQ_SILU) DQ_GATE_GRAD(F32, DQ_SILU);
    else DQ_GATE_GRAD(F32, DQ_GELU);
  } else {
    if (kind == DQ_SILU) DQ_GATE_GRAD(Bf16, DQ_SILU);
    else DQ_GATE_GRAD(Bf16, DQ_GELU);
  }
  return hip_status(hipGetLastError());
}

}  // extern "C"
