// norm.hip -- layer norm and RMS norm of rows, with an optional SiLU gate, and
// their gradients.
//
//   xh = (x - mean) rstd, n = xh w + b, y = n silu(z)
//   dn = dy silu(z), dz = dy n silu'(z), dh = dn w,
//   dx = rstd (dh - mean(dh) - xh mean(dh xh))     (RMS: without mean(dh))
//   dw = sum over rows of dn xh, db = sum over rows of dn
//
// Bound: HBM.  A row is read once and held in registers as fp32 by TPR threads
// with NV 16-byte pieces each, so that mean and variance are two passes over
// registers, not over memory; a workgroup walks rows with its weights, and
// in the backward pass its sums for dw and db, in registers.  The sums of the
// workgroups go through a workspace and are added up by a second launch in a
// fixed order (no atomics: the same call gives the same bits).  Rows too long for
// the registers are read from memory in every pass, by one workgroup each.
// Measured: RMS norm with gate of 262144 rows of 128 in bf16, 202 MB, 32 us, 6.3 TB/s;
// layer norm of 3001 rows of 1537 in fp32, 37 MB, 8.5 us; gradients of the first,
// 337 MB, 69 us and 4 for the sums, 4.9 TB/s; of layer norm with bias of 8192 rows of
// 4096 in bf16, 201 MB, 39 us and 4, 5.2 TB/s.
#include "lanes.hpp"
#include "launch.hpp"
#include "layer.hpp"
#include "tile16.hpp"

namespace gdn {

namespace {

constexpr int kParts = 256;  // workgroups of the backward pass: one a CU

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));

template <typename T> struct Piece;  // 16 bytes of a row of any alignment
template <> struct Piece<float> {
  static constexpr int E = 4;
  f32x4u v;
};
template <> struct Piece<__bf16> {
  static constexpr int E = 8;
  bf16x8u v;
};

// a piece as it lies in memory (0 past the row's end), and its values
template <typename T>
__device__ __forceinline__ auto load_raw(const T* __restrict__ row, int e, int D) {
  constexpr int E = Piece<T>::E;
  decltype(Piece<T>::v) p;
  if (e + E <= D) {
    p = *(const decltype(Piece<T>::v)*)(row + e);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) p[i] = e + i < D ? row[e + i] : (T)0.f;
  }
  return p;
}
// elements e .. e + E - 1 of a row of D (0 past its end)
template <typename T, int E = Piece<T>::E>
__device__ __forceinline__ void load_piece(float (&x)[E], const T* __restrict__ row, int e, int D) {
  if (e + E <= D) {
    if constexpr (E == Piece<T>::E) {
      const auto p = *(const decltype(Piece<T>::v)*)(row + e);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = (float)p[i];
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = (float)row[e + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = e + i < D ? (float)row[e + i] : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_piece(T* __restrict__ row, const float (&x)[Piece<T>::E],
                                            int e, int D) {
  constexpr int E = Piece<T>::E;
  if (e + E <= D) {
    decltype(Piece<T>::v) p;
#pragma unroll
    for (int i = 0; i < E; ++i) p[i] = (T)x[i];
    *(decltype(Piece<T>::v)*)(row + e) = p;
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (e + i < D) row[e + i] = (T)x[i];
  }
}
// a weight or bias in either dtype; `none` where there is none
template <int E>
__device__ __forceinline__ void load_param(float (&x)[E], const void* p, bool bf, float none,
                                           int e, int D) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = none;
  } else if (bf) {
    load_piece<__bf16, E>(x, (const __bf16*)p, e, D);
  } else {
    load_piece<float, E>(x, (const float*)p, e, D);
  }
}

// 1 / (1 + e^-z).  The exponential and the reciprocal are the hardware's (1
// ulp, and |z| 6e-8 from the scaled argument): the exact ones made the
// vector operations as long as the memory traffic.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __expf(-z));
}

// Sums over the TPR threads of a row, the same in each of them.  Past one wave
// they meet in LDS: `red` holds two values a wave, in two buffers that the
// calls take in turn, so that one barrier a call is enough.
template <int TPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float* red, int& buf) {
  a = sum_lanes<(TPR < 64 ? TPR : 64)>(a);
  b = sum_lanes<(TPR < 64 ? TPR : 64)>(b);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* r = red + buf * 32;
    buf ^= 1;
    const int w = threadIdx.x >> 6;
    if (lane_id() == 0) {
      r[2 * w] = a;
      r[2 * w + 1] = b;
    }
    __syncthreads();
    const int w0 = w / W * W;
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      a += r[2 * (w0 + i)];
      b += r[2 * (w0 + i) + 1];
    }
  }
}

struct NormArgs {
  const void *dy, *x, *w, *b, *z;
  const float *mean_in, *rstd_in;
  void *out, *dz;
  float *mean, *rstd, *ws;
  int64_t rows;
  int D;
  float eps;
  bool rms, wbf;
};

}  // namespace

// A workgroup of B threads: B / TPR rows at a time.
template <typename T, int TPR, int NV, int B>
__global__ __launch_bounds__(B) void k_norm(const NormArgs a) {
  constexpr int E = Piece<T>::E, RPB = B / TPR;
  __shared__ float red[64];
  int buf = 0;
  const int t = threadIdx.x % TPR, r = threadIdx.x / TPR, D = a.D;
  float w[NV][E], bias[NV][E];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    load_param<E>(w[k], a.w, a.wbf, 1.f, (t + k * TPR) * E, D);
    load_param<E>(bias[k], a.b, a.wbf, 0.f, (t + k * TPR) * E, D);
  }
  const float inv = 1.f / (float)D;
  for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < a.rows; row0 += (int64_t)gridDim.x * RPB) {
    const bool live = row0 + r < a.rows;
    const int64_t row = live ? row0 + r : a.rows - 1;
    const T* xr = (const T*)a.x + row * D;
    float x[NV][E], z[NV][E];
#pragma unroll
    for (int k = 0; k < NV; ++k) load_piece<T>(x[k], xr, (t + k * TPR) * E, D);
    if (a.z)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        load_piece<T>(z[k], (const T*)a.z + row * D, (t + k * TPR) * E, D);
    float mean = 0.f, var = 0.f, none = 0.f;
    if (!a.rms) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) mean += x[k][i];
      row_sums<TPR>(mean, none, red, buf);
      mean *= inv;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[k][i] = (t + k * TPR) * E + i < D ? x[k][i] - mean : 0.f;
        var = __builtin_fmaf(x[k][i], x[k][i], var);
      }
    none = 0.f;
    row_sums<TPR>(var, none, red, buf);
    const float rstd = 1.f / sqrtf(var * inv + a.eps);
    if (!live) continue;
    if (t == 0) {
      if (a.mean && !a.rms) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float y[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        y[i] = __builtin_fmaf(x[k][i] * rstd, w[k][i], bias[k][i]);
        if (a.z) y[i] *= z[k][i] * sigmoid(z[k][i]);
      }
      store_piece<T>((T*)a.out + row * D, y, (t + k * TPR) * E, D);
    }
  }
}

// Rows of any length, a workgroup of 1024 each, read from memory in every pass.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_long(const NormArgs a) {
  constexpr int E = Piece<T>::E;
  __shared__ float red[64];
  int buf = 0;
  const int D = a.D;
  const float inv = 1.f / (float)D;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* xr = (const T*)a.x + row * D;
    float mean = 0.f, var = 0.f, none = 0.f;
    if (!a.rms) {
      for (int e = threadIdx.x * E; e < D; e += 1024 * E) {
        float x[E];
        load_piece<T>(x, xr, e, D);
#pragma unroll
        for (int i = 0; i < E; ++i) mean += x[i];
      }
      row_sums<1024>(mean, none, red, buf);
      mean *= inv;
    }
    for (int e = threadIdx.x * E; e < D; e += 1024 * E) {
      float x[E];
      load_piece<T>(x, xr, e, D);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = e + i < D ? x[i] - mean : 0.f;
        var = __builtin_fmaf(x[i], x[i], var);
      }
    }
    none = 0.f;
    row_sums<1024>(var, none, red, buf);
    const float rstd = 1.f / sqrtf(var * inv + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean && !a.rms) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (int e = threadIdx.x * E; e < D; e += 1024 * E) {
      float x[E], w[E], b[E], z[E];
      load_piece<T>(x, xr, e, D);
      load_param<E>(w, a.w, a.wbf, 1.f, e, D);
      load_param<E>(b, a.b, a.wbf, 0.f, e, D);
      if (a.z) load_piece<T>(z, (const T*)a.z + row * D, e, D);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = __builtin_fmaf((x[i] - mean) * rstd, w[i], b[i]);
        if (a.z) x[i] *= z[i] * sigmoid(z[i]);
      }
      store_piece<T>((T*)a.out + row * D, x, e, D);
    }
  }
}

// What a piece of a row gives: xh, dn (the gradient of n, 0 past the row) and dz.
template <typename T>
struct GradPiece {
  static constexpr int E = Piece<T>::E;
  float h[E], dn[E], dz[E];
  __device__ __forceinline__ void form(const NormArgs& a, int64_t row, int e, const float (&w)[E],
                                       const float (&b)[E], float mean, float rstd) {
    float z[E];
    load_piece<T>(h, (const T*)a.x + row * a.D, e, a.D);
    load_piece<T>(dn, (const T*)a.dy + row * a.D, e, a.D);
    if (a.z) load_piece<T>(z, (const T*)a.z + row * a.D, e, a.D);
#pragma unroll
    for (int i = 0; i < E; ++i) h[i] = (h[i] - mean) * rstd;
    if (a.z) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float s = sigmoid(z[i]), dy = dn[i];
        dz[i] = dy * __builtin_fmaf(h[i], w[i], b[i]) * (s * __builtin_fmaf(z[i], 1.f - s, 1.f));
        dn[i] = dy * (z[i] * s);
      }
    }
  }
};

// A row's pieces as they lie in memory, asked for two rows ahead.
template <typename T, int NV, bool GATE>
struct RawRow {
  decltype(Piece<T>::v) x[NV], dy[NV], z[GATE ? NV : 1];
  float mean, rstd;
};

// Workgroups of B threads, B / TPR rows at a time; each leaves its sums of dw
// and db in row blockIdx.x of the workspace: ws [parts][D], then the same for
// db.  want: bit 0 dw, bit 1 db.  GATE: z is given; BIAS: b or db is.
template <typename T, int TPR, int NV, int B, bool GATE, bool BIAS>
__global__ __launch_bounds__(B) void k_norm_grad(const NormArgs a, int want) {
  constexpr int E = Piece<T>::E, RPB = B / TPR;
  extern __shared__ float part[];  // 64 values of row_sums, then the sums [2][D]
  float* red = part;
  float* sum = part + 64;
  int buf = 0;
  const int t = threadIdx.x % TPR, r = threadIdx.x / TPR, D = a.D;
  float w[NV][E], bias[GATE && BIAS ? NV : 1][E], dw[NV][E], db[BIAS ? NV : 1][E];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    load_param<E>(w[k], a.w, a.wbf, 1.f, (t + k * TPR) * E, D);
    if constexpr (GATE && BIAS) load_param<E>(bias[k], a.b, a.wbf, 0.f, (t + k * TPR) * E, D);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      dw[k][i] = 0.f;
      if constexpr (BIAS) db[k][i] = 0.f;
    }
  }
  const float inv = 1.f / (float)D;
  const int64_t step = (int64_t)gridDim.x * RPB;
  typedef RawRow<T, NV, GATE> Row;
  auto fetch = [&](Row& x, int64_t row) __attribute__((always_inline)) {
    row = row < a.rows ? row : a.rows - 1;
    const int64_t at = row * D;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = (t + k * TPR) * E;
      x.x[k] = load_raw<T>((const T*)a.x + at, e, D);
      x.dy[k] = load_raw<T>((const T*)a.dy + at, e, D);
      if constexpr (GATE) x.z[k] = load_raw<T>((const T*)a.z + at, e, D);
    }
    x.mean = a.rms ? 0.f : a.mean_in[row];
    x.rstd = a.rstd_in[row];
  };
  auto rows = [&](const Row& cur, int64_t row0) __attribute__((always_inline)) {
    const bool live = row0 + r < a.rows;
    const int64_t at = (live ? row0 + r : a.rows - 1) * D;
    // dn (dy without a gate) and dz, then the row's two sums
    float dn[NV][E], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float dz[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float h = ((float)cur.x[k][i] - cur.mean) * cur.rstd;
        float d = (float)cur.dy[k][i];
        if constexpr (GATE) {
          const float z = (float)cur.z[k][i], s = sigmoid(z);
          float n = h * w[k][i];
          if constexpr (BIAS) n += bias[k][i];
          dz[i] = d * n * (s * __builtin_fmaf(z, 1.f - s, 1.f));
          d *= z * s;
        }
        dn[k][i] = d;
        const float dh = d * w[k][i];
        s1 += dh;
        s2 = __builtin_fmaf(dh, h, s2);  // (past the row's end d is 0)
      }
      if constexpr (GATE)
        if (live) store_piece<T>((T*)a.dz + at, dz, (t + k * TPR) * E, D);
    }
    row_sums<TPR>(s1, s2, red, buf);
    if (live) {
      s1 = a.rms ? 0.f : s1 * inv;
      s2 *= inv;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float dx[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float h = ((float)cur.x[k][i] - cur.mean) * cur.rstd;
          dx[i] = cur.rstd * (dn[k][i] * w[k][i] - s1 - h * s2);
          dw[k][i] = __builtin_fmaf(dn[k][i], h, dw[k][i]);
          if constexpr (BIAS) db[k][i] += dn[k][i];
        }
        store_piece<T>((T*)a.out + at, dx, (t + k * TPR) * E, D);
      }
    }
  };
  // two sets in turn, each asked for again when it has been used: copied from one to the
  // other they were waited for before the next ones were asked for
  Row r0, r1;
  int64_t row0 = (int64_t)blockIdx.x * RPB;
  fetch(r0, row0 + r);
  fetch(r1, row0 + step + r);
  for (; row0 < a.rows; row0 += 2 * step) {
    rows(r0, row0);
    fetch(r0, row0 + 2 * step + r);
    if (row0 + step >= a.rows) break;
    rows(r1, row0 + step);
    fetch(r1, row0 + 3 * step + r);
  }
  if (!want) return;
  // the sums of the rows that ran side by side: within a wave by exchange,
  // then wave after wave into LDS
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < E; ++i)
#pragma unroll
      for (int o = TPR; o < 64; o <<= 1) {
        dw[k][i] += __shfl_xor(dw[k][i], o);
        if constexpr (BIAS) db[k][i] += __shfl_xor(db[k][i], o);
      }
  constexpr int GROUPS = TPR < 64 ? B / 64 : RPB;
  const int64_t at = (int64_t)blockIdx.x * D, half = (int64_t)gridDim.x * D;
  if constexpr (GROUPS == 1) {  // one row at a time: the sums are whole
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int e = (t + k * TPR) * E + i;
        if (e < D && (want & 1)) a.ws[at + e] = dw[k][i];
        if constexpr (BIAS)
          if (e < D && (want & 2)) a.ws[half + at + e] = db[k][i];
      }
    return;
  }
  const int mine = TPR < 64 ? threadIdx.x >> 6 : r;
  for (int gi = 0; gi < GROUPS; ++gi) {
    if (mine == gi && (TPR >= 64 || lane_id() < TPR))
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const int e = (t + k * TPR) * E + i;
          if (e < D) {
            sum[e] = gi ? sum[e] + dw[k][i] : dw[k][i];
            if constexpr (BIAS) sum[D + e] = gi ? sum[D + e] + db[k][i] : db[k][i];
          }
        }
    __syncthreads();
  }
  for (int e = threadIdx.x; e < D; e += B) {
    if (want & 1) a.ws[at + e] = sum[e];
    if (BIAS && (want & 2)) a.ws[half + at + e] = sum[D + e];
  }
}

// The same for rows of any length: one row at a time, read twice; the sums
// stay in the workspace.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_grad_long(const NormArgs a, int want) {
  constexpr int E = Piece<T>::E;
  __shared__ float red[64];
  int buf = 0;
  const int D = a.D;
  const float inv = 1.f / (float)D;
  float* dw = a.ws + (int64_t)blockIdx.x * D;
  float* db = dw + (int64_t)gridDim.x * D;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.rms ? 0.f : a.mean_in[row], rstd = a.rstd_in[row];
    float s1 = 0.f, s2 = 0.f, w[E], b[E];
    GradPiece<T> p;
    for (int e = threadIdx.x * E; e < D; e += 1024 * E) {
      load_param<E>(w, a.w, a.wbf, 1.f, e, D);
      load_param<E>(b, a.z ? a.b : nullptr, a.wbf, 0.f, e, D);
      p.form(a, row, e, w, b, mean, rstd);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        s1 += p.dn[i] * w[i];
        s2 = __builtin_fmaf(p.dn[i] * w[i], p.h[i], s2);
      }
    }
    row_sums<1024>(s1, s2, red, buf);
    s1 = a.rms ? 0.f : s1 * inv;
    s2 *= inv;
    const bool first = row == blockIdx.x;
    for (int e = threadIdx.x * E; e < D; e += 1024 * E) {
      load_param<E>(w, a.w, a.wbf, 1.f, e, D);
      load_param<E>(b, a.z ? a.b : nullptr, a.wbf, 0.f, e, D);
      p.form(a, row, e, w, b, mean, rstd);
      float dx[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        dx[i] = rstd * (p.dn[i] * w[i] - s1 - p.h[i] * s2);
        if (e + i < D) {
          if (want & 1) dw[e + i] = p.dn[i] * p.h[i] + (first ? 0.f : dw[e + i]);
          if (want & 2) db[e + i] = p.dn[i] + (first ? 0.f : db[e + i]);
        }
      }
      store_piece<T>((T*)a.out + row * D, dx, e, D);
      if (a.z) store_piece<T>((T*)a.dz + row * D, p.dz, e, D);
    }
  }
}

// out[d] = sum over the parts, 16 threads a column and 16 columns a workgroup
__global__ __launch_bounds__(256) void k_norm_parts(const float* __restrict__ ws, float* dw,
                                                    float* db, int parts, int D) {
  __shared__ float s[16][17];
  const float* from = ws + (blockIdx.y ? (int64_t)parts * D : 0);
  float* to = blockIdx.y ? db : dw;
  if (!to) return;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, d = blockIdx.x * 16 + c;
  float x = 0.f;
  if (d < D)
#pragma unroll 8
    for (int p = r; p < parts; p += 16) x += from[(int64_t)p * D + d];
  s[r][c] = x;
  __syncthreads();
  if (r == 0 && d < D) {
#pragma unroll
    for (int i = 1; i < 16; ++i) x += s[i][c];
    to[d] = x;
  }
}

int norm_backward_parts(int64_t rows) { return (int)(rows < kParts ? rows : kParts); }

// TPR threads and NV pieces a thread for a row of n 16-byte pieces: a short
// row takes part of a wave, so that a wave's loads stay 16 bytes a lane
#define GDN_NORM_SHAPES(X) \
  X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(256, 1) X(256, 2) X(1024, 1) X(1024, 2)

template <typename T>
static hipError_t norm_forward(const NormArgs& a, hipStream_t st) {
  const int n = (a.D + Piece<T>::E - 1) / Piece<T>::E;
#define GDN_X(TPR, NV)                                                                       \
  if (n <= TPR * NV) {                                                                       \
    constexpr int B = TPR > 256 ? TPR : 256, R = B / TPR;                                    \
    const int64_t need = (a.rows + R - 1) / R, most = 256 * (2048 / B);                      \
    hipLaunchKernelGGL((k_norm<T, TPR, NV, B>), dim3((unsigned)(need < most ? need : most)), \
                       dim3(B), 0, st, a);                                                   \
    return hipGetLastError();                                                                \
  }
  GDN_NORM_SHAPES(GDN_X)
#undef GDN_X
  hipLaunchKernelGGL((k_norm_long<T>), dim3((unsigned)(a.rows < 512 ? a.rows : 512)), dim3(1024),
                     0, st, a);
  return hipGetLastError();
}

template <typename T>
static hipError_t norm_backward(const NormArgs& a, int want, hipStream_t st) {
  const int n = (a.D + Piece<T>::E - 1) / Piece<T>::E;
  const int parts = norm_backward_parts(a.rows);
  const bool bias = a.b || (want & 2);
#define GDN_G(TPR, NV, GATE, BIAS)                                                          \
  hipLaunchKernelGGL((k_norm_grad<T, TPR, NV, 1024, GATE, BIAS>), dim3((unsigned)parts),    \
                     dim3(1024), (64 + (TPR < 1024 ? 2 * a.D : 0)) * sizeof(float), st, a, want)
#define GDN_X(TPR, NV)                                        \
  if (n <= TPR * NV) {                                        \
    if (a.z && bias) GDN_G(TPR, NV, true, true);              \
    else if (a.z) GDN_G(TPR, NV, true, false);                \
    else if (bias) GDN_G(TPR, NV, false, true);               \
    else GDN_G(TPR, NV, false, false);                        \
    return hipGetLastError();                                 \
  }
  // one piece a thread: two with their sums pass the 128 registers that a workgroup
  // of 1024 threads has for each (with fp32's four values a piece they do not)
  GDN_X(16, 1) GDN_X(32, 1) GDN_X(64, 1) GDN_X(128, 1) GDN_X(256, 1) GDN_X(512, 1) GDN_X(1024, 1)
  if constexpr (sizeof(T) == 4) {
    GDN_X(1024, 2)
  }
#undef GDN_X
#undef GDN_G
  hipLaunchKernelGGL((k_norm_grad_long<T>), dim3((unsigned)parts), dim3(1024), 0, st, a, want);
  return hipGetLastError();
}

hipError_t launch_norm_forward(const void* x, const void* w, const void* b, const void* z, void* y,
                               float* mean, float* rstd, int64_t rows, int D, float eps, bool rms,
                               int dtype, int w_dtype, hipStream_t st) {
  NormArgs a{};
  a.x = x, a.w = w, a.b = b, a.z = z, a.out = y, a.mean = mean, a.rstd = rstd;
  a.rows = rows, a.D = D, a.eps = eps, a.rms = rms, a.wbf = w_dtype == 1;
  return dtype == 0 ? norm_forward<float>(a, st) : norm_forward<__bf16>(a, st);
}

hipError_t launch_norm_backward(const void* dy, const void* x, const void* w, const void* b,
                                const void* z, const float* mean, const float* rstd, void* dx,
                                float* dw, float* db, void* dz, float* ws, int64_t rows, int D,
                                bool rms, int dtype, int w_dtype, hipStream_t st) {
  NormArgs a{};
  a.dy = dy, a.x = x, a.w = w, a.b = b, a.z = z, a.mean_in = mean, a.rstd_in = rstd;
  a.out = dx, a.dz = dz, a.ws = ws, a.rows = rows, a.D = D, a.rms = rms, a.wbf = w_dtype == 1;
  const int want = (dw ? 1 : 0) | (db ? 2 : 0);
  if (rows > 0) {
    const hipError_t e =
        dtype == 0 ? norm_backward<float>(a, want, st) : norm_backward<__bf16>(a, want, st);
    if (e != hipSuccess) return e;
  }
  if (want) {
    hipLaunchKernelGGL(k_norm_parts, dim3((unsigned)((D + 15) / 16), 2), dim3(256), 0, st, ws, dw,
                       db, norm_backward_parts(rows), D);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace gdn
