// group_norm.hip -- group norm, channels last, with an activation and a gate, and its
// gradients.
//
// x [N, S, C], the channels in G groups of Cg: mean and rstd of each (n, group) over S Cg
// values, and with h = (x - mean) rstd, n = h w + b (w, b of each channel),
//   y = act(n) silu(z),   act(n) = n or silu(n),
//   dz = dy act(n) silu'(z),  dn = dy silu(z) act'(n),  dh = dn w,
//   dx = rstd (dh - mean(dh) - h mean(dh h)),  dw = sum dn h, db = sum dn  (over n and s).
//
// Bound: HBM.  A group that fits the registers of a workgroup, or of part of a wave, is read
// once (k_gn_rows; the gradients where S = 1, k_gn_rows_grad).  Others are read twice: the sums
// of parts of the positions first, then the results.  A thread has V neighbouring channels
// of one group all along, so that its weights and its sums of dw and db stay in registers.
// Everything is added up in a fixed order (no atomics: the same call gives the same bits).
// (8192 rows of 32 groups of 128 with a gate, bf16: 37 us, 5.4 TB/s; gradients 69 and 4 us,
// 4.9 TB/s.  4 x 4096 positions of 32 groups of 16, SiLU: 8 us for the sums, 12 for the
// results.  Gradients of 3 x 3001 positions of 8 groups of 41, fp32, a value a load: 10 and 14.)
#include <algorithm>

#include "group_norm.hpp"
#include "lanes.hpp"
#include "launch.hpp"
#include "norm.hpp"
#include "tile16.hpp"

namespace gdn {

namespace {

template <typename T, int V> struct Vals {
  typedef T type __attribute__((ext_vector_type(V)));
};
template <typename T> struct Vals<T, 1> { typedef T type; };

template <typename T, int V>
__device__ __forceinline__ void get(float (&x)[V], const T* __restrict__ p) {
  if constexpr (V == 1) {
    x[0] = (float)*p;
  } else {
    const auto v = *(const typename Vals<T, V>::type*)p;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)v[i];
  }
}
template <typename T, int V>
__device__ __forceinline__ void put(T* __restrict__ p, const float (&x)[V]) {
  if constexpr (V == 1) {
    *p = (T)x[0];
  } else {
    typename Vals<T, V>::type v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)x[i];
    *(typename Vals<T, V>::type*)p = v;
  }
}
// V values as they lie in memory, and as floats
template <typename T, int V> struct Raw {
  typename Vals<T, V>::type v;
  __device__ __forceinline__ void load(const T* __restrict__ p) {
    v = *(const typename Vals<T, V>::type*)p;
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (V == 1) return (float)v; else return (float)v[i];
  }
};
// a weight or bias in either dtype; `none` where there is none
template <int V>
__device__ __forceinline__ void get_param(float (&x)[V], const void* p, bool bf, float none,
                                          int at) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = none;
  } else if (bf) {
    get<__bf16, V>(x, (const __bf16*)p + at);
  } else {
    get<float, V>(x, (const float*)p + at);
  }
}

__device__ __forceinline__ float silu_grad(float t) {
  const float s = sigmoid(t);
  return s * __builtin_fmaf(t, 1.f - s, 1.f);
}

// what follows n: bit 0 SiLU, bit 1 a gate
constexpr int kAct = 1, kGate = 2;

// the results of one value
template <int OPS>
__device__ __forceinline__ float result(float h, float w, float b, float z) {
  float n = __builtin_fmaf(h, w, b);
  if (OPS & kAct) n *= sigmoid(n);
  if (OPS & kGate) n *= z * sigmoid(z);
  return n;
}
// dn (and dz) of one value
template <int OPS>
__device__ __forceinline__ float grad(float h, float w, float b, float z, float dy, float& dz) {
  const float n = __builtin_fmaf(h, w, b);
  if (OPS & kGate) {
    const float s = sigmoid(z);
    dz = dy * (OPS & kAct ? n * sigmoid(n) : n) * (s * __builtin_fmaf(z, 1.f - s, 1.f));
    dy *= z * s;
  }
  return OPS & kAct ? dy * silu_grad(n) : dy;
}

// sums over the `tpi` neighbouring threads (a power of two) of a group; past a wave they
// meet in LDS, in two buffers that the calls take in turn
struct Sums {
  float* red;
  int buf, tpi;
  __device__ __forceinline__ void operator()(float& a) {
    if (tpi >= 2) a += lane_moved<0xB1>(a);
    if (tpi >= 4) a += lane_moved<0x4E>(a);
    if (tpi >= 8) a += lane_moved<0x141>(a);
    if (tpi >= 16) a += lane_moved<0x140>(a);
    if (tpi >= 32) a = sum_apart16(a);
    if (tpi >= 64) a = sum_apart32(a);
    if (tpi > 64) {
      float* r = red + buf * 32;
      buf ^= 1;
      if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = a;
      __syncthreads();
      a = 0.f;
      for (int i = 0; i < tpi >> 6; ++i) a += r[i];
    }
  }
  __device__ __forceinline__ void operator()(float& a, float& b) {
    if (tpi >= 2) a += lane_moved<0xB1>(a), b += lane_moved<0xB1>(b);
    if (tpi >= 4) a += lane_moved<0x4E>(a), b += lane_moved<0x4E>(b);
    if (tpi >= 8) a += lane_moved<0x141>(a), b += lane_moved<0x141>(b);
    if (tpi >= 16) a += lane_moved<0x140>(a), b += lane_moved<0x140>(b);
    if (tpi >= 32) a = sum_apart16(a), b = sum_apart16(b);
    if (tpi >= 64) a = sum_apart32(a), b = sum_apart32(b);
    if (tpi > 64) {  // (the whole workgroup)
      float* r = red + buf * 32;
      buf ^= 1;
      const int w = threadIdx.x >> 6, n = tpi >> 6;
      if ((threadIdx.x & 63) == 0) r[2 * w] = a, r[2 * w + 1] = b;
      __syncthreads();
      a = b = 0.f;
      for (int i = 0; i < n; ++i) a += r[2 * i], b += r[2 * i + 1];
    }
  }
};

}  // namespace

// Groups in registers.  A workgroup has gw groups of nw n's at a time, tpi threads each, and
// walks the n's, the next ones asked for ahead; piece k of thread t of a group is its
// (t + k tpi)-th piece of V values.
template <typename T, int V, int NV, int OPS>
__global__ __launch_bounds__(256) void k_gn_rows(const GroupArgs a) {
  __shared__ float red[64];
  Sums sums{red, 0, a.tpi};
  const int slot = (int)threadIdx.x / a.tpi, t = (int)threadIdx.x - slot * a.tpi;
  const int blocks = a.G / a.gw, gb = (int)(blockIdx.x % blocks), nb = (int)(blockIdx.x / blocks);
  const int ni = slot / a.gw, g = gb * a.gw + slot - ni * a.gw;
  const bool mine = ni < a.nw;
  const int pr = a.Cg / V, pieces = a.S * pr;
  float w[NV][V], b[NV][V];
  int at[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int p = t + k * a.tpi, s = p / pr, ch = g * a.Cg + (p - s * pr) * V;
    at[k] = mine && p < pieces ? s * a.C + ch : -1;
    get_param<V>(w[k], at[k] < 0 ? nullptr : a.w, a.wbf, 1.f, ch);
    get_param<V>(b[k], at[k] < 0 ? nullptr : a.b, a.wbf, 0.f, ch);
  }
  const float inv = 1.f / (float)(a.S * a.Cg);
  const int64_t step = (int64_t)(gridDim.x / blocks) * a.nw, size = (int64_t)a.S * a.C;
  Raw<T, V> x[NV], z[NV];
  auto fetch = [&](int64_t n) __attribute__((always_inline)) {
    n = n < a.N ? n : a.N - 1;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t p = n * size + max(at[k], 0);
      x[k].load((const T*)a.x + p);
      if (OPS & kGate) z[k].load((const T*)a.z + p);
    }
  };
  int64_t n0 = (int64_t)nb * a.nw;
  fetch(n0 + ni);
  for (; n0 < a.N; n0 += step) {
    const int64_t n = n0 + ni;
    const bool live = mine && n < a.N;
    float h[NV][V], f[NV][V], mean = 0.f, var = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[k][i] = x[k][i];
        f[k][i] = OPS & kGate ? z[k][i] : 0.f;
        mean += at[k] >= 0 ? h[k][i] : 0.f;
      }
    fetch(n + step);
    sums(mean);
    mean *= inv;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[k][i] = at[k] >= 0 ? h[k][i] - mean : 0.f;
        var = __builtin_fmaf(h[k][i], h[k][i], var);
      }
    sums(var);
    const float rstd = 1.f / sqrtf(var * inv + a.eps);
    if (!live) continue;
    if (t == 0) {
      if (a.mean) a.mean[n * a.G + g] = mean;
      if (a.rstd) a.rstd[n * a.G + g] = rstd;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at[k] >= 0) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = result<OPS>(h[k][i] * rstd, w[k][i], b[k][i], f[k][i]);
        put<T, V>((T*)a.out + n * size + at[k], y);
      }
  }
}

// the largest power of two below n (0 for one)
__host__ __device__ inline int half_of(int n) {
  int h = 0;
  for (int p = 1; p < n; p *= 2) h = p;
  return h;
}
// most n's whose sums lie in LDS at once
inline int of_sums(int nw) { return std::max(nw - half_of(nw), half_of(nw) / 2); }

// The gradients where S = 1.  The n's that run side by side add up their dw and db in LDS, the
// workgroups' sums go to row nb of the workspace: [parts][C], then the same for db.
template <typename T, int V, int NV, int B, int OPS>
__global__ __launch_bounds__(B) void k_gn_rows_grad(const GroupArgs a, int parts) {
  extern __shared__ float lds[];  // 64 values of the sums, then [of_sums][2][gw Cg]
  Sums sums{lds, 0, a.tpi};
  const int slot = (int)threadIdx.x / a.tpi, t = (int)threadIdx.x - slot * a.tpi;
  const int blocks = a.G / a.gw, gb = (int)(blockIdx.x % blocks), nb = (int)(blockIdx.x / blocks);
  const int ni = slot / a.gw, gi = slot - ni * a.gw, g = gb * a.gw + gi;
  const bool mine = ni < a.nw;
  const int pr = a.Cg / V;
  float w[NV][V], b[NV][V], dw[NV][V], db[NV][V];
  int at[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int p = t + k * a.tpi;
    at[k] = mine && p < pr ? g * a.Cg + p * V : -1;
    get_param<V>(w[k], at[k] < 0 ? nullptr : a.w, a.wbf, 1.f, at[k]);
    get_param<V>(b[k], at[k] < 0 ? nullptr : a.b, a.wbf, 0.f, at[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.f;
  }
  const float inv = 1.f / (float)a.Cg;
  const int64_t step = (int64_t)parts * a.nw;
  struct Row {
    Raw<T, V> x[NV], dy[NV], z[NV];
    float mean, rstd;
  };
  auto fetch = [&](Row& r, int64_t n) __attribute__((always_inline)) {
    n = n < a.N ? n : a.N - 1;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t p = n * a.C + max(at[k], 0);
      r.x[k].load((const T*)a.x + p);
      r.dy[k].load((const T*)a.dy + p);
      if (OPS & kGate) r.z[k].load((const T*)a.z + p);
    }
    r.mean = a.mean_in[n * a.G + (mine ? g : 0)];
    r.rstd = a.rstd_in[n * a.G + (mine ? g : 0)];
  };
  auto row = [&](const Row& r, int64_t n) __attribute__((always_inline)) {
    const bool live = mine && n < a.N;
    float h[NV][V], dn[NV][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float dz[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[k][i] = ((float)r.x[k][i] - r.mean) * r.rstd;
        dn[k][i] = grad<OPS>(h[k][i], w[k][i], b[k][i], OPS & kGate ? r.z[k][i] : 0.f, r.dy[k][i],
                             dz[i]);
        const float dh = at[k] >= 0 ? dn[k][i] * w[k][i] : 0.f;
        s1 += dh;
        s2 += at[k] >= 0 ? dh * h[k][i] : 0.f;
      }
      if ((OPS & kGate) && live && at[k] >= 0) put<T, V>((T*)a.dz + n * a.C + at[k], dz);
    }
    sums(s1, s2);
    s1 *= inv, s2 *= inv;
    if (!live) return;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at[k] >= 0) {
        float dx[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dx[i] = r.rstd * (dn[k][i] * w[k][i] - s1 - h[k][i] * s2);
          dw[k][i] = __builtin_fmaf(dn[k][i], h[k][i], dw[k][i]);
          db[k][i] += dn[k][i];
        }
        put<T, V>((T*)a.out + n * a.C + at[k], dx);
      }
  };
  // two sets in turn, each asked for again when it has been used
  Row r0, r1;
  int64_t n0 = (int64_t)nb * a.nw;
  fetch(r0, n0 + ni);
  fetch(r1, n0 + step + ni);
  for (; n0 < a.N; n0 += 2 * step) {
    row(r0, n0 + ni);
    fetch(r0, n0 + 2 * step + ni);
    if (n0 + step >= a.N) break;
    row(r1, n0 + step + ni);
    fetch(r1, n0 + 3 * step + ni);
  }
  if (!a.dw && !a.db) return;
  float* sum = lds + 64;
  const int width = a.gw * a.Cg;
  float* to = a.ws + (int64_t)nb * a.C + (int64_t)gb * width;
  auto write = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at[k] >= 0)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          to[at[k] - gb * width + i] = dw[k][i];
          to[(int64_t)parts * a.C + at[k] - gb * width + i] = db[k][i];
        }
  };
  // halves of the n's onto each other (one after the other, 128 n's of a small group took 40 us)
  for (int half = half_of(a.nw); half > 0; half /= 2) {
    auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (at[k] >= 0)
#pragma unroll
          for (int i = 0; i < V; ++i) f(at[k] - gb * width + i, dw[k][i], db[k][i]);
    };
    if (mine && ni >= half && ni < 2 * half) {
      float* x = sum + (ni - half) * 2 * width;
      each([&](int c, float& u, float& v) { x[c] = u, x[width + c] = v; });
    }
    __syncthreads();
    if (mine && ni < half && ni + half < a.nw) {
      const float* x = sum + ni * 2 * width;
      each([&](int c, float& u, float& v) { u += x[c], v += x[width + c]; });
    }
    __syncthreads();
  }
  if (mine && ni == 0) write();
}

// ---- groups read twice.  A workgroup has the positions s0 .. s1 of one n and a block of
// `cols` pieces of V channels: whole groups where a group has up to 256 pieces, else a part of
// one.  Thread t has piece t % cols, and every (256 / cols)-th position.
struct Tile {
  int64_t n, row0;  // row0: n S
  int part, s0, s1, cols, c0, col, row, step, g0, ng, per, piece;
  bool mine;
  template <int V>
  static __device__ __forceinline__ Tile of(const GroupArgs& a, uint32_t block = blockIdx.x) {
    Tile t;
    const uint32_t pn = (uint32_t)a.sparts * (uint32_t)a.cblocks;
    t.n = block / pn;
    const int at = (int)(block - (uint32_t)t.n * pn);
    t.part = at / a.cblocks;
    const int cb = at - t.part * a.cblocks, pr = a.Cg / V;
    t.s0 = (int)((int64_t)a.S * t.part / a.sparts);
    t.s1 = (int)((int64_t)a.S * (t.part + 1) / a.sparts);
    if (pr <= 256) {
      const int most = 256 / pr;  // groups a block
      t.g0 = cb * most;
      t.ng = min(most, a.G - t.g0);
      t.cols = t.ng * pr;
      t.c0 = t.g0 * a.Cg;
      t.per = 1, t.piece = 0;
    } else {
      t.per = (pr + 255) / 256;  // blocks a group
      t.g0 = cb / t.per;
      t.ng = 1;
      t.piece = cb - t.g0 * t.per;
      const int p0 = t.piece * 256;
      t.cols = min(256, pr - p0);
      t.c0 = t.g0 * a.Cg + p0 * V;
    }
    t.step = 256 / t.cols;
    t.row = (int)threadIdx.x / t.cols;
    t.col = t.c0 + ((int)threadIdx.x - t.row * t.cols) * V;
    t.mine = t.row < t.step;
    t.row0 = t.n * a.S;
    return t;
  }
  // a power of two within a wave, all groups at once where they are few enough
  __device__ __forceinline__ int threads_a_group() const {
    return ng <= 4 ? 64 : ng <= 8 ? 32 : ng <= 16 ? 16 : ng <= 32 ? 8 : 4;
  }
  // parts of a group, and which one this is (of one in many column blocks too)
  __device__ __forceinline__ int parts(const GroupArgs& a) const { return a.sparts * per; }
  __device__ __forceinline__ int at(const GroupArgs& a) const { return part * per + piece; }
  __device__ __forceinline__ int64_t base(const GroupArgs& a, int s) const {
    return (row0 + s) * a.C + col;
  }
};

// sum over the threads of each of the tile's groups: 16 threads a group, 16 groups at a time;
// f(group, sum) is called by one of them
template <typename F, typename G>
__device__ __forceinline__ void sum_groups(const Tile& t, F value, G f) {
  const int per = t.cols / t.ng, lane = threadIdx.x & 15;
  for (int g0 = 0; g0 < t.ng; g0 += 16) {
    const int g = g0 + (int)(threadIdx.x >> 4);
    float x = 0.f;
    if (g < t.ng)
      for (int i = lane; i < per * t.step; i += 16) {
        const int r = i / per;
        x += value(r * t.cols + g * per + i - r * per);
      }
    x = sum_lanes<16>(x);
    if (lane == 0 && g < t.ng) f(g, x);
  }
}

// count, mean and sum of squares about it, of a part of a group: [N][G][parts][4]
template <typename T, int V>
__global__ __launch_bounds__(256) void k_gn_stats(const GroupArgs a) {
  __shared__ float sm[256], sq[256], sc[256], gm[256], gn[256];
  const Tile t = Tile::of<V>(a);
  // runs of R positions: their mean and squares in two passes over registers, joined to
  // those before them
  constexpr int R = 8;
  float cnt = 0.f, mean = 0.f, m2 = 0.f;
  if (t.mine)
    for (int s = t.s0 + t.row; s < t.s1; s += R * t.step) {
      float x[R][V], sum = 0.f, q = 0.f;
      const int k = min(R, (t.s1 - s + t.step - 1) / t.step);
#pragma unroll
      for (int r = 0; r < R; ++r)
        get<T, V>(x[r], (const T*)a.x + t.base(a, min(s + r * t.step, t.s1 - 1)));
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) sum += r < k ? x[r][i] : 0.f;
      const float nb = (float)(k * V), mb = sum / nb;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = r < k ? x[r][i] - mb : 0.f;
          q = __builtin_fmaf(d, d, q);
        }
      const float d = mb - mean, n = cnt + nb;
      mean += d * (nb / n);
      m2 += q + d * d * (cnt * nb / n);
      cnt = n;
    }
  sm[threadIdx.x] = mean, sq[threadIdx.x] = m2, sc[threadIdx.x] = cnt;
  __syncthreads();
  sum_groups(t, [&](int i) { return sc[i]; }, [&](int g, float x) { gn[g] = x; });
  sum_groups(t, [&](int i) { return sc[i] * sm[i]; }, [&](int g, float x) { gm[g] = x; });
  __syncthreads();
  const int per = t.cols / t.ng, parts = t.parts(a);
  sum_groups(
      t,
      [&](int i) {
        const int g = i % t.cols / per;
        const float d = sm[i] - gm[g] / gn[g];
        return sq[i] + sc[i] * d * d;
      },
      [&](int g, float x) {
        *(f32x4*)(a.ws + ((t.n * a.G + t.g0 + g) * parts + t.at(a)) * 4) =
            f32x4{gn[g], gm[g] / gn[g], x, 0.f};
      });
}

template <typename T, int V, int OPS>
__global__ __launch_bounds__(256) void k_gn_apply(const GroupArgs a) {
  __shared__ float sm[256], sr[256];
  const Tile t = Tile::of<V>(a);
  const int parts = t.parts(a);
  const int each = t.threads_a_group(), lane = (int)threadIdx.x % each;
  for (int g0 = 0; g0 < t.ng; g0 += 256 / each) {  // join the parts: pairwise, then over threads
    const int g = g0 + (int)threadIdx.x / each;
    const f32x4* p = (const f32x4*)a.ws + (t.n * a.G + t.g0 + min(g, t.ng - 1)) * parts;
    float c = 0.f, m = 0.f, q = 0.f;
#pragma unroll 4
    for (int i = lane; i < parts; i += each) {
      const f32x4 v = p[i];
      const float n = c + v[0], d = v[1] - m;
      m += d * (v[0] / n);
      q += v[2] + d * d * (c * v[0] / n);
      c = n;
    }
    Sums sums{nullptr, 0, each};
    float n = c, mean = c * m;
    sums(n, mean);
    mean /= n;
    q += c * (m - mean) * (m - mean);
    sums(q);
    if (lane == 0 && g < t.ng) {
      sm[g] = mean;
      sr[g] = 1.f / sqrtf(q / n + a.eps);
      if (t.at(a) == 0) {
        if (a.mean) a.mean[t.n * a.G + t.g0 + g] = mean;
        if (a.rstd) a.rstd[t.n * a.G + t.g0 + g] = sr[g];
      }
    }
  }
  __syncthreads();
  if (!t.mine) return;
  const int g = t.col / a.Cg - t.g0;
  const float mean = sm[g], rstd = sr[g];
  float w[V], b[V];
  get_param<V>(w, a.w, a.wbf, 1.f, t.col);
  get_param<V>(b, a.b, a.wbf, 0.f, t.col);
#pragma unroll 4
  for (int s = t.s0 + t.row; s < t.s1; s += t.step) {
    const int64_t at = t.base(a, s);
    float x[V], z[V], y[V];
    get<T, V>(x, (const T*)a.x + at);
    if (OPS & kGate) get<T, V>(z, (const T*)a.z + at);
#pragma unroll
    for (int i = 0; i < V; ++i)
      y[i] = result<OPS>((x[i] - mean) * rstd, w[i], b[i], OPS & kGate ? z[i] : 0.f);
    put<T, V>((T*)a.out + at, y);
  }
}

// The sums of dn h and dn of a part of the positions, of every nrows-th n: [nrows sparts][C], then
// the same for dn; behind them what the groups' means need of each n, the sums of dh h and dh:
// [N][G][parts][2].  (A row of each n is as long as a few positions of it, and the rows are added
// up one after the other.  8192 rows of 16384, bf16: 763 us and 34 MB, with a row each 897 and
// 1.1 GB; 65536 n's of 4 positions, 8 groups of 8: 250 and 310 us.)
template <typename T, int V, int OPS>
__global__ __launch_bounds__(256) void k_gn_sums(const GroupArgs a) {
  __shared__ float s1[256 * V], s2[256 * V];
  Tile t = Tile::of<V>(a);
  float w[V], b[V], sw[V], sb[V];  // sw, sb: of channel c0 + threadIdx.x + 256 i, over the n's
#pragma unroll
  for (int i = 0; i < V; ++i) sw[i] = sb[i] = 0.f;
  get_param<V>(w, t.mine ? a.w : nullptr, a.wbf, 1.f, t.col);
  get_param<V>(b, t.mine ? a.b : nullptr, a.wbf, 0.f, t.col);
  float* to = a.ws + (t.n * a.sparts + t.part) * a.C + t.c0;
  const int64_t half = (int64_t)a.nrows * a.sparts * a.C;
  const int per = t.cols * V / t.ng, lane = threadIdx.x & 15, parts = t.parts(a);
  for (; t.n < a.N; t.n += a.nrows, t.row0 = t.n * a.S) {
    float dw[V], db[V];
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
    if (t.mine) {
      const int g = t.col / a.Cg;
      const float mean = a.mean_in[t.n * a.G + g], rstd = a.rstd_in[t.n * a.G + g];
#pragma unroll 4
      for (int s = t.s0 + t.row; s < t.s1; s += t.step) {
        const int64_t at = t.base(a, s);
        float x[V], dy[V], z[V];
        get<T, V>(x, (const T*)a.x + at);
        get<T, V>(dy, (const T*)a.dy + at);
        if (OPS & kGate) get<T, V>(z, (const T*)a.z + at);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float dz;
          const float h = (x[i] - mean) * rstd;
          const float dn = grad<OPS>(h, w[i], b[i], OPS & kGate ? z[i] : 0.f, dy[i], dz);
          dw[i] = __builtin_fmaf(dn, h, dw[i]);
          db[i] += dn;
        }
      }
    }
    __syncthreads();  // (the groups' sums of the n before have been read)
#pragma unroll
    for (int i = 0; i < V; ++i) s1[threadIdx.x * V + i] = dw[i], s2[threadIdx.x * V + i] = db[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = threadIdx.x + 256 * i;
      if (c < t.cols * V) {
        float x = 0.f, y = 0.f, f[1];
        for (int r = 0; r < t.step; ++r) x += s1[r * t.cols * V + c], y += s2[r * t.cols * V + c];
        sw[i] += x;
        sb[i] += y;
        get_param<1>(f, a.w, a.wbf, 1.f, t.c0 + c);
        s1[c] = f[0] * x, s2[c] = f[0] * y;  // (read by this thread alone until here)
      }
    }
    __syncthreads();
    for (int g0 = 0; g0 < t.ng; g0 += 16) {
      const int g = g0 + (int)(threadIdx.x >> 4);
      float x = 0.f, y = 0.f;
      if (g < t.ng)
        for (int i = lane; i < per; i += 16) x += s1[g * per + i], y += s2[g * per + i];
      x = sum_lanes<16>(x), y = sum_lanes<16>(y);
      if (lane == 0 && g < t.ng) {
        float* m = a.ws + 2 * half + ((t.n * a.G + t.g0 + g) * parts + t.at(a)) * 2;
        m[0] = x, m[1] = y;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = threadIdx.x + 256 * i;
    if (c < t.cols * V) to[c] = sw[i], to[half + c] = sb[i];
  }
}

// dw[c] (dn h) and db[c]: sums over the parts, 16 threads a column and 16 columns a workgroup
__device__ __forceinline__ void sum_parts(const GroupArgs& a, int64_t parts, int block) {
  __shared__ float s[16][17];
  const int blocks = (a.C + 15) / 16, second = block >= blocks;
  const float* from = a.ws + (second ? parts * a.C : 0);
  float* to = second ? a.db : a.dw;
  if (!to) return;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, d = (block - second * blocks) * 16 + c;
  float x = 0.f;
  if (d < a.C)
#pragma unroll 8
    for (int64_t p = r; p < parts; p += 16) x += from[p * a.C + d];
  s[r][c] = x;
  __syncthreads();
  if (r == 0 && d < a.C) {
#pragma unroll
    for (int i = 1; i < 16; ++i) x += s[i][c];
    to[d] = x;
  }
}
__global__ __launch_bounds__(256) void k_gn_parts(const GroupArgs a, int64_t parts) {
  sum_parts(a, parts, (int)blockIdx.x);
}

// (the first blocks add up dw and db)
template <typename T, int V, int OPS>
__global__ __launch_bounds__(256) void k_gn_dx(const GroupArgs a, int adding) {
  if ((int)blockIdx.x < adding) return sum_parts(a, a.nrows * a.sparts, (int)blockIdx.x);
  __shared__ float m1[256], m2[256];
  const Tile t = Tile::of<V>(a, blockIdx.x - adding);
  const float* sums = a.ws + 2 * ((int64_t)a.nrows * a.sparts * a.C);
  const int parts = t.parts(a);
  const float inv = 1.f / ((float)a.S * (float)a.Cg);
  const int each = t.threads_a_group(), lane = (int)threadIdx.x % each;
  for (int g0 = 0; g0 < t.ng; g0 += 256 / each) {
    const int g = g0 + (int)threadIdx.x / each;
    const float* p = sums + (t.n * a.G + t.g0 + min(g, t.ng - 1)) * parts * 2;
    float x = 0.f, y = 0.f;
#pragma unroll 4
    for (int i = lane; i < parts; i += each) x += p[2 * i], y += p[2 * i + 1];
    Sums{nullptr, 0, each}(x, y);
    if (lane == 0 && g < t.ng) m2[g] = x * inv, m1[g] = y * inv;
  }
  __syncthreads();
  if (!t.mine) return;
  const int g = t.col / a.Cg;
  const int64_t ng = t.n * a.G + g;
  const float mean = a.mean_in[ng], rstd = a.rstd_in[ng], s1 = m1[g - t.g0], s2 = m2[g - t.g0];
  float w[V], b[V];
  get_param<V>(w, a.w, a.wbf, 1.f, t.col);
  get_param<V>(b, a.b, a.wbf, 0.f, t.col);
#pragma unroll 4
  for (int s = t.s0 + t.row; s < t.s1; s += t.step) {
    const int64_t at = t.base(a, s);
    float x[V], dy[V], z[V], dz[V];
    get<T, V>(x, (const T*)a.x + at);
    get<T, V>(dy, (const T*)a.dy + at);
    if (OPS & kGate) get<T, V>(z, (const T*)a.z + at);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float h = (x[i] - mean) * rstd;
      const float dn = grad<OPS>(h, w[i], b[i], OPS & kGate ? z[i] : 0.f, dy[i], dz[i]);
      x[i] = rstd * (dn * w[i] - s1 - h * s2);
    }
    put<T, V>((T*)a.out + at, x);
    if (OPS & kGate) put<T, V>((T*)a.dz + at, dz);
  }
}

// ---------------------------------------------------------------------------
// launch shapes

namespace {

int pow2_up(int64_t x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}
int largest_divisor(int n, int most) {
  for (int d = std::min(n, most); d > 1; --d)
    if (n % d == 0) return d;
  return 1;
}

// values a thread takes at once
int vec_of(int Cg, int dtype) {
  if (dtype == 0) return Cg % 4 == 0 ? 4 : 1;
  return Cg % 8 == 0 ? 8 : Cg % 2 == 0 ? 2 : 1;
}

// pieces a thread holds, threads of a workgroup and of a group; 0 where a group is read twice.
// (4 x 4096 positions of 32 groups of 16 channels in bf16, the groups in registers of 1024
// threads, 32 bytes of a position each: 45 us, read twice 20.)
struct RowShape { int nv, b, tpi; };
RowShape row_shape(int64_t pieces, int S, bool grad) {
  if (grad && S > 1) return {0, 0, 0};
  if (pieces <= 64) return {1, grad ? 1024 : 256, pow2_up(pieces)};
  if (pieces <= 128) return {2, 256, 64};
  if (pieces <= 256) return {4, 256, 64};
  if (S == 1 && pieces <= 1024) return {4, 256, 256};
  return {0, 0, 0};
}

// the groups of a workgroup, how many n's side by side, and the parts of the n's
int row_parts(GroupArgs& a, const RowShape& r, bool grad) {
  const int ipb = r.b / r.tpi;
  a.tpi = r.tpi;
  a.gw = largest_divisor(a.G, ipb);
  a.nw = std::max(1, ipb / a.gw);
  const int64_t blocks = a.G / a.gw, rounds = (a.N + a.nw - 1) / a.nw;
  const int64_t most = std::max<int64_t>(1, (grad ? 1024 : 2048) * 256 / r.b / blocks);
  return (int)std::max<int64_t>(1, std::min(rounds, most));
}

// groups read twice: column blocks, parts of the positions, and n's that have sums of dw and db of
// their own (the others are added to these: 2048 workgroups are as many as run at a time)
void tile_parts(GroupArgs& a, int V) {
  const int64_t pr = a.Cg / V;
  a.cblocks = (int)(pr <= 256 ? (a.G + 256 / pr - 1) / (256 / pr) : a.G * ((pr + 255) / 256));
  const int64_t cols = pr <= 256 ? pr * std::min<int64_t>(a.G, 256 / pr) : 256;
  const int64_t step = std::max<int64_t>(1, 256 / cols);
  const int64_t want = std::max<int64_t>(1, 768 / std::max<int64_t>(1, a.N * a.cblocks));
  const int64_t most = std::max<int64_t>(1, a.S / (8 * step));  // eight positions a thread
  a.sparts = (int)std::min<int64_t>(std::min(want, most), 256);
  a.nrows = (int)std::min<int64_t>(a.N, std::max(1, 2048 / (a.sparts * a.cblocks)));
}

}  // namespace

namespace {
GroupArgs sizes(int64_t N, int S, int G, int Cg) {
  GroupArgs a{};
  a.N = N, a.S = S, a.G = G, a.Cg = Cg, a.C = G * Cg;
  return a;
}
RowShape shape_of(int S, int Cg, int V, bool grad) {
  return row_shape((int64_t)S * (Cg / V), S, grad);
}
int64_t parts_a_group(const GroupArgs& a, int V) {
  const int pr = a.Cg / V;
  return (int64_t)a.sparts * (pr > 256 ? (pr + 255) / 256 : 1);
}
}  // namespace

int64_t group_forward_blocks(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  if (shape_of(S, Cg, V, false).nv) return 0;
  tile_parts(a, V);
  return N * a.sparts * a.cblocks;
}
int64_t group_forward_workspace(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  if (shape_of(S, Cg, V, false).nv) return 0;
  tile_parts(a, V);
  return N * G * parts_a_group(a, V) * 4;
}

int64_t group_backward_blocks(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  if (shape_of(S, Cg, V, true).nv) return 0;
  tile_parts(a, V);
  return N * a.sparts * a.cblocks + 2 * ((a.C + 15) / 16);
}
int64_t group_backward_workspace(int64_t N, int S, int G, int Cg, int dtype, bool sums) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  const RowShape r = shape_of(S, Cg, V, true);
  if (r.nv) return sums ? 2ll * row_parts(a, r, true) * a.C : 0;
  tile_parts(a, V);
  return 2ll * a.nrows * a.sparts * a.C + 2 * N * G * parts_a_group(a, V);
}

template <typename T, int V, int OPS>
static hipError_t group_forward(GroupArgs a, hipStream_t st) {
  const RowShape r = shape_of(a.S, a.Cg, V, false);
  if (r.nv) {
    const dim3 grid((unsigned)(row_parts(a, r, false) * (a.G / a.gw)));
    if (r.nv == 1)
      hipLaunchKernelGGL((k_gn_rows<T, V, 1, OPS>), grid, dim3(256), 0, st, a);
    else if (r.nv == 2)
      hipLaunchKernelGGL((k_gn_rows<T, V, 2, OPS>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((k_gn_rows<T, V, 4, OPS>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
  }
  tile_parts(a, V);
  const dim3 grid((unsigned)(a.N * a.sparts * a.cblocks));
  hipLaunchKernelGGL((k_gn_stats<T, V>), grid, dim3(256), 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((k_gn_apply<T, V, OPS>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T, int V, int OPS>
static hipError_t group_backward(GroupArgs a, hipStream_t st) {
  const RowShape r = shape_of(a.S, a.Cg, V, true);
  const unsigned adding = a.dw || a.db ? 2 * ((a.C + 15) / 16) : 0;
  int64_t parts = 0;
  if (a.N > 0 && !r.nv) {
    tile_parts(a, V);
    const unsigned each = (unsigned)(a.sparts * a.cblocks);
    hipLaunchKernelGGL((k_gn_sums<T, V, OPS>), dim3(a.nrows * each), dim3(256), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((k_gn_dx<T, V, OPS>), dim3((unsigned)a.N * each + adding), dim3(256), 0, st,
                       a, (int)adding);
    return hipGetLastError();
  }
  if (a.N > 0) {
    parts = row_parts(a, r, true);
    const dim3 grid((unsigned)(parts * (a.G / a.gw)));
    const size_t lds = (64 + (a.nw > 1 ? of_sums(a.nw) * 2 * (size_t)a.gw * a.Cg : 0)) * sizeof(float);
    if (r.nv == 1)
      hipLaunchKernelGGL((k_gn_rows_grad<T, V, 1, 1024, OPS>), grid, dim3(1024), lds, st, a, (int)parts);
    else if (r.nv == 2)
      hipLaunchKernelGGL((k_gn_rows_grad<T, V, 2, 256, OPS>), grid, dim3(256), lds, st, a, (int)parts);
    else
      hipLaunchKernelGGL((k_gn_rows_grad<T, V, 4, 256, OPS>), grid, dim3(256), lds, st, a, (int)parts);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (!adding) return hipSuccess;
  hipLaunchKernelGGL(k_gn_parts, dim3(adding), dim3(256), 0, st, a, parts);
  return hipGetLastError();
}

// by type, values a piece and what follows n
template <int OPS>
static hipError_t by_width(const GroupArgs& a, int dtype, bool grad, hipStream_t st) {
  const int v = vec_of(a.Cg, dtype);
#define GDN_X(T, V) return grad ? group_backward<T, V, OPS>(a, st) : group_forward<T, V, OPS>(a, st)
  if (dtype == 0) {
    if (v == 4) GDN_X(float, 4);
    GDN_X(float, 1);
  }
  if (v == 8) GDN_X(__bf16, 8);
  if (v == 2) GDN_X(__bf16, 2);
  GDN_X(__bf16, 1);
#undef GDN_X
}
static hipError_t by_ops(const GroupArgs& a, int dtype, bool grad, hipStream_t st) {
  switch ((a.act ? kAct : 0) | (a.z ? kGate : 0)) {
    case 0: return by_width<0>(a, dtype, grad, st);
    case kAct: return by_width<kAct>(a, dtype, grad, st);
    case kGate: return by_width<kGate>(a, dtype, grad, st);
    default: return by_width<kAct | kGate>(a, dtype, grad, st);
  }
}

hipError_t launch_group_forward(const GroupArgs& a, int dtype, hipStream_t st) {
  return by_ops(a, dtype, false, st);
}
hipError_t launch_group_backward(const GroupArgs& a, int dtype, hipStream_t st) {
  return by_ops(a, dtype, true, st);
}

}  // namespace gdn
