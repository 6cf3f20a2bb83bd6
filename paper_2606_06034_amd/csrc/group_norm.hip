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
#include <algorithm>

#include "group_norm.hpp"
#include "lanes.hpp"
#include "launch.hpp"
#include "norm.hpp"

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
// a weight or bias in either dtype; `none` where there is none.  (Its rows need no more than
// an element's alignment.)
template <int V>
__device__ __forceinline__ void get_param(float (&x)[V], const void* p, bool bf, float none,
                                          int at) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    x[i] = !p ? none : bf ? (float)((const __bf16*)p)[at + i] : ((const float*)p)[at + i];
}

__device__ __forceinline__ float silu_grad(float t) {
  const float s = sigmoid(t);
  return s * __builtin_fmaf(t, 1.f - s, 1.f);
}

// the results of one value
__device__ __forceinline__ float result(const GroupArgs& a, float h, float w, float b, float z) {
  float n = __builtin_fmaf(h, w, b);
  if (a.act) n *= sigmoid(n);
  if (a.z) n *= z * sigmoid(z);
  return n;
}
// dn (and dz) of one value
__device__ __forceinline__ float grad(const GroupArgs& a, float h, float w, float b, float z,
                                      float dy, float& dz) {
  const float n = __builtin_fmaf(h, w, b);
  if (a.z) {
    const float s = sigmoid(z);
    dz = dy * (a.act ? n * sigmoid(n) : n) * (s * __builtin_fmaf(z, 1.f - s, 1.f));
    dy *= z * s;
  }
  return a.act ? dy * silu_grad(n) : dy;
}

// sums over the `tpi` neighbouring threads (a power of two) of a group; past a wave they
// meet in LDS, in two buffers that the calls take in turn
struct Sums {
  float* red;
  int buf, tpi;
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
// walks the n's; piece k of thread t of a group is its (t + k tpi)-th piece of V values.
template <typename T, int V, int NV, int B>
__global__ __launch_bounds__(B) void k_gn_rows(const GroupArgs a) {
  __shared__ float red[64];
  Sums sums{red, 0, a.tpi};
  const int slot = (int)threadIdx.x / a.tpi, t = (int)threadIdx.x - slot * a.tpi;
  const int blocks = a.G / a.gw, gb = (int)(blockIdx.x % blocks), nb = (int)(blockIdx.x / blocks);
  const int ni = slot / a.gw, g = gb * a.gw + slot - ni * a.gw;
  const bool mine = ni < a.nw;
  const int pr = a.Cg / V, pieces = a.S * pr;
  constexpr bool HOLD = NV <= 2;  // (weights and gates past that are read where they are used)
  constexpr int H = HOLD ? NV : 1;
  float w[H][V], b[H][V];
  int at[NV], ch[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int p = t + k * a.tpi, s = p / pr;
    ch[k] = g * a.Cg + (p - s * pr) * V;
    at[k] = mine && p < pieces ? s * a.C + ch[k] : -1;
    if constexpr (HOLD) {
      get_param<V>(w[k], at[k] < 0 ? nullptr : a.w, a.wbf, 1.f, ch[k]);
      get_param<V>(b[k], at[k] < 0 ? nullptr : a.b, a.wbf, 0.f, ch[k]);
    }
  }
  const float inv = 1.f / (float)(a.S * a.Cg);
  const int parts = (int)(gridDim.x / blocks);
  for (int64_t n0 = (int64_t)nb * a.nw; n0 < a.N; n0 += (int64_t)parts * a.nw) {
    const int64_t n = n0 + ni, base = n * a.S * a.C;
    const bool live = mine && n < a.N;
    float x[NV][V], z[H][V], mean = 0.f, var = 0.f, none = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) x[k][i] = 0.f;
      if (live && at[k] >= 0) {
        get<T, V>(x[k], (const T*)a.x + base + at[k]);
        if constexpr (HOLD)
          if (a.z) get<T, V>(z[k], (const T*)a.z + base + at[k]);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) mean += x[k][i];
    }
    sums(mean, none);
    mean *= inv;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] = at[k] >= 0 ? x[k][i] - mean : 0.f;
        var = __builtin_fmaf(x[k][i], x[k][i], var);
      }
    sums(var, none);
    const float rstd = 1.f / sqrtf(var * inv + a.eps);
    if (!live) continue;
    if (t == 0) {
      if (a.mean) a.mean[n * a.G + g] = mean;
      if (a.rstd) a.rstd[n * a.G + g] = rstd;
    }
    const void *wp = a.w, *bp = a.b;
    if constexpr (!HOLD) asm volatile("" : "+s"(wp), "+s"(bp));  // (not read ahead of the loop)
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at[k] >= 0) {
        constexpr int O = HOLD ? 1 : 0;
        float y[V];
        if constexpr (!HOLD) {
          get_param<V>(w[0], wp, a.wbf, 1.f, ch[k]);
          get_param<V>(b[0], bp, a.wbf, 0.f, ch[k]);
          if (a.z) get<T, V>(z[0], (const T*)a.z + base + at[k]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
          y[i] = result(a, x[k][i] * rstd, w[O * k][i], b[O * k][i], a.z ? z[O * k][i] : 0.f);
        put<T, V>((T*)a.out + base + at[k], y);
      }
  }
}

// The gradients where S = 1.  The n's that run side by side add up their dw and db in LDS, the
// workgroups' sums go to row nb of the workspace: [parts][C], then the same for db.
template <typename T, int V, int NV, int B>
__global__ __launch_bounds__(B) void k_gn_rows_grad(const GroupArgs a, int parts) {
  extern __shared__ float lds[];  // 64 values of the sums, then [2][gw Cg]
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
  for (int64_t n0 = (int64_t)nb * a.nw; n0 < a.N; n0 += (int64_t)parts * a.nw) {
    const int64_t n = n0 + ni, base = n * a.C;
    const bool live = mine && n < a.N;
    const float mean = live ? a.mean_in[n * a.G + g] : 0.f;
    const float rstd = live ? a.rstd_in[n * a.G + g] : 0.f;
    float h[NV][V], dn[NV][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] = dn[k][i] = 0.f;
      if (live && at[k] >= 0) {
        float z[V], dz[V];
        get<T, V>(h[k], (const T*)a.x + base + at[k]);
        get<T, V>(dn[k], (const T*)a.dy + base + at[k]);
        if (a.z) get<T, V>(z, (const T*)a.z + base + at[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          h[k][i] = (h[k][i] - mean) * rstd;
          dn[k][i] = grad(a, h[k][i], w[k][i], b[k][i], a.z ? z[i] : 0.f, dn[k][i], dz[i]);
          const float dh = dn[k][i] * w[k][i];
          s1 += dh;
          s2 = __builtin_fmaf(dh, h[k][i], s2);
        }
        if (a.z) put<T, V>((T*)a.dz + base + at[k], dz);
      }
    }
    sums(s1, s2);
    s1 *= inv, s2 *= inv;
    if (!live) continue;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at[k] >= 0) {
        float dx[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dx[i] = rstd * (dn[k][i] * w[k][i] - s1 - h[k][i] * s2);
          dw[k][i] = __builtin_fmaf(dn[k][i], h[k][i], dw[k][i]);
          db[k][i] += dn[k][i];
        }
        put<T, V>((T*)a.out + base + at[k], dx);
      }
  }
  if (!a.dw && !a.db) return;
  float* sum = lds + 64;
  const int width = a.gw * a.Cg;
  float* to = a.ws + (int64_t)nb * a.C + (int64_t)gb * width;
  if (a.nw == 1) {  // the sums are whole
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (at[k] >= 0)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          to[at[k] - gb * width + i] = dw[k][i];
          to[(int64_t)parts * a.C + at[k] - gb * width + i] = db[k][i];
        }
    return;
  }
  for (int r = 0; r < a.nw; ++r) {
    if (mine && ni == r)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (at[k] >= 0)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int c = at[k] - gb * width + i;
            sum[c] = r ? sum[c] + dw[k][i] : dw[k][i];
            sum[width + c] = r ? sum[width + c] + db[k][i] : db[k][i];
          }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < width; c += B) {
    to[c] = sum[c];
    to[(int64_t)parts * a.C + c] = sum[width + c];
  }
}

// ---- groups read twice.  A workgroup has the positions s0 .. s1 of one n and a block of
// `cols` pieces of V channels: whole groups where a group has up to 256 pieces, else a part of
// one.  Thread t has piece t % cols, and every (256 / cols)-th position.
struct Tile {
  int64_t n, row0;  // row0: n S
  int part, s0, s1, cols, c0, col, row, step, g0, ng;
  bool mine;
  template <int V> static __device__ __forceinline__ Tile of(const GroupArgs& a) {
    Tile t;
    const uint32_t pn = (uint32_t)a.sparts * (uint32_t)a.cblocks;
    t.n = blockIdx.x / pn;
    const int at = (int)(blockIdx.x - (uint32_t)t.n * pn);
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
    } else {
      const int per = (pr + 255) / 256;  // blocks a group
      t.g0 = cb / per;
      t.ng = 1;
      const int p0 = (cb - t.g0 * per) * 256;
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
  const int per = t.cols / t.ng, cb = a.Cg / V > 256 ? (t.c0 - t.g0 * a.Cg) / (256 * V) : 0;
  const int cparts = a.Cg / V > 256 ? (a.Cg / V + 255) / 256 : 1, parts = a.sparts * cparts;
  sum_groups(
      t,
      [&](int i) {
        const int g = i % t.cols / per;
        const float d = gn[g] > 0.f ? sm[i] - gm[g] / gn[g] : 0.f;
        return sq[i] + sc[i] * d * d;
      },
      [&](int g, float x) {
        float* to = a.ws + ((t.n * a.G + t.g0 + g) * parts + t.part * cparts + cb) * 4;
        to[0] = gn[g], to[1] = gn[g] > 0.f ? gm[g] / gn[g] : 0.f, to[2] = x;
      });
}

template <typename T, int V>
__global__ __launch_bounds__(256) void k_gn_apply(const GroupArgs a) {
  __shared__ float sm[256], sr[256];
  const Tile t = Tile::of<V>(a);
  const int parts = a.sparts * (a.Cg / V > 256 ? (a.Cg / V + 255) / 256 : 1);
  for (int g0 = 0; g0 < t.ng; g0 += 16) {  // 16 threads a group join its parts
    const int g = g0 + (int)(threadIdx.x >> 4), lane = threadIdx.x & 15;
    const float* p = a.ws + (t.n * a.G + t.g0 + min(g, t.ng - 1)) * parts * 4;
    float c = 0.f, m = 0.f, q = 0.f;
    for (int i = lane; i < parts; i += 16) c += p[4 * i], m += p[4 * i] * p[4 * i + 1];
    c = sum_lanes<16>(c);
    m = sum_lanes<16>(m) / c;
    for (int i = lane; i < parts; i += 16) {
      const float d = p[4 * i + 1] - m;
      q += p[4 * i + 2] + p[4 * i] * d * d;
    }
    q = sum_lanes<16>(q) / c;
    if (lane == 0 && g < t.ng) {
      sm[g] = m;
      sr[g] = 1.f / sqrtf(q + a.eps);
      if (t.part == 0 && t.c0 == t.g0 * a.Cg) {
        if (a.mean) a.mean[t.n * a.G + t.g0 + g] = m;
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
    if (a.z) get<T, V>(z, (const T*)a.z + at);
#pragma unroll
    for (int i = 0; i < V; ++i)
      y[i] = result(a, (x[i] - mean) * rstd, w[i], b[i], a.z ? z[i] : 0.f);
    put<T, V>((T*)a.out + at, y);
  }
}

// the sums of dn h and dn of a part of the positions: [N sparts][C], then the same for dn
template <typename T, int V>
__global__ __launch_bounds__(256) void k_gn_sums(const GroupArgs a) {
  __shared__ float s1[256 * V], s2[256 * V];
  const Tile t = Tile::of<V>(a);
  float dw[V], db[V], w[V], b[V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
  if (t.mine) {
    const int g = t.col / a.Cg;
    const float mean = a.mean_in[t.n * a.G + g], rstd = a.rstd_in[t.n * a.G + g];
    get_param<V>(w, a.w, a.wbf, 1.f, t.col);
    get_param<V>(b, a.b, a.wbf, 0.f, t.col);
#pragma unroll 4
    for (int s = t.s0 + t.row; s < t.s1; s += t.step) {
      const int64_t at = t.base(a, s);
      float x[V], dy[V], z[V];
      get<T, V>(x, (const T*)a.x + at);
      get<T, V>(dy, (const T*)a.dy + at);
      if (a.z) get<T, V>(z, (const T*)a.z + at);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float dz;
        const float h = (x[i] - mean) * rstd;
        const float dn = grad(a, h, w[i], b[i], a.z ? z[i] : 0.f, dy[i], dz);
        dw[i] = __builtin_fmaf(dn, h, dw[i]);
        db[i] += dn;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) s1[threadIdx.x * V + i] = dw[i], s2[threadIdx.x * V + i] = db[i];
  __syncthreads();
  float* to = a.ws + (t.n * a.sparts + t.part) * a.C + t.c0;
  const int64_t half = a.N * a.sparts * a.C;
  for (int c = threadIdx.x; c < t.cols * V; c += 256) {
    float x = 0.f, y = 0.f;
    for (int r = 0; r < t.step; ++r) x += s1[r * t.cols * V + c], y += s2[r * t.cols * V + c];
    to[c] = x;
    to[half + c] = y;
  }
}

// what the groups' means need of them: mean(dh h) and mean(dh) of each (n, group), behind the
// sums in the workspace
__global__ __launch_bounds__(256) void k_gn_means(const GroupArgs a) {
  __shared__ float red[64];
  Sums sums{red, 0, 256};
  const int64_t n = blockIdx.x / (uint32_t)a.G, half = a.N * a.sparts * a.C;
  const int g = (int)(blockIdx.x - (uint32_t)n * (uint32_t)a.G);
  const float* from = a.ws + n * a.sparts * a.C + g * a.Cg;
  float x = 0.f, y = 0.f;
  for (int i = threadIdx.x; i < a.Cg * a.sparts; i += 256) {
    const int p = i / a.Cg, c = i - p * a.Cg;
    float w[1];
    get_param<1>(w, a.w, a.wbf, 1.f, g * a.Cg + c);
    x += w[0] * from[(int64_t)p * a.C + c];
    y += w[0] * from[half + (int64_t)p * a.C + c];
  }
  sums(x, y);
  if (threadIdx.x == 0) {
    const float inv = 1.f / ((float)a.S * (float)a.Cg);
    a.ws[2 * half + 2 * blockIdx.x] = x * inv;
    a.ws[2 * half + 2 * blockIdx.x + 1] = y * inv;
  }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void k_gn_dx(const GroupArgs a) {
  const Tile t = Tile::of<V>(a);
  if (!t.mine) return;
  const int g = t.col / a.Cg;
  const int64_t ng = t.n * a.G + g;
  const float mean = a.mean_in[ng], rstd = a.rstd_in[ng];
  const float* m = a.ws + 2 * (a.N * a.sparts * a.C) + 2 * ng;
  const float s2 = m[0], s1 = m[1];
  float w[V], b[V];
  get_param<V>(w, a.w, a.wbf, 1.f, t.col);
  get_param<V>(b, a.b, a.wbf, 0.f, t.col);
#pragma unroll 4
  for (int s = t.s0 + t.row; s < t.s1; s += t.step) {
    const int64_t at = t.base(a, s);
    float x[V], dy[V], z[V], dz[V];
    get<T, V>(x, (const T*)a.x + at);
    get<T, V>(dy, (const T*)a.dy + at);
    if (a.z) get<T, V>(z, (const T*)a.z + at);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float h = (x[i] - mean) * rstd;
      const float dn = grad(a, h, w[i], b[i], a.z ? z[i] : 0.f, dy[i], dz[i]);
      x[i] = rstd * (dn * w[i] - s1 - h * s2);
    }
    put<T, V>((T*)a.out + at, x);
    if (a.z) put<T, V>((T*)a.dz + at, dz);
  }
}

// dw[c] (dn h) and db[c]: sums over the parts, 16 threads a column and 16 columns a workgroup
__global__ __launch_bounds__(256) void k_gn_parts(const float* __restrict__ ws, float* dw,
                                                  float* db, int64_t parts, int C) {
  __shared__ float s[16][17];
  const float* from = ws + (blockIdx.y ? parts * C : 0);
  float* to = blockIdx.y ? db : dw;
  if (!to) return;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, d = blockIdx.x * 16 + c;
  float x = 0.f;
  if (d < C)
#pragma unroll 8
    for (int64_t p = r; p < parts; p += 16) x += from[p * C + d];
  s[r][c] = x;
  __syncthreads();
  if (r == 0 && d < C) {
#pragma unroll
    for (int i = 1; i < 16; ++i) x += s[i][c];
    to[d] = x;
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

// pieces a thread holds, threads of a workgroup and of a group; 0 where a group is too long
struct RowShape { int nv, b, tpi; };
RowShape row_shape(int64_t pieces, bool grad) {
  if (pieces <= 64) return {1, 256, pow2_up(pieces)};
  if (pieces <= 128) return {2, 256, 64};
  if (pieces <= 256) return {4, 256, 64};
  if (pieces <= 1024) return {4, 256, 256};
  if (!grad && pieces <= 4096) return {4, 1024, 1024};
  if (!grad && pieces <= 8192) return {8, 1024, 1024};
  return {0, 0, 0};
}

// the groups of a workgroup, how many n's side by side, and the parts of the n's
int row_parts(GroupArgs& a, const RowShape& r, bool grad) {
  const int ipb = r.b / r.tpi;
  a.tpi = r.tpi;
  a.gw = largest_divisor(a.G, ipb);
  a.nw = std::max(1, ipb / a.gw);
  const int64_t blocks = a.G / a.gw, rounds = (a.N + a.nw - 1) / a.nw;
  const int64_t most = std::max<int64_t>(1, (grad ? 1024 : 8192) * 256 / r.b / blocks);
  return (int)std::max<int64_t>(1, std::min(rounds, most));
}

// groups read twice: column blocks, and parts of the positions
void tile_parts(GroupArgs& a, int V) {
  const int64_t pr = a.Cg / V;
  a.cblocks = pr <= 256 ? (int)((a.G + 256 / pr - 1) / (256 / pr)) : (int)(a.G * ((pr + 255) / 256));
  const int step = pr <= 256 ? (int)std::max<int64_t>(1, 256 / (pr * std::min<int64_t>(a.G, 256 / pr))) : 1;
  const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(1, a.N * a.cblocks));
  const int64_t most = std::max<int64_t>(1, a.S / (8ll * step));  // eight positions a thread
  a.sparts = (int)std::min<int64_t>(std::min(want, most), 256);
}

}  // namespace

namespace {
GroupArgs sizes(int64_t N, int S, int G, int Cg) {
  GroupArgs a{};
  a.N = N, a.S = S, a.G = G, a.Cg = Cg, a.C = G * Cg;
  return a;
}
bool in_registers(int S, int Cg, int V, bool grad) {
  return grad ? S == 1 && row_shape(Cg / V, true).nv : row_shape((int64_t)S * (Cg / V), false).nv;
}
}  // namespace

int64_t group_forward_blocks(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  if (in_registers(S, Cg, V, false)) return 0;
  tile_parts(a, V);
  return N * a.sparts * a.cblocks;
}
int64_t group_forward_workspace(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype), pr = Cg / V;
  if (in_registers(S, Cg, V, false)) return 0;
  tile_parts(a, V);
  return N * G * a.sparts * (pr > 256 ? (pr + 255) / 256 : 1) * 4;
}

int64_t group_backward_blocks(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  if (in_registers(S, Cg, V, true)) return 0;
  tile_parts(a, V);
  return N * std::max<int64_t>((int64_t)a.sparts * a.cblocks, G);
}
int64_t group_backward_workspace(int64_t N, int S, int G, int Cg, int dtype) {
  GroupArgs a = sizes(N, S, G, Cg);
  const int V = vec_of(Cg, dtype);
  if (in_registers(S, Cg, V, true)) return 2ll * row_parts(a, row_shape(Cg / V, true), true) * a.C;
  tile_parts(a, V);
  return 2 * N * a.sparts * a.C + 2 * N * G;
}

#define GDN_GN_ROWS(X) X(1, 256) X(2, 256) X(4, 256)

template <typename T, int V>
static hipError_t group_forward(GroupArgs a, hipStream_t st) {
  const RowShape r = row_shape((int64_t)a.S * (a.Cg / V), false);
  if (r.nv) {
    const unsigned grid = (unsigned)(row_parts(a, r, false) * (a.G / a.gw));
#define GDN_X(NV, B)                                                              \
  if (r.nv == NV && r.b == B) {                                                   \
    hipLaunchKernelGGL((k_gn_rows<T, V, NV, B>), dim3(grid), dim3(B), 0, st, a);  \
    return hipGetLastError();                                                     \
  }
    GDN_GN_ROWS(GDN_X) GDN_X(4, 1024) GDN_X(8, 1024)
#undef GDN_X
    return hipErrorNotSupported;
  }
  tile_parts(a, V);
  const unsigned grid = (unsigned)(a.N * a.sparts * a.cblocks);
  hipLaunchKernelGGL((k_gn_stats<T, V>), dim3(grid), dim3(256), 0, st, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((k_gn_apply<T, V>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T, int V>
static hipError_t group_backward(GroupArgs a, hipStream_t st) {
  int64_t parts = 0;
  if (a.N == 0) {
  } else if (in_registers(a.S, a.Cg, V, true)) {
    const RowShape r = row_shape(a.Cg / V, true);
    parts = row_parts(a, r, true);
    const unsigned grid = (unsigned)(parts * (a.G / a.gw));
    const size_t lds = (64 + (a.nw > 1 ? 2 * (size_t)a.gw * a.Cg : 0)) * sizeof(float);
#define GDN_X(NV, B)                                                                         \
  if (r.nv == NV && r.b == B)                                                                \
    hipLaunchKernelGGL((k_gn_rows_grad<T, V, NV, B>), dim3(grid), dim3(B), lds, st, a, (int)parts);
    GDN_GN_ROWS(GDN_X)
#undef GDN_X
  } else {
    tile_parts(a, V);
    parts = a.N * a.sparts;
    const unsigned grid = (unsigned)(parts * a.cblocks);
    hipLaunchKernelGGL((k_gn_sums<T, V>), dim3(grid), dim3(256), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL(k_gn_means, dim3((unsigned)(a.N * a.G)), dim3(256), 0, st, a);
    if (hipError_t e = hipGetLastError()) return e;
    hipLaunchKernelGGL((k_gn_dx<T, V>), dim3(grid), dim3(256), 0, st, a);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (!a.dw && !a.db) return hipSuccess;
  hipLaunchKernelGGL(k_gn_parts, dim3((unsigned)((a.C + 15) / 16), 2), dim3(256), 0, st, a.ws, a.dw,
                     a.db, parts, a.C);
  return hipGetLastError();
}

hipError_t launch_group_forward(const GroupArgs& a, int dtype, hipStream_t st) {
  const int v = vec_of(a.Cg, dtype);
  if (dtype == 0) return v == 4 ? group_forward<float, 4>(a, st) : group_forward<float, 1>(a, st);
  return v == 8   ? group_forward<__bf16, 8>(a, st)
         : v == 2 ? group_forward<__bf16, 2>(a, st)
                  : group_forward<__bf16, 1>(a, st);
}
hipError_t launch_group_backward(const GroupArgs& a, int dtype, hipStream_t st) {
  const int v = vec_of(a.Cg, dtype);
  if (dtype == 0) return v == 4 ? group_backward<float, 4>(a, st) : group_backward<float, 1>(a, st);
  return v == 8   ? group_backward<__bf16, 8>(a, st)
         : v == 2 ? group_backward<__bf16, 2>(a, st)
                  : group_backward<__bf16, 1>(a, st);
}

}  // namespace gdn
