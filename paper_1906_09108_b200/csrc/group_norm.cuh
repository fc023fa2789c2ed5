// Group normalisation with an activation, channels last, forward and backward.
//
// x [N][P][C] (P = H * W pixels); group g of image n is channels [g*Cg, (g+1)*Cg) at all pixels, m = P * Cg values:
//   mean = sum x / m,  var = sum (x - mean)^2 / m,  rstd = 1/sqrt(var + eps),  xhat = (x - mean)*rstd,
//   z = gamma*xhat + beta [+ res],  y = act(z);
//   dz = dy*act'(z),  A[n][c] = sum_p dz*xhat,  B[n][c] = sum_p dz:  dgamma = sum_n A,  dbeta = sum_n B,
//   S1 = sum over the group's channels of gamma*B,  S2 = of gamma*A,
//   dx = rstd*(gamma*dz - (S1 + xhat*S2)/m) [+ res].
// Bound by memory: 10 to 25 operations on each value against 2 to 9 bytes of traffic.  What can be won is reading each tensor
// once although every output needs sums over its whole group, and keeping enough loads in flight.
//
// Layout.  A row of a pixel's channels is cut into columns of 8 channels; a thread keeps one column and walks the pixels, rp of
// them side by side in a CTA of 256 threads, so a warp's accesses are contiguous for every channel count, and a group may start
// and end anywhere inside a column (5 channels of 160, say): sums are formed per channel and thread and added per group from
// shared memory.
//
// Two forms, chosen by gn_plan_*:
//   resident  a cluster of up to 8 CTAs takes an image, each a share of its pixels, which it copies to shared memory at once
//             (cp.async, every thread its own vectors, so nothing but a thread's own wait stands between copy and use).  The
//             statistics are formed there, exchanged through distributed shared memory, and applied from there: one launch, one
//             read, one write.
//   streamed  images that no cluster holds: a CTA per chunk of pixels leaves its sums in scratch, a small kernel adds them in a
//             fixed order, and a third pass reads the tensor again, the last chunks first, which are still in L2.
//
// Variance: within a CTA from the CTA's own mean (two sweeps over shared memory), across CTAs by Chan's formula in fp64; no
// difference of large sums is formed, so an offset of a thousand standard deviations costs no more than the inputs' own
// rounding.  All sums are fp32 within a CTA (chains of at most a few dozen values a thread, then a tree), in a fixed order.
#pragma once
#include <cooperative_groups.h>

#include "ckpt8.cuh"
#include "kernel_common.cuh"

namespace fdg {
namespace gn {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kMaxCols = kThreads;          // columns of 8 channels that a CTA addresses; wider rows go in tiles (streamed)
constexpr int kMaxCluster = 8;
enum { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2 };

struct Geom {
  int N, P, C, G, Cg;
  int cols, rp;             // columns of a CTA's tile, pixels side by side
  int parts, pix;           // CTAs per image, pixels per CTA
  int iters;                // pixels per thread: ceil(pix / rp)
  int lanes_g, lanes_c;     // lanes that add up one group / one channel
  int tiles;                // tiles of columns (1 unless streamed with more than 2048 channels)
};

// ---- device helpers -------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float silu(float z);
template <> __device__ __forceinline__ float silu<float>(float z) { return z / (1.f + expf(-z)); }
template <> __device__ __forceinline__ float silu<__nv_bfloat16>(float z) { return __fdividef(z, 1.f + __expf(-z)); }
template <typename T> __device__ __forceinline__ float silu_slope(float z) {
  const float s = sizeof(T) == 4 ? 1.f / (1.f + expf(-z)) : __fdividef(1.f, 1.f + __expf(-z));
  return s * (1.f + z * (1.f - s));
}
// NaN stays NaN.
__device__ __forceinline__ float relu(float z) { return z < 0.f ? 0.f : z; }

__device__ __forceinline__ void copy16_async(void* smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}
__device__ __forceinline__ void copy8_async(void* smem, const void* gmem) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Vectors a thread keeps in shared memory: its own [iters] of them, 16 bytes of consecutive threads side by side.
template <typename T> struct Slots {
  static constexpr int Q = sizeof(T) / 2;
  uint4* base;                // + threadIdx.x
  __device__ __forceinline__ Slots(void* smem) : base(static_cast<uint4*>(smem) + threadIdx.x) {}
  template <bool VEC> __device__ __forceinline__ void fetch(int k, const T* __restrict__ p, int left) const {
    if constexpr (VEC) {
#pragma unroll
      for (int j = 0; j < Q; ++j) copy16_async(base + (k * Q + j) * kThreads, reinterpret_cast<const uint4*>(p) + j);
    } else {
      put(k, raw8_load<T, false>(p, left));
    }
  }
  __device__ __forceinline__ Raw8<T> get(int k) const {
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < Q; ++j) r.q[j] = base[(k * Q + j) * kThreads];
    return r;
  }
  __device__ __forceinline__ void put(int k, const Raw8<T>& r) const {
#pragma unroll
    for (int j = 0; j < Q; ++j) base[(k * Q + j) * kThreads] = r.q[j];
  }
};

// This thread's place in a CTA's tile.
struct Place {
  int col, r;
  bool active;
  int c0, left;               // first channel, channels of the column that exist
  __device__ __forceinline__ Place(const Geom& g, int tile) {
    col = threadIdx.x % g.cols; r = threadIdx.x / g.cols;
    active = r < g.rp;
    c0 = (tile * kMaxCols + col) * 8;
    left = min(8, g.C - c0);
  }
  __device__ __forceinline__ int channel(int i) const { return i < left ? c0 + i : c0; }
};

// red[r][8 * cols] = the 8 sums of each thread.
__device__ __forceinline__ void put_sums(float* red, const Geom& g, const Place& at, const float (&v)[8]) {
  if (!at.active) return;
  float4* d = reinterpret_cast<float4*>(red + (at.r * g.cols + at.col) * 8);
  d[0] = make_float4(v[0], v[1], v[2], v[3]);
  d[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// done(s, sum of value(r, s*size + j) over r < rows, j < size) for s < sets: `lanes` consecutive lanes (a power of two up
// to 32) share a set.  To be called by the whole CTA.
template <typename Value, typename Done>
__device__ __forceinline__ void add_sets(int rows, int sets, int size, int lanes, Value value, Done done) {
  const int sub = threadIdx.x & (lanes - 1), per_pass = kThreads / lanes, mine = threadIdx.x / lanes;
  const int dr = lanes / size, dj = lanes - dr * size;
  const int r0 = sub / size, j0 = sub - r0 * size;
  for (int s0 = 0; s0 < sets; s0 += per_pass) {
    const int s = s0 + mine;
    float a = 0.f;
    if (s < sets) {
      int r = r0, j = j0;
      while (r < rows) {
        a += value(r, s * size + j);
        r += dr; j += dj;
        if (j >= size) { j -= size; ++r; }
      }
    }
    for (int o = lanes >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    if (s < sets && sub == 0) done(s, a);
  }
}

// ---- forward ------------------------------------------------------------------------------------------------
template <typename T> struct Forward {
  Geom g;
  const T* x;
  const float* gamma;
  const float* beta;
  const T* res;
  T* y;
  float* stats;               // mean [N][G], rstd [N][G]
  uint8_t* gate;              // bits of [y > 0], a byte per column
  int8_t* codes;              // x in 8 bits
  uint8_t* scales;
  float* partial;             // streamed: [N][parts][2][C]
  float eps;
  int act;
  int ckpt_lanes;
};

// Sums over this CTA's `count` pixels in `slots`: done(set, mean, sum of squared deviations from that mean) for sets of `size`
// consecutive channels.  `red`: 2048 floats, `mean`: a float per set.
template <typename T, typename Done>
__device__ __forceinline__ void cta_moments(const Geom& g, const Place& at, const Slots<T>& slots, int count, int sets, int size, int lanes,
                                            float* red, float* mean, Done done) {
  const int width = g.cols * 8;
  const float inv = count > 0 ? 1.f / ((float)count * (float)size) : 0.f;
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = 0.f;
  if (at.active)
#pragma unroll 4
    for (int k = 0; k < g.iters; ++k) {
      if (at.r + k * g.rp >= count) break;
      float v[8];
      raw8_to_f(slots.get(k), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] += v[i];
    }
  put_sums(red, g, at, a);
  __syncthreads();
  auto value = [&](int r, int c) { return red[r * width + c]; };
  add_sets(g.rp, sets, size, lanes, value, [&](int s, float sum) { mean[s] = sum * inv; });
  __syncthreads();
  float mu[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mu[i] = mean[min((at.col * 8 + i) / size, sets - 1)];
    a[i] = 0.f;
  }
  if (at.active)
#pragma unroll 4
    for (int k = 0; k < g.iters; ++k) {
      if (at.r + k * g.rp >= count) break;
      float v[8];
      raw8_to_f(slots.get(k), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) { const float d = v[i] - mu[i]; a[i] += d * d; }
    }
  put_sums(red, g, at, a);
  __syncthreads();
  add_sets(g.rp, sets, size, lanes, value, [&](int s, float sum) { done(s, mean[s], sum); });
}

// y (and the gate's bits, and x in 8 bits) of this CTA's pixels: fetch(k) gives the thread's k-th vector of x.
// Every lane takes every turn, since the lanes of a block of 32 channels exchange its maximum.
template <typename T, bool VEC, typename Fetch>
__device__ __forceinline__ void emit(const Forward<T>& p, const Place& at, size_t row0, int count, const float (&mean)[8],
                                     const float (&scale)[8], const float (&shift)[8], Fetch fetch) {
  const Geom& g = p.g;
  const int all_cols = (g.C + 7) >> 3;
#pragma unroll 2
  for (int k = 0; k < g.iters; ++k) {
    const int pixel = at.r + k * g.rp;
    const bool live = at.active && pixel < count;
    const size_t row = row0 + pixel, off = row * g.C + at.c0;
    float v[8], z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (live) {
      raw8_to_f(fetch(k, off), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = fmaf(v[i] - mean[i], scale[i], shift[i]);
      if (p.res) {
        float r[8];
        raw8_to_f(raw8_load<T, VEC>(p.res + off, at.left), r);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += r[i];
      }
      if (p.act == ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = relu(z[i]);
      } else if (p.act == ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = silu<T>(z[i]);
      }
      const Raw8<T> out = raw8_of<T>(z);
      raw8_put<T, VEC>(p.y + off, at.left, out);
      if (p.gate) {
        uint32_t b = 0;
        raw8_to_f(out, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) b |= (i < at.left && z[i] > 0.f ? 1u : 0u) << i;
        p.gate[row * all_cols + (at.c0 >> 3)] = (uint8_t)b;
      }
    }
    if (p.codes) {
      const CkptScale s = ckpt_scale(ckpt_top_of_lanes(ckpt_top(v), p.ckpt_lanes));
      if (live) {
        store_codes<VEC>(p.codes, off, at.left, ckpt_codes(v, s));
        if ((at.col & (p.ckpt_lanes - 1)) == 0) p.scales[row * ((g.C + kCkptBlock - 1) / kCkptBlock) + at.c0 / kCkptBlock] = (uint8_t)s.byte;
      }
    }
  }
}

// The resident form: blockIdx.x = image * parts + share of its pixels, a cluster per image.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 3) forward_kernel(const __grid_constant__ Forward<T> p) {
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  float* red = reinterpret_cast<float*>(smem + (size_t)g.iters * Slots<T>::Q * kThreads);      // [2048]
  float* own = red + kThreads * 8;            // mean [G], squared deviations [G] of this CTA's pixels
  float* mom = own + 2 * g.G;                 // mean [G], rstd [G] of the image
  const int rank = blockIdx.x % g.parts, n = blockIdx.x / g.parts;
  const int p0 = rank * g.pix, count = max(0, min(g.pix, g.P - p0));
  const size_t row0 = (size_t)n * g.P + p0;
  const Place at(g, 0);
  const Slots<T> slots(smem);
  grid_dependency_wait();
  if (at.active) {
    const T* src = p.x + (row0 + at.r) * g.C + at.c0;
    for (int k = 0; k < g.iters && at.r + k * g.rp < count; ++k) slots.template fetch<VEC>(k, src + (size_t)k * g.rp * g.C, at.left);
  }
  float scale[8], shift[8], mean[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { scale[i] = p.gamma[at.channel(i)]; shift[i] = p.beta[at.channel(i)]; }
  copies_done();
  cta_moments(g, at, slots, count, g.G, g.Cg, g.lanes_g, red, own, [&](int s, float, float m2) { own[g.G + s] = m2; });
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  // Chan: the CTAs' moments about the image's mean
  const double m = (double)g.P * g.Cg;
  for (int s = threadIdx.x; s < g.G; s += kThreads) {
    double mu = 0.0, m2 = 0.0;
    for (int j = 0; j < g.parts; ++j) {
      const double cnt = (double)max(0, min(g.pix, g.P - j * g.pix)) * g.Cg;
      mu += cnt * (double)cluster.map_shared_rank(own, j)[s];
    }
    mu /= m;
    for (int j = 0; j < g.parts; ++j) {
      const double cnt = (double)max(0, min(g.pix, g.P - j * g.pix)) * g.Cg;
      const float* other = cluster.map_shared_rank(own, j);
      const double d = (double)other[s] - mu;
      m2 += (double)other[g.G + s] + cnt * d * d;
    }
    const float rstd = (float)(1.0 / sqrt(m2 / m + (double)p.eps));
    mom[s] = (float)mu;
    mom[g.G + s] = rstd;
    if (rank == 0) {
      p.stats[(size_t)n * g.G + s] = (float)mu;
      p.stats[(size_t)(g.N + n) * g.G + s] = rstd;
    }
  }
  cg::cluster_group::arrival_token token = cluster.barrier_arrive();      // this CTA reads its neighbours' sums no more
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = at.channel(i) / g.Cg;
    mean[i] = mom[s];
    scale[i] *= mom[g.G + s];
  }
  emit<T, VEC>(p, at, row0, count, mean, scale, shift, [&](int k, size_t) { return slots.get(k); });
  cluster.barrier_wait(std::move(token));                                 // nor do they read its own
}

// Streamed, first pass: mean and squared deviations of each channel over a chunk of pixels.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 3) moments_kernel(const __grid_constant__ Forward<T> p) {
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  float* red = reinterpret_cast<float*>(smem + (size_t)g.iters * Slots<T>::Q * kThreads);
  float* mean = red + kThreads * 8;
  const int part = blockIdx.x % g.parts, n = blockIdx.x / g.parts;
  const int p0 = part * g.pix, count = min(g.pix, g.P - p0);
  const size_t row0 = (size_t)n * g.P + p0;
  Place at(g, blockIdx.y);
  at.active = at.active && at.left > 0;
  const Slots<T> slots(smem);
  grid_dependency_wait();
  if (at.active) {
    const T* src = p.x + (row0 + at.r) * g.C + at.c0;
    for (int k = 0; k < g.iters && at.r + k * g.rp < count; ++k) slots.template fetch<VEC>(k, src + (size_t)k * g.rp * g.C, at.left);
  }
  copies_done();
  const int c_first = blockIdx.y * kMaxCols * 8, sets = min(g.cols * 8, g.C - c_first);
  float* out = p.partial + (size_t)blockIdx.x * 2 * g.C + c_first;
  cta_moments(g, at, slots, count, sets, 1, g.lanes_c, red, mean, [&](int s, float mu, float m2) {
    out[s] = mu;
    out[g.C + s] = m2;
  });
}

// Streamed, second pass: the statistics of group blockIdx.x from the moments of its channels in every chunk.
template <typename T>
__global__ void __launch_bounds__(1024) combine_kernel(const __grid_constant__ Forward<T> p) {
  __shared__ double part[32];
  __shared__ double total;
  const Geom& g = p.g;
  const int n = blockIdx.x / g.G, s = blockIdx.x % g.G, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const float* src = p.partial + (size_t)n * g.parts * 2 * g.C + (size_t)s * g.Cg;
  grid_dependency_wait();
  auto sum = [&](double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
      double a = 0.0;
      for (int w = 0; w < warps; ++w) a += part[w];
      total = a;
    }
    __syncthreads();
    return total;
  };
  auto each = [&](auto take) {
    const int step = blockDim.x / g.Cg, over = blockDim.x - step * g.Cg;
    int chunk = threadIdx.x / g.Cg, c = threadIdx.x - chunk * g.Cg;
    while (chunk < g.parts) {
      const float* row = src + (size_t)chunk * 2 * g.C + c;
      take((double)min(g.pix, g.P - chunk * g.pix), (double)row[0], row + g.C);
      chunk += step; c += over;
      if (c >= g.Cg) { c -= g.Cg; ++chunk; }
    }
  };
  const double m = (double)g.P * g.Cg;
  double a = 0.0;
  each([&](double cnt, double mu, const float*) { a += cnt * mu; });
  const double mean = sum(a) / m;
  a = 0.0;
  each([&](double cnt, double mu, const float* m2) { a += (double)*m2 + cnt * (mu - mean) * (mu - mean); });
  const double var = sum(a) / m;
  if (threadIdx.x == 0) {
    p.stats[(size_t)n * g.G + s] = (float)mean;
    p.stats[(size_t)(g.N + n) * g.G + s] = (float)(1.0 / sqrt(var + (double)p.eps));
  }
}

// Streamed, last pass: y from x and the statistics, the last chunks first.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 3) apply_kernel(const __grid_constant__ Forward<T> p) {
  const Geom& g = p.g;
  const int block = gridDim.x - 1 - blockIdx.x, part = block % g.parts, n = block / g.parts;
  const int p0 = part * g.pix, count = min(g.pix, g.P - p0);
  const size_t row0 = (size_t)n * g.P + p0;
  Place at(g, blockIdx.y);
  at.active = at.active && at.left > 0;
  float scale[8], shift[8], mean[8];
  grid_dependency_wait();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = at.active ? at.channel(i) : 0, s = c / g.Cg;
    mean[i] = p.stats[(size_t)n * g.G + s];
    scale[i] = p.gamma[c] * p.stats[(size_t)(g.N + n) * g.G + s];
    shift[i] = p.beta[c];
  }
  emit<T, VEC>(p, at, row0, count, mean, scale, shift, [&](int, size_t off) { return raw8_load<T, VEC>(p.x + off, at.left); });
}

// ---- backward -----------------------------------------------------------------------------------------------
template <typename T> struct Backward {
  Geom g;
  const T* dy;
  const T* x;
  const int8_t* codes;        // x in 8 bits, in place of x
  const uint8_t* scales;
  const float* stats;
  const float* gamma;
  const float* beta;          // SiLU only
  const T* mask;              // ReLU: y, or the bits of [y > 0]
  const uint8_t* gate;
  const T* res;
  T* dx;
  float* partial;             // streamed: [N][parts][2][C]
  float* totals;              // [N][2][C]: A, B
  int act;
};

// The operands of one column of 8 channels at a pixel, raw.
template <typename T, bool CK> struct Held {
  Raw8<T> dy;
  Raw8<T> x;
  uint2 codes;
  uint32_t scale, open;       // scale byte of the codes, bits of the ReLU gate
};

template <typename T, bool VEC> __device__ __forceinline__ uint32_t open_bits(const Backward<T>& p, const Place& at, size_t row) {
  if (p.gate) return p.gate[row * ((p.g.C + 7) >> 3) + (at.c0 >> 3)];
  float m[8];
  raw8_to_f(raw8_load<T, VEC>(p.mask + row * p.g.C + at.c0, at.left), m);
  uint32_t b = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) b |= (m[i] > 0.f ? 1u : 0u) << i;
  return b;
}
__device__ __forceinline__ size_t scale_index(const Geom& g, const Place& at, size_t row) {
  return row * ((g.C + kCkptBlock - 1) / kCkptBlock) + at.c0 / kCkptBlock;
}

// A thread's 8 channels: mean, gamma * rstd, beta.
struct Channels {
  float mean[8], scale[8], shift[8];
};

// dz and x - mean of one vector.
template <typename T, bool CK>
__device__ __forceinline__ void gated(const Held<T, CK>& h, int act, const Channels& ch, float (&dz)[8], float (&d)[8]) {
  raw8_to_f(h.dy, dz);
  if constexpr (CK) ckpt_values(h.codes, ckpt_step(h.scale), d); else raw8_to_f(h.x, d);
#pragma unroll
  for (int i = 0; i < 8; ++i) d[i] -= ch.mean[i];
  if (act == ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dz[i] = (h.open >> i & 1u) ? dz[i] : 0.f;
  } else if (act == ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dz[i] *= silu_slope<T>(fmaf(d[i], ch.scale[i], ch.shift[i]));
  }
}

// dx of this CTA's pixels: fetch(k, row) gives the thread's k-th operands; k1 = rstd*S1/m, k2 = rstd^2*S2/m.
template <typename T, bool VEC, bool CK, typename Fetch>
__device__ __forceinline__ void emit_dx(const Backward<T>& p, const Place& at, size_t row0, int count, const Channels& ch,
                                        const float (&k1)[8], const float (&k2)[8], Fetch fetch) {
  const Geom& g = p.g;
  if (!at.active) return;
#pragma unroll 2
  for (int k = 0; k < g.iters; ++k) {
    const int pixel = at.r + k * g.rp;
    if (pixel >= count) break;
    const size_t row = row0 + pixel, off = row * g.C + at.c0;
    float dz[8], d[8];
    gated<T, CK>(fetch(k, row), p.act, ch, dz, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) dz[i] = fmaf(ch.scale[i], dz[i], fmaf(-d[i], k2[i], -k1[i]));
    if (p.res) {
      raw8_to_f(raw8_load<T, VEC>(p.res + off, at.left), d);
#pragma unroll
      for (int i = 0; i < 8; ++i) dz[i] += d[i];
    }
    raw8_store<T, VEC>(p.dx + off, at.left, dz);
  }
}

template <typename T, bool VEC, bool CK>
__device__ __forceinline__ Held<T, CK> load_held(const Backward<T>& p, const Place& at, size_t row) {
  Held<T, CK> h;
  const size_t off = row * p.g.C + at.c0;
  h.dy = raw8_load<T, VEC>(p.dy + off, at.left);
  if constexpr (CK) {
    h.codes = load_codes<VEC>(p.codes, off, at.left);
    h.scale = p.scales[scale_index(p.g, at, row)];
  } else {
    h.x = raw8_load<T, VEC>(p.x + off, at.left);
  }
  h.open = p.act == ACT_RELU ? open_bits<T, VEC>(p, at, row) : 0u;
  return h;
}

// The resident form.  Shared memory: the thread's vectors of dy and x (or its codes), a byte per vector for the gate's bits and
// one for the scale; then per-thread sums, per-channel sums A, B and per-group sums S1, S2 of this CTA, and k1, k2 of the image.
template <typename T, bool VEC, bool CK>
__global__ void __launch_bounds__(kThreads, 3) backward_kernel(const __grid_constant__ Backward<T> p) {
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  const size_t vecs = (size_t)g.iters * kThreads;
  uint4* xs = smem + vecs * Slots<T>::Q;
  uint2* cs = reinterpret_cast<uint2*>(xs);
  float* red = reinterpret_cast<float*>(CK ? reinterpret_cast<uint4*>(cs + vecs) : xs + vecs * Slots<T>::Q);   // [2][2048]
  float* chan = red + 2 * kThreads * 8;       // [2][C]
  float* own = chan + 2 * g.C;                // [2][G]
  float* coef = own + 2 * g.G;                // [2][G]
  uint8_t* open = reinterpret_cast<uint8_t*>(coef + 2 * g.G);
  uint8_t* scale_bytes = open + vecs;
  const int rank = blockIdx.x % g.parts, n = blockIdx.x / g.parts, tid = threadIdx.x;
  const int p0 = rank * g.pix, count = max(0, min(g.pix, g.P - p0));
  const size_t row0 = (size_t)n * g.P + p0;
  const Place at(g, 0);
  const Slots<T> dys(smem), xslots(xs);
  grid_dependency_wait();
  if (at.active) {
#pragma unroll 4
    for (int k = 0; k < g.iters; ++k) {
      const int pixel = at.r + k * g.rp;
      if (pixel >= count) break;
      const size_t row = row0 + pixel, off = row * g.C + at.c0;
      dys.template fetch<VEC>(k, p.dy + off, at.left);
      if constexpr (CK) {
        if constexpr (VEC) copy8_async(cs + k * kThreads + tid, p.codes + off); else cs[k * kThreads + tid] = load_codes<false>(p.codes, off, at.left);
      } else {
        xslots.template fetch<VEC>(k, p.x + off, at.left);
      }
    }
#pragma unroll 4
    for (int k = 0; k < g.iters; ++k) {
      const int pixel = at.r + k * g.rp;
      if (pixel >= count) break;
      if (p.act == ACT_RELU) open[k * kThreads + tid] = (uint8_t)open_bits<T, VEC>(p, at, row0 + pixel);
      if constexpr (CK) scale_bytes[k * kThreads + tid] = p.scales[scale_index(g, at, row0 + pixel)];
    }
  }
  Channels ch;
  float rstd[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = at.channel(i), s = c / g.Cg;
    ch.mean[i] = p.stats[(size_t)n * g.G + s];
    rstd[i] = p.stats[(size_t)(g.N + n) * g.G + s];
    ch.scale[i] = p.gamma[c] * rstd[i];
    ch.shift[i] = p.act == ACT_SILU ? p.beta[c] : 0.f;
  }
  copies_done();
  auto held = [&](int k) {
    Held<T, CK> h;
    h.dy = dys.get(k);
    if constexpr (CK) {
      h.codes = cs[k * kThreads + tid];
      h.scale = scale_bytes[k * kThreads + tid];
    } else {
      h.x = xslots.get(k);
    }
    h.open = p.act == ACT_RELU ? open[k * kThreads + tid] : 0u;
    return h;
  };
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
  if (at.active)
#pragma unroll 2
    for (int k = 0; k < g.iters; ++k) {
      if (at.r + k * g.rp >= count) break;
      float dz[8], d[8];
      gated<T, CK>(held(k), p.act, ch, dz, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) { a[i] = fmaf(dz[i], d[i], a[i]); b[i] += dz[i]; }
    }
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] *= rstd[i];
  put_sums(red, g, at, a);
  put_sums(red + kThreads * 8, g, at, b);
  __syncthreads();
  const int width = g.cols * 8;
  for (int s = 0; s < 2; ++s) {
    const float* from = red + s * kThreads * 8;
    add_sets(g.rp, g.C, 1, g.lanes_c, [&](int r, int c) { return from[r * width + c]; }, [&](int c, float sum) { chan[s * g.C + c] = sum; });
  }
  __syncthreads();
  add_sets(1, g.G, g.Cg, g.lanes_g, [&](int, int c) { return p.gamma[c] * chan[g.C + c]; }, [&](int s, float sum) { own[s] = sum; });
  add_sets(1, g.G, g.Cg, g.lanes_g, [&](int, int c) { return p.gamma[c] * chan[c]; }, [&](int s, float sum) { own[g.G + s] = sum; });
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  const float inv_m = (float)(1.0 / ((double)g.P * g.Cg));
  for (int s = tid; s < g.G; s += kThreads) {
    float s1 = 0.f, s2 = 0.f;
    for (int j = 0; j < g.parts; ++j) {
      const float* other = cluster.map_shared_rank(own, j);
      s1 += other[s]; s2 += other[g.G + s];
    }
    const float r = p.stats[(size_t)(g.N + n) * g.G + s];
    coef[s] = r * s1 * inv_m;
    coef[g.G + s] = r * r * s2 * inv_m;
  }
  // each CTA of the cluster adds up a share of the channels for the parameter gradients
  const int share = (2 * g.C + g.parts - 1) / g.parts;
  for (int c = rank * share + tid; c < min((rank + 1) * share, 2 * g.C); c += kThreads) {
    float t = 0.f;
    for (int j = 0; j < g.parts; ++j) t += cluster.map_shared_rank(chan, j)[c];
    p.totals[(size_t)n * 2 * g.C + c] = t;
  }
  cg::cluster_group::arrival_token token = cluster.barrier_arrive();
  __syncthreads();
  grid_dependency_release();
  float k1[8], k2[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = at.channel(i) / g.Cg;
    k1[i] = coef[s]; k2[i] = coef[g.G + s];
  }
  emit_dx<T, VEC, CK>(p, at, row0, count, ch, k1, k2, [&](int k, size_t) { return held(k); });
  cluster.barrier_wait(std::move(token));
}

// Streamed, first pass: A and B of each channel over a chunk of pixels.
template <typename T, bool VEC, bool CK>
__global__ void __launch_bounds__(kThreads, 2) backward_sums_kernel(const __grid_constant__ Backward<T> p) {
  __shared__ __align__(16) float red[2][kThreads * 8];
  const Geom& g = p.g;
  const int part = blockIdx.x % g.parts, n = blockIdx.x / g.parts;
  const int p0 = part * g.pix, count = min(g.pix, g.P - p0);
  const size_t row0 = (size_t)n * g.P + p0;
  const Place at(g, blockIdx.y);
  const bool active = at.active && at.left > 0;
  grid_dependency_wait();
  Channels ch;
  float rstd[8], a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = active ? at.channel(i) : 0, s = c / g.Cg;
    ch.mean[i] = p.stats[(size_t)n * g.G + s];
    rstd[i] = p.stats[(size_t)(g.N + n) * g.G + s];
    ch.scale[i] = p.gamma[c] * rstd[i];
    ch.shift[i] = p.act == ACT_SILU ? p.beta[c] : 0.f;
    a[i] = b[i] = 0.f;
  }
  auto add = [&](const Held<T, CK>& h) {
    float dz[8], d[8];
    gated<T, CK>(h, p.act, ch, dz, d);
#pragma unroll
    for (int i = 0; i < 8; ++i) { a[i] = fmaf(dz[i], d[i], a[i]); b[i] += dz[i]; }
  };
  if (active) {
    constexpr int U = sizeof(T) == 4 ? 2 : 4;             // vectors in flight
    int pixel = at.r;
    for (; pixel + (U - 1) * g.rp < count; pixel += U * g.rp) {
      Held<T, CK> h[U];
#pragma unroll
      for (int u = 0; u < U; ++u) h[u] = load_held<T, VEC, CK>(p, at, row0 + pixel + u * g.rp);
#pragma unroll
      for (int u = 0; u < U; ++u) add(h[u]);
    }
    for (; pixel < count; pixel += g.rp) add(load_held<T, VEC, CK>(p, at, row0 + pixel));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] *= rstd[i];
  put_sums(red[0], g, at, a);
  put_sums(red[1], g, at, b);
  __syncthreads();
  const int width = g.cols * 8, c_first = blockIdx.y * kMaxCols * 8, sets = min(width, g.C - c_first);
  for (int s = 0; s < 2; ++s) {
    float* out = p.partial + ((size_t)blockIdx.x * 2 + s) * g.C + c_first;
    add_sets(g.rp, sets, 1, g.lanes_c, [&](int r, int c) { return red[s][r * width + c]; }, [&](int c, float sum) { out[c] = sum; });
  }
}

// out[j][i] = the sum of `rows` rows of `width` floats from in[j * rows] on, j = blockIdx.x / blocks; a block takes 32 of
// the width, its warps every 32nd row, and adds in fp64.  Streamed, second pass (a row per chunk), and, for all forms, the
// parameter gradients (a row per image; `split` > 0: values from there on go to out2).
__global__ void __launch_bounds__(1024) add_rows_kernel(const float* __restrict__ in, int rows, int width, float* __restrict__ out,
                                                        float* __restrict__ out2, int split) {
  __shared__ double fin[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int blocks = (width + 31) / 32, j = blockIdx.x / blocks, first = (blockIdx.x - j * blocks) * 32;
  const int i = first + lane;
  in += (size_t)j * rows * width;
  out += (size_t)j * width;
  grid_dependency_wait();
  double t = 0.0;
  if (i < width)
#pragma unroll 4
    for (int r = warp; r < rows; r += 32) t += (double)in[(size_t)r * width + i];
  fin[warp][lane] = t;
  __syncthreads();
  const int ii = first + warp;
  t = fin[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (lane != 0 || ii >= width) return;
  if (split > 0 && ii >= split) out2[ii - split] = (float)t; else out[ii] = (float)t;
}

// Streamed, last pass: dx, the last chunks first.  Every CTA forms S1 and S2 of its tile's groups from the image's totals.
template <typename T, bool VEC, bool CK>
__global__ void __launch_bounds__(kThreads, 3) backward_apply_kernel(const __grid_constant__ Backward<T> p) {
  __shared__ float coef[2][kMaxCols * 8];
  const Geom& g = p.g;
  const int block = gridDim.x - 1 - blockIdx.x, part = block % g.parts, n = block / g.parts;
  const int p0 = part * g.pix, count = min(g.pix, g.P - p0);
  const size_t row0 = (size_t)n * g.P + p0;
  Place at(g, blockIdx.y);
  at.active = at.active && at.left > 0;
  const int c_first = blockIdx.y * kMaxCols * 8, c_last = min(g.C, c_first + g.cols * 8) - 1;
  const int g_first = c_first / g.Cg, sets = c_last / g.Cg - g_first + 1;
  const float inv_m = (float)(1.0 / ((double)g.P * g.Cg));
  grid_dependency_wait();
  const float* tot = p.totals + (size_t)n * 2 * g.C;
  const float* rs = p.stats + (size_t)(g.N + n) * g.G + g_first;
  const int c_base = g_first * g.Cg;
  add_sets(1, sets, g.Cg, g.lanes_g, [&](int, int c) { return p.gamma[c_base + c] * tot[g.C + c_base + c]; },
           [&](int s, float sum) { coef[0][s] = rs[s] * sum * inv_m; });
  add_sets(1, sets, g.Cg, g.lanes_g, [&](int, int c) { return p.gamma[c_base + c] * tot[c_base + c]; },
           [&](int s, float sum) { coef[1][s] = rs[s] * rs[s] * sum * inv_m; });
  __syncthreads();
  Channels ch;
  float k1[8], k2[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = at.active ? at.channel(i) : c_first, s = c / g.Cg;
    ch.mean[i] = p.stats[(size_t)n * g.G + s];
    ch.scale[i] = p.gamma[c] * p.stats[(size_t)(g.N + n) * g.G + s];
    ch.shift[i] = p.act == ACT_SILU ? p.beta[c] : 0.f;
    k1[i] = coef[0][s - g_first]; k2[i] = coef[1][s - g_first];
  }
  emit_dx<T, VEC, CK>(p, at, row0, count, ch, k1, k2, [&](int, size_t row) { return load_held<T, VEC, CK>(p, at, row); });
}

// ---- host side: plans ----------------------------------------------------------------------------------------
struct Plan {
  Geom g;
  bool resident;
  size_t smem;                // dynamic shared memory of the resident kernel, or of moments_kernel
};
inline int pow2_up_to(int64_t most, int cap) {
  int v = 1;
  while (2 * v <= cap && 2 * (int64_t)v <= most) v *= 2;
  return v;
}
constexpr size_t kSmemMost = 220 * 1024;        // of 227 KB
constexpr size_t kSmemShare = 72 * 1024;        // three CTAs on an SM: one's copies run beside another's arithmetic
constexpr int kStreamIters = 16;                // pixels per thread and chunk of the streamed form, 16-bit storage

// `vec_bytes`: shared memory per vector of 8 channels; `fixed`: besides the vectors.
inline Plan plan(int N, int P, int C, int G, size_t vec_bytes, size_t fixed, int stream_iters) {
  Plan pl{};
  Geom& g = pl.g;
  g.N = N; g.P = P; g.C = C; g.G = G; g.Cg = C / G;
  const int all_cols = C / 8 + (C % 8 != 0);
  g.cols = std::min(all_cols, kMaxCols);
  g.tiles = (all_cols + kMaxCols - 1) / kMaxCols;
  g.rp = kThreads / g.cols;
  g.lanes_g = pow2_up_to(kThreads / std::min(G, kThreads), 32);
  g.lanes_c = pow2_up_to(kThreads / std::min(g.cols * 8, kThreads), 32);
  auto split = [&](int parts) {
    g.parts = parts;
    g.pix = P / parts + (P % parts != 0);
    g.iters = g.pix / g.rp + (g.pix % g.rp != 0);
    return (size_t)g.iters * kThreads * vec_bytes + fixed;
  };
  if (g.tiles == 1) {
    int parts = 1;
    while (parts < kMaxCluster && split(parts) > kSmemShare) parts *= 2;
    // few images: more SMs, while every thread keeps two pixels
    while (parts < kMaxCluster && (int64_t)N * parts * 2 <= 2 * kSms && (split(parts), g.iters) >= 4) parts *= 2;
    pl.smem = split(parts);
    pl.resident = pl.smem <= kSmemMost && (int64_t)N * parts <= INT32_MAX;
    if (pl.resident) return pl;
  }
  g.iters = stream_iters;
  g.pix = std::min(P, g.rp * stream_iters);
  g.iters = (g.pix + g.rp - 1) / g.rp;
  g.parts = P / g.pix + (P % g.pix != 0);
  pl.smem = (size_t)g.iters * kThreads * vec_bytes + fixed;
  return pl;
}
inline Plan plan_forward(int elem_bytes, int N, int P, int C, int G) {
  const size_t red = kThreads * 8 * 4;
  Plan pl = plan(N, P, C, G, 8 * (size_t)elem_bytes, red + 16 * (size_t)G, elem_bytes == 4 ? kStreamIters / 2 : kStreamIters);
  if (!pl.resident) pl.smem = (size_t)pl.g.iters * kThreads * 8 * elem_bytes + red + (size_t)pl.g.cols * 8 * 4;     // moments_kernel
  return pl;
}
inline Plan plan_backward(int elem_bytes, int N, int P, int C, int G, bool ckpt) {
  const size_t vec = 8 * (size_t)elem_bytes + (ckpt ? 8 : 8 * (size_t)elem_bytes) + 2;      // dy, x, a byte each for gate and scale
  return plan(N, P, C, G, vec, 2 * kThreads * 8 * 4 + 8 * (size_t)C + 16 * (size_t)G, elem_bytes == 4 ? kStreamIters / 2 : kStreamIters);
}
// Whether every launch's grid can be given.
inline bool grid_ok(const Plan& pl) {
  const Geom& g = pl.g;
  return pl.resident || ((int64_t)g.N * g.parts <= INT32_MAX && (int64_t)g.N * g.G <= INT32_MAX && g.tiles <= 65535 &&
                         (int64_t)g.N * ((2 * (int64_t)g.C + 31) / 32) <= INT32_MAX);
}
inline size_t partial_floats(const Plan& pl) { return pl.resident ? 0 : (size_t)pl.g.N * pl.g.parts * 2 * pl.g.C; }

// ---- host side: launches ---------------------------------------------------------------------------------------
template <typename Kernel, typename Params>
inline cudaError_t launch_cluster(Kernel kernel, int blocks, int cluster, size_t smem, cudaStream_t st, const Params& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T, bool VEC> inline cudaError_t launch_forward_as(cudaStream_t st, const Plan& pl, const Forward<T>& p) {
  const Geom& g = pl.g;
  static OncePerDevice once;
  cudaError_t e = once_per_device(&once, []() {
    const cudaError_t f = set_smem_limit(forward_kernel<T, VEC>, kSmemMost);
    return f != cudaSuccess ? f : set_smem_limit(moments_kernel<T, VEC>, kSmemMost);
  });
  if (e != cudaSuccess) return e;
  if (pl.resident) return launch_cluster(forward_kernel<T, VEC>, g.N * g.parts, g.parts, pl.smem, st, p);
  const dim3 grid((unsigned)(g.N * g.parts), (unsigned)g.tiles);
  e = launch_chained(moments_kernel<T, VEC>, grid, dim3(kThreads), pl.smem, st, p);
  const int warps = pow2_up_to((int64_t)g.parts * g.Cg / 64, 32);
  if (e == cudaSuccess) e = launch_chained(combine_kernel<T>, dim3((unsigned)(g.N * g.G)), dim3(32 * warps), 0, st, p);
  if (e == cudaSuccess) e = launch_chained(apply_kernel<T, VEC>, grid, dim3(kThreads), 0, st, p);
  return e;
}

template <typename T>
inline cudaError_t launch_forward(cudaStream_t st, const Plan& pl, Forward<T> p) {
  p.g = pl.g;
  const int C = p.g.C;
  p.ckpt_lanes = p.codes ? ckpt_block_lanes(C) : 0;
  int8_t* codes = p.codes;
  if (p.ckpt_lanes == 0) p.codes = nullptr;       // blocks that do not fall on groups of lanes: a pass of their own
  const bool vec = C % 8 == 0 && aligned_to(p.x, 16) && aligned_to(p.y, 16) && aligned_to(p.res, 16) && aligned_to(p.codes, 8);
  cudaError_t e = vec ? launch_forward_as<T, true>(st, pl, p) : launch_forward_as<T, false>(st, pl, p);
  if (e == cudaSuccess && codes && !p.codes) e = launch_ckpt_encode<T>(st, p.x, (size_t)p.g.N * p.g.P, C, codes, p.scales);
  return e;
}

template <typename T, bool VEC, bool CK> inline cudaError_t launch_backward_as(cudaStream_t st, const Plan& pl, const Backward<T>& p) {
  const Geom& g = pl.g;
  static OncePerDevice once;
  cudaError_t e = once_per_device(&once, []() { return set_smem_limit(backward_kernel<T, VEC, CK>, kSmemMost); });
  if (e != cudaSuccess) return e;
  if (pl.resident) return launch_cluster(backward_kernel<T, VEC, CK>, g.N * g.parts, g.parts, pl.smem, st, p);
  const dim3 grid((unsigned)(g.N * g.parts), (unsigned)g.tiles);
  e = launch_chained(backward_sums_kernel<T, VEC, CK>, grid, dim3(kThreads), 0, st, p);
  if (e == cudaSuccess)
    e = launch_chained(add_rows_kernel, dim3((unsigned)(g.N * ((2 * g.C + 31) / 32))), dim3(1024), 0, st, (const float*)p.partial,
                       g.parts, 2 * g.C, p.totals, (float*)nullptr, 0);
  if (e == cudaSuccess) e = launch_chained(backward_apply_kernel<T, VEC, CK>, grid, dim3(kThreads), 0, st, p);
  return e;
}

template <typename T>
inline cudaError_t launch_backward(cudaStream_t st, const Plan& pl, Backward<T> p, float* dgamma, float* dbeta) {
  p.g = pl.g;
  const Geom& g = p.g;
  const bool vec = g.C % 8 == 0 && aligned_to(p.dy, 16) && aligned_to(p.x, 16) && aligned_to(p.codes, 8) && aligned_to(p.mask, 16) &&
                   aligned_to(p.res, 16) && aligned_to(p.dx, 16);
  cudaError_t e = p.codes ? (vec ? launch_backward_as<T, true, true>(st, pl, p) : launch_backward_as<T, false, true>(st, pl, p))
                          : (vec ? launch_backward_as<T, true, false>(st, pl, p) : launch_backward_as<T, false, false>(st, pl, p));
  if (e == cudaSuccess)
    e = launch_chained(add_rows_kernel, dim3((unsigned)((2 * g.C + 31) / 32)), dim3(1024), 0, st, (const float*)p.totals, g.N, 2 * g.C,
                       dgamma, dbeta, g.C);
  return e;
}

}  // namespace gn
}  // namespace fdg
