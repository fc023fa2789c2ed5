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
// 1/(1 + exp(-z)).  For tensors in 16 bits from the approximate exponential and reciprocal (relative error below 2^-20 for
// |z| < 16, growing with |z| as the rounding of z*log2(e) does), for fp32 ones from expf and a division.
template <typename T> __device__ __forceinline__ float sigmoid(float z) {
  if constexpr (sizeof(T) == 2) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
  } else {
    return 1.f / (1.f + expf(-z));
  }
}
template <typename T> __device__ __forceinline__ float silu_slope(float z) {
  const float s = sigmoid<T>(z);
  return s * fmaf(z, 1.f - s, 1.f);
}

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

// take(i, channel, group) for the 8 channels of a column; those past the last channel stand in for the first.
template <typename Take> __device__ __forceinline__ void each_channel(const Place& at, int Cg, Take take) {
  const int first = at.c0 / Cg;
  int s = first, rem = at.c0 - first * Cg;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    take(i, at.channel(i), i < at.left ? s : first);
    if (++rem == Cg) { rem = 0; ++s; }
  }
}

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

// Moments of this CTA's `count` pixels in `slots`: done(set, mean, sum of squared deviations from that mean) for sets of `size`
// consecutive channels.  `red`: 2048 floats, `mean`: a float per set.
// A thread sums its values of a channel, and their squares, less the first of them: the square of the distance from that value
// to the mean is at most n times the spread of the n values, so what cancels when the sum is taken out again is at most n times
// the result, whatever the offset (n is a few dozen at most).  The threads' moments are then brought about the CTA's mean.
template <typename T, typename Done>
__device__ __forceinline__ void cta_moments(const Geom& g, const Place& at, const Slots<T>& slots, int count, int sets, int size, int lanes,
                                            float* red, float* mean, Done done) {
  const int width = g.cols * 8;
  const float inv = count > 0 ? 1.f / ((float)count * (float)size) : 0.f;
  F8 first, sum, square;
#pragma unroll
  for (int j = 0; j < 4; ++j) first.p[j] = sum.p[j] = square.p[j] = 0;
  int n = 0;
  if (at.active && at.r < count) {
    F8 less;
    first = raw8_to_f8(slots.get(0));
#pragma unroll
    for (int j = 0; j < 4; ++j) less.p[j] = mul2(first.p[j], pair(-1.f));
    n = 1;
#pragma unroll 4
    for (int k = 1; k < g.iters; ++k) {
      if (at.r + k * g.rp >= count) break;
      const F8 x = raw8_to_f8(slots.get(k));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 d = add2(x.p[j], less.p[j]);
        sum.p[j] = add2(sum.p[j], d);
        square.p[j] = fma2(d, d, square.p[j]);
      }
      ++n;
    }
  }
  const float fn = (float)n, over = n > 0 ? 1.f / fn : 0.f;
  float a[8], mu[8];                  // the thread's mean and squared deviations
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = halves(first.p[j]), s1 = halves(sum.p[j]), s2 = halves(square.p[j]);
    mu[2 * j] = fmaf(s1.x, over, f.x);
    mu[2 * j + 1] = fmaf(s1.y, over, f.y);
    a[2 * j] = max_nan(fmaf(-s1.x * over, s1.x, s2.x), 0.f);
    a[2 * j + 1] = max_nan(fmaf(-s1.y * over, s1.y, s2.y), 0.f);
  }
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = mu[i] * fn;
  put_sums(red, g, at, t);
  __syncthreads();
  auto value = [&](int r, int c) { return red[r * width + c]; };
  add_sets(g.rp, sets, size, lanes, value, [&](int s, float total) { mean[s] = total * inv; });
  __syncthreads();
  if (at.active) {
    int s = at.col * 8 / size, rem = at.col * 8 - s * size;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = mu[i] - mean[min(s, sets - 1)];
      t[i] = fmaf(fn * d, d, a[i]);
      if (++rem == size) { rem = 0; ++s; }
    }
    put_sums(red, g, at, t);
  }
  __syncthreads();
  add_sets(g.rp, sets, size, lanes, value, [&](int s, float total) { done(s, mean[s], total); });
}

// What a thread multiplies its 8 channels by: scale = gamma*rstd and shift = beta, and the mean with its sign turned.  16-bit
// tensors take the mean into the shift: that rounds |mean|*scale to 24 bits where x itself has 8.
template <typename T> struct Affine {
  static constexpr bool kFolded = sizeof(T) == 2;
  f32x2 scale[4], shift[4], less[kFolded ? 1 : 4];
  __device__ __forceinline__ void set(int j, float2 mean, float2 sc, float2 sh) {
    scale[j] = pair(sc.x, sc.y);
    if constexpr (kFolded) {
      shift[j] = pair(fmaf(-mean.x, sc.x, sh.x), fmaf(-mean.y, sc.y, sh.y));
    } else {
      shift[j] = pair(sh.x, sh.y);
      less[j] = pair(-mean.x, -mean.y);
    }
  }
  __device__ __forceinline__ f32x2 of(int j, f32x2 x) const {
    if constexpr (kFolded) return fma2(x, scale[j], shift[j]); else return fma2(add2(x, less[j]), scale[j], shift[j]);
  }
};

// Bits of [y > 0] of 8 stored values.
__device__ __forceinline__ uint32_t positive_bits(const Raw8<__nv_bfloat16>& y) {
  const uint32_t w[4] = {y.q[0].x, y.q[0].y, y.q[0].z, y.q[0].w};
  uint32_t b = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&w[j]);
    b |= __hgt2_mask(v, __nv_bfloat162{__nv_bfloat16_raw{0}, __nv_bfloat16_raw{0}}) & ((1u << (2 * j)) | (1u << (2 * j + 17)));
  }
  return (b | b >> 16) & 0xFFu;
}
__device__ __forceinline__ uint32_t positive_bits(const Raw8<float>& y) {
  const uint32_t w[8] = {y.q[0].x, y.q[0].y, y.q[0].z, y.q[0].w, y.q[1].x, y.q[1].y, y.q[1].z, y.q[1].w};
  uint32_t b = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) b |= (__uint_as_float(w[i]) > 0.f ? 1u : 0u) << i;
  return b;
}

// y (and the gate's bits, and x in 8 bits) of this CTA's pixels: fetch(k, offset) gives the thread's k-th vector of x; U of them
// (and of res) are fetched before the first is used.  Every lane takes every turn, since the lanes of a block of 32 channels
// exchange its maximum.  Offsets inside a CTA's pixels fit 32 bits.
template <typename T, bool VEC, int U, typename Fetch>
__device__ __forceinline__ void emit(const Forward<T>& p, const Place& at, size_t row0, int count, const Affine<T>& affine, Fetch fetch) {
  const Geom& g = p.g;
  const int all_cols = (g.C + 7) >> 3, per_row = (g.C + kCkptBlock - 1) / kCkptBlock;
  const size_t row = row0 + at.r, off = row * g.C + at.c0;
  T* const y = p.y + off;
  const T* const res = p.res + off;
  int8_t* const codes = p.codes + off;
  uint8_t* const gate = p.gate + (row * all_cols + (at.c0 >> 3));
  uint8_t* const scales = p.scales + (row * per_row + at.c0 / kCkptBlock);
  const bool has_res = p.res != nullptr, has_gate = p.gate != nullptr, has_codes = p.codes != nullptr;
  const bool leads = (at.col & (p.ckpt_lanes - 1)) == 0;
  const uint32_t step = (uint32_t)g.rp * g.C;
  for (int k0 = 0; k0 < g.iters; k0 += U) {
    Raw8<T> xs[U], rs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u;
      const bool live = at.active && at.r + k * g.rp < count;
      xs[u] = live ? fetch(k, (uint32_t)k * step) : Raw8<T>{};
      if (has_res) rs[u] = live ? raw8_load<T, VEC>(res + (uint32_t)k * step, at.left) : Raw8<T>{};
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u;
      const bool live = at.active && at.r + k * g.rp < count;
      const uint32_t o = (uint32_t)k * step;
      const F8 x = raw8_to_f8(xs[u]);
      if (live) {
        F8 z;
#pragma unroll
        for (int j = 0; j < 4; ++j) z.p[j] = affine.of(j, x.p[j]);
        if (has_res) {
          const F8 r = raw8_to_f8(rs[u]);
#pragma unroll
          for (int j = 0; j < 4; ++j) z.p[j] = add2(z.p[j], r.p[j]);
        }
        if (p.act == ACT_RELU) {
          const Raw8<T> out = f8_to_raw8<T, true>(z);
          raw8_put<T, VEC>(y + o, at.left, out);
          if (has_gate) gate[(uint32_t)(k * g.rp) * all_cols] = (uint8_t)(positive_bits(out) & (VEC ? 0xFFu : (1u << at.left) - 1));
        } else {
          if (p.act == ACT_SILU) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 h = halves(z.p[j]);
              z.p[j] = mul2(z.p[j], pair(sigmoid<T>(h.x), sigmoid<T>(h.y)));
            }
          }
          raw8_put<T, VEC>(y + o, at.left, f8_to_raw8<T>(z));
        }
      }
      if (has_codes) {
        const CkptScale s = ckpt_scale(ckpt_top_of_lanes(ckpt_top(xs[u]), p.ckpt_lanes));
        if (live) {
          store_codes<VEC>(codes + o, 0, at.left, ckpt_codes(x, s));
          if (leads) scales[(uint32_t)(k * g.rp) * per_row] = (uint8_t)s.byte;
        }
      }
    }
  }
}

// The resident form: blockIdx.x = image * parts + share of its pixels, a cluster per image.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) forward_kernel(const __grid_constant__ Forward<T> p) {
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  float* red = reinterpret_cast<float*>(smem + (size_t)g.iters * Slots<T>::Q * kThreads);      // [2048]
  float* own = red + kThreads * 8;            // mean [G], squared deviations [G] of this CTA's pixels
  float2* mom = reinterpret_cast<float2*>(own + 2 * g.G);                 // mean, rstd [G] of the image
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
  float scale[8], shift[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { scale[i] = p.gamma[at.channel(i)]; shift[i] = p.beta[at.channel(i)]; }
  copies_done();
  cta_moments(g, at, slots, count, g.G, g.Cg, g.lanes_g, red, own, [&](int s, float, float m2) { own[g.G + s] = m2; });
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  // Chan: the CTAs' moments about the image's mean; a lane per CTA and group
  const int j = threadIdx.x & (g.parts - 1);
  const float in_j = (float)max(0, min(g.pix, g.P - j * g.pix)), inv_p = 1.f / (float)g.P;
  const float* other = cluster.map_shared_rank(own, j);
  for (int s0 = 0; s0 < g.G; s0 += kThreads / g.parts) {
    const int s = s0 + threadIdx.x / g.parts;
    const float mean_j = s < g.G ? other[s] : 0.f, m2_j = s < g.G ? other[g.G + s] : 0.f;
    float mu = mean_j * (in_j * inv_p);
    for (int o = g.parts >> 1; o > 0; o >>= 1) mu += __shfl_xor_sync(0xffffffffu, mu, o);
    const float d = mean_j - mu;
    float var = fmaf(in_j * d, d, m2_j / (float)g.Cg);
    for (int o = g.parts >> 1; o > 0; o >>= 1) var += __shfl_xor_sync(0xffffffffu, var, o);
    const float rstd = 1.f / sqrtf(fmaf(var, inv_p, p.eps));
    if (j == 0 && s < g.G) {
      mom[s] = make_float2(mu, rstd);
      if (rank == 0) {
        p.stats[(size_t)n * g.G + s] = mu;
        p.stats[(size_t)(g.N + n) * g.G + s] = rstd;
      }
    }
  }
  cg::cluster_group::arrival_token token = cluster.barrier_arrive();      // this CTA reads its neighbours' sums no more
  __syncthreads();
  Affine<T> affine;
  float2 m[8];
  each_channel(at, g.Cg, [&](int i, int, int s) { m[i] = mom[s]; });
#pragma unroll
  for (int i = 0; i < 4; ++i)
    affine.set(i, make_float2(m[2 * i].x, m[2 * i + 1].x), make_float2(scale[2 * i] * m[2 * i].y, scale[2 * i + 1] * m[2 * i + 1].y),
               make_float2(shift[2 * i], shift[2 * i + 1]));
  emit<T, VEC, 2>(p, at, row0, count, affine, [&](int k, uint32_t) { return slots.get(k); });
  cluster.barrier_wait(std::move(token));                                 // nor do they read its own
}

// Streamed, first pass: mean and squared deviations of each channel over a chunk of pixels.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) moments_kernel(const __grid_constant__ Forward<T> p) {
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
__global__ void __launch_bounds__(kThreads, 2) apply_kernel(const __grid_constant__ Forward<T> p) {
  const Geom& g = p.g;
  const int block = gridDim.x - 1 - blockIdx.x, part = block % g.parts, n = block / g.parts;
  const int p0 = part * g.pix, count = min(g.pix, g.P - p0);
  const size_t row0 = (size_t)n * g.P + p0;
  Place at(g, blockIdx.y);
  at.active = at.active && at.left > 0;
  if (!at.active) at.c0 = 0;
  Affine<T> affine;
  float mean[8], scale[8], shift[8];
  grid_dependency_wait();
  each_channel(at, g.Cg, [&](int i, int c, int s) {
    c = at.active ? c : 0;
    s = at.active ? s : 0;
    mean[i] = p.stats[(size_t)n * g.G + s];
    scale[i] = p.gamma[c] * p.stats[(size_t)(g.N + n) * g.G + s];
    shift[i] = p.beta[c];
  });
#pragma unroll
  for (int j = 0; j < 4; ++j)
    affine.set(j, make_float2(mean[2 * j], mean[2 * j + 1]), make_float2(scale[2 * j], scale[2 * j + 1]), make_float2(shift[2 * j], shift[2 * j + 1]));
  const T* x = p.x + (row0 + at.r) * g.C + at.c0;
  emit<T, VEC, sizeof(T) == 2 ? 4 : 2>(p, at, row0, count, affine, [&](int, uint32_t o) { return raw8_load<T, VEC>(x + o, at.left); });
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
  uint32_t scale, open;       // scale byte of the codes, bits of the gate (all set without ReLU)
};

template <typename T, bool VEC> __device__ __forceinline__ uint32_t open_bits(const Backward<T>& p, const Place& at, size_t row) {
  if (p.gate) return p.gate[row * ((p.g.C + 7) >> 3) + (at.c0 >> 3)];
  return positive_bits(raw8_load<T, VEC>(p.mask + row * p.g.C + at.c0, at.left));
}
__device__ __forceinline__ size_t scale_index(const Geom& g, const Place& at, size_t row) {
  return row * ((g.C + kCkptBlock - 1) / kCkptBlock) + at.c0 / kCkptBlock;
}

// A thread's 8 channels: the mean with its sign turned, gamma * rstd, beta.
struct Channels {
  f32x2 less[4], scale[4], shift[4];
};

// dz where the gate's bits are set, 0 elsewhere.  A product by 0x10204080 moves 4 bits to the tops of 4 bytes, from where a
// byte permutation spreads each over 16 bits.
template <uint32_t SELECT> __device__ __forceinline__ uint32_t spread_signs(uint32_t v) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(d) : "r"(v), "n"(SELECT));      // (__byte_perm has no sign-spreading selectors)
  return d;
}
__device__ __forceinline__ Raw8<__nv_bfloat16> opened(const Raw8<__nv_bfloat16>& dy, uint32_t open) {
  const uint32_t lo = (open & 15u) * 0x10204080u, hi = (open >> 4) * 0x10204080u;
  Raw8<__nv_bfloat16> r;
  r.q[0] = make_uint4(dy.q[0].x & spread_signs<0x9988>(lo), dy.q[0].y & spread_signs<0xBBAA>(lo),
                      dy.q[0].z & spread_signs<0x9988>(hi), dy.q[0].w & spread_signs<0xBBAA>(hi));
  return r;
}
__device__ __forceinline__ Raw8<float> opened(const Raw8<float>& dy, uint32_t open) {
  Raw8<float> r;
  const uint32_t* from = reinterpret_cast<const uint32_t*>(&dy);
  uint32_t* to = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
  for (int i = 0; i < 8; ++i) to[i] = (open >> i & 1u) ? from[i] : 0u;
  return r;
}

// x - mean and dz of one vector; h.dy is gated already where the gate is ReLU's.
template <typename T, bool CK>
__device__ __forceinline__ void operands(const Held<T, CK>& h, int act, const Channels& ch, F8& dz, F8& d) {
  dz = raw8_to_f8(h.dy);
  if constexpr (CK) {
    d = ckpt_numbers(h.codes);
    const f32x2 step = pair(ckpt_step(h.scale));
#pragma unroll
    for (int j = 0; j < 4; ++j) d.p[j] = fma2(d.p[j], step, ch.less[j]);
  } else {
    d = raw8_to_f8(h.x);
#pragma unroll
    for (int j = 0; j < 4; ++j) d.p[j] = add2(d.p[j], ch.less[j]);
  }
  if (act == ACT_SILU) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 z = halves(fma2(d.p[j], ch.scale[j], ch.shift[j]));
      dz.p[j] = mul2(dz.p[j], pair(silu_slope<T>(z.x), silu_slope<T>(z.y)));
    }
  }
}

// dx of this CTA's pixels: fetch(k) gives the thread's k-th operands; k1 = -rstd*S1/m, k2 = -rstd^2*S2/m.
template <typename T, bool VEC, bool CK, int U, typename Fetch>
__device__ __forceinline__ void emit_dx(const Backward<T>& p, const Place& at, size_t row0, int count, const Channels& ch,
                                        const f32x2 (&k1)[4], const f32x2 (&k2)[4], Fetch fetch) {
  const Geom& g = p.g;
  if (!at.active) return;
  const size_t off = (row0 + at.r) * g.C + at.c0;
  T* const dx = p.dx + off;
  const T* const res = p.res + off;
  const bool has_res = p.res != nullptr;
  const uint32_t step = (uint32_t)g.rp * g.C;
  for (int k0 = 0; k0 < g.iters; k0 += U) {
    if (at.r + k0 * g.rp >= count) break;
    Held<T, CK> hs[U];
    Raw8<T> rs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at.r + (k0 + u) * g.rp >= count) continue;
      hs[u] = fetch(k0 + u);
      if (has_res) rs[u] = raw8_load<T, VEC>(res + (uint32_t)(k0 + u) * step, at.left);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at.r + (k0 + u) * g.rp >= count) continue;
      F8 dz, d;
      operands<T, CK>(hs[u], p.act, ch, dz, d);
#pragma unroll
      for (int j = 0; j < 4; ++j) dz.p[j] = fma2(ch.scale[j], dz.p[j], fma2(d.p[j], k2[j], k1[j]));
      if (has_res) {
        const F8 r = raw8_to_f8(rs[u]);
#pragma unroll
        for (int j = 0; j < 4; ++j) dz.p[j] = add2(dz.p[j], r.p[j]);
      }
      raw8_put<T, VEC>(dx + (uint32_t)(k0 + u) * step, at.left, f8_to_raw8<T>(dz));
    }
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
  h.open = p.act == ACT_RELU ? open_bits<T, VEC>(p, at, row) : 0xFFu;
  return h;
}
// The constants of a thread's channels from the saved statistics.
template <typename T>
__device__ __forceinline__ void load_channels(const Backward<T>& p, const Place& at, int n, Channels& ch, float (&rstd)[8]) {
  const Geom& g = p.g;
  float mean[8], scale[8], shift[8];
  each_channel(at, g.Cg, [&](int i, int c, int s) {
    mean[i] = p.stats[(size_t)n * g.G + s];
    rstd[i] = p.stats[(size_t)(g.N + n) * g.G + s];
    scale[i] = p.gamma[c] * rstd[i];
    shift[i] = p.act == ACT_SILU ? p.beta[c] : 0.f;
  });
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    ch.less[j] = pair(-mean[2 * j], -mean[2 * j + 1]);
    ch.scale[j] = pair(scale[2 * j], scale[2 * j + 1]);
    ch.shift[j] = pair(shift[2 * j], shift[2 * j + 1]);
  }
}
// k1, k2 of a thread's channels from those of the groups, the first of which is `first`.
__device__ __forceinline__ void load_coefficients(const Place& at, int Cg, const float* c1, const float* c2, int first, f32x2 (&k1)[4], f32x2 (&k2)[4]) {
  float a[8], b[8];
  each_channel(at, Cg, [&](int i, int, int s) { a[i] = -c1[s - first]; b[i] = -c2[s - first]; });
#pragma unroll
  for (int j = 0; j < 4; ++j) { k1[j] = pair(a[2 * j], a[2 * j + 1]); k2[j] = pair(b[2 * j], b[2 * j + 1]); }
}
// A thread's sums of dz*(x - mean) and of dz.
struct Sums {
  F8 a, b;
  __device__ __forceinline__ Sums() {
#pragma unroll
    for (int j = 0; j < 4; ++j) a.p[j] = b.p[j] = 0;
  }
  __device__ __forceinline__ void add(const F8& dz, const F8& d) {
#pragma unroll
    for (int j = 0; j < 4; ++j) { a.p[j] = fma2(dz.p[j], d.p[j], a.p[j]); b.p[j] = add2(b.p[j], dz.p[j]); }
  }
  // A = rstd * sum dz*(x - mean) and B, to red[0..2048) and red[2048..4096)
  __device__ __forceinline__ void put(float* red, const Geom& g, const Place& at, const float (&rstd)[8]) const {
    float v[8], w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 x = halves(a.p[j]), y = halves(b.p[j]);
      v[2 * j] = x.x * rstd[2 * j]; v[2 * j + 1] = x.y * rstd[2 * j + 1];
      w[2 * j] = y.x; w[2 * j + 1] = y.y;
    }
    put_sums(red, g, at, v);
    put_sums(red + kThreads * 8, g, at, w);
  }
};

// The resident form.  Shared memory: the thread's vectors of dy and x (or its codes), a byte per vector for the gate's bits and
// one for the scale; then per-thread sums, per-channel sums A, B and per-group sums S1, S2 of this CTA, and k1, k2 of the image.
template <typename T, bool VEC, bool CK>
__global__ void __launch_bounds__(kThreads, 2) backward_kernel(const __grid_constant__ Backward<T> p) {
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
  load_channels(p, at, n, ch, rstd);
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
    return h;
  };
  Sums sums;
  if (at.active)
#pragma unroll 2
    for (int k = 0; k < g.iters; ++k) {
      if (at.r + k * g.rp >= count) break;
      Held<T, CK> h = held(k);
      if (p.act == ACT_RELU) {
        h.dy = opened(h.dy, open[k * kThreads + tid]);
        dys.put(k, h.dy);                           // gated once, for the second sweep too
      }
      F8 dz, d;
      operands<T, CK>(h, p.act, ch, dz, d);
      sums.add(dz, d);
    }
  sums.put(red, g, at, rstd);
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
  f32x2 k1[4], k2[4];
  load_coefficients(at, g.Cg, coef, coef + g.G, 0, k1, k2);
  emit_dx<T, VEC, CK, 2>(p, at, row0, count, ch, k1, k2, held);
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
  Place at(g, blockIdx.y);
  at.active = at.active && at.left > 0;
  if (!at.active) at.c0 = blockIdx.y * kMaxCols * 8;
  grid_dependency_wait();
  Channels ch;
  float rstd[8];
  load_channels(p, at, n, ch, rstd);
  Sums sums;
  auto add = [&](const Held<T, CK>& h) {
    F8 dz, d;
    operands<T, CK>(h, p.act, ch, dz, d);
    sums.add(dz, d);
  };
  if (at.active) {
    constexpr int U = sizeof(T) == 4 ? 2 : 4;             // vectors in flight
    int pixel = at.r;
    for (; pixel + (U - 1) * g.rp < count; pixel += U * g.rp) {
      Held<T, CK> h[U];
#pragma unroll
      for (int u = 0; u < U; ++u) h[u] = load_held<T, VEC, CK>(p, at, row0 + pixel + u * g.rp);
#pragma unroll
      for (int u = 0; u < U; ++u) { h[u].dy = opened(h[u].dy, h[u].open); add(h[u]); }
    }
    for (; pixel < count; pixel += g.rp) {
      Held<T, CK> h = load_held<T, VEC, CK>(p, at, row0 + pixel);
      h.dy = opened(h.dy, h.open);
      add(h);
    }
  }
  sums.put(red[0], g, at, rstd);
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
__global__ void __launch_bounds__(kThreads, 2) backward_apply_kernel(const __grid_constant__ Backward<T> p) {
  __shared__ float coef[2][kMaxCols * 8];
  const Geom& g = p.g;
  const int block = gridDim.x - 1 - blockIdx.x, part = block % g.parts, n = block / g.parts;
  const int p0 = part * g.pix, count = min(g.pix, g.P - p0);
  const size_t row0 = (size_t)n * g.P + p0;
  Place at(g, blockIdx.y);
  at.active = at.active && at.left > 0;
  if (!at.active) at.c0 = blockIdx.y * kMaxCols * 8;
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
  float rstd[8];
  f32x2 k1[4], k2[4];
  load_channels(p, at, n, ch, rstd);
  load_coefficients(at, g.Cg, coef[0], coef[1], g_first, k1, k2);
  emit_dx<T, VEC, CK, 2>(p, at, row0, count, ch, k1, k2, [&](int k) {
    Held<T, CK> h = load_held<T, VEC, CK>(p, at, row0 + at.r + k * g.rp);
    h.dy = opened(h.dy, h.open);
    return h;
  });
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
