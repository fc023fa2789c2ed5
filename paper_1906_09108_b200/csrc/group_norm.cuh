// Group normalisation with an activation, channels last, forward and backward.
//
// x [N][P][C] (P = H * W pixels); group g of image n is channels [g*Cg, (g+1)*Cg) at all pixels, m = P * Cg values:
//   mean = sum x / m,  var = sum (x - mean)^2 / m,  rstd = 1/sqrt(var + eps),  xhat = (x - mean)*rstd,
//   z = gamma*xhat + beta [+ res],  y = act(z);
//   dz = dy*act'(z),  A[n][c] = sum_p dz*xhat,  B[n][c] = sum_p dz:  dgamma = sum_n A,  dbeta = sum_n B,
//   S1 = sum over the group's channels of gamma*B,  S2 = of gamma*A,
//   dx = rstd*(gamma*dz - (S1 + xhat*S2)/m) [+ res].
// Bound by memory: 10 to 25 operations on each value against 2 to 9 bytes of traffic, which is close enough to the rate at which
// instructions issue that these count too: values go through the arithmetic in pairs (kernel_common.cuh), and what a call does
// not ask for (activation, gate, residual, checkpoint) is compiled out.
//
// Layout.  A row of a pixel's channels is cut into columns of 8 channels; a thread keeps one column and walks the pixels, rp of
// them side by side in a CTA of 256 threads, so a warp's accesses are contiguous for every channel count, and a group may start
// and end anywhere inside a column (5 channels of 160, say): sums are formed per channel and thread and added per group from
// shared memory.
//
// Streamed, both passes: as many CTAs as run at once, each a contiguous share of an image's pixels.  One kernel forms the sums
// and leaves a row of them per CTA in scratch; a second adds the rows up and applies them, walking its pixels backwards, so that
// it starts with what L2 holds, and starting its copies before the first has ended.  Vectors come through rings in shared memory.
// Resident, forward only (plan_forward): a cluster of up to 8 CTAs takes an image, each a share of its pixels, which it copies to
// shared memory at once (every thread its own vectors, so nothing but a thread's own wait stands between copy and use).  The
// moments are formed there, exchanged through distributed shared memory, and applied from there: one launch, one read, one write.
// (A backward pass by clusters was no faster anywhere: its parameter gradients need a second launch all the same.)
// In teams (plan_teams): small images, several to a CTA, one after the other.
//
// Variance: a thread sums its values and their squares less a pivot that follows their mean (Moments), brings them about a common
// value of the CTA (a mean over at least a 64th of the channel's values), then about the CTA's group mean, and CTAs are combined by Chan's
// formula.  The square of the distance from a mean over a share f of the values to the mean over all is at most var*(1 - f)/f, so what
// cancels in each step is bounded by the data itself, whatever offset x has.  The team form has the image at hand and takes the mean first.
// All sums are fp32 within a CTA (a thread's values in chains of 64 that are added up in turn, then rows of threads, then a tree), in a
// fixed order; what many CTAs leave is added in fp64.
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
  int iters;                // pixels per thread at most: ceil(pix / rp)
  int whole, whole_last;    // pixels that each of a thread's rows has at least: in a full share, in the last one with pixels
  int lanes_g, lanes_c;     // lanes that add up one group / one channel
  uint32_t col_mul, cg_mul; // tid / cols = tid * col_mul >> 16;  c / Cg = the high word of c * cg_mul (0: Cg = 1)
  int tiles;                // tiles of columns (1 unless streamed with more than 2048 channels)
  float inv_m;              // 1 / (P * Cg)
  int team;                 // team form: threads that take an image
  int entries, per_row;     // what a group's sums add in a row of threads: its columns or, where columns are cut, its channels
  int lanes_log, rows_on, cols_on;      // of a group's lanes: how many (log2), and how far apart in rows and entries a lane's terms are
  int buffers;              // images that a team has room for
  int slices, slice, Gs;    // a team's part of an image: of how many, its channels and groups (whole ones)
};
constexpr int kMergeParts = 16;             // rows of sums that the second streamed pass adds up itself
constexpr int kForwardPerSm = 3, kBackwardPerSm = 2;      // CTAs on an SM: 80 and 128 registers a thread

// ---- device helpers -------------------------------------------------------------------------------------
// 1/(1 + exp(-z)) of two values.  Exponentials and reciprocals run at 16 values per SM and cycle, a quarter of what a streaming
// pass asks for.
// For tensors in 16 bits from the approximate ones (relative error below 2^-20 for |z| < 16, growing with |z| as the rounding of
// z*log2(e) does), down to the smallest normal number and 0 below it; infinities and NaN come out as a division gives them.  us, 128
// images of 32x32x160, forward / backward / backward from codes: 29.9 / 39.6 / 42.8; two values sharing a reciprocal, 1/a = b * 1/(ab),
// 27.9 / 39.7 / 43.7, but that ends at exp(-z) = 2^62, from where SiLU came out as z * 2^-62; made good below by a factor, 29.3 / 43.0 / 47.7.
// For fp32 ones from expf and the approximate reciprocal r of d = 1 + exp(-z), which a step of Newton's iteration, r + r(1 - dr),
// brings from 2^-23 to the rounding of its last sum.  Below the smallest normal number the value is 0; d stops short of infinity,
// which the step would turn into NaN.  A division here branches: forward 22.8 us with it and 14.6 with this, 128 images of
// 16x16x160; backward 151 and 109 at 2048 pixels of 160 channels.
template <typename T> __device__ __forceinline__ f32x2 sigmoid(f32x2 z) {
  if constexpr (sizeof(T) == 2) {
    const float2 t = halves(mul2(z, pair(-1.44269504f)));
    float a, b, ra, rb;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(b) : "f"(t.y));
    const float2 d = halves(add2(pair(a, b), pair(1.f)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ra) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rb) : "f"(d.y));
    return pair(ra, rb);
  } else {
    const float2 h = halves(z);
    const float a = fminf(1.f + expf(-h.x), 3e38f), b = fminf(1.f + expf(-h.y), 3e38f);
    float ra, rb;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ra) : "f"(a));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rb) : "f"(b));
    const f32x2 r = pair(ra, rb);
    return fma2(r, fma2(pair(-a, -b), r, pair(1.f)), r);
  }
}
template <typename T> __device__ __forceinline__ f32x2 silu_slope(f32x2 z) {
  const f32x2 s = sigmoid<T>(z);
  return mul2(s, fma2(z, fma2(s, pair(-1.f), pair(1.f)), pair(1.f)));
}

__device__ __forceinline__ void copy16_async(void* smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}
__device__ __forceinline__ void copy8_async(void* smem, const void* gmem) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}
// Through L1, for pieces of a sector: the accesses that follow to the same sector find it there.
template <int W> __device__ __forceinline__ void copy_piece_async(void* smem, const void* gmem, bool exists) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem), "n"(W), "r"(exists ? W : 0)
               : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void prefetch_l2(const void* gmem) { asm volatile("prefetch.global.L2 [%0];" ::"l"(gmem)); }

// Vectors a thread keeps in shared memory: its own [iters] of them, 16 bytes of consecutive threads side by side.
template <typename T> struct Slots {
  static constexpr int Q = sizeof(T) / 2;
  uint4* base;                // + threadIdx.x
  __device__ __forceinline__ Slots(void* smem) : base(static_cast<uint4*>(smem) + threadIdx.x) {}
  template <int W> __device__ __forceinline__ void fetch(int k, const T* __restrict__ p, int left) const {
    if constexpr (W == kWhole && sizeof(T) == 2) {
      copy16_async(base + k * kThreads, p);
    } else if constexpr (W >= 4) {
      constexpr int B = W, PER = B / (int)sizeof(T);
#pragma unroll
      for (int i = 0; i < 8 / PER; ++i)
        copy_piece_async<B>(reinterpret_cast<char*>(base + (k * Q + i * B / 16) * kThreads) + i * B % 16, p + i * PER, W == kWhole || i * PER < left);
    } else {
      put(k, raw8_load<T, W>(p, left));
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

// The streamed passes copy to shared memory ahead of what they use, every thread its own vectors, B of them to a commit group
// (32 bytes) and kAhead groups under way: 96 to 128 bytes per thread are on their way at any time, which costs no registers and
// needs no barrier.  start(mine, issue) begins; run() calls turn(k, slot, full) for k = 0, B, ... < n once vectors k .. k + B - 1 have
// come to slots slot .. slot + B - 1; issue(slot) starts the copy of the thread's next vector (of `mine`) into a slot.  The loop is
// unrolled over the ring, so that slots are constants.
constexpr int kAhead = 3;
template <typename T> __host__ __device__ constexpr int batch_of() { return sizeof(T) == 2 ? 2 : 1; }
template <typename T> __host__ __device__ constexpr int ring_of() { return batch_of<T>() * (kAhead + 1); }
template <bool FULL> struct Full { static constexpr bool value = FULL; };      // whether every vector of a turn exists
template <int B> struct Stream {
  static constexpr int R = B * (kAhead + 1);
  template <typename Issue> static __device__ __forceinline__ void start(int mine, Issue issue) {
#pragma unroll
    for (int k = 0; k < B * kAhead; ++k) {
      if (k < mine) issue(k);
      if (k % B == B - 1) asm volatile("cp.async.commit_group;" ::: "memory");
    }
  }
  // `after`(k), once k vectors have been used, k a multiple of R: after whole rounds of the ring, which ask nothing of a single vector.
  // Fewer than R + B * kAhead vectors follow the last of them.
  template <typename Issue, typename Turn, typename After>
  static __device__ __forceinline__ void run(int n, int mine, Issue issue, Turn turn, After after) {
    int k0 = 0;
    for (; k0 + R + B * kAhead <= mine; k0 += R) {
      round<true>(k0, n, mine, issue, turn);
      after(k0 + R);
    }
    for (; k0 < n; k0 += R) round<false>(k0, n, mine, issue, turn);
  }
  template <typename Issue, typename Turn> static __device__ __forceinline__ void run(int n, int mine, Issue issue, Turn turn) {
    run(n, mine, issue, turn, [](int) {});
  }
  // The same in a loop of single turns, for turns whose code unrolled over the ring does not fit the instruction caches.
  template <typename Issue, typename Turn> static __device__ __forceinline__ void run_rolled(int n, int mine, Issue issue, Turn turn) {
#pragma unroll 1
    for (int k = 0; k < n; k += B) {
#pragma unroll
      for (int u = 0; u < B; ++u)
        if (k + B * kAhead + u < mine) issue((k + B * kAhead + u) & (R - 1));
      asm volatile("cp.async.commit_group;" ::: "memory");
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
      turn(k, k & (R - 1), Full<false>());
    }
  }

 private:
  template <bool FULL, typename Issue, typename Turn>
  static __device__ __forceinline__ void round(int k0, int n, int mine, Issue& issue, Turn& turn) {
#pragma unroll
    for (int b = 0; b < R; b += B) {
      if (FULL || k0 + b < n) {
#pragma unroll
        for (int u = 0; u < B; ++u)
          if (FULL || k0 + b + B * kAhead + u < mine) issue((b + B * kAhead + u) % R);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
        turn(k0 + b, b, Full<FULL>());
      }
    }
  }
};

// Whether copies of these vectors may begin before a kernel's grid_dependency_wait(), see moments_kernel: those that go past L1.  (L1 is
// not coherent: a line that it holds from before the wait may be older than what the wait makes visible.)
template <typename T, int W> constexpr bool kEarly = W == kWhole && sizeof(T) == 2;

// This thread's place in a CTA's tile.
struct Place {
  int col, r;
  bool active;
  int c0, left;               // first channel, channels of the column that exist
  __device__ __forceinline__ Place(const Geom& g, int tile, uint32_t tid = threadIdx.x) {
    r = (int)(tid * g.col_mul >> 16); col = (int)tid - r * g.cols;
    active = r < g.rp;
    c0 = (tile * kMaxCols + col) * 8;
    left = min(8, g.C - c0);
  }
  __device__ __forceinline__ int channel(int i) const { return i < left ? c0 + i : c0; }
};

// take(i, channel, group) for the 8 channels of a column; those past the last channel stand in for the first.
__device__ __forceinline__ int group_of(const Geom& g, int c) { return g.cg_mul ? (int)__umulhi((uint32_t)c, g.cg_mul) : c; }
template <typename Take> __device__ __forceinline__ void each_channel(const Geom& g, const Place& at, Take take) {
  const int Cg = g.Cg, first = group_of(g, at.c0);
  int s = first, rem = at.c0 - first * Cg;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    take(i, at.channel(i), i < at.left ? s : first);
    if (++rem == Cg) { rem = 0; ++s; }
  }
}

// This CTA's pixels: `count` from pixel `row0` of the tensor on; a thread has `mine` of them, `whole` or one more.
struct Share {
  size_t row0;
  int count, whole, mine;
  int turns;                  // of the CTA's threads, the most that one has
  __device__ __forceinline__ Share(const Geom& g, const Place& at, int n, int part) {
    const int p0 = part * g.pix;
    row0 = (size_t)n * g.P + p0;
    count = max(0, min(g.pix, g.P - p0));
    whole = count == g.pix ? g.whole : count > 0 ? g.whole_last : 0;
    turns = whole + (count > whole * g.rp ? 1 : 0);
    mine = at.active ? whole + (at.r < count - whole * g.rp ? 1 : 0) : 0;
  }
};

// red[r][8 * cols] = the 8 sums of each thread.
__device__ __forceinline__ void put_sums(float* red, const Geom& g, const Place& at, const float (&v)[8]) {
  if (!at.active) return;
  float4* d = reinterpret_cast<float4*>(red + (at.r * g.cols + at.col) * 8);
  d[0] = make_float4(v[0], v[1], v[2], v[3]);
  d[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Sums over the rows of threads of two such arrays (the second 2048 floats behind the first): done(c, sum, sum) for the tile's
// first `sets` channels; `lanes` consecutive lanes (a power of two up to 32) share a channel.  For the whole CTA.
template <typename Done>
__device__ __forceinline__ void channel_sums(const float* red, const Geom& g, int sets, int lanes, Done done) {
  const int sub = threadIdx.x & (lanes - 1), per_pass = kThreads / lanes, width = g.cols * 8;
  for (int c0 = 0; c0 < sets; c0 += per_pass) {
    const int c = c0 + threadIdx.x / lanes;
    float a = 0.f, b = 0.f;
    if (c < sets) {
      const float* v = red + c + sub * width;
#pragma unroll 4
      for (int r = sub; r < g.rp; r += lanes, v += lanes * width) { a += v[0]; b += v[kThreads * 8]; }
    }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (c < sets && sub == 0) done(c, a, b);
  }
}
// The sum of v over the `lanes` lanes that share a group.
__device__ __forceinline__ float lane_sum(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// done(s, sum of first(c), sum of second(c) over the group's channels) for groups s < sets of `size` channels from c = 0 on; chains of
// at most 64 and then of at most 32 for 65536 channels.
template <typename Value, typename Done>
__device__ __forceinline__ void group_sums(int sets, int size, int lanes, Value value, Done done) {
  const int sub = threadIdx.x & (lanes - 1), per_pass = kThreads / lanes;
  for (int s0 = 0; s0 < sets; s0 += per_pass) {
    const int s = s0 + threadIdx.x / lanes;
    float2 a = make_float2(0.f, 0.f);
    if (s < sets)
      for (int j0 = 0; j0 < size; j0 += 64 * lanes) {
        float2 b = make_float2(0.f, 0.f);
        const int end = min(size, j0 + 64 * lanes);
#pragma unroll 8
        for (int j = j0 + sub; j < end; j += lanes) {
          const float2 v = value(s * size + j);
          b.x += v.x; b.y += v.y;
        }
        a.x += b.x; a.y += b.y;
      }
    a.x = lane_sum(a.x, lanes);
    a.y = lane_sum(a.y, lanes);
    if (s < sets && sub == 0) done(s, a.x, a.y);
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
  float* partial;             // streamed: [N][parts][2][sets]: means and squared deviations; sets = groups, or channels with tiles > 1
  float eps;
  int act;
  int ckpt_lanes;
  bool combined;              // streamed: `stats` holds the statistics when the second pass starts
};

// A thread's moments of its 8 channels: sums of its values and of their squares less a pivot, at first the first of them.
// close(n), n values so far, moves the pivot to their mean and puts their squared deviations from it with those of earlier values, at
// every doubling and then every kChain values (closes()).  With M = sum (x - mean)^2 over all n values of the thread, the mean of the
// first k differs from that of all by at most sqrt(M/k): the squares of the next min(k, kChain) values about it add up to no
// more than a few M whatever the first value is, and no chain of additions is longer than kChain, or than the number of chains.
// (From the first value alone: n M, which at 2048 values of spread 1 around 100, the first one 0, cost rstd its second digit.)
constexpr int kChain = 64;
struct Moments {
  F8 pivot, sum, square, closed;                 // the pivot with its sign turned
  __device__ __forceinline__ Moments() {
#pragma unroll
    for (int j = 0; j < 4; ++j) pivot.p[j] = sum.p[j] = square.p[j] = closed.p[j] = 0;
  }
  __device__ __forceinline__ void start(const F8& x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) pivot.p[j] = mul2(x.p[j], pair(-1.f));
  }
  __device__ __forceinline__ void add(const F8& x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 d = add2(x.p[j], pivot.p[j]);
      sum.p[j] = add2(sum.p[j], d);
      square.p[j] = fma2(d, d, square.p[j]);
    }
  }
  static __device__ __forceinline__ int after(int n) { return n + min(n, kChain); }      // when to close next
  // The pivot moves by t as rounded, and what the sum is not exactly 0 by then stays in it: roundings of the pivot do not add up.
  __device__ __forceinline__ void close(int n) {
    const f32x2 over = pair(-1.f / (float)n), less_n = pair(-(float)n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 to = fma2(sum.p[j], over, pivot.p[j]);
      const f32x2 t = fma2(to, pair(-1.f), pivot.p[j]), rest = fma2(t, less_n, sum.p[j]);
      closed.p[j] = add2(closed.p[j], fma2(mul2(t, pair(-1.f)), add2(sum.p[j], rest), square.p[j]));
      sum.p[j] = rest; square.p[j] = 0; pivot.p[j] = to;
    }
  }
};

// The CTA's moments from its threads' (each over n values): chan[c] = mean and squared deviations from it of the tile's first
// `sets` channels.  `red`: 4096 floats, `common`: 2048 floats.  Ends with a barrier.
// A channel's rows of threads are summed about a common value.  That value's distance from the mean, where it is a mean over a share f
// of the values, is at most sqrt(var (1 - f)/f), so the sums lose a factor of up to 1/f: a row of the rp.  Beyond 64 rows (three columns
// or fewer) eight of them, far apart, give it: with the first of 256 alone, a map whose first column is blank cost rstd 4e-5 of itself.
constexpr int kRowsAbout = 8;
__device__ __forceinline__ void cta_moments(const Geom& g, const Place& at, const Moments& m, int n, int count, int sets, float* red, float* common,
                                            float2* chan) {
  const float fn = (float)n, over = n > 0 ? 1.f / fn : 0.f;
  float mu[8], dev[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = halves(m.pivot.p[j]), s1 = halves(m.sum.p[j]), s2 = halves(m.square.p[j]), s3 = halves(m.closed.p[j]);
    mu[2 * j] = fmaf(s1.x, over, -f.x);
    mu[2 * j + 1] = fmaf(s1.y, over, -f.y);
    dev[2 * j] = fmaf(-s1.x * over, s1.x, s2.x) + s3.x;
    dev[2 * j + 1] = fmaf(-s1.y * over, s1.y, s2.y) + s3.y;
  }
  if (at.r == 0) put_sums(common, g, at, mu);
  const int filled = min(g.rp, count);                   // rows of threads with values
  if (filled > 64) {
    const int apart = filled / kRowsAbout, row = at.r / apart, w = g.cols * 8;
    if (at.r == row * apart && row < kRowsAbout) put_sums(red + (row - at.r) * w, g, at, mu);          // rows 0 to 7 of red
    __syncthreads();
    if (threadIdx.x < w) {
      const float* v = red + threadIdx.x;                  // in pairs, so that equal ones give themselves exactly
      common[threadIdx.x] = 0.125f * (((v[0] + v[w]) + (v[2 * w] + v[3 * w])) + ((v[4 * w] + v[5 * w]) + (v[6 * w] + v[7 * w])));
    }
  }
  __syncthreads();
  const float4* k = reinterpret_cast<const float4*>(common + at.col * 8);
  const float4 k0 = k[0], k1 = k[1];
  const float about[8] = {k0.x, k0.y, k0.z, k0.w, k1.x, k1.y, k1.z, k1.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float d = n > 0 ? mu[i] - about[i] : 0.f;
    mu[i] = fn * d;
    dev[i] = n > 0 ? fmaf(fn * d, d, max_nan(dev[i], 0.f)) : 0.f;
  }
  put_sums(red, g, at, mu);
  put_sums(red + kThreads * 8, g, at, dev);
  __syncthreads();
  const float inv = count > 0 ? 1.f / (float)count : 0.f;
  channel_sums(red, g, sets, g.lanes_c, [&](int c, float s, float q) {
    const float d = s * inv;
    chan[c] = make_float2(common[c] + d, max_nan(fmaf(-s, d, q), 0.f));
  });
  __syncthreads();
}
// done(s, mean, squared deviations) of this CTA's groups from its channels' moments over `count` pixels.
template <typename Done>
__device__ __forceinline__ void group_moments(const Geom& g, int count, const float2* chan, Done done) {
  const int lanes = g.lanes_g, sub = threadIdx.x & (lanes - 1), per_pass = kThreads / lanes;
  const float inv = 1.f / (float)g.Cg;
  for (int s0 = 0; s0 < g.G; s0 += per_pass) {
    const int s = s0 + threadIdx.x / lanes;
    float a = 0.f, q = 0.f;
    const float first = chan[min(s, g.G - 1) * g.Cg].x;          // differences from it: equal means give themselves exactly
    if (s < g.G)
      for (int j = sub; j < g.Cg; j += lanes) a += chan[s * g.Cg + j].x - first;
    const float mu = fmaf(lane_sum(a, lanes), inv, first);
    if (s < g.G)
      for (int j = sub; j < g.Cg; j += lanes) {
        const float2 c = chan[s * g.Cg + j];
        const float d = c.x - mu;
        q += fmaf((float)count * d, d, c.y);
      }
    q = lane_sum(q, lanes);
    if (s < g.G && sub == 0) done(s, mu, q);
  }
}
// Chan: done(s, mean, rstd) of the image's groups from the moments of its `rows` CTAs, row(j)[s] their means and row(j)[G + s] their
// squared deviations; up to 8 lanes share a group.
template <typename Row, typename Done>
__device__ __forceinline__ void image_moments(const Geom& g, int rows, float eps, Row row, Done done) {
  const int lanes = rows >= 8 ? 8 : rows >= 4 ? 4 : rows >= 2 ? 2 : 1, sub = threadIdx.x & (lanes - 1), per_pass = kThreads / lanes;
  const float inv_p = 1.f / (float)g.P, inv_cg = 1.f / (float)g.Cg;
  auto pixels = [&](int j) { return (float)max(0, min(g.pix, g.P - j * g.pix)); };
  for (int s0 = 0; s0 < g.G; s0 += per_pass) {
    const int s = s0 + threadIdx.x / lanes;
    float a = 0.f, q = 0.f;
    const float first = row(0)[min(s, g.G - 1)];
    if (s < g.G)
      for (int j = sub; j < rows; j += lanes) a = fmaf(row(j)[s] - first, pixels(j) * inv_p, a);
    const float mu = lane_sum(a, lanes) + first;
    if (s < g.G)
      for (int j = sub; j < rows; j += lanes) {
        const float d = row(j)[s] - mu;
        q = fmaf(pixels(j) * d, d, fmaf(row(j)[g.G + s], inv_cg, q));
      }
    q = lane_sum(q, lanes);
    if (s < g.G && sub == 0) done(s, mu, 1.f / sqrtf(fmaf(q, inv_p, eps)));
  }
}

// What a thread multiplies its 8 channels by: scale = gamma*rstd and shift = beta, and the mean with its sign turned.  The mean is
// subtracted before anything is rounded: in a group without spread, where rstd is 1/sqrt(eps), x - mean is 0 and y is act(beta) exactly.
// (Taken into the shift, it is rounded at the size of |mean|*scale: blank groups of 100 came out up to 2e-3 beside beta, ReLU's
// gate of a whole group with them.)
struct Affine {
  f32x2 scale[4], shift[4], less[4];
  __device__ __forceinline__ void set(int j, float2 mean, float2 sc, float2 sh) {
    scale[j] = pair(sc.x, sc.y);
    shift[j] = pair(sh.x, sh.y);
    less[j] = pair(-mean.x, -mean.y);
  }
  __device__ __forceinline__ f32x2 of(int j, f32x2 x) const { return fma2(add2(x, less[j]), scale[j], shift[j]); }
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

// y (and the gate's bits, and x in 8 bits) of a thread's pixels.  ACT < 0: p.act.  EXTRA 1: res and gate may be asked for; 2: and
// codes.  Offsets inside a CTA's pixels fit 32 bits.
enum { PLAIN = 0, WITH_RES_GATE = 1, WITH_CODES = 2 };
template <typename T, int W, int ACT, int EXTRA> struct Emitter {
  T* y;                       // of the CTA's first pixel, as the others: the same for all threads
  const T* res;
  int8_t* codes;
  uint8_t *gate, *scales;
  uint32_t first, step, gate_first, gate_step, scale_first, scale_step;      // the thread's first pixel, and the next from each
  int act, left, lanes;
  bool leads;
  __device__ __forceinline__ Emitter(const Forward<T>& p, const Place& at, const Share& sh) {
    const Geom& g = p.g;
    const size_t off = sh.row0 * g.C;
    act = ACT < 0 ? p.act : ACT;
    left = at.left;
    y = p.y + off;
    first = (uint32_t)at.r * g.C + at.c0;
    step = (uint32_t)g.rp * g.C;
    res = nullptr; gate = nullptr; codes = nullptr;
    if constexpr (EXTRA >= WITH_RES_GATE) {
      const int all_cols = (g.C + 7) >> 3;
      if (p.res) res = p.res + off;
      if (p.gate) gate = p.gate + sh.row0 * all_cols;
      gate_first = (uint32_t)at.r * all_cols + (at.c0 >> 3);
      gate_step = (uint32_t)g.rp * all_cols;
    }
    if constexpr (EXTRA == WITH_CODES) {
      const int per_row = (g.C + kCkptBlock - 1) / kCkptBlock;
      if (W == kWhole || p.codes) codes = p.codes + off;             // the form for any alignment is compiled once, for all options
      scales = p.scales + sh.row0 * per_row;
      scale_first = (uint32_t)at.r * per_row + at.c0 / kCkptBlock;
      scale_step = (uint32_t)g.rp * per_row;
      lanes = p.ckpt_lanes;
      leads = (at.col & (lanes - 1)) == 0;
    }
  }
  // Pixel k of the thread, at element offset o.
  __device__ __forceinline__ void value(uint32_t k, uint32_t o, const Affine& affine, const F8& x, const Raw8<T>& raw_res) const {
    F8 z;
#pragma unroll
    for (int j = 0; j < 4; ++j) z.p[j] = affine.of(j, x.p[j]);
    if constexpr (EXTRA >= WITH_RES_GATE)
      if (res) {
        const F8 r = raw8_to_f8(raw_res);
#pragma unroll
        for (int j = 0; j < 4; ++j) z.p[j] = add2(z.p[j], r.p[j]);
      }
    if (act == ACT_RELU) {
      const Raw8<T> out = f8_to_raw8<T, true>(z);
      raw8_put<T, W>(y + o, left, out);
      if constexpr (EXTRA >= WITH_RES_GATE)
        if (gate) gate[gate_first + k * gate_step] = (uint8_t)(positive_bits(out) & (W == kWhole ? 0xFFu : (1u << left) - 1));
    } else {
      if (act == ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 4; ++j) z.p[j] = mul2(z.p[j], sigmoid<T>(z.p[j]));
      }
      raw8_put<T, W>(y + o, left, f8_to_raw8<T>(z));
    }
  }
  // A turn of B pixels, raw, k counting from the thread's first pixel or (back) its last; for the whole warp where codes are
  // formed, since the lanes that share a block of 32 channels (they have the same pixels) exchange its maximum.
  template <bool FULL, int B>
  __device__ __forceinline__ void turn(int k, int mine, bool back, const Affine& affine, const Raw8<T> (&raw)[B], const Raw8<T>* raw_res) const {
    uint32_t top[B];
    if constexpr (EXTRA == WITH_CODES)
      if (W == kWhole || codes) block_tops<B>(raw, top);
#pragma unroll
    for (int u = 0; u < B; ++u)
      if (FULL || k + u < mine) {
        const uint32_t kk = (uint32_t)(back ? mine - 1 - (k + u) : k + u), o = first + kk * step;
        const F8 x = raw8_to_f8(raw[u]);
        value(kk, o, affine, x, raw_res[EXTRA >= WITH_RES_GATE ? u : 0]);
        if constexpr (EXTRA == WITH_CODES)
          if (W == kWhole || codes) {
            const CkptScale s = ckpt_scale(top[u]);
            store_codes<kCodeWidth<T, W>>(codes + o, left, ckpt_codes(x, s));
            if (leads) scales[scale_first + kk * scale_step] = (uint8_t)s.byte;
          }
      }
  }
  // The largest magnitudes of the blocks of B vectors: 16-bit ones travel two to a word.
  template <int B> __device__ __forceinline__ void block_tops(const Raw8<T> (&raw)[B], uint32_t (&top)[B]) const {
    if constexpr (sizeof(T) == 2 && B == 2) {
      const uint32_t a = ckpt_top2(raw[0]), b = ckpt_top2(raw[1]);
      uint32_t m = max_u16x2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
      if (lanes >= 2) m = max_u16x2(m, __shfl_xor_sync(0xffffffffu, m, 1));
      if (lanes >= 4) m = max_u16x2(m, __shfl_xor_sync(0xffffffffu, m, 2));
      top[0] = m << 16;
      top[1] = m & 0xFFFF0000u;
    } else {
#pragma unroll
      for (int u = 0; u < B; ++u) top[u] = ckpt_top_of_lanes(ckpt_top(raw[u]), lanes);
    }
  }
};
// The constants of a thread's channels from their groups' statistics.
template <typename T, typename Stat>
__device__ __forceinline__ void load_affine(const Forward<T>& p, const Place& at, const float (&gamma)[8], const float (&beta)[8], Stat stat, Affine& affine) {
  float2 m[8];
  each_channel(p.g, at, [&](int i, int, int s) { m[i] = stat(s); });
#pragma unroll
  for (int j = 0; j < 4; ++j)
    affine.set(j, make_float2(m[2 * j].x, m[2 * j + 1].x), make_float2(gamma[2 * j] * m[2 * j].y, gamma[2 * j + 1] * m[2 * j + 1].y),
               make_float2(beta[2 * j], beta[2 * j + 1]));
}

// The resident form: blockIdx = image, share of its pixels, tile of columns: a cluster per image.
template <typename T, int W, int ACT, int EXTRA>
__global__ void __launch_bounds__(kThreads, kForwardPerSm) forward_kernel(const __grid_constant__ Forward<T> p) {
  constexpr int kBatch = W == kWhole ? 2 : 1;           // pieces of a vector take registers of their own: 16x16384x36 35.4 us with 2, 33.1 with 1
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  float* red = reinterpret_cast<float*>(smem + (size_t)g.iters * Slots<T>::Q * kThreads);      // [4096]
  float* common = red + 2 * kThreads * 8;                                                       // [2048]
  float2* chan = reinterpret_cast<float2*>(common + kThreads * 8);                               // [C]
  float* own = reinterpret_cast<float*>(chan + g.C);      // mean [G], squared deviations [G] of this CTA's pixels
  float2* mom = reinterpret_cast<float2*>(own + 2 * g.G);                                        // mean, rstd [G] of the image
  const int rank = blockIdx.y, n = blockIdx.x;
  const Place at(g, 0);
  const Share sh(g, at, n, rank);
  const Slots<T> slots(smem);
  grid_dependency_wait();
  const T* src = p.x + (sh.row0 + at.r) * g.C + at.c0;
  const uint32_t step = (uint32_t)g.rp * g.C;
#pragma unroll 4
  for (int k = 0; k < sh.mine; ++k) slots.template fetch<W>(k, src + (uint32_t)k * step, at.left);
  const Emitter<T, W, ACT, EXTRA> out(p, at, sh);
  if constexpr (EXTRA >= WITH_RES_GATE)
    if (out.res)
      for (int k = 0; k < sh.mine; ++k) prefetch_l2(out.res + (out.first + (uint32_t)k * step));
  float gamma[8], beta[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { gamma[i] = p.gamma[at.channel(i)]; beta[i] = p.beta[at.channel(i)]; }
  copies_done();
  Moments m;
  if (sh.mine > 0) m.start(raw8_to_f8(slots.get(0)));
  int k = 0, close_at = 8;
  for (; k + 8 <= sh.mine; k += 8) {
#pragma unroll 4
    for (int u = 0; u < 8; ++u) m.add(raw8_to_f8(slots.get(k + u)));
    if (k + 8 == close_at) { m.close(k + 8); close_at = Moments::after(k + 8); }
  }
  for (; k < sh.mine; ++k) m.add(raw8_to_f8(slots.get(k)));
  cta_moments(g, at, m, sh.mine, sh.count, g.C, red, common, chan);
  group_moments(g, sh.count, chan, [&](int s, float mu, float q) { own[s] = mu; own[g.G + s] = q; });
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  image_moments(g, g.parts, p.eps, [&](int j) { return cluster.map_shared_rank(own, j); }, [&](int s, float mu, float rstd) {
    mom[s] = make_float2(mu, rstd);
    if (rank == 0) {
      p.stats[(size_t)n * g.G + s] = mu;
      p.stats[(size_t)(g.N + n) * g.G + s] = rstd;
    }
  });
  cg::cluster_group::arrival_token token = cluster.barrier_arrive();      // this CTA reads its neighbours' sums no more
  __syncthreads();
  Affine affine;
  load_affine(p, at, gamma, beta, [&](int s) { return mom[s]; }, affine);
  Raw8<T> next_res{};
  if constexpr (EXTRA >= WITH_RES_GATE && kBatch == 1)
    if (out.res && sh.mine > 0) next_res = raw8_load<T, W>(out.res + out.first, at.left);
  for (int k = 0; k < (EXTRA == WITH_CODES ? sh.turns : sh.mine); k += kBatch) {
    Raw8<T> xs[kBatch], rs[EXTRA >= WITH_RES_GATE ? kBatch : 1];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (EXTRA == WITH_CODES || k + u < sh.mine) xs[u] = slots.get(min(k + u, g.iters - 1));
      if constexpr (EXTRA >= WITH_RES_GATE && kBatch > 1)
        if (out.res && k + u < sh.mine) rs[u] = raw8_load<T, W>(out.res + (out.first + (uint32_t)(k + u) * step), at.left);
    }
    if constexpr (EXTRA >= WITH_RES_GATE && kBatch == 1) {
      rs[0] = next_res;
      if (out.res && k + 1 < sh.mine) next_res = raw8_load<T, W>(out.res + (out.first + (uint32_t)(k + 1) * step), at.left);
    }
    out.template turn<false>(k, sh.mine, false, affine, xs, rs);
  }
  cluster.barrier_wait(std::move(token));                                 // nor do they read its own
}

// The team form, for small images: `team` threads (32 to 256, whole warps) take an image, a CTA the images that its teams have room
// for, each team one after the other with the next one's copy under way; a team waits for nobody else.  An image is in shared
// memory, so its mean comes first and the squares of what is left of it after, from sums over groups (a value per thread where
// columns lie in one group each).  What a CTA per image spends on starting, on exchanging sums and on its end is the time of these
// calls: us, with the other forms / with this one, 16-bit storage: 4096x2x2x64 54 / 5.0, 4096x4x4x256 66 / 15, 1024x8x8x160 23 / 11,
// 20000x1x512 284 / 28, 128x8x8x160 6.4 / 4.3, one image of 8x8x64 4.9 / 3.0.  Bound by issue slots at one pixel per image (a quarter of the
// copy rate), by memory from a few kilobytes per image on (60 to 72 %).  A pixel at a time: two cost more spilled registers (14.3 against
// 16.4).  At 80 registers the forms with a residual, gate or codes, and those for rows that are no whole vectors, spill 16 to 88 bytes.
struct Team {
  int first, tid, size;       // its first thread, this thread's number in it
  int sub, set, r0, j0;       // which of a group's lanes, of which of the first groups; where that lane's terms start
  __device__ __forceinline__ explicit Team(const Geom& g)
      : first(threadIdx.x & ~(g.team - 1)), tid(threadIdx.x & (g.team - 1)), size(g.team), sub(tid & (g.lanes_g - 1)), set(tid >> g.lanes_log),
        r0(sub / g.entries), j0(sub - r0 * g.entries) {}
  __device__ __forceinline__ void sync() const {
    if (size == 32) __syncwarp();
    else asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + first / 32), "r"(size) : "memory");
  }
};
// Where a thread's entries of a group's sums are: one where its column is in one group, else one per channel.
__device__ __forceinline__ float* team_at(float* red, const Geom& g, const Place& at) {
  return red + (at.r * g.per_row) + at.col * (g.entries == g.Cg ? 8 : 1);
}
// red = what a thread adds to its groups' sums.
__device__ __forceinline__ void team_put(float* red, const Geom& g, const Place& at, const F8& v) {
  if (!at.active) return;
  float* d = team_at(red, g, at);
  if (g.entries == g.Cg) {
    reinterpret_cast<ulonglong2*>(d)[0] = make_ulonglong2(v.p[0], v.p[1]);
    reinterpret_cast<ulonglong2*>(d)[1] = make_ulonglong2(v.p[2], v.p[3]);
  } else {
    const float2 t = halves(add2(add2(v.p[0], v.p[1]), add2(v.p[2], v.p[3])));
    *d = t.x + t.y;
  }
}
// done(s, the sum over group s).
template <typename Done> __device__ __forceinline__ void team_group_sums(const Geom& g, const Team& t, const float* red, Done done) {
  const int n = g.entries;
  for (int s0 = 0; s0 < g.Gs; s0 += t.size >> g.lanes_log) {
    const int s = s0 + t.set;
    float a = 0.f;
    if (s < g.Gs) {
      const float* v = red + s * n;
      for (int r = t.r0, j = t.j0; r < g.rp;) {
        a += v[r * g.per_row + j];
        r += g.rows_on; j += g.cols_on;
        if (j >= n) { j -= n; ++r; }
      }
    }
    a = lane_sum(a, g.lanes_g);
    if (s < g.Gs && t.sub == 0) done(s, a);
  }
}
// The same of threads' means, weighted by the pixels of their rows: done(s, the mean over group s), as differences from the first of
// them, so that a group without spread has exactly its value.  over: 1 / (entries * pixels).
template <typename Done> __device__ __forceinline__ void team_group_means(const Geom& g, const Team& t, const float* red, float over, Done done) {
  const int n = g.entries, more = g.P - g.whole * g.rp;
  const float cnt = (float)g.whole;
  for (int s0 = 0; s0 < g.Gs; s0 += t.size >> g.lanes_log) {
    const int s = s0 + t.set;
    float a = 0.f, first = 0.f;
    if (s < g.Gs) {
      const float* v = red + s * n;
      first = v[0];
      for (int r = t.r0, j = t.j0; r < g.rp;) {
        a = fmaf(v[r * g.per_row + j] - first, r < more ? cnt + 1.f : cnt, a);
        r += g.rows_on; j += g.cols_on;
        if (j >= n) { j -= n; ++r; }
      }
    }
    a = lane_sum(a, g.lanes_g);
    if (s < g.Gs && t.sub == 0) done(s, fmaf(a, over, first));
  }
}
// A group's value for each channel of a thread's column.
template <typename Value> __device__ __forceinline__ void team_values(const Geom& g, const Place& at, Value value, float (&m)[8]) {
  if (g.entries == g.Cg) {
    each_channel(g, at, [&](int i, int, int s) { m[i] = value(s); });
  } else {
    const float v = value(group_of(g, at.c0));
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = v;
  }
}
template <typename T, int W, int ACT, int EXTRA>
__global__ void __launch_bounds__(kThreads, kForwardPerSm) forward_teams_kernel(const __grid_constant__ Forward<T> p) {
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  const Team t(g);
  const Place at(g, 0, (uint32_t)t.tid);                                                        // in the slice, and
  Place whole = at;                                                                             // in the image
  whole.c0 += blockIdx.y * g.slice;
  const int g_first = blockIdx.y * g.Gs;
  const Slots<T> slots(smem);                                                                   // two images, iters of each
  float* red = reinterpret_cast<float*>(smem + (size_t)g.buffers * g.iters * Slots<T>::Q * kThreads) + t.first * 8;      // [8 * team]
  float2* mom = reinterpret_cast<float2*>(reinterpret_cast<float*>(smem + (size_t)g.buffers * g.iters * Slots<T>::Q * kThreads) + 8 * kThreads) +
                (t.first / t.size) * g.Gs;                                                      // [Gs]: mean, rstd
  const int teams = kThreads / t.size, stride = gridDim.x * teams;
  const uint32_t first = (uint32_t)at.r * g.C + whole.c0, step = (uint32_t)g.rp * g.C;
  const int mine = Share(g, at, 0, 0).mine;
  const bool cut = g.entries == g.Cg;                                                           // columns lie in more than one group
  const float over = mine > 0 ? 1.f / (float)(cut ? mine : 8 * mine) : 0.f, m = (float)(g.P * g.Cg);
  auto fetch = [&](int n, int buf) {
    const T* src = p.x + (size_t)n * g.P * g.C + first;
    for (int k = 0; k < mine; ++k) slots.template fetch<W>(buf * g.iters + k, src + (uint32_t)k * step, at.left);
    if constexpr (EXTRA >= WITH_RES_GATE)
      if (p.res)
        for (int k = 0; k < mine; ++k) prefetch_l2(p.res + (size_t)n * g.P * g.C + (first + (uint32_t)k * step));
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int n = blockIdx.x * teams + t.first / t.size, buf = 0;
  grid_dependency_wait();
  if (n < g.N) fetch(n, 0);
  float gamma[8], beta[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { gamma[i] = p.gamma[whole.channel(i)]; beta[i] = p.beta[whole.channel(i)]; }
  for (; n < g.N; n += stride, buf ^= 1) {
    if (n < g.N - stride) fetch(n + stride, buf ^ 1);
    else asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    const int at0 = buf * g.iters;
    F8 v;
    if constexpr (sizeof(T) == 2) {
      // Sums of values.  Those of equal 16-bit values are exact (a group has at most 48 * 1024 here, plan_teams), so with a quotient
      // rounded once the mean of a group without spread is its value.
#pragma unroll
      for (int j = 0; j < 4; ++j) v.p[j] = 0;
      for (int k = 0; k < mine; ++k) {
        const F8 x = raw8_to_f8(slots.get(at0 + k));
#pragma unroll
        for (int j = 0; j < 4; ++j) v.p[j] = add2(v.p[j], x.p[j]);
      }
      team_put(red, g, at, v);
      t.sync();
      team_group_sums(g, t, red, [&](int s, float a) { mom[s].x = __fdiv_rn(a, m); });
    } else {
      // Means of a thread's values, from sums of their differences from its first pixel; then of the group's, alike.
      float* const d = team_at(red, g, at);
      F8 x{}, first;
      if (mine > 0) x = raw8_to_f8(slots.get(at0));
      if (cut) {
#pragma unroll
        for (int j = 0; j < 4; ++j) { first.p[j] = mul2(x.p[j], pair(-1.f)); v.p[j] = 0; }
      } else {
        const f32x2 f = pair(-halves(x.p[0]).x);
#pragma unroll
        for (int j = 0; j < 4; ++j) { first.p[j] = f; v.p[j] = add2(x.p[j], f); }
      }
      for (int k = 1; k < mine; ++k) {
        x = raw8_to_f8(slots.get(at0 + k));
#pragma unroll
        for (int j = 0; j < 4; ++j) v.p[j] = add2(v.p[j], add2(x.p[j], first.p[j]));
      }
      if (cut) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v.p[j] = fma2(v.p[j], pair(over), mul2(first.p[j], pair(-1.f)));
        if (at.active) {
          reinterpret_cast<ulonglong2*>(d)[0] = make_ulonglong2(v.p[0], v.p[1]);
          reinterpret_cast<ulonglong2*>(d)[1] = make_ulonglong2(v.p[2], v.p[3]);
        }
      } else if (at.active) {
        const float2 a = halves(add2(add2(v.p[0], v.p[1]), add2(v.p[2], v.p[3])));
        *d = fmaf(a.x + a.y, over, -halves(first.p[0]).x);
      }
      t.sync();
      team_group_means(g, t, red, cut ? g.inv_m : 8.f * g.inv_m, [&](int s, float mu) { mom[s].x = mu; });
    }
    t.sync();
    F8 less;
    {
      float mu[8];
      team_values(g, at, [&](int s) { return mom[s].x; }, mu);
#pragma unroll
      for (int j = 0; j < 4; ++j) { less.p[j] = pair(-mu[2 * j], -mu[2 * j + 1]); v.p[j] = 0; }
    }
    for (int k = 0; k < mine; ++k) {
      const F8 x = raw8_to_f8(slots.get(at0 + k));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 d = add2(x.p[j], less.p[j]);
        v.p[j] = fma2(d, d, v.p[j]);
      }
    }
    team_put(red, g, at, v);
    t.sync();
    team_group_sums(g, t, red, [&](int s, float a) {
      const float rstd = 1.f / sqrtf(fmaf(a, g.inv_m, p.eps));
      mom[s].y = rstd;
      p.stats[(size_t)n * g.G + g_first + s] = mom[s].x;
      p.stats[(size_t)(g.N + n) * g.G + g_first + s] = rstd;
    });
    t.sync();
    Affine affine;
    float rstd[8];
    team_values(g, at, [&](int s) { return mom[s].y; }, rstd);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 m = halves(less.p[j]);
      affine.set(j, make_float2(-m.x, -m.y), make_float2(gamma[2 * j] * rstd[2 * j], gamma[2 * j + 1] * rstd[2 * j + 1]), make_float2(beta[2 * j], beta[2 * j + 1]));
    }
    const Share sh(g, at, n, 0);
    const Emitter<T, W, ACT, EXTRA> out(p, whole, sh);
    Raw8<T> next_res{};
    if constexpr (EXTRA >= WITH_RES_GATE)
      if (out.res && mine > 0) next_res = raw8_load<T, W>(out.res + out.first, at.left);
    for (int k = 0; k < (EXTRA == WITH_CODES ? sh.turns : mine); ++k) {
      const Raw8<T> xs[1] = {slots.get(at0 + min(k, g.iters - 1))}, rs[1] = {next_res};
      if constexpr (EXTRA >= WITH_RES_GATE)
        if (out.res && k + 1 < mine) next_res = raw8_load<T, W>(out.res + (out.first + (uint32_t)(k + 1) * step), at.left);
      out.template turn<false>(k, mine, false, affine, xs, rs);
    }
  }
}

// Streamed, first pass: moments of each group (with tiles > 1: of each channel) over a CTA's pixels.
template <typename T, int W>
__global__ void __launch_bounds__(kThreads, kForwardPerSm) moments_kernel(const __grid_constant__ Forward<T> p) {
  constexpr int kBatch = batch_of<T>(), kRing = ring_of<T>();
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  float* red = reinterpret_cast<float*>(smem + kRing * Slots<T>::Q * kThreads);   // [4096]
  float* common = red + 2 * kThreads * 8;                                      // [2048]
  float2* chan = reinterpret_cast<float2*>(common + kThreads * 8);             // [8 * cols]
  const int part = blockIdx.y, n = blockIdx.x;
  Place at(g, blockIdx.z);
  at.active = at.active && at.left > 0;
  const Share sh(g, at, n, part);
  // The next kernel may start once every CTA is past the wait: what this kernel's inputs come from is complete then, so the
  // next one copies from them (and from nothing that this kernel writes) before its own wait.
  grid_dependency_wait();
  grid_dependency_release();
  const T* const src = p.x + sh.row0 * g.C;
  uint32_t next = (uint32_t)at.r * g.C + at.c0;
  const uint32_t step = (uint32_t)g.rp * g.C;
  const Slots<T> ring(smem);
  Moments m;
  Raw8<T> first{};
  if (sh.mine > 0) first = raw8_load<T, W>(src + next, at.left);
  auto issue = [&](int slot) {
    ring.template fetch<W>(slot, src + next, at.left);
    next += step;
  };
  Stream<kBatch>::start(sh.mine, issue);
  m.start(raw8_to_f8(first));
  int close_at = kRing;
  Stream<kBatch>::run(sh.mine, sh.mine, issue, [&](int k, int slot, auto full) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (full.value || k + u < sh.mine) m.add(raw8_to_f8(ring.get(slot + u)));
  }, [&](int n) {
    if (n == close_at) { m.close(n); close_at = Moments::after(n); }
  });
  const int c_first = blockIdx.z * kMaxCols * 8, sets = min(g.cols * 8, g.C - c_first);
  cta_moments(g, at, m, sh.mine, sh.count, sets, red, common, chan);
  if (g.tiles == 1) {
    float* out = p.partial + ((size_t)n * g.parts + part) * 2 * g.G;
    group_moments(g, sh.count, chan, [&](int s, float mu, float q) { out[s] = mu; out[g.G + s] = q; });
  } else {
    float* out = p.partial + ((size_t)n * g.parts + part) * 2 * g.C + c_first;
    for (int c = threadIdx.x; c < sets; c += kThreads) { out[c] = chan[c].x; out[g.C + c] = chan[c].y; }
  }
}

// Streamed, between the passes where an image has many rows: the statistics of every gridDim.x-th group from blockIdx.x on, from the
// moments of its channels (tiles > 1) or its own in every row, in fp64.
template <typename T>
__global__ void __launch_bounds__(1024) combine_kernel(const __grid_constant__ Forward<T> p) {
  __shared__ double part[32];
  __shared__ double total;
  const Geom& g = p.g;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int width = g.tiles == 1 ? g.G : g.C, size = g.tiles == 1 ? 1 : g.Cg;      // of a row, of the group's share of it
  grid_dependency_wait();
  grid_dependency_release();
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
  const double values = (double)g.P * size;
  const double per = g.tiles == 1 ? (double)g.Cg : 1.0;                            // values behind a pixel of a row's entry
  for (size_t item = blockIdx.x; item < (size_t)g.N * g.G; item += gridDim.x) {
    const int n = (int)(item / g.G), s = (int)(item - (size_t)n * g.G);
    const float* src = p.partial + (size_t)n * g.parts * 2 * width + (size_t)s * size;
    auto each = [&](auto take) {
      const int step = blockDim.x / size, over = blockDim.x - step * size;
      int j = threadIdx.x / size, c = threadIdx.x - j * size;
      while (j < g.parts) {
        const float* row = src + (size_t)j * 2 * width + c;
        take((double)min(g.pix, g.P - j * g.pix), (double)row[0], row + width);
        j += step; c += over;
        if (c >= size) { c -= size; ++j; }
      }
    };
    double a = 0.0;
    each([&](double cnt, double mu, const float*) { a += cnt * mu; });
    const double mean = sum(a) / values;
    a = 0.0;
    each([&](double cnt, double mu, const float* m2) { a += (double)*m2 + cnt * per * (mu - mean) * (mu - mean); });
    const double var = sum(a) / ((double)g.P * g.Cg);
    if (threadIdx.x == 0) {
      p.stats[(size_t)n * g.G + s] = (float)mean;
      p.stats[(size_t)(g.N + n) * g.G + s] = (float)(1.0 / sqrt(var + (double)p.eps));
    }
  }
}

// Streamed, second pass: y from x and the statistics, which every CTA of an image forms from the rows of sums itself (the same
// bits everywhere; its first CTA writes them out) unless combine_kernel has.
template <typename T, int W, int ACT, int EXTRA>
__global__ void __launch_bounds__(kThreads, kForwardPerSm) apply_kernel(const __grid_constant__ Forward<T> p) {
  constexpr int kBatch = batch_of<T>(), kRing = ring_of<T>();
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  const Slots<T> ring(smem), res_ring(smem + kRing * Slots<T>::Q * kThreads);
  float2* mom = reinterpret_cast<float2*>(smem + (EXTRA >= WITH_RES_GATE && p.res ? 2 : 1) * kRing * Slots<T>::Q * kThreads);    // [G], unless combined
  const int part = blockIdx.y, n = blockIdx.x;
  Place at(g, blockIdx.z);
  at.active = at.active && at.left > 0;
  if (at.left <= 0) { at.c0 = 0; at.left = 1; }
  const Share sh(g, at, n, part);
  const Emitter<T, W, ACT, EXTRA> out(p, at, sh);
  const T* const x = p.x + sh.row0 * g.C;
  uint32_t next = out.first + (uint32_t)max(sh.mine - 1, 0) * out.step;
  auto issue = [&](int slot) {
    ring.template fetch<W>(slot, x + next, at.left);
    if constexpr (EXTRA >= WITH_RES_GATE)
      if (out.res) res_ring.template fetch<W>(slot, out.res + next, at.left);
    next -= out.step;
  };
  float gamma[8], beta[8];
  if constexpr (kEarly<T, W>) Stream<kBatch>::start(sh.mine, issue);      // see grid_dependency_release in moments_kernel
  grid_dependency_wait();
  grid_dependency_release();
  if constexpr (!kEarly<T, W>) Stream<kBatch>::start(sh.mine, issue);
#pragma unroll
  for (int i = 0; i < 8; ++i) { gamma[i] = p.gamma[at.channel(i)]; beta[i] = p.beta[at.channel(i)]; }
  if (!p.combined) {
    const float* rows = p.partial + (size_t)n * g.parts * 2 * g.G;
    image_moments(g, g.parts, p.eps, [&](int j) { return rows + (size_t)j * 2 * g.G; }, [&](int s, float mu, float rstd) {
      mom[s] = make_float2(mu, rstd);
      if (part == 0) {
        p.stats[(size_t)n * g.G + s] = mu;
        p.stats[(size_t)(g.N + n) * g.G + s] = rstd;
      }
    });
    __syncthreads();
  }
  Affine affine;
  if (p.combined)
    load_affine(p, at, gamma, beta, [&](int s) { return make_float2(p.stats[(size_t)n * g.G + s], p.stats[(size_t)(g.N + n) * g.G + s]); }, affine);
  else
    load_affine(p, at, gamma, beta, [&](int s) { return mom[s]; }, affine);
  auto turn = [&](int k, int slot, auto full) {
    Raw8<T> xs[kBatch], rs[EXTRA >= WITH_RES_GATE ? kBatch : 1];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (EXTRA == WITH_CODES || full.value || k + u < sh.mine) xs[u] = ring.get(slot + u);
      if constexpr (EXTRA >= WITH_RES_GATE)
        if (out.res && (full.value || k + u < sh.mine)) rs[u] = res_ring.get(slot + u);
    }
    out.template turn<full.value>(k, sh.mine, true, affine, xs, rs);
  };
  if constexpr (EXTRA == WITH_CODES) Stream<kBatch>::run_rolled(sh.turns, sh.mine, issue, turn);
  else Stream<kBatch>::run(sh.mine, sh.mine, issue, turn);
}

// ---- backward -----------------------------------------------------------------------------------------------
enum { SLOPE_ONE = 0, SLOPE_MASK = 1, SLOPE_BITS = 2, SLOPE_SILU = 3 };      // act' from nothing, from y, from y's bits, from z
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
  float* partial;             // [N][parts][2][C]: A, B of each CTA
  float* totals;              // [N][2][C]: A, B of each image, or null if the second pass adds up the rows itself
  float* dgamma;
  float* dbeta;
  int extra;                  // of the second pass: ceil(2C / 32 / parts)
  int slope;
};

// The operands of one column of 8 channels at a pixel, raw.
template <typename T, bool CK> struct Held {
  Raw8<T> dy;
  Raw8<T> x;                  // the column of x, or
  uint2 codes;                // its codes and
  uint32_t scale;             // their scale byte
  Raw8<T> mask;               // SLOPE_MASK
  uint32_t open;              // SLOPE_BITS
};
// Where a CTA's pixels start in the tensors (the same for all threads), where a thread's columns do, and how far apart its
// pixels are.
template <typename T> struct Columns {
  const T *dy, *x, *mask;
  const int8_t* codes;
  const uint8_t *scales, *gate;
  uint32_t first, step, gate_first, gate_step, scale_first, scale_step;
  __device__ __forceinline__ Columns(const Backward<T>& p, const Place& at, const Share& sh) {
    const Geom& g = p.g;
    const int all_cols = (g.C + 7) >> 3, per_row = (g.C + kCkptBlock - 1) / kCkptBlock;
    const size_t off = sh.row0 * g.C;
    dy = p.dy + off; x = p.x + off; mask = p.mask + off; codes = p.codes + off;
    scales = p.scales + sh.row0 * per_row;
    gate = p.gate + sh.row0 * all_cols;
    first = (uint32_t)at.r * g.C + at.c0;
    scale_first = (uint32_t)at.r * per_row + at.c0 / kCkptBlock;
    gate_first = (uint32_t)at.r * all_cols + (at.c0 >> 3);
    step = (uint32_t)g.rp * g.C; gate_step = (uint32_t)g.rp * all_cols; scale_step = (uint32_t)g.rp * per_row;
  }
};

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

// dy where it passes ReLU.
template <typename T, bool CK> __device__ __forceinline__ Raw8<T> passed(const Held<T, CK>& h, int slope) {
  if (slope == SLOPE_MASK) return opened(h.dy, positive_bits(h.mask));
  if (slope == SLOPE_BITS) return opened(h.dy, h.open);
  return h.dy;
}
// x - mean, and dz from the dy that passes.
template <typename T, bool CK>
__device__ __forceinline__ void operands(const Raw8<T>& dy, const Held<T, CK>& h, int slope, const Channels& ch, F8& dz, F8& d) {
  dz = raw8_to_f8(dy);
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
  if (slope == SLOPE_SILU) {
#pragma unroll
    for (int j = 0; j < 4; ++j) dz.p[j] = mul2(dz.p[j], silu_slope<T>(fma2(d.p[j], ch.scale[j], ch.shift[j])));
  }
}

// dx of one vector: k1 = -rstd*S1/m, k2 = -rstd^2*S2/m.
template <typename T, bool CK>
__device__ __forceinline__ Raw8<T> dx_of(const Raw8<T>& dy, const Held<T, CK>& h, int slope, const Channels& ch, const f32x2 (&k1)[4],
                                         const f32x2 (&k2)[4], const Raw8<T>* res) {
  F8 dz, d;
  operands<T, CK>(dy, h, slope, ch, dz, d);
#pragma unroll
  for (int j = 0; j < 4; ++j) dz.p[j] = fma2(ch.scale[j], dz.p[j], fma2(d.p[j], k2[j], k1[j]));
  if (res) {
    const F8 r = raw8_to_f8(*res);
#pragma unroll
    for (int j = 0; j < 4; ++j) dz.p[j] = add2(dz.p[j], r.p[j]);
  }
  return f8_to_raw8<T>(dz);
}

// The operands of a pass: rings of dy, x (or its codes), the mask and res, as far as a pass has them; the bytes
// (scales, gate bits) come through registers, as many turns ahead.
template <typename T, int W, bool CK> struct Feed {
  static constexpr int kBatch = batch_of<T>(), kRing = ring_of<T>();
  const Columns<T> from;
  const Slots<T> dys, xs, masks, ress;
  uint2* codes;
  const T* res;
  int left, slope, n;
  bool reverse;
  uint32_t scale[kAhead + 1][kBatch], open[kAhead + 1][kBatch];     // by turn, as the ring
  uint32_t next, next_scale, next_gate, step, scale_step, gate_step;       // offsets of the next vector and bytes to be fetched
  static constexpr int kVec = kRing * Slots<T>::Q * kThreads;        // 16-byte words of a ring
  // words of shared memory of a pass, in 16 bytes
  static __host__ __device__ __forceinline__ int words(bool mask, bool res) {
    return kVec + (CK ? kRing * kThreads / 2 : kVec) + (mask ? kVec : 0) + (res ? kVec : 0);
  }
  __device__ __forceinline__ Feed(const Backward<T>& p, const Place& at, const Share& sh, int slope_, const T* res_, bool reverse_, uint4* smem)
      : from(p, at, sh), dys(smem), xs(smem + kVec), masks(smem + kVec + (CK ? kRing * kThreads / 2 : kVec)),
        ress(smem + words(slope_ == SLOPE_MASK, false)), codes(reinterpret_cast<uint2*>(smem + kVec) + threadIdx.x),
        res(res_ ? res_ + sh.row0 * p.g.C : nullptr), left(at.left), slope(slope_), n(sh.mine), reverse(reverse_) {
    step = reverse ? 0u - from.step : from.step;
    scale_step = reverse ? 0u - from.scale_step : from.scale_step;
    gate_step = reverse ? 0u - from.gate_step : from.gate_step;
    const uint32_t k = reverse && n > 0 ? (uint32_t)(n - 1) : 0u;
    next = from.first + k * from.step; next_scale = from.scale_first + k * from.scale_step; next_gate = from.gate_first + k * from.gate_step;
  }
  __device__ __forceinline__ void start_bytes() {
#pragma unroll
    for (int t = 0; t < kAhead; ++t) bytes<false>(t * kBatch, t * kBatch);
  }
  // The bytes of the turn that begins with vector k, to be used kAhead turns later.
  template <bool FULL> __device__ __forceinline__ void bytes(int k, int slot) {
    const int to = slot / kBatch % (kAhead + 1);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (FULL || k + u < n) {
        if constexpr (CK) { scale[to][u] = from.scales[next_scale]; next_scale += scale_step; }
        if (slope == SLOPE_BITS) { open[to][u] = from.gate[next_gate]; next_gate += gate_step; }
      }
  }
  __device__ __forceinline__ void issue(int s) {
    vectors(s, next);
    if constexpr (CK) bytes_of_x(s, next);
    next += step;
  }
  __device__ __forceinline__ void vectors(int s, uint32_t o) {
    dys.template fetch<W>(s, from.dy + o, left);
    if constexpr (!CK) xs.template fetch<W>(s, from.x + o, left);
    if (slope == SLOPE_MASK) masks.template fetch<W>(s, from.mask + o, left);
    if (res) ress.template fetch<W>(s, res + o, left);
  }
  __device__ __forceinline__ void bytes_of_x(int s, uint32_t o) {           // 8 of them: there is no copy of that size past L1
    if constexpr (W == kWhole) copy8_async(codes + s * kThreads, from.codes + o); else codes[s * kThreads] = load_codes<kCodeWidth<T, W>>(from.codes + o, left);
  }
  // Stream::start in two parts: what goes past L1, and what does not (with the first group all of the former).
  __device__ __forceinline__ void start_past_l1() {
#pragma unroll
    for (int k = 0; k < kBatch * kAhead; ++k)
      if (k < n) vectors(k, next + (uint32_t)k * step);
  }
  __device__ __forceinline__ void start_rest() {
#pragma unroll
    for (int k = 0; k < kBatch * kAhead; ++k) {
      if constexpr (CK)
        if (k < n) bytes_of_x(k, next + (uint32_t)k * step);
      if (k % kBatch == kBatch - 1) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    next += (uint32_t)(kBatch * kAhead) * step;
  }
  __device__ __forceinline__ Held<T, CK> get(int slot, int u) const {
    Held<T, CK> h;
    const int s = slot + u;
    h.dy = dys.get(s);
    if constexpr (CK) { h.codes = codes[s * kThreads]; h.scale = scale[slot / kBatch][u]; } else { h.x = xs.get(s); }
    if (slope == SLOPE_MASK) h.mask = masks.get(s);
    if (slope == SLOPE_BITS) h.open = open[slot / kBatch][u];
    return h;
  }
};

// The constants of a thread's channels from the saved statistics.
template <typename T>
__device__ __forceinline__ void load_channels(const Backward<T>& p, const Place& at, int n, int slope, Channels& ch, float (&rstd)[8]) {
  const Geom& g = p.g;
  float mean[8], scale[8], shift[8];
  each_channel(g, at, [&](int i, int c, int s) {
    mean[i] = p.stats[(size_t)n * g.G + s];
    rstd[i] = p.stats[(size_t)(g.N + n) * g.G + s];
    scale[i] = p.gamma[c] * rstd[i];
    shift[i] = slope == SLOPE_SILU ? p.beta[c] : 0.f;
  });
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    ch.less[j] = pair(-mean[2 * j], -mean[2 * j + 1]);
    ch.scale[j] = pair(scale[2 * j], scale[2 * j + 1]);
    ch.shift[j] = pair(shift[2 * j], shift[2 * j + 1]);
  }
}
// k1, k2 of a thread's channels from those of the groups, the first of which is `first`.
__device__ __forceinline__ void load_coefficients(const Geom& g, const Place& at, const float* c1, const float* c2, int first, f32x2 (&k1)[4], f32x2 (&k2)[4]) {
  float a[8], b[8];
  each_channel(g, at, [&](int i, int, int s) { a[i] = -c1[s - first]; b[i] = -c2[s - first]; });
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

// What chains of kChain vectors have come to, so that no chain is longer (one of 4096 equal gradients was off by 6e-5 of its sum): in
// registers, or, in the forms that have none left, in 16 floats of the thread's own in shared memory, which a call asks for where its
// threads have that many vectors.  (All forms there: fp32 with a mask 112 -> 137 us, 128 images of 32x32x160, for want of L1.)
template <bool REGISTERS> struct Closed;
template <> struct Closed<true> {
  Sums all;
  __device__ __forceinline__ Closed(uint4*) {}
  __device__ __forceinline__ void take(Sums& s, bool) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      all.a.p[j] = add2(all.a.p[j], s.a.p[j]); all.b.p[j] = add2(all.b.p[j], s.b.p[j]);
      s.a.p[j] = s.b.p[j] = 0;
    }
  }
  __device__ __forceinline__ void give(Sums& s) { take(s, false); s = all; }
};
template <> struct Closed<false> {
  ulonglong2* own;
  __device__ __forceinline__ Closed(uint4* smem) : own(reinterpret_cast<ulonglong2*>(smem) + threadIdx.x) {}
  __device__ __forceinline__ void take(Sums& s, bool first) {
    if (!first) give(s);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      own[j * kThreads] = make_ulonglong2(s.a.p[2 * j], s.a.p[2 * j + 1]);
      own[(2 + j) * kThreads] = make_ulonglong2(s.b.p[2 * j], s.b.p[2 * j + 1]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s.a.p[j] = s.b.p[j] = 0;
  }
  __device__ __forceinline__ void give(Sums& s) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const ulonglong2 a = own[j * kThreads], b = own[(2 + j) * kThreads];
      s.a.p[2 * j] = add2(s.a.p[2 * j], a.x); s.a.p[2 * j + 1] = add2(s.a.p[2 * j + 1], a.y);
      s.b.p[2 * j] = add2(s.b.p[2 * j], b.x); s.b.p[2 * j + 1] = add2(s.b.p[2 * j + 1], b.y);
    }
  }
};
template <typename T> constexpr int kClosedFrom = kChain + batch_of<T>() * kAhead;       // vectors from which a chain is closed, see Stream::run
constexpr size_t kClosedBytes = (size_t)kThreads * 16 * sizeof(float);
template <int SLOPE> constexpr bool kClosedInRegisters = SLOPE == SLOPE_ONE || SLOPE == SLOPE_MASK;

// First pass: A and B of each channel over a CTA's pixels.
template <typename T, int W, bool CK, int SLOPE>
__global__ void __launch_bounds__(kThreads, kBackwardPerSm) backward_sums_kernel(const __grid_constant__ Backward<T> p) {
  constexpr int kBatch = batch_of<T>(), kRing = ring_of<T>();
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  const int slope = SLOPE < 0 ? p.slope : SLOPE;
  const int part = blockIdx.y, n = blockIdx.x;
  Place at(g, blockIdx.z);
  at.active = at.active && at.left > 0;
  if (at.left <= 0) { at.c0 = blockIdx.z * kMaxCols * 8; at.left = 1; }
  const Share sh(g, at, n, part);
  grid_dependency_wait();
  grid_dependency_release();
  Feed<T, W, CK> feed(p, at, sh, slope, nullptr, false, smem);
  feed.start_bytes();
  Channels ch;
  float rstd[8];
  Sums sums;
  Closed<kClosedInRegisters<SLOPE>> closed(smem + Feed<T, W, CK>::words(slope == SLOPE_MASK, false));
  auto issue = [&](int slot) { feed.issue(slot); };
  Stream<kBatch>::start(sh.mine, issue);
  load_channels(p, at, n, slope, ch, rstd);
  Stream<kBatch>::run(sh.mine, sh.mine, issue, [&](int k, int slot, auto full) {
    feed.template bytes<full.value>(k + kAhead * kBatch, slot + kAhead * kBatch);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (full.value || k + u < sh.mine) {
        const Held<T, CK> h = feed.get(slot, u);
        F8 dz, d;
        operands<T, CK>(passed<T, CK>(h, slope), h, slope, ch, dz, d);
        sums.add(dz, d);
      }
  }, [&](int k) {
    if ((k & (kChain - 1)) == 0) closed.take(sums, k == kChain);
  });
  if (sh.mine >= kClosedFrom<T>) closed.give(sums);
  __syncthreads();                    // the sums go where the rings were
  float* red = reinterpret_cast<float*>(smem);
  sums.put(red, g, at, rstd);
  __syncthreads();
  const int c_first = blockIdx.z * kMaxCols * 8, sets = min(g.cols * 8, g.C - c_first);
  float* out = p.partial + ((size_t)n * g.parts + part) * 2 * g.C + c_first;
  channel_sums(red, g, sets, g.lanes_c, [&](int c, float a, float b) { out[c] = a; out[g.C + c] = b; });
}

// Sums of `rows` rows of `width` floats, 32 of the width from `first` on: done(i, sum).  The CTA's warps take every `warps`-th
// row and add in fp64; fin: [warps][33].
template <typename Done>
__device__ __forceinline__ void add_rows(const float* __restrict__ in, int rows, int width, int first, double (*fin)[33], Done done) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int i = first + lane;
  double t = 0.0;
  if (i < width)
#pragma unroll 8
    for (int r = warp; r < rows; r += warps) t += (double)in[(size_t)r * width + i];
  fin[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && i < width) {
    for (int w = 1; w < warps; ++w) t += fin[w][lane];
    done(i, (float)t);
  }
  __syncthreads();
}
// Between the passes where an image has many rows: totals[n][i] = the sum of image n's rows of sums, 32 of `width` at a time, every
// gridDim.x-th of them from blockIdx.x on.
__global__ void __launch_bounds__(1024) totals_kernel(const float* __restrict__ partial, int images, int rows, int width, float* __restrict__ totals) {
  __shared__ double fin[32][33];
  const int blocks = (width + 31) / 32;
  grid_dependency_wait();
  grid_dependency_release();
  for (size_t item = blockIdx.x; item < (size_t)images * blocks; item += gridDim.x) {
    const int n = (int)(item / blocks);
    add_rows(partial + (size_t)n * rows * width, rows, width, (int)(item - (size_t)n * blocks) * 32, fin,
             [&](int i, float v) { totals[(size_t)n * width + i] = v; });
  }
}

// The team form of the backward pass: both passes over an image from shared memory.  A team adds its images' A and B up in registers (at
// most kTeamImages of them, so that sums stay short), a CTA leaves one row of its teams' in scratch for parameters_kernel.  What ReLU
// passes of dy replaces it in shared memory, so that the mask or its bits are read once.  us, streamed / this form, 16-bit storage, no
// activation: 4096x2x2x64 62 / 9, 4096x4x4x256 74 / 28, 2000x7x7x128 39 / 35, 20000x1x512 365 / 37; from codes and bits 75 / 10, 90 / 39,
// 48 / 42, 437 / 44.  Bound by issue slots, at one pixel per image by what an image costs beside its values.
constexpr int kTeamImages = 128;
template <typename T, int W, bool CK, int SLOPE>
__global__ void __launch_bounds__(kThreads, kBackwardPerSm) backward_teams_kernel(const __grid_constant__ Backward<T> p) {
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  const int slope = SLOPE < 0 ? p.slope : SLOPE;
  const Team t(g);
  const Place at(g, 0, (uint32_t)t.tid);                                     // in the slice, and
  Place whole = at;                                                          // in the image
  whole.c0 += blockIdx.y * g.slice;
  const int g_first = blockIdx.y * g.Gs;
  const int vectors = g.buffers * g.iters * Slots<T>::Q * kThreads;          // 16-byte words of an operand
  const Slots<T> dys(smem), xs(smem + vectors);
  uint2* const codes = reinterpret_cast<uint2*>(smem + vectors) + threadIdx.x;
  float* const all = reinterpret_cast<float*>(smem + 2 * vectors);           // [2][kThreads * 8]
  float* const red = all + t.first * 8;
  float* const own = all + 2 * kThreads * 8 + (t.first / t.size) * 6 * g.Gs; // [2][2][Gs]: mean, rstd of two images
  float* const coef = own + 4 * g.Gs;                                        // [2][Gs]
  const int teams = kThreads / t.size, stride = gridDim.x * teams;
  const uint32_t first = (uint32_t)at.r * g.C + whole.c0, step = (uint32_t)g.rp * g.C;
  const int mine = Share(g, at, 0, 0).mine;
  auto fetch = [&](int n, int buf) {
    const size_t off = (size_t)n * g.P * g.C + first;
    for (int k = 0; k < mine; ++k) {
      const size_t o = off + (uint32_t)k * step;
      const int slot = buf * g.iters + k;
      dys.template fetch<W>(slot, p.dy + o, at.left);
      if constexpr (CK) {
        if constexpr (W == kWhole) copy8_async(codes + slot * kThreads, p.codes + o);
        else codes[slot * kThreads] = load_codes<kCodeWidth<T, W>>(p.codes + o, at.left);
      } else {
        xs.template fetch<W>(slot, p.x + o, at.left);
      }
      if (slope == SLOPE_MASK) prefetch_l2(p.mask + o);
      if (p.res) prefetch_l2(p.res + o);
    }
    for (int s = t.tid; s < g.Gs; s += t.size) {
      copy_piece_async<4>(own + buf * 2 * g.Gs + s, p.stats + (size_t)n * g.G + g_first + s, true);
      copy_piece_async<4>(own + (buf * 2 + 1) * g.Gs + s, p.stats + (size_t)(g.N + n) * g.G + g_first + s, true);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int n = blockIdx.x * teams + t.first / t.size, buf = 0;
  grid_dependency_wait();
  grid_dependency_release();
  if (n < g.N) fetch(n, 0);
  float gamma[8], beta[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    gamma[i] = p.gamma[whole.channel(i)];
    beta[i] = slope == SLOPE_SILU ? p.beta[whole.channel(i)] : 0.f;
  }
  float A[8], B[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) A[i] = B[i] = 0.f;
  for (; n < g.N; n += stride, buf ^= 1) {
    if (n < g.N - stride) fetch(n + stride, buf ^ 1);
    else asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    t.sync();                         // the statistics are the team's
    const int at0 = buf * g.iters;
    const float *means = own + buf * 2 * g.Gs, *rstds = means + g.Gs;
    Channels ch;
    float rstd[8];
    {
      float mean[8];
      team_values(g, at, [&](int s) { return means[s]; }, mean);
      team_values(g, at, [&](int s) { return rstds[s]; }, rstd);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ch.less[j] = pair(-mean[2 * j], -mean[2 * j + 1]);
        ch.scale[j] = pair(gamma[2 * j] * rstd[2 * j], gamma[2 * j + 1] * rstd[2 * j + 1]);
        ch.shift[j] = pair(beta[2 * j], beta[2 * j + 1]);
      }
    }
    const Share sh(g, at, n, 0);
    const Columns<T> from(p, whole, sh);
    auto held = [&](int k) {
      Held<T, CK> h;
      h.dy = dys.get(at0 + k);
      if constexpr (CK) {
        h.codes = codes[(at0 + k) * kThreads];
        h.scale = from.scales[from.scale_first + (uint32_t)k * from.scale_step];
      } else {
        h.x = xs.get(at0 + k);
      }
      return h;
    };
    Sums sums;
    for (int k = 0; k < mine; ++k) {
      Held<T, CK> h = held(k);
      if (slope == SLOPE_MASK) h.mask = raw8_load<T, W>(from.mask + (from.first + (uint32_t)k * from.step), at.left);
      if (slope == SLOPE_BITS) h.open = from.gate[from.gate_first + (uint32_t)k * from.gate_step];
      const Raw8<T> dy = passed<T, CK>(h, slope);
      if (slope == SLOPE_MASK || slope == SLOPE_BITS) dys.put(at0 + k, dy);
      F8 dz, d;
      operands<T, CK>(dy, h, slope, ch, dz, d);
      sums.add(dz, d);
    }
    F8 w1, w2;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a = halves(sums.a.p[j]), b = halves(sums.b.p[j]);
      const float a0 = a.x * rstd[2 * j], a1 = a.y * rstd[2 * j + 1];
      A[2 * j] += a0; A[2 * j + 1] += a1;
      B[2 * j] += b.x; B[2 * j + 1] += b.y;
      w1.p[j] = pair(gamma[2 * j] * b.x, gamma[2 * j + 1] * b.y);
      w2.p[j] = pair(gamma[2 * j] * a0, gamma[2 * j + 1] * a1);
    }
    team_put(red, g, at, w1);
    team_put(red + kThreads * 8, g, at, w2);
    t.sync();
    team_group_sums(g, t, red, [&](int s, float v) { coef[s] = -(rstds[s] * v * g.inv_m); });
    team_group_sums(g, t, red + kThreads * 8, [&](int s, float v) { coef[g.Gs + s] = -(rstds[s] * rstds[s] * v * g.inv_m); });
    t.sync();
    f32x2 k1[4], k2[4];
    {
      float c1[8], c2[8];
      team_values(g, at, [&](int s) { return coef[s]; }, c1);
      team_values(g, at, [&](int s) { return coef[g.Gs + s]; }, c2);
#pragma unroll
      for (int j = 0; j < 4; ++j) { k1[j] = pair(c1[2 * j], c1[2 * j + 1]); k2[j] = pair(c2[2 * j], c2[2 * j + 1]); }
    }
    T* const dx = p.dx + sh.row0 * g.C;
    const T* const res = p.res ? p.res + sh.row0 * g.C : nullptr;
    Raw8<T> next{};
    if (res && mine > 0) next = raw8_load<T, W>(res + first, at.left);
    for (int k = 0; k < mine; ++k) {
      const Raw8<T> r = next;
      if (res && k + 1 < mine) next = raw8_load<T, W>(res + (first + (uint32_t)(k + 1) * step), at.left);
      const Held<T, CK> h = held(k);
      raw8_put<T, W>(dx + (first + (uint32_t)k * step), at.left, dx_of<T, CK>(h.dy, h, slope, ch, k1, k2, res ? &r : nullptr));
    }
  }
  __syncthreads();
  put_sums(red, g, at, A);
  put_sums(red + kThreads * 8, g, at, B);
  __syncthreads();
  float* const out = p.partial + (size_t)blockIdx.x * 2 * g.C + blockIdx.y * g.slice;
  const int lanes = g.lanes_c, sub = threadIdx.x & (lanes - 1), rows = teams * g.rp;
  for (int c0 = 0; c0 < g.slice; c0 += kThreads / lanes) {
    const int c = c0 + threadIdx.x / lanes;
    float a = 0.f, b = 0.f;
    if (c < g.slice)
      for (int i = sub; i < rows; i += lanes) {
        const int team = i / g.rp;
        const float* v = all + (team * t.size + (i - team * g.rp) * g.cols) * 8 + c;
        a += v[0]; b += v[kThreads * 8];
      }
    a = lane_sum(a, lanes);
    b = lane_sum(b, lanes);
    if (c < g.slice && sub == 0) { out[c] = a; out[g.C + c] = b; }
  }
}
// dgamma and dbeta, 32 of them, from `rows` rows of sums.
__global__ void __launch_bounds__(1024) parameters_kernel(const float* __restrict__ partial, int rows, int C, float* __restrict__ dgamma,
                                                          float* __restrict__ dbeta) {
  __shared__ double fin[32][33];
  grid_dependency_wait();
  grid_dependency_release();
  add_rows(partial, rows, 2 * C, blockIdx.x * 32, fin, [&](int i, float v) { (i < C ? dgamma + i : dbeta + (i - C))[0] = v; });
}

// Second pass: dx.  Every CTA forms S1 and S2 of its tile's groups from the image's totals, or from its rows of sums.
// The first `extra` CTAs of a share add up the parameter gradients, 32 values each.
template <typename T, int W, bool CK, int SLOPE>
__global__ void __launch_bounds__(kThreads, kBackwardPerSm) backward_apply_kernel(const __grid_constant__ Backward<T> p) {
  constexpr int kBatch = batch_of<T>(), kRing = ring_of<T>();
  extern __shared__ uint4 smem[];
  const Geom& g = p.g;
  float* coef = reinterpret_cast<float*>(smem + Feed<T, W, CK>::words((SLOPE < 0 ? p.slope : SLOPE) == SLOPE_MASK, p.res != nullptr));   // [2][sets]
  const int slope = SLOPE < 0 ? p.slope : SLOPE;
  const int part = blockIdx.y, n = (int)blockIdx.x - p.extra;
  const int c_first = blockIdx.z * kMaxCols * 8;
  if (n < 0) {
    const int first = ((int)blockIdx.x * g.parts + part) * 32;
    grid_dependency_wait();
    grid_dependency_release();
    if (blockIdx.z == 0 && first < 2 * g.C)
      add_rows(p.partial, g.N * g.parts, 2 * g.C, first, reinterpret_cast<double(*)[33]>(smem),
               [&](int i, float v) { (i < g.C ? p.dgamma + i : p.dbeta + (i - g.C))[0] = v; });
    return;
  }
  Place at(g, blockIdx.z);
  at.active = at.active && at.left > 0;
  if (at.left <= 0) { at.c0 = c_first; at.left = 1; }
  const Share sh(g, at, n, part);
  const int c_last = min(g.C, c_first + g.cols * 8) - 1;
  const int g_first = c_first / g.Cg, sets = c_last / g.Cg - g_first + 1, c_base = g_first * g.Cg;
  Feed<T, W, CK> feed(p, at, sh, slope, p.res, true, smem);
  if constexpr (kEarly<T, W>) feed.start_past_l1();
  grid_dependency_wait();
  grid_dependency_release();
  auto issue = [&](int slot) { feed.issue(slot); };
  if constexpr (kEarly<T, W>) feed.start_rest(); else Stream<kBatch>::start(sh.mine, issue);
  feed.start_bytes();
  Channels ch;
  float rstd[8];
  load_channels(p, at, n, slope, ch, rstd);
  const int rows = p.totals ? 1 : g.parts;
  const float* src = p.totals ? p.totals + (size_t)n * 2 * g.C : p.partial + (size_t)n * g.parts * 2 * g.C;
  const float* rs = p.stats + (size_t)(g.N + n) * g.G + g_first;
  auto weighted = [&](int c) {
    float a = 0.f, b = 0.f;
#pragma unroll 4
    for (int j = 0; j < rows; ++j) { a += src[(size_t)j * 2 * g.C + c]; b += src[(size_t)j * 2 * g.C + g.C + c]; }
    const float w = p.gamma[c];
    return make_float2(w * b, w * a);
  };
  auto done = [&](int s, float s1, float s2) {
    coef[s] = rs[s] * s1 * g.inv_m;
    coef[sets + s] = rs[s] * rs[s] * s2 * g.inv_m;
  };
  if (g.tiles == 1) {
    float2* chan = reinterpret_cast<float2*>(coef + 2 * sets);                // [C]
    for (int c = threadIdx.x; c < g.C; c += kThreads) chan[c] = weighted(c);
    __syncthreads();
    group_sums(sets, g.Cg, g.lanes_g, [&](int c) { return chan[c]; }, done);
  } else if (rows == 1) {             // loads that do not wait for one another (4096x1x4096, one group: 505 us for 2576)
    group_sums(sets, g.Cg, g.lanes_g, [&](int c) {
      const float w = p.gamma[c_base + c];
      return make_float2(w * src[g.C + c_base + c], w * src[c_base + c]);
    }, done);
  } else {
    group_sums(sets, g.Cg, g.lanes_g, [&](int c) { return weighted(c_base + c); }, done);
  }
  __syncthreads();
  f32x2 k1[4], k2[4];
  load_coefficients(g, at, coef, coef + sets, g_first, k1, k2);
  uint32_t o = feed.from.first + (uint32_t)max(sh.mine - 1, 0) * feed.from.step;
  T* const dx = p.dx + sh.row0 * g.C;
  Stream<kBatch>::run(sh.mine, sh.mine, issue, [&](int k, int slot, auto full) {
    feed.template bytes<full.value>(k + kAhead * kBatch, slot + kAhead * kBatch);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (full.value || k + u < sh.mine) {
        const Held<T, CK> h = feed.get(slot, u);
        Raw8<T> r;
        if (feed.res) r = feed.ress.get(slot + u);
        raw8_put<T, W>(dx + o, at.left, dx_of<T, CK>(passed<T, CK>(h, slope), h, slope, ch, k1, k2, feed.res ? &r : nullptr));
        o += feed.step;
      }
  });
}

// ---- host side: plans ----------------------------------------------------------------------------------------
struct Plan {
  Geom g;
  bool resident;              // one launch and no scratch: a cluster per image, or (g.team) the team form
  size_t smem;                // dynamic shared memory of the resident kernels
  int ctas;                   // of the team form
  int64_t rows;               // of sums in scratch
};
inline int pow2_up_to(int64_t most, int cap) {
  int v = 1;
  while (2 * v <= cap && 2 * (int64_t)v <= most) v *= 2;
  return v;
}
constexpr size_t kSmemMost = 220 * 1024;        // of 227 KB that a CTA can have
constexpr size_t kSmemOfSm = 227 * 1024;

inline void split(Geom& g, int parts) {
  g.parts = parts;
  g.pix = g.P / parts + (g.P % parts != 0);
  g.iters = g.pix / g.rp + (g.pix % g.rp != 0);
  g.whole = g.pix / g.rp;
  const int last = g.P % g.pix;
  g.whole_last = last ? last / g.rp : g.whole;
}
// One wave of CTAs (`per_sm` on an SM), each with at least one batch of pixels in flight.  More waves of smaller shares cost
// their start and end each, about 2.5 us: 23.2, 28.3 and 32.9 us with one, two and three waves (forward, 128 images of 32x32x160).
inline Plan plan_streamed(int N, int P, int C, int G, int per_sm) {
  Plan pl{};
  Geom& g = pl.g;
  g.N = N; g.P = P; g.C = C; g.G = G; g.Cg = C / G;
  g.inv_m = (float)(1.0 / ((double)P * g.Cg));
  const int all_cols = C / 8 + (C % 8 != 0);
  g.cols = std::min(all_cols, kMaxCols);
  g.tiles = (all_cols + kMaxCols - 1) / kMaxCols;
  g.rp = kThreads / g.cols;
  g.col_mul = (65536 + g.cols - 1) / g.cols;              // exact for tid < 256: the excess is below 256 / 65536 <= 1 / cols
  g.cg_mul = g.Cg == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + g.Cg - 1) / g.Cg);      // exact for c * Cg < 2^32 (C <= 2^16)
  g.lanes_g = pow2_up_to(kThreads / std::min(G, kThreads), 32);
  g.lanes_c = pow2_up_to(kThreads / std::min(g.cols * 8, kThreads), 32);
  split(g, (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)per_sm * kSms / N, P / (4 * g.rp))));
  g.parts = P / g.pix + (P % g.pix != 0);         // none without pixels
  pl.rows = (int64_t)N * g.parts;
  return pl;
}
// The team form: the slices of an image (whole groups and blocks of 32 channels) and the size of a team that give the least of
// (rounds of images per team) * (pixels per thread + 4, the fixed part of a round, in pixels), the fewest slices and the largest team
// where some are alike; none where an image does not fit.  vec_bytes: of a thread's pixel in shared memory; shared, per_group: bytes of
// a CTA, of a team's group beside them.
// Slices are for rows wider than a CTA (us, streamed / sliced: 4096x1x4096 263 / 49, 512x4x4x4096 63 / 29) and, forward, for images that
// all run at once then (16x16x16x256 6.8 / 3.4, 64x7x7x512 7.1 / 4.5, 128x8x8x640 8.7 / 7.2; in rounds 512x8x8x640 30 / 28 and with codes
// 38 / 44; backward 512x16x16x64 16.5 / 20.3).
// Forward (`most` = 12): teams smaller than a CTA only where they leave no SM without one (37x28x28x30 on 19 SMs: 12 us for 8.4); with
// a CTA per image at most 12 pixels a thread, beyond which a cluster or the streamed form is as fast without codes and faster with
// them (128x16x16x160, 22 pixels: 7.5 / 8.2 and 13 / 10.5).
// Backward (`most` = 4, `fill`): with fewer CTAs than SMs the streamed form is faster (8x16x16x8 4.9 / 6.9 us), and where only one CTA
// fits an SM too (1024x8x8x160 from codes and bits 31.8 / 35, fp32 41.8 / 59); with a CTA per image, 8 pixels a thread 14.9 / 20.0 (400x32x32x16).
inline Plan plan_teams(int vec_bytes, bool fill, int per_sm, size_t shared, int per_group, int most, int N, int P, int C, int G) {
  Plan best{};
  int64_t least = INT64_MAX;
  for (int slices = 1; slices == 1 || (G % slices == 0 && C % (32 * slices) == 0); slices *= 2) {
    const int slice = C / slices, cols = slice / 8 + (slice % 8 != 0), Gs = G / slices;
    for (int team = kThreads; team >= 32 && team >= cols; team /= 2) {
      const int rp = team / cols, iters = P / rp + (P % rp != 0), teams = kThreads / team;
      const int64_t all = N / teams + (N % teams != 0);
      if ((fill || team < kThreads) && all * slices < kSms) continue;
      if (team == kThreads && iters > most) continue;
      if (iters > 48) break;        // no room
      const size_t own = shared + (size_t)per_group * teams * Gs, image = (size_t)vec_bytes * iters * kThreads;
      int64_t at_once = 0;          // CTAs of a slice
      int buffers = 0;
      for (; at_once < all && buffers < 2; ++buffers) {           // a second one where a team has a second image
        const size_t ctas = std::min<size_t>(per_sm, kSmemOfSm / (image * (buffers + 1) + own + 1024));
        at_once = ctas < (fill ? per_sm : 1) ? 0 : std::max<int64_t>(1, (int64_t)kSms * ctas / slices);
      }
      const size_t smem = image * buffers + own;
      if (smem > kSmemMost || at_once == 0) continue;
      if (slices > 1 && C <= 8 * kMaxCols && (fill || at_once < all)) continue;
      const int64_t cost = (all + at_once - 1) / at_once * (iters + 4);
      if (cost >= least) continue;
      least = cost;
      best = Plan{};
      best.resident = true;
      best.smem = smem;
      best.ctas = (int)std::min(all, at_once);
      Geom& g = best.g;
      g.N = N; g.P = P; g.C = C; g.G = G; g.Cg = C / G;
      g.cols = cols; g.rp = rp; g.team = team; g.tiles = 1; g.buffers = buffers;
      g.slices = slices; g.slice = slice; g.Gs = Gs;
    }
  }
  Geom& g = best.g;
  if (g.team == 0) return best;
  g.inv_m = (float)(1.0 / ((double)P * g.Cg));
  g.col_mul = (65536 + g.cols - 1) / g.cols;
  g.cg_mul = g.Cg == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + g.Cg - 1) / g.Cg);
  g.lanes_g = pow2_up_to(g.team / std::min(g.Gs, g.team), 32);
  g.lanes_c = pow2_up_to(kThreads / std::min(g.slice, kThreads), 32);
  while (1 << g.lanes_log < g.lanes_g) ++g.lanes_log;
  g.entries = g.Cg % 8 ? g.Cg : g.Cg / 8;
  g.per_row = g.Cg % 8 ? g.cols * 8 : g.cols;
  g.rows_on = g.lanes_g / g.entries;
  g.cols_on = g.lanes_g % g.entries;
  split(g, 1);
  return best;
}
// The team form for small images, else a cluster where an image fits one and all of a call's CTAs run at once (two on an SM, if their shared memory allows), with
// as many CTAs per image as that gives, and where they fill at least half of the SMs or a thread has few pixels.
// us, cluster / streamed, 16-bit storage: 128x16x16x160 8.2 / 10.3, 128x8x8x640 8.7 / 10.8; on the other side of the rule
// 2x64x64x128 with SiLU 12.2 / 10.0, and 128 images of 32x32x160 in more than one wave 31.5 / 23.4.
inline Plan plan_forward(int elem_bytes, int N, int P, int C, int G) {
  const Plan small = plan_teams(8 * elem_bytes, false, kForwardPerSm, 32 * kThreads, 8, 12, N, P, C, G);
  if (small.g.team) return small;
  Plan pl = plan_streamed(N, P, C, G, kForwardPerSm);
  if (pl.g.tiles > 1) return pl;
  Plan res = pl;
  res.rows = 0;
  for (int parts = kMaxCluster; parts >= 1; parts /= 2) {
    split(res.g, parts);
    if (parts > 1 && res.g.iters < 2) continue;
    res.smem = (size_t)res.g.iters * kThreads * 8 * elem_bytes + 3 * kThreads * 8 * 4 + 8 * (size_t)C + 16 * (size_t)G;
    const int64_t per = std::min<size_t>(kSmemOfSm / (res.smem + 1024), 2), ctas = (int64_t)N * parts;
    if (res.smem > kSmemMost || ctas > per * kSms) continue;
    res.resident = ctas >= kSms / 2 || res.g.iters <= 4;
    return res.resident ? res : pl;
  }
  return pl;
}
inline Plan plan_backward(int elem_bytes, int N, int P, int C, int G) {
  Plan small = plan_teams(2 * 8 * elem_bytes, true, kBackwardPerSm, 64 * kThreads, 24, 4, N, P, C, G);
  if (small.g.team) {
    const int64_t images = (int64_t)(kThreads / small.g.team) * kTeamImages;
    small.ctas = std::max(small.ctas, (int)((N + images - 1) / images));
    small.rows = small.ctas;
    return small;
  }
  return plan_streamed(N, P, C, G, kBackwardPerSm);
}
inline size_t partial_floats(const Plan& pl) { return (size_t)pl.rows * 2 * pl.g.C; }
// Whether a second streamed pass adds up an image's rows of sums itself.  (Backward also with tiles: a launch that forms the totals of
// many images of one row each took 5 of 5.8 ms for 4096 of 4096 channels.)
inline bool merges(const Geom& g) { return g.tiles == 1 && g.parts <= kMergeParts; }
inline bool merges_backward(const Geom& g) { return g.parts <= kMergeParts; }
// CTAs of a launch whose items are as many as groups or images times blocks of channels, more than a grid may have.
constexpr size_t kItemCtas = 16 * kSms;
inline unsigned item_ctas(size_t items) { return (unsigned)std::min(items, kItemCtas); }

// ---- host side: launches ---------------------------------------------------------------------------------------
template <typename Kernel, typename Params>
inline cudaError_t launch_cluster(Kernel kernel, int images, int cluster, size_t smem, cudaStream_t st, const Params& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)images, (unsigned)cluster); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 1; at[1].val.clusterDim.y = (unsigned)cluster; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T, int W, int ACT, int EXTRA> inline cudaError_t launch_forward_as(cudaStream_t st, const Plan& pl, Forward<T> p) {
  const Geom& g = pl.g;
  if (g.team) {
    static OncePerDevice once;
    const cudaError_t e = once_per_device(&once, []() { return set_smem_limit(forward_teams_kernel<T, W, ACT, EXTRA>, kSmemMost); });
    return e != cudaSuccess ? e : launch_chained(forward_teams_kernel<T, W, ACT, EXTRA>, dim3((unsigned)pl.ctas, (unsigned)g.slices), dim3(kThreads), pl.smem, st, p);
  }
  if (pl.resident) {
    static OncePerDevice once;
    const cudaError_t e = once_per_device(&once, []() { return set_smem_limit(forward_kernel<T, W, ACT, EXTRA>, kSmemMost); });
    return e != cudaSuccess ? e : launch_cluster(forward_kernel<T, W, ACT, EXTRA>, g.N, g.parts, pl.smem, st, p);
  }
  static OncePerDevice once;
  cudaError_t e = once_per_device(&once, []() {
    const cudaError_t f = set_smem_limit(moments_kernel<T, W>, kSmemMost);
    return f != cudaSuccess ? f : set_smem_limit(apply_kernel<T, W, ACT, EXTRA>, kSmemMost);
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)g.N, (unsigned)g.parts, (unsigned)g.tiles);
  const size_t ring = (size_t)ring_of<T>() * kThreads * 8 * sizeof(T);
  e = launch_chained(moments_kernel<T, W>, grid, dim3(kThreads), ring + 3 * kThreads * 8 * 4 + 64 * (size_t)g.cols, st, p);
  p.combined = !merges(g);
  if (e == cudaSuccess && p.combined) {
    const int64_t entries = (int64_t)g.parts * (g.tiles == 1 ? 1 : g.Cg);
    e = launch_chained(combine_kernel<T>, dim3(item_ctas((size_t)g.N * g.G)), dim3(32 * pow2_up_to(entries / 64, 32)), 0, st, p);
  }
  if (e == cudaSuccess)
    e = launch_chained(apply_kernel<T, W, ACT, EXTRA>, grid, dim3(kThreads), (p.res ? 2 : 1) * ring + (p.combined ? 0 : 8 * (size_t)g.G), st, p);
  return e;
}

template <typename T, int ACT> inline cudaError_t launch_forward_act(cudaStream_t st, const Plan& pl, const Forward<T>& p) {
  return p.codes ? launch_forward_as<T, kWhole, ACT, WITH_CODES>(st, pl, p)
                 : p.res || p.gate ? launch_forward_as<T, kWhole, ACT, WITH_RES_GATE>(st, pl, p) : launch_forward_as<T, kWhole, ACT, PLAIN>(st, pl, p);
}
template <typename T>
inline cudaError_t launch_forward(cudaStream_t st, const Plan& pl, Forward<T> p) {
  p.g = pl.g;
  const int C = p.g.C;
  p.ckpt_lanes = p.codes ? ckpt_block_lanes(C) : 0;
  int8_t* codes = p.codes;
  if (p.ckpt_lanes == 0) p.codes = nullptr;       // blocks that do not fall on groups of lanes: a pass of their own
  const int w = access_width<T>(C, {p.x, p.y, p.res}, p.codes);
  cudaError_t e = w == 8 ? launch_forward_as<T, 8, -1, WITH_CODES>(st, pl, p)
                  : w == 4 ? launch_forward_as<T, 4, -1, WITH_CODES>(st, pl, p)
                  : w != kWhole ? launch_forward_as<T, sizeof(T), -1, WITH_CODES>(st, pl, p)
                  : p.act == ACT_RELU ? launch_forward_act<T, ACT_RELU>(st, pl, p)
                  : p.act == ACT_SILU ? launch_forward_act<T, ACT_SILU>(st, pl, p) : launch_forward_act<T, ACT_NONE>(st, pl, p);
  if (e == cudaSuccess && codes && !p.codes) e = launch_ckpt_encode<T>(st, p.x, (size_t)p.g.N * p.g.P, C, codes, p.scales);
  return e;
}

template <typename T, int W, bool CK, int SLOPE>
inline cudaError_t launch_backward_as(cudaStream_t st, const Plan& pl, Backward<T> p) {
  const Geom& g = pl.g;
  const int width = 2 * g.C, blocks = (width + 31) / 32;
  if (g.team) {
    static OncePerDevice once;
    cudaError_t e = once_per_device(&once, []() { return set_smem_limit(backward_teams_kernel<T, W, CK, SLOPE>, kSmemMost); });
    if (e == cudaSuccess) e = launch_chained(backward_teams_kernel<T, W, CK, SLOPE>, dim3((unsigned)pl.ctas, (unsigned)g.slices), dim3(kThreads), pl.smem, st, p);
    if (e == cudaSuccess)
      e = launch_chained(parameters_kernel, dim3((unsigned)blocks), dim3(1024), 0, st, (const float*)p.partial, (int)pl.rows, g.C, p.dgamma, p.dbeta);
    return e;
  }
  static OncePerDevice once;
  cudaError_t e = once_per_device(&once, []() {
    const cudaError_t f = set_smem_limit(backward_sums_kernel<T, W, CK, SLOPE>, kSmemMost);
    return f != cudaSuccess ? f : set_smem_limit(backward_apply_kernel<T, W, CK, SLOPE>, kSmemMost);
  });
  if (e != cudaSuccess) return e;
  auto rings = [&](bool res) { return 16 * (size_t)Feed<T, W, CK>::words(p.slope == SLOPE_MASK, res); };
  e = launch_chained(backward_sums_kernel<T, W, CK, SLOPE>, dim3((unsigned)g.N, (unsigned)g.parts, (unsigned)g.tiles), dim3(kThreads),
                     rings(false) + (kClosedInRegisters<SLOPE> || g.iters < kClosedFrom<T> ? 0 : kClosedBytes), st, p);
  if (merges_backward(g)) p.totals = nullptr;
  else if (e == cudaSuccess)
    e = launch_chained(totals_kernel, dim3(item_ctas((size_t)g.N * blocks)), dim3(1024), 0, st, (const float*)p.partial, g.N, g.parts, width, p.totals);
  // coefficients of the tile's groups; with one tile also the channels' sums
  const size_t own = 8 * (size_t)std::min(g.G, g.cols * 8) + (g.tiles == 1 ? 8 * (size_t)g.C : 0);
  p.extra = (blocks + g.parts - 1) / g.parts;
  if (e == cudaSuccess)
    e = launch_chained(backward_apply_kernel<T, W, CK, SLOPE>, dim3((unsigned)(g.N + p.extra), (unsigned)g.parts, (unsigned)g.tiles), dim3(kThreads),
                       rings(p.res != nullptr) + own, st, p);
  return e;
}
template <typename T, bool CK> inline cudaError_t launch_backward_of(cudaStream_t st, const Plan& pl, const Backward<T>& p) {
  switch (access_width<T>(p.g.C, {p.dy, p.x, p.mask, p.res, p.dx}, p.codes)) {
    case kWhole: break;
    case 8: return launch_backward_as<T, 8, CK, -1>(st, pl, p);
    case 4: return launch_backward_as<T, 4, CK, -1>(st, pl, p);
    default: return launch_backward_as<T, sizeof(T), CK, -1>(st, pl, p);
  }
  switch (p.slope) {
    case SLOPE_MASK: return launch_backward_as<T, kWhole, CK, SLOPE_MASK>(st, pl, p);
    case SLOPE_BITS: return launch_backward_as<T, kWhole, CK, SLOPE_BITS>(st, pl, p);
    case SLOPE_SILU: return launch_backward_as<T, kWhole, CK, SLOPE_SILU>(st, pl, p);
    default: return launch_backward_as<T, kWhole, CK, SLOPE_ONE>(st, pl, p);
  }
}
template <typename T> inline cudaError_t launch_backward(cudaStream_t st, const Plan& pl, Backward<T> p) {
  p.g = pl.g;
  return p.codes ? launch_backward_of<T, true>(st, pl, p) : launch_backward_of<T, false>(st, pl, p);
}

}  // namespace gn
}  // namespace fdg
