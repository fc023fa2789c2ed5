// Activations held in 8 bits between the forward and the backward pass ("checkpoints").
//
// A tensor [rows][C] is held as one signed byte per value and one scale byte per block of 32 consecutive channels of a row
// (the last block of a row may be shorter):
//   step  = 2^e with e the smallest integer >= -126 for which the block's largest magnitude rounds to at most 127 steps,
//   code  = x / step rounded to the nearest integer, ties to even;   value held = code * step;   scale byte = e + 127.
// A step that is a power of two makes the division and the product exact, so a value is rounded once (by at most half a
// step), every reader forms the same number, and that number has 7 significant bits: a bf16 tensor decoded from a
// checkpoint is the checkpoint, and the tensor-core weight gradients multiply it without a further rounding.  The step is
// up to twice amax/127; blocks as short as 32 (1/32 byte per value for the scale) give most of that back against one fp32
// scale per row.  Two borders: a block that holds an infinity or a NaN gets scale byte 255 and codes 0 and reads back as NaN
// throughout; where e would be 122 (magnitudes from 127.5/128 * 2^128 on, bf16's largest among them) e stays 121, so that
// every value held is finite, and codes stop at +-127.
#pragma once
#include "kernel_common.cuh"

namespace fdg {

constexpr int kCkptBlock = 32;
constexpr int kCkptThreads = 256;

// ---- one block's scale, 8 values at a time --------------------------------------------------------
// `top`: the largest magnitude of the block as its bit pattern (the order of the patterns is that of the magnitudes, with
// infinity and then NaN above them).  Adding 2^16 carries into the exponent exactly when the mantissa is 255/128 or more,
// i.e. when the magnitude is 127.5 steps of the lower exponent or more (127.5 itself rounds to 128).
struct CkptScale {
  uint32_t byte;        // e + 127
  float inv_step;       // 2^-e; 0 for a block that is not finite
  bool clamp;           // codes past +-127 are possible
};
__device__ __forceinline__ CkptScale ckpt_scale(uint32_t top) {
  CkptScale s;
  const uint32_t t = max(top + 0x10000u, 7u << 23);                 // its exponent is e + 127 + 6, 7 at least
  s.byte = (t >> 23) - 6u;
  s.inv_step = __uint_as_float((260u << 23) - (t & 0x7F800000u));    // exponent 254 - (e + 127)
  s.clamp = top >= 0x7F7F0000u;
  if (s.clamp) {
    s.byte = top >= 0x7F800000u ? 255u : 248u;
    s.inv_step = top >= 0x7F800000u ? 0.f : __uint_as_float(6u << 23);
  }
  return s;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The largest magnitude of 8 values, in the storage type's own bits where it has 16 (two at a time), as fp32 bits.
__device__ __forceinline__ uint32_t ckpt_top2(const Raw8<__nv_bfloat16>& r) {
  return max_u16x2(max_u16x2(r.q[0].x & 0x7FFF7FFFu, r.q[0].y & 0x7FFF7FFFu), max_u16x2(r.q[0].z & 0x7FFF7FFFu, r.q[0].w & 0x7FFF7FFFu));
}
__device__ __forceinline__ uint32_t ckpt_top(const Raw8<__nv_bfloat16>& r) {
  const uint32_t m = ckpt_top2(r);
  return max(m & 0xFFFF0000u, m << 16);
}
__device__ __forceinline__ uint32_t ckpt_top(const Raw8<float>& r) {
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    m = max_nan(m, max_nan(fabsf(__uint_as_float(r.q[j].x)), fabsf(__uint_as_float(r.q[j].y))));
    m = max_nan(m, max_nan(fabsf(__uint_as_float(r.q[j].z)), fabsf(__uint_as_float(r.q[j].w))));
  }
  return __float_as_uint(m);
}
// x / step rounded to the nearest even integer, in the low byte: the product is exact, and adding 1.5 * 2^23 rounds it.
constexpr float kCkptRound = 12582912.f;
__device__ __forceinline__ uint32_t ckpt_code(float x, const CkptScale& s) {
  float t = x * s.inv_step;
  if (s.clamp) {
    if (s.byte == 255u) return 0;
    t = fminf(fmaxf(t, -127.f), 127.f);
  }
  return __float_as_uint(t + kCkptRound);
}
__device__ __forceinline__ uint2 ckpt_codes(const F8& v, const CkptScale& s) {
  uint32_t q[8];
  const f32x2 inv = pair(s.inv_step), round = pair(kCkptRound);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 t = halves(fma2(v.p[j], inv, round));
    q[2 * j] = __float_as_uint(t.x);
    q[2 * j + 1] = __float_as_uint(t.y);
  }
  if (s.clamp) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 t = halves(v.p[j]);
      q[2 * j] = ckpt_code(t.x, s);
      q[2 * j + 1] = ckpt_code(t.y, s);
    }
  }
  uint2 r;
  r.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
  r.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
  return r;
}
__device__ __forceinline__ float ckpt_step(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}
// The codes as fp32 numbers: code + 128 in the mantissa of 2^23, then the offset off, an integer conversion on the fp32 pipe.
__device__ __forceinline__ F8 ckpt_numbers(uint2 codes) {
  const uint32_t lo = codes.x ^ 0x80808080u, hi = codes.y ^ 0x80808080u;
  const f32x2 off = pair(-8388736.f);
  F8 f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f.p[j] = add2(pair(__uint_as_float(__byte_perm(lo, 0x4B000000u, 0x7540u + 2 * j)), __uint_as_float(__byte_perm(lo, 0x4B000000u, 0x7541u + 2 * j))), off);
    f.p[2 + j] = add2(pair(__uint_as_float(__byte_perm(hi, 0x4B000000u, 0x7540u + 2 * j)), __uint_as_float(__byte_perm(hi, 0x4B000000u, 0x7541u + 2 * j))), off);
  }
  return f;
}
__device__ __forceinline__ F8 ckpt_values(uint2 codes, float step) {
  F8 f = ckpt_numbers(codes);
  const f32x2 st = pair(step);
#pragma unroll
  for (int j = 0; j < 4; ++j) f.p[j] = mul2(f.p[j], st);
  return f;
}

// 8 codes in pieces of CW bytes (8, 4, 2, 1), the first `left` of them.
template <int CW> struct CodePiece;
template <> struct CodePiece<4> { typedef uint32_t Type; };
template <> struct CodePiece<2> { typedef uint16_t Type; };
template <> struct CodePiece<1> { typedef uint8_t Type; };
template <int CW> __device__ __forceinline__ uint2 load_codes(const int8_t* codes, int left) {
  if constexpr (CW == 8) {
    return *reinterpret_cast<const uint2*>(codes);
  } else {
    typedef typename CodePiece<CW>::Type P;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8 / CW; ++i)
      if (i * CW < left) w[i * CW / 4] |= (uint32_t) reinterpret_cast<const P*>(codes)[i] << (8 * (i * CW % 4));
    return make_uint2(w[0], w[1]);
  }
}
template <int CW> __device__ __forceinline__ void store_codes(int8_t* codes, int left, uint2 q) {
  if constexpr (CW == 8) {
    *reinterpret_cast<uint2*>(codes) = q;
  } else {
    typedef typename CodePiece<CW>::Type P;
#pragma unroll
    for (int i = 0; i < 8 / CW; ++i)
      if (i * CW < left) reinterpret_cast<P*>(codes)[i] = (P)((i * CW < 4 ? q.x : q.y) >> (8 * (i * CW % 4)));
  }
}

// Lanes that share a block when consecutive lanes hold consecutive vectors of 8 channels, 0 if blocks do not fall on
// aligned groups of lanes: rows of whole groups of four vectors, or of one or two vectors (one block).
inline int ckpt_block_lanes(int C) {
  const int cols = (C + 7) / 8;
  return cols % 4 == 0 ? 4 : (cols <= 2 ? cols : 0);
}
__device__ __forceinline__ uint32_t ckpt_top_of_lanes(uint32_t top, int lanes, uint32_t taking_part = 0xffffffffu) {
  if (lanes >= 2) top = max(top, __shfl_xor_sync(taking_part, top, 1));
  if (lanes >= 4) top = max(top, __shfl_xor_sync(taking_part, top, 2));
  return top;
}

// ---- whole tensors -----------------------------------------------------------------------------------
// Encode, rows of whole vectors on aligned lane groups: a thread takes vectors of 8 values, consecutive lanes consecutive
// vectors, kCkptUnroll of them in flight.  Nothing is shared but the shuffles of a block's maximum.
constexpr int kCkptUnroll = 4;
template <typename T>
__global__ void __launch_bounds__(kCkptThreads) ckpt_encode_kernel(const T* __restrict__ x, size_t vecs, int lanes, int8_t* __restrict__ codes,
                                                                   uint8_t* __restrict__ scales) {
  const int shift = lanes >> 1;                       // 1, 2, 4 lanes
  grid_dependency_wait();
  const size_t first = (size_t)blockIdx.x * (kCkptThreads * kCkptUnroll) + threadIdx.x;
  Raw8<T> raw[kCkptUnroll];
#pragma unroll
  for (int u = 0; u < kCkptUnroll; ++u) {
    const size_t i = first + (size_t)u * kCkptThreads;
    raw[u] = i < vecs ? raw8_load<T, kWhole>(x + i * 8, 8) : Raw8<T>{};
  }
#pragma unroll
  for (int u = 0; u < kCkptUnroll; ++u) {
    const size_t i = first + (size_t)u * kCkptThreads;
    const CkptScale s = ckpt_scale(ckpt_top_of_lanes(ckpt_top(raw[u]), lanes));
    if (i < vecs) {
      *reinterpret_cast<uint2*>(codes + i * 8) = ckpt_codes(raw8_to_f8(raw[u]), s);
      if ((i & (unsigned)(lanes - 1)) == 0) scales[i >> shift] = (uint8_t)s.byte;
    }
  }
}

// Bytes of a piece of 8 codes, beside vectors that move in pieces of W bytes.
template <typename T, int W> constexpr int kCodeWidth = W == kWhole ? 8 : W / (int)sizeof(T);

// Where a thread's block is: its row, its first column of 8 channels, its columns.
struct BlockPlace {
  size_t off;               // first value
  int col, n;
  __device__ __forceinline__ BlockPlace(size_t b, int C, int per_row) {
    const size_t row = b / (unsigned)per_row;
    col = (int)(b - row * (unsigned)per_row) * 4;
    n = min(4, (C + 7) / 8 - col);
    off = row * (unsigned)C + col * 8;
  }
};
// Encode and decode, rows that do not fall on lanes so, or are no whole vectors: a thread takes a block, up to 4 vectors.
template <typename T, int W>
__global__ void __launch_bounds__(kCkptThreads) ckpt_encode_blocks_kernel(const T* __restrict__ x, size_t blocks, int C, int per_row,
                                                                          int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  grid_dependency_wait();
  const size_t b = (size_t)blockIdx.x * kCkptThreads + threadIdx.x;
  if (b >= blocks) return;
  const BlockPlace at(b, C, per_row);
  Raw8<T> raw[4];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < at.n) raw[i] = raw8_load<T, W>(x + at.off + 8 * i, C - 8 * (at.col + i));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < at.n) top = max(top, ckpt_top(raw[i]));
  const CkptScale s = ckpt_scale(top);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < at.n) store_codes<kCodeWidth<T, W>>(codes + at.off + 8 * i, C - 8 * (at.col + i), ckpt_codes(raw8_to_f8(raw[i]), s));
  scales[b] = (uint8_t)s.byte;
}
template <typename T, int W>
__global__ void __launch_bounds__(kCkptThreads) ckpt_decode_blocks_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                          size_t blocks, int C, int per_row, T* __restrict__ x) {
  grid_dependency_wait();
  const size_t b = (size_t)blockIdx.x * kCkptThreads + threadIdx.x;
  if (b >= blocks) return;
  const BlockPlace at(b, C, per_row);
  uint2 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < at.n) q[i] = load_codes<kCodeWidth<T, W>>(codes + at.off + 8 * i, C - 8 * (at.col + i));
  const float step = ckpt_step(scales[b]);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < at.n) raw8_put<T, W>(x + at.off + 8 * i, C - 8 * (at.col + i), f8_to_raw8<T>(ckpt_values(q[i], step)));
}

// Encode, any row length and alignment: a lane takes a value, a warp a block, kCkptBlocks of them in flight.
constexpr int kCkptBlocks = 8;
template <typename T>
__global__ void __launch_bounds__(kCkptThreads) ckpt_encode_any_kernel(const T* __restrict__ x, size_t blocks, int C, int per_row,
                                                                       int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  grid_dependency_wait();
  const int lane = threadIdx.x & 31;
  const size_t b0 = ((size_t)blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5)) * kCkptBlocks;
  if (b0 >= blocks) return;
  const size_t row0 = b0 / (unsigned)per_row;
  const int first = (int)(b0 - row0 * (unsigned)per_row);
  x += row0 * C; codes += row0 * C;                      // the same for the warp; what follows is a few rows on
  const int n = (int)min((size_t)kCkptBlocks, blocks - b0);
  float v[kCkptBlocks];
  int off[kCkptBlocks];                                  // of the lane's value, -1 behind the row's end
  int row = 0, in_row = first;
#pragma unroll
  for (int i = 0; i < kCkptBlocks; ++i) {
    const int c = in_row * kCkptBlock + lane;
    off[i] = i < n && c < C ? row * C + c : -1;
    v[i] = off[i] >= 0 ? to_f(x[off[i]]) : 0.f;
    if (++in_row == per_row) { in_row = 0; ++row; }
  }
  uint32_t byte = 0;
#pragma unroll
  for (int i = 0; i < kCkptBlocks; ++i) {
    const CkptScale s = ckpt_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(v[i]) & 0x7FFFFFFFu));
    if (off[i] >= 0) codes[off[i]] = (int8_t)ckpt_code(v[i], s);
    if (lane == i) byte = s.byte;
  }
  if (lane < n) scales[b0 + lane] = (uint8_t)byte;
}

// Decode, rows of whole vectors (C a multiple of 8): a thread takes vectors of 8 values.  `lanes` as in the encoder; 0: the
// place of a vector in its row is found by one division and then by steps (step_rows rows and step_cols columns are
// kCkptThreads vectors).
template <typename T>
__global__ void __launch_bounds__(kCkptThreads) ckpt_decode_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                   size_t vecs, int lanes, int cols, int per_row, int step_rows, int step_cols,
                                                                   T* __restrict__ x) {
  grid_dependency_wait();
  const size_t first = (size_t)blockIdx.x * (kCkptThreads * kCkptUnroll) + threadIdx.x;
  const int shift = lanes >> 1;
  size_t row = 0;
  int col = 0;
  if (lanes == 0) { row = first / (unsigned)cols; col = (int)(first - row * (unsigned)cols); }
  uint2 q[kCkptUnroll];
  uint32_t k[kCkptUnroll];
#pragma unroll
  for (int u = 0; u < kCkptUnroll; ++u) {
    const size_t i = first + (size_t)u * kCkptThreads;
    if (i < vecs) {
      q[u] = *reinterpret_cast<const uint2*>(codes + i * 8);
      k[u] = scales[lanes ? i >> shift : row * (unsigned)per_row + (unsigned)col / 4];
    }
    if (lanes == 0) {
      row += (unsigned)step_rows; col += step_cols;
      if (col >= cols) { col -= cols; ++row; }
    }
  }
#pragma unroll
  for (int u = 0; u < kCkptUnroll; ++u) {
    const size_t i = first + (size_t)u * kCkptThreads;
    if (i >= vecs) break;
    raw8_put<T, kWhole>(x + i * 8, 8, f8_to_raw8<T>(ckpt_values(q[u], ckpt_step(k[u]))));
  }
}
// Decode, any row length and alignment: as the encoder.
template <typename T>
__global__ void __launch_bounds__(kCkptThreads) ckpt_decode_any_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                       size_t blocks, int C, int per_row, T* __restrict__ x) {
  grid_dependency_wait();
  const int lane = threadIdx.x & 31;
  const size_t b0 = ((size_t)blockIdx.x * (kCkptThreads / 32) + (threadIdx.x >> 5)) * kCkptBlocks;
  if (b0 >= blocks) return;
  const size_t row0 = b0 / (unsigned)per_row;
  const int first = (int)(b0 - row0 * (unsigned)per_row);
  x += row0 * C; codes += row0 * C;
  const int n = (int)min((size_t)kCkptBlocks, blocks - b0);
  const uint32_t byte = lane < n ? scales[b0 + lane] : 0;
  int8_t q[kCkptBlocks];
  int off[kCkptBlocks];
  int row = 0, in_row = first;
#pragma unroll
  for (int i = 0; i < kCkptBlocks; ++i) {
    const int c = in_row * kCkptBlock + lane;
    off[i] = i < n && c < C ? row * C + c : -1;
    q[i] = off[i] >= 0 ? codes[off[i]] : (int8_t)0;
    if (++in_row == per_row) { in_row = 0; ++row; }
  }
#pragma unroll
  for (int i = 0; i < kCkptBlocks; ++i) {
    const float step = ckpt_step(__shfl_sync(0xffffffffu, byte, i));
    if (off[i] >= 0) x[off[i]] = from_f<T>((float)q[i] * step);
  }
}

// ---- host side (at most 2^36 values and 2^28 channels: grids below 2^31, offsets inside a warp's blocks in 32 bits) ----------
inline size_t ceil_div(size_t n, size_t d) { return (n + d - 1) / d; }
template <typename T>
inline cudaError_t launch_ckpt_encode(cudaStream_t st, const T* x, size_t rows, int C, int8_t* codes, uint8_t* scales) {
  const int lanes = ckpt_block_lanes(C), per_row = (C + kCkptBlock - 1) / kCkptBlock;
  const size_t blocks = rows * (size_t)per_row;
  const dim3 threads(kCkptThreads);
  const int w = access_width<T>(C, {x}, codes);
  auto by_blocks = [&](auto kernel) {
    return launch_chained(kernel, dim3((unsigned)ceil_div(blocks, kCkptThreads)), threads, 0, st, x, blocks, C, per_row, codes, scales);
  };
  // us, blocks by threads / values by lanes: bf16 [160000, 100] 16.6 / 40.8, [262144, 30] (pieces of 4 bytes) 23.1 / 17.5; fp32
  // [160000, 100] 52.3 / 39.5
  if (w == 8 && sizeof(T) == 2) return by_blocks(ckpt_encode_blocks_kernel<T, 8>);
  if (w != kWhole)
    return launch_chained(ckpt_encode_any_kernel<T>, dim3((unsigned)ceil_div(blocks, kCkptThreads / 32 * kCkptBlocks)), threads, 0, st, x, blocks, C,
                          per_row, codes, scales);
  if (!lanes) return by_blocks(ckpt_encode_blocks_kernel<T, kWhole>);
  const size_t vecs = rows * (size_t)(C / 8);
  return launch_chained(ckpt_encode_kernel<T>, dim3((unsigned)ceil_div(vecs, kCkptThreads * kCkptUnroll)), threads, 0, st, x, vecs, lanes, codes, scales);
}
template <typename T>
inline cudaError_t launch_ckpt_decode(cudaStream_t st, const int8_t* codes, const uint8_t* scales, size_t rows, int C, T* x) {
  const int per_row = (C + kCkptBlock - 1) / kCkptBlock;
  const dim3 threads(kCkptThreads);
  const int w = access_width<T>(C, {x}, codes);
  const size_t blocks = rows * (size_t)per_row;
  auto by_blocks = [&](auto kernel) {
    return launch_chained(kernel, dim3((unsigned)ceil_div(blocks, kCkptThreads)), threads, 0, st, codes, scales, blocks, C, per_row, x);
  };
  if (w == 8 && sizeof(T) == 2) return by_blocks(ckpt_decode_blocks_kernel<T, 8>);
  if (w == kWhole) {
    const size_t vecs = rows * (size_t)(C / 8);
    return launch_chained(ckpt_decode_kernel<T>, dim3((unsigned)ceil_div(vecs, kCkptThreads * kCkptUnroll)), threads, 0, st, codes, scales, vecs,
                          ckpt_block_lanes(C), C / 8, per_row, kCkptThreads / (C / 8), kCkptThreads % (C / 8), x);
  }
  return launch_chained(ckpt_decode_any_kernel<T>, dim3((unsigned)ceil_div(blocks, kCkptThreads / 32 * kCkptBlocks)), threads, 0, st, codes, scales,
                        blocks, C, per_row, x);
}

}  // namespace fdg
