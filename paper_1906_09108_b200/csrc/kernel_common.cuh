// What the kernels of the library share: programmatic dependent launch, settings made once per device, conversion between
// storage types and fp32, and vectors of 8 channels.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "once_per_device.h"

namespace fdg {

// ------------------------------------------------ programmatic dependent launch --
// The kernels that follow one another in a module's chain (convolution, batch-norm apply, batch-norm
// backward apply) are launched with programmatic stream serialisation: the next kernel of the stream may be
// scheduled while this one still runs, does the part of its start-up that needs nothing from global
// memory (barriers, tensor-memory allocation, descriptor prefetch), and then blocks in grid_dependency_wait()
// until the preceding kernel has completed and its writes are visible.  Nothing may be written to global memory
// before that wait, and nothing read, but for copies past L1 (cp.async.cg) of what was complete before the
// preceding kernel released this one: a kernel that releases after its own wait vouches for everything
// before itself, though not for what it writes (the second passes of group_norm.cuh).  grid_dependency_release() tells the scheduler that, as far as this
// block is concerned, the next kernel may start being scheduled (it fires once every block has called it or
// exited).  Both are no-ops in a kernel launched the ordinary way.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dependency_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Launch with the attribute that allows the overlap described above.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_chained(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Makes a setting of the current device (see OncePerDevice).  Setting a function attribute is no stream operation: a launch
// may be a recorded one.
template <typename Work>
inline cudaError_t once_per_device(OncePerDevice* once, Work work) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  return e != cudaSuccess ? e : once->run(dev, work);
}
template <typename Kernel>
inline cudaError_t set_smem_limit(Kernel kernel, size_t bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

// SMs of a B200.  Splits whose rows need scratch are planned for this number, not for the device's own: the size of the
// workspace is asked for without a device.
constexpr int kSms = 148;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Eight consecutive values of a row in the storage type (16 or 32 bytes), as the kernels on columns of 8 channels move them.
// W = kWhole: rows are whole numbers of such vectors, aligned to their size.  Otherwise rows and bases are multiples of W bytes
// (8, 4, or an element), the first `left` values exist, and the rest read as zero.
constexpr int kWhole = 16;
template <typename T> struct alignas(8 * sizeof(T)) Raw8 { uint4 q[sizeof(T) / 2]; };
template <int W> struct Piece;
template <> struct Piece<8> { typedef uint2 Type; };
template <> struct Piece<4> { typedef uint32_t Type; };
template <> struct Piece<2> { typedef uint16_t Type; };
template <typename T, int W> __device__ __forceinline__ Raw8<T> raw8_load(const T* __restrict__ p, int left) {
  Raw8<T> r;
  if constexpr (W == kWhole && sizeof(T) == 4) {         // one 256-bit access: two of 128 bits would each touch every sector
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.q[0].x), "=r"(r.q[0].y), "=r"(r.q[0].z), "=r"(r.q[0].w), "=r"(r.q[1].x), "=r"(r.q[1].y), "=r"(r.q[1].z), "=r"(r.q[1].w)
                 : "l"(p));
  } else if constexpr (W == kWhole) {
    r.q[0] = *reinterpret_cast<const uint4*>(p);
  } else {
    typedef typename Piece<W>::Type P;
    constexpr int PER = W / (int)sizeof(T);
    P* e = reinterpret_cast<P*>(&r);
#pragma unroll
    for (int i = 0; i < 8 / PER; ++i) e[i] = i * PER < left ? reinterpret_cast<const P*>(p)[i] : P{};
  }
  return r;
}
template <typename T, int W> __device__ __forceinline__ void raw8_put(T* __restrict__ p, int left, const Raw8<T>& r) {
  if constexpr (W == kWhole && sizeof(T) == 4) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r.q[0].x), "r"(r.q[0].y), "r"(r.q[0].z), "r"(r.q[0].w),
                 "r"(r.q[1].x), "r"(r.q[1].y), "r"(r.q[1].z), "r"(r.q[1].w), "l"(p)
                 : "memory");
  } else if constexpr (W == kWhole) {
    *reinterpret_cast<uint4*>(p) = r.q[0];
  } else {
    typedef typename Piece<W>::Type P;
    constexpr int PER = W / (int)sizeof(T);
    const P* e = reinterpret_cast<const P*>(&r);
#pragma unroll
    for (int i = 0; i < 8 / PER; ++i)
      if (i * PER < left) reinterpret_cast<P*>(p)[i] = e[i];
  }
}
inline bool aligned_to(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
// W for rows of C values and these tensors (null ones do not count); `bytes`: a tensor of rows of C bytes, which is moved in
// pieces of W / sizeof(T).
template <typename T> inline int access_width(int C, std::initializer_list<const void*> tensors, const void* bytes = nullptr) {
  uintptr_t bits = (uintptr_t)C * sizeof(T) | reinterpret_cast<uintptr_t>(bytes) * sizeof(T);
  for (const void* t : tensors) bits |= reinterpret_cast<uintptr_t>(t);
  return bits % (8 * sizeof(T)) == 0 ? kWhole : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : (int)sizeof(T);
}

// Pairs of fp32 values in one 64-bit register pair.  sm_100a adds, multiplies and multiply-adds both halves with one
// instruction (each half rounded as the scalar instruction rounds it), which halves the arithmetic issued by kernels that have
// a handful of operations on every value they stream.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ f32x2 pair(float v) { return pair(v, v); }
__device__ __forceinline__ float2 halves(f32x2 v) {
  float2 d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(v));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// Eight fp32 values as pairs, and the way from and to the storage type.
struct F8 { f32x2 p[4]; };
__device__ __forceinline__ F8 raw8_to_f8(const Raw8<__nv_bfloat16>& r) {
  const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
  F8 f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f.p[j] = pair(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
  return f;
}
__device__ __forceinline__ F8 raw8_to_f8(const Raw8<float>& r) {
  F8 f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f.p[2 * j] = pair(__uint_as_float(r.q[j].x), __uint_as_float(r.q[j].y));
    f.p[2 * j + 1] = pair(__uint_as_float(r.q[j].z), __uint_as_float(r.q[j].w));
  }
  return f;
}
// The storage type's values, and with RELU those of max(v, 0), NaN staying NaN.
template <bool RELU> __device__ __forceinline__ uint32_t pack_bf16x2(f32x2 v) {
  const float2 h = halves(v);
  uint32_t d;
  if (RELU) asm("cvt.rn.relu.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(h.y), "f"(h.x));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(h.y), "f"(h.x));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
template <typename T, bool RELU = false> __device__ __forceinline__ Raw8<T> f8_to_raw8(const F8& f) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 2) {
    r.q[0] = make_uint4(pack_bf16x2<RELU>(f.p[0]), pack_bf16x2<RELU>(f.p[1]), pack_bf16x2<RELU>(f.p[2]), pack_bf16x2<RELU>(f.p[3]));
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float2 a = halves(f.p[2 * j]), b = halves(f.p[2 * j + 1]);
      if (RELU) { a.x = max_nan(a.x, 0.f); a.y = max_nan(a.y, 0.f); b.x = max_nan(b.x, 0.f); b.y = max_nan(b.y, 0.f); }
      r.q[j] = make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
  }
  return r;
}

}  // namespace fdg
