// dmx_rows.cuh — what the operators on rows share: 16-byte or single-element accesses, programmatic dependent launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dmx.h"
#include "dmx_host.h"

namespace dmx_rows {

typedef __nv_bfloat16 bf16;

template <typename T, int V>
struct Vec;                                            // V elements as one access
template <> struct Vec<float, 4> { using type = uint4; };
template <> struct Vec<float, 1> { using type = unsigned; };
template <> struct Vec<bf16, 8> { using type = uint4; };
template <> struct Vec<bf16, 1> { using type = unsigned short; };

template <typename T> constexpr int kWide = 16 / (int)sizeof(T);      // elements of a 16-byte access

template <typename T>
__device__ __forceinline__ void widen(const uint4& r, float* x) {
  if constexpr (sizeof(T) == 4) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  } else {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
  }
}
template <typename T>
__device__ __forceinline__ void widen(const unsigned& r, float* x) { x[0] = __uint_as_float(r); }
template <typename T>
__device__ __forceinline__ void widen(const unsigned short& r, float* x) { x[0] = __uint_as_float((unsigned)r << 16); }

__device__ __forceinline__ unsigned pack2(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&t);
}
template <typename T, int V>
__device__ __forceinline__ typename Vec<T, V>::type narrow(const float* x) {
  if constexpr (V == 1 && sizeof(T) == 4) return __float_as_uint(x[0]);
  else if constexpr (V == 1) return __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
  else if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  else return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}

// A load where `live`, else zeros, issued where it stands (a plain conditional load may move towards its use).
__device__ __forceinline__ void load_if(uint4& r, const void* p, bool live) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "=&r"(r.x), "=&r"(r.y), "=&r"(r.z), "=&r"(r.w) : "l"(p), "r"((unsigned)live) : "memory");
}
__device__ __forceinline__ void load_if(uint2& r, const void* p, bool live) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\t@p ld.global.v2.u32 {%0, %1}, [%2];\n\t}"
               : "=&r"(r.x), "=&r"(r.y) : "l"(p), "r"((unsigned)live) : "memory");
}
__device__ __forceinline__ void load_if(unsigned& r, const void* p, bool live) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\tmov.u32 %0, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "=&r"(r) : "l"(p), "r"((unsigned)live) : "memory");
}
__device__ __forceinline__ void load_if(unsigned short& r, const void* p, bool live) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\tmov.u16 %0, 0;\n\t@p ld.global.u16 %0, [%1];\n\t}" : "=&h"(r) : "l"(p), "r"((unsigned)live) : "memory");
}

// Launched as programmatic dependents: what needs no data is set up while the kernel before still runs; then all of its
// (and earlier) writes are waited for. The kernel after may begin likewise.
// Inputs are read behind the wait and with ordinary loads: a read-only one promises that its data do not change while the kernel is resident, which is
// while the one before still writes them.
__device__ __forceinline__ void start_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... V>
int start(dim3 grid, int threads, int cluster, size_t shared, cudaStream_t st, void (*kernel)(P...), V... args) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return dmxh::cuda_ok(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...)) ? DMX_OK : DMX_ERR_CUDA;
}

inline bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int64_t pad256(int64_t n) { return (n + 255) & ~(int64_t)255; }
inline int element_size(int dtype) { return dtype == DMX_F32 ? 4 : 2; }
// rows of D elements that 16-byte accesses reach
inline bool wide_rows(const void* p, int64_t rows, int64_t ld, int64_t D, int dtype) {
  const int V = 16 / element_size(dtype);
  return aligned(p, 16) && D % V == 0 && (rows <= 1 || ld % V == 0);
}

}  // namespace dmx_rows
