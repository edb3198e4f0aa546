// Device-side helpers of the training operators (not installed): 16-byte loads and stores of fp32 or
// bf16 runs as fp32 registers, block reductions in a fixed order, and the launch-overlap controls.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace dlm {

// Elements of T in 16 bytes.
template <typename T>
constexpr int kRun = 16 / (int)sizeof(T);

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&t);
}

// One 16-byte run, held as the four words it came in.
struct Words {
    uint32_t w[4];
};
__device__ __forceinline__ Words ld_words(const void* p) {
    uint4 t = *reinterpret_cast<const uint4*>(p);
    return {{t.x, t.y, t.z, t.w}};
}
__device__ __forceinline__ void st_words(void* p, const Words& a) {
    *reinterpret_cast<uint4*>(p) = make_uint4(a.w[0], a.w[1], a.w[2], a.w[3]);
}
template <typename T>
__device__ __forceinline__ void unpack(const Words& a, float* v);
template <>
__device__ __forceinline__ void unpack<float>(const Words& a, float* v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = __uint_as_float(a.w[u]);
}
template <>
__device__ __forceinline__ void unpack<__nv_bfloat16>(const Words& a, float* v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        v[2 * u] = __uint_as_float(a.w[u] << 16);
        v[2 * u + 1] = __uint_as_float(a.w[u] & 0xffff0000u);
    }
}
template <typename T>
__device__ __forceinline__ Words pack(const float* v);
template <>
__device__ __forceinline__ Words pack<float>(const float* v) {
    return {{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}};
}
template <>
__device__ __forceinline__ Words pack<__nv_bfloat16>(const float* v) {
    return {{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}};
}

// Sum over the warp, the same value in every lane (butterfly: a fixed order).
template <typename V>
__device__ __forceinline__ V warp_sum(V v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Programmatic dependent launch: a kernel launched with the overlap attribute may start while its
// predecessor drains and must not touch what the predecessor wrote before pdl_wait() has returned.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Launch with the overlap attribute, in clusters of `cluster` CTAs.
template <typename... K, typename... A>
inline cudaError_t launch_overlapped(void (*kernel)(K...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, int cluster,
                                     A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<K>(args)...);
}

}  // namespace dlm
