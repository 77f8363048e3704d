// What the block-cache kernels share: the paged cache's addressing, 16-bit element types, status codes.
//
// A cache holds keys and values of many requests in pages of `page_size` tokens; the pages of one request
// are listed, block by block, in its row of the block table.  Offsets are 64-bit throughout: a long cache
// passes 2^31 elements.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "check.cuh"
#include "ptx.cuh"

namespace ivf {

constexpr int kKvStatusBadId = -6;
constexpr int kKvStatusNoPages = -8;
// status[1] of a block-cache call: which operator met the first bad value
enum KvSite { KV_SITE_TABLES = 601, KV_SITE_APPEND, KV_SITE_SUMMARIZE, KV_SITE_SELECT, KV_SITE_ATTEND };

constexpr int kKvMaxDim = 256;
constexpr int kKvMaxGroup = 64;     // query heads per kv head
constexpr int kKvMaxSelect = 1024;  // selected blocks per token and kv head

__device__ __forceinline__ void kv_report(int* status, int code, int site) {
    if (atomicCAS(status, 0, code) == 0) {
        status[1] = site;
        status[2] = static_cast<int>(blockIdx.x);
    }
}

// One side (keys or values) of a cache: element (page, head, token, i) is at
// base + page * page_stride + head * head_stride + token * token_stride + i.
struct KvPlane {
    void* base;
    int64_t page_stride, head_stride, token_stride;
};

template <typename T>
struct Pair16;
template <>
struct Pair16<__half> {
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return __half22float2(*reinterpret_cast<const __half2*>(&w));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <>
struct Pair16<__nv_bfloat16> {
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

template <typename T>
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    float2 p;
    p = Pair16<T>::unpack(v.x); f[0] = p.x; f[1] = p.y;
    p = Pair16<T>::unpack(v.y); f[2] = p.x; f[3] = p.y;
    p = Pair16<T>::unpack(v.z); f[4] = p.x; f[5] = p.y;
    p = Pair16<T>::unpack(v.w); f[6] = p.x; f[7] = p.y;
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(Pair16<T>::pack(f[0], f[1]), Pair16<T>::pack(f[2], f[3]), Pair16<T>::pack(f[4], f[5]),
                      Pair16<T>::pack(f[6], f[7]));
}

// Sum of x[0..N), N a power of two: the second half is added onto the first until one value is left.  The
// order is fixed so that what is rounded to 8 bits afterwards does not depend on the launch.
template <int N>
__device__ __forceinline__ float halving_sum(float (&x)[N]) {
#pragma unroll
    for (int s = N / 2; s > 0; s >>= 1) {
#pragma unroll
        for (int i = 0; i < s; ++i) x[i] = __fadd_rn(x[i], x[i + s]);
    }
    return x[0];
}

// Largest magnitude so far: NaN stays NaN (fmaxf would drop it, and the row would be coded as if the number were not there).
__device__ __forceinline__ float max_magnitude(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
// Row of 32-bit numbers with largest magnitude `amax` -> codes in [-127, 127] and a scale; a scale below the
// normal range, and a scale that is not finite (NaN too), becomes 0 and all codes 0.
__device__ __forceinline__ float code_scale(float amax) {
    const float s = __fmul_rn(amax, 1.0f / 127.0f);
    return s >= 1.17549435e-38f && s <= 3.4e38f ? s : 0.0f;
}
__device__ __forceinline__ int code_of(float x, float scale) {
    if (!(scale > 0.0f)) return 0;
    return static_cast<int>(fminf(fmaxf(rintf(__fdiv_rn(x, scale)), -127.0f), 127.0f));
}

// ------------------------------------------------------------------ clusters: shared memory of the other CTAs
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {  // the same place in another CTA of the cluster
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_store(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The two halves of it: what lies between them need not wait for the other CTAs.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float4 cluster_load4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 cluster_load2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

}  // namespace ivf
