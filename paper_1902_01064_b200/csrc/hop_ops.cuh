// Shared by the layer operators (hop_norm.cu, hop_linear.cu): element types, error messages, group lookup.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <type_traits>

#include "hop.h"

constexpr int kHopSMs = 148;        // the B200's; launch plans (and so workspace sizes) use it on hosts without a GPU too

// Message into the caller's buffer; no allocation, nothing thrown.
template <typename... A>
static inline int hop_op_fail(char* errbuf, int64_t len, int code, const char* fmt, A... a) {
    if (errbuf && len > 0) {
        if constexpr (sizeof...(A) == 0) snprintf(errbuf, (size_t)len, "%s", fmt);
        else snprintf(errbuf, (size_t)len, fmt, a...);
    }
    return code;
}
static inline int hop_op_cuda(char* errbuf, int64_t len, const char* who, cudaError_t e) {
    if (e == cudaSuccess) return HOP_OK;
    return hop_op_fail(errbuf, len, HOP_E_CUDA, "%s: %s", who, cudaGetErrorString(e));
}
static inline bool hop_op_dtype_ok(int d) { return d == HOP_DT_F32 || d == HOP_DT_F16 || d == HOP_DT_BF16; }
static inline int hop_op_size(int d) { return d == HOP_DT_F32 ? 4 : 2; }

__device__ __forceinline__ float op_f(float v) { return v; }
__device__ __forceinline__ float op_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float op_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T op_t(float v);
template <> __device__ __forceinline__ float op_t<float>(float v) { return v; }
template <> __device__ __forceinline__ __half op_t<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 op_t<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight consecutive elements, the first n of which exist; VEC: the address is 16-byte aligned.
template <typename T, bool VEC>
__device__ __forceinline__ void op_load8(const T* p, int n, float (&v)[8]) {
    if (VEC && n >= 8) {
        union { uint4 q[sizeof(T) / 2]; T t[8]; } u;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) u.q[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = op_f(u.t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? op_f(p[i]) : 0.f;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void op_store8(T* p, int n, const float (&v)[8]) {
    if (VEC && n >= 8) {
        union { uint4 q[sizeof(T) / 2]; T t[8]; } u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.t[i] = op_t<T>(v[i]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = u.q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = op_t<T>(v[i]);
    }
}

// Group that owns `row`, by a whole warp: the number of groups that end at or before it (32 ends per load; `groups` when
// the row lies behind the last group).  No entry of offsets is used as an address.
__device__ __forceinline__ int op_group_of(const int32_t* offsets, int groups, int64_t row, int lane) {
    if (!offsets) return 0;
    int g = 0;
    for (int i = 0; i < groups; i += 32) {
        const bool before = i + lane < groups && (int64_t)offsets[i + lane + 1] <= row;
        g += __popc(__ballot_sync(0xffffffffu, before));
    }
    return g;
}

// Shifts a lane's words (its own units and the next) down by m bytes.
template <int W>
__device__ __forceinline__ void op_shift_words(uint32_t (&w)[W], uint32_t m) {
    if (m & 8) {
#pragma unroll
        for (int i = 0; i < W - 2; ++i) w[i] = w[i + 2];
    }
    if (m & 4) {
#pragma unroll
        for (int i = 0; i < W - 3; ++i) w[i] = w[i + 1];
    }
    if (m & 2) {
#pragma unroll
        for (int i = 0; i < W - 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
}

// Programmatic dependent launch: every kernel of the layer operators is launched so that it sets itself up while the one in
// front on the stream finishes, and waits for that one -- which has itself waited for its own -- before it reads or writes
// anything of the caller's.  A product of 4 x 32 rows of 64 columns, one after the other: 7.3 -> 5.0 us.  None of their pointers is
// __restrict__: what such a pointer reads may come by the path for data that nobody writes while the kernel lives, and the kernel
// in front may still be writing (and dropout's y may be its x).
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... P, typename... A>
static inline cudaError_t hop_launch_dependent(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
