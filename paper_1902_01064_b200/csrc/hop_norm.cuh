// Device side of the layer operators on rows: dropout's mask, rows at any alignment, and the norm kernels (hop_norm.cu
// holds the entries; hop_norm_f32 / f16 / bf16.cu instantiate the kernels for one element type each).
#pragma once
#include "hop_internal.h"
#include "hop_ops.cuh"
#include "hop_philox.cuh"

struct DropRng { uint32_t thr, last, step, site; float scale; uint32_t k0[10], k1[10]; };      // round keys: operands from constant memory
struct NormPlan { int threads, nv, teams_per_block, rows_per_team, teams, stages; size_t smem; };

struct NormDev {
    hop_norm_args a;
    DropRng d;
    int rows_per_team, drop, stages;
    float* partial;             // backward: [team + group][two sums, layer norms four][cols]
};

// Blocks an SM is to hold, forward and backward, of the kernels for one warp a row (128 threads a block), of up to 256 and
// of up to 512 threads: what bounds their registers.  Measured in bf16 with dropout, us: forward 16384 x 1024 with 2 / 3 / 4
// small blocks 41 / 51 / 45, 8192 x 4096 73 / 74 / 76; backward 16384 x 2048 with 1 / 2 / 3 small blocks 139 / 129 / 292 (spills),
// 32768 x 512 with 3 / 4 blocks of warps 72 / 86.
constexpr int kWarpBlocks[2] = {4, 3}, kSmallBlocks[2] = {2, 2}, kLargeBlocks[2] = {1, 1};
constexpr int kNormSmem = 220 * 1024;       // most dynamic shared memory of a block (the sums' buffer is static)


// Kernels for one element type: rows of any alignment when askew
cudaError_t hop_norm_launch_f32(const NormDev& P, const NormPlan& pl, bool backward, bool askew, cudaStream_t st);
cudaError_t hop_norm_launch_f16(const NormDev& P, const NormPlan& pl, bool backward, bool askew, cudaStream_t st);
cudaError_t hop_norm_launch_bf16(const NormDev& P, const NormPlan& pl, bool backward, bool askew, cudaStream_t st);

namespace {


// ------------------------------------------------------------------------------------------------ dropout
// A column is dropped when its 16-bit number is below thr = floor(65536 p + 1/2).  Sixteen bits decide a column and not
// 32: one Philox block (10 rounds) then serves eight columns, and p is off by at most 2^-17.

__device__ __forceinline__ void drop_words(const DropRng& d, uint32_t c, uint32_t row, uint32_t (&o)[4]) { philox4x32_10(c, row, d.step, d.site, d.k0, d.k1, o); }
// Values of columns 8c .. 8c+7 of a row: dropped ones become 0 whatever they hold (infinities and NaN too).  A 16-bit
// number is compared in the upper half of its word, so the odd ones need no extraction.
__device__ __forceinline__ void drop8(const DropRng& d, const uint32_t (&o)[4], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = v[2 * i] * d.scale, y = v[2 * i + 1] * d.scale;
        v[2 * i] = (o[i] << 16) > d.last ? x : 0.f;
        v[2 * i + 1] = o[i] > d.last ? y : 0.f;         // (the low half cannot lift a smaller high half over it)
    }
}

// ------------------------------------------------------------------------------------------------ rows at any alignment
// A warp covers 256 columns of a row, eight consecutive ones a lane (one Philox block).  Rows need not start on a 16-byte
// boundary: the warp fetches the whole 16-byte units that its columns touch -- a unit that holds a byte of the row lies in
// the row's own allocation -- and a lane takes its eight values out of its own units and the next one, shifted by the m
// bytes its address is off.  m is the same for the whole warp, so the shifts are uniform branches.
template <typename T> constexpr int kUnits = (int)sizeof(T) / 2;              // 16-byte units of eight values
template <typename T> constexpr int kWindow = (32 * kUnits<T> + 1) * 16;      // bytes a warp can touch

template <typename T>
__device__ __forceinline__ void unpack8(const uint32_t* w, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    } else if constexpr (std::is_same_v<T, __half>) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}
template <typename T>
__device__ __forceinline__ void pack8(const float (&v)[8], uint32_t* w) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
    } else if constexpr (std::is_same_v<T, __half>) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&h); }
    }
}
// A lane's eight values out of the warp's window in shared memory; those behind the row's end are 0.
template <typename T, bool ASKEW>
__device__ __forceinline__ void window_read(const unsigned char* window, int lane, uint32_t m, float (&v)[8]) {
    constexpr int U = kUnits<T>;
    uint32_t w[4 * U + 4];
    const uint4* q = reinterpret_cast<const uint4*>(window) + lane * U;
#pragma unroll
    for (int i = 0; i < U; ++i) { const uint4 x = q[i]; w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w; }
    if (ASKEW && m) {
        const uint4 x = q[U];
        w[4 * U] = x.x; w[4 * U + 1] = x.y; w[4 * U + 2] = x.z; w[4 * U + 3] = x.w;
        op_shift_words(w, m);
    }
    unpack8<T>(w, v);
}
// Copies the first n <= 16 bytes of a unit, zeros for the rest (n <= 0: zeros, the source is not touched)
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, int n) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(max(0, min(16, n))) : "memory");
}
// Starts the copy of the units that `bytes` bytes at base + off (the warp's columns; off m bytes past the grid) touch; what
// lies behind them in the window becomes 0.
template <typename T, bool ASKEW>
__device__ __forceinline__ void window_fetch(uint32_t window, const char* base, uint32_t off, uint32_t m, int bytes, int lane) {
    const char* first = base + (ASKEW ? (int64_t)off - m : (int64_t)off);
    const int total = bytes > 0 ? bytes + (ASKEW ? (int)m : 0) : 0;
#pragma unroll
    for (int k = 0; k < kUnits<T>; ++k)
        cp16(window + (lane + 32 * k) * 16, first + (lane + 32 * k) * 16, total - (lane + 32 * k) * 16);
    if (ASKEW && lane == 0) cp16(window + 32 * kUnits<T> * 16, first + 32 * kUnits<T> * 16, total - 32 * kUnits<T> * 16);
}
// Stores a warp's values (lane: eight from p + 8 * lane, n of them exist; `cols` exist in the whole warp).  Rows off the
// 16-byte grid go through shared memory, so that the warp's element stores are consecutive.
template <typename T, bool ASKEW>
__device__ __forceinline__ void warp_store(T* p, int lane, int n, int cols, const float (&v)[8], unsigned char* scratch) {
    constexpr int U = kUnits<T>;
    uint32_t w[4 * U];
    pack8<T>(v, w);
    if (!ASKEW || (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        if (n == 8) {
#pragma unroll
            for (int i = 0; i < U; ++i) reinterpret_cast<uint4*>(p + lane * 8)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[lane * 8 + i] = op_t<T>(v[i]);
        }
        return;
    }
    uint4* q = reinterpret_cast<uint4*>(scratch);
#pragma unroll
    for (int i = 0; i < U; ++i) q[lane * U + i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    __syncwarp();
    if (sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = (i * 32 + lane) * 2;
            if (e + 1 < cols) reinterpret_cast<uint32_t*>(p)[i * 32 + lane] = reinterpret_cast<const uint32_t*>(scratch)[i * 32 + lane];
            else if (e < cols) p[e] = reinterpret_cast<const T*>(scratch)[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i * 32 + lane < cols) p[i * 32 + lane] = reinterpret_cast<const T*>(scratch)[i * 32 + lane];
    }
    __syncwarp();
}

// ------------------------------------------------------------------------------------------------ norms
// A team of threads owns a row at a time, eight consecutive columns per thread and piece, and walks rows_per_team
// consecutive rows: the group's vectors stay in shared memory, each thread's own values in its own places, and, backward, the
// column sums in its registers.  The rows ahead are on their way into shared memory (cp.async, `stages` rows deep), each warp its own columns, so a row costs no barrier but those of
// its sums.
// Sums of N <= 3 values over the team; everyone gets them.  Within a warp the values share their shuffles: after the first
// two exchanges an eight-lane group holds one value, so three sums take 6 shuffles and not 15.  buf: two halves used in
// turn, so one barrier per reduction.
template <int N, bool WARP>
__device__ __forceinline__ void team_sum(float (&v)[N], float* buf, int& turn) {
    constexpr uint32_t kAll = 0xffffffffu;
    const int lane = threadIdx.x & 31;
    float c;
    if constexpr (N == 1) {
        c = v[0];
        c += __shfl_xor_sync(kAll, c, 16);
        c += __shfl_xor_sync(kAll, c, 8);
    } else {
        const bool hi = lane & 16, odd = lane & 8;
        float p = hi ? (N > 2 ? v[N - 1] : 0.f) : v[0], q = hi ? 0.f : v[1];
        p += __shfl_xor_sync(kAll, hi ? v[0] : (N > 2 ? v[N - 1] : 0.f), 16);       // lanes 0-15: value 0, 16-31: value 2
        q += __shfl_xor_sync(kAll, hi ? v[1] : 0.f, 16);                            // lanes 0-15: value 1
        c = (odd ? q : p) + __shfl_xor_sync(kAll, odd ? p : q, 8);
    }
    c += __shfl_xor_sync(kAll, c, 4);
    c += __shfl_xor_sync(kAll, c, 2);
    c += __shfl_xor_sync(kAll, c, 1);
    if constexpr (!WARP) {
        float* b = buf + turn;
        turn ^= 32 * 4;
        const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, k = N == 1 ? 0 : lane >> 3;
        if ((lane & 7) == 0 && (lane >> 3) < N) b[(lane >> 3) * 32 + warp] = c;
        __syncthreads();
        c = 0.f;
        for (int w = lane & 7; w < warps; w += 8) c += b[k * 32 + w];
        c += __shfl_xor_sync(kAll, c, 4);
        c += __shfl_xor_sync(kAll, c, 2);
        c += __shfl_xor_sync(kAll, c, 1);
    }
    if constexpr (N == 1) {
        v[0] = c;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(kAll, c, i * 8);
    }
}

// Eight values of a group's vector (float32, at any address): `none` where there is no vector
__device__ __forceinline__ void vec8(const float* base, int64_t stride, int g, int c, int n, float none, float (&v)[8]) {
    const float* p = base + (int64_t)g * stride + c;
    if (base && n == 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        const float4 x = reinterpret_cast<const float4*>(p)[0], y = reinterpret_cast<const float4*>(p)[1];
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = base && i < n ? p[i] : none;
}

// Eight values as four pairs: one instruction for two float32 operations (each rounded as by itself), which halves what the
// kernels, bound by the instructions they issue, spend on arithmetic.
__device__ __forceinline__ void mul2(float& d0, float& d1, float a0, float a1, float b0, float b1) {
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}" : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b0, float b1, float c0, float c1) {
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void mul8(float (&d)[8], const float (&a)[8], const float (&b)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) mul2(d[i], d[i + 1], a[i], a[i + 1], b[i], b[i + 1]);
}
__device__ __forceinline__ void scale8(float (&d)[8], const float (&a)[8], float s) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) mul2(d[i], d[i + 1], a[i], a[i + 1], s, s);
}
// d = a * b + c
__device__ __forceinline__ void fma8(float (&d)[8], const float (&a)[8], const float (&b)[8], const float (&c)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) fma2(d[i], d[i + 1], a[i], a[i + 1], b[i], b[i + 1], c[i], c[i + 1]);
}
__device__ __forceinline__ void fmas8(float (&d)[8], const float (&a)[8], float s, const float (&c)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) fma2(d[i], d[i + 1], a[i], a[i + 1], s, s, c[i], c[i + 1]);
}
// sum of a * b, added to s
__device__ __forceinline__ void dot8(float& s, const float (&a)[8], const float (&b)[8]) {
    float p, q;
    mul2(p, q, a[0], a[1], b[0], b[1]);
#pragma unroll
    for (int i = 2; i < 8; i += 2) fma2(p, q, a[i], a[i + 1], b[i], b[i + 1], p, q);
    s += p + q;
}

#define HOP_FOR_PIECES _Pragma("unroll") for (int j = 0; j < NV; ++j)
#define HOP_FOR_8 _Pragma("unroll") for (int i = 0; i < 8; ++i)

// mean and 1 / deviation of the team's row
template <int NV, bool LAYER, bool WARP>
__device__ __forceinline__ void row_stats(const float (&v)[NV][8], const int (&n)[NV], float icols, float eps, float* buf, int& turn, float& mean, float& inv) {
    float s[1] = {0.f};
    mean = 0.f;
    if constexpr (LAYER) {
        HOP_FOR_PIECES HOP_FOR_8 s[0] += v[j][i];
        team_sum<1, WARP>(s, buf, turn);
        mean = s[0] * icols;
        s[0] = 0.f;
        HOP_FOR_PIECES HOP_FOR_8 { const float u = i < n[j] ? v[j][i] - mean : 0.f; s[0] = fmaf(u, u, s[0]); }
    } else {
        HOP_FOR_PIECES dot8(s[0], v[j], v[j]);       // what lies behind the row's end is 0
    }
    team_sum<1, WARP>(s, buf, turn);
    inv = rsqrtf(fmaf(s[0], icols, eps));
}

// One of the row arrays as a team reads it: staged ahead through the warp's windows, or straight from memory where the plan finds
// no room for a row: above 8192 columns, in float32 gradients of layer norms above 7168 (with a token gate 6144) and of RMS norms
// with a token gate above 7168.  Those forms are held to 64 registers by their 1024 threads and spill (backward 1.0 to 2.8 KB a
// thread, forward 0.1 to 0.3): 4096 x 12288 forward bf16 177 us (2.9 times the bytes' time; layer 3.9), float32 193 (1.6), backward
// 375 (4.1; layer 5.7) and 452 (2.5).  Offsets from the team's first row fit 32 bits (the plan sees to it).
template <typename T, int NV, bool ASKEW, bool STAGED>
struct RowIn {
    const char* base;           // the warp's (unstaged: this thread's) first column in the team's first row
    uint32_t stride, ahead, here;       // bytes; offsets of the row to fetch next and of the row to read next
    __device__ __forceinline__ void open(const void* p, int64_t stride_elems, int64_t row0, int col) {
        base = p ? reinterpret_cast<const char*>(p) + (row0 * stride_elems + col) * (int64_t)sizeof(T) : nullptr;
        stride = (uint32_t)(stride_elems * (int64_t)sizeof(T));
        ahead = here = 0;
    }
    __device__ __forceinline__ uint32_t skew(uint32_t off) const { return ((uint32_t)reinterpret_cast<uintptr_t>(base) + off) & 15u; }
    __device__ __forceinline__ void fetch(uint32_t window, const int (&wide)[NV], int piece_cols, int lane) {
        if (base) HOP_FOR_PIECES {
            const uint32_t off = ahead + j * piece_cols * (uint32_t)sizeof(T);      // (256 columns, so pieces share the row's skew)
            window_fetch<T, ASKEW>(window + j * kWindow<T>, base, off, skew(ahead), wide[j] * (int)sizeof(T), lane);
        }
        ahead += stride;
    }
    __device__ __forceinline__ void read(const unsigned char* window, int lane, int piece_cols, const int (&n)[NV], float (&v)[NV][8]) {
        if constexpr (STAGED) {
            HOP_FOR_PIECES window_read<T, ASKEW>(window + j * kWindow<T>, lane, skew(here), v[j]);
        } else {
            const T* p = reinterpret_cast<const T*>(base + here);
            HOP_FOR_PIECES {
                if (n[j] == 8 && (!ASKEW || (reinterpret_cast<uintptr_t>(p) & 15) == 0)) op_load8<T, true>(p + j * piece_cols, n[j], v[j]);
                else op_load8<T, false>(p + j * piece_cols, n[j], v[j]);
            }
        }
    }
};
// A row array that is written: base as above, always the warp's first column
template <typename T, int NV, bool ASKEW>
struct RowOut {
    char* base;
    uint32_t stride, here;
    __device__ __forceinline__ void open(void* p, int64_t stride_elems, int64_t row0, int wcol) {
        base = p ? reinterpret_cast<char*>(p) + (row0 * stride_elems + wcol) * (int64_t)sizeof(T) : nullptr;
        stride = (uint32_t)(stride_elems * (int64_t)sizeof(T));
        here = 0;
    }
    __device__ __forceinline__ void write(int lane, int piece_cols, const int (&n)[NV], const int (&wide)[NV], const float (&v)[NV][8], unsigned char* scratch) const {
        HOP_FOR_PIECES if (!ASKEW || wide[j] > 0) warp_store<T, ASKEW>(reinterpret_cast<T*>(base + here) + j * piece_cols, lane, n[j], wide[j], v[j], scratch);
    }
};

// What both passes set up: columns, windows, the team's rows and the group of the first one
#define HOP_TEAM_SETUP(ARRAYS, VECTORS)                                                                                                                  \
    extern __shared__ __align__(16) unsigned char smem[];                                                                                       \
    __shared__ float buf[2 * 32 * 4];                                                                                                           \
    int turn = 0;                                                                                                                               \
    const hop_norm_args& a = P.a;                                                                                                               \
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = WARP ? lane : threadIdx.x, width = WARP ? 32 : blockDim.x;                 \
    const int64_t team = WARP ? (int64_t)blockIdx.x * (blockDim.x >> 5) + warp : blockIdx.x;                                                     \
    const int64_t row0 = team * P.rows_per_team, row1 = min(row0 + P.rows_per_team, a.rows);                                                     \
    if (row0 >= a.rows) { dependency_wait(); return; }                                                                                          \
    const int rows = (int)(row1 - row0), warps = blockDim.x >> 5, pcols = width * 8;                                                             \
    const float icols = 1.f / a.cols;                                                                                                           \
    int col[NV], n[NV], wide[NV];                                                                                                               \
    HOP_FOR_PIECES {                                                                                                                            \
        col[j] = (tid + j * width) * 8;                                                                                                         \
        n[j] = max(0, min(8, a.cols - col[j]));                                                                                                 \
        wide[j] = max(0, min(256, a.cols - (col[j] - lane * 8)));                                                                               \
    }                                                                                                                                           \
    const int wcol = col[0] - lane * 8, icol = STAGED ? wcol : col[0];                                                                          \
    /* shared memory: the group's vectors (each thread's own values, in its own places), store buffers, stages of windows */                     \
    float4* vecs = reinterpret_cast<float4*>(smem) + (WARP ? warp * 32 * 2 * NV * (VECTORS) : 0) + tid;                                          \
    unsigned char* after = smem + (STAGED ? (size_t)blockDim.x * 32 * NV * (VECTORS) : 0);                                                       \
    unsigned char* scratch = after + warp * (kWindow<T> - 16);                                                                                  \
    constexpr uint32_t kArray = NV * kWindow<T>;                                                                                                \
    const uint32_t stage_size = warps * (ARRAYS) * kArray, ring = P.stages * stage_size;                                                         \
    unsigned char* windows = after + warps * (kWindow<T> - 16) + warp * (ARRAYS) * kArray;                                                        \
    const uint32_t windows_at = (uint32_t)__cvta_generic_to_shared(windows);                                                                    \
    uint32_t to = 0, from = 0;      /* stages being filled and read */                                                                          \
    int fetched = 0;                                                                                                                            \
    dependency_wait();                                                                                                                          \
    launch_dependents();                                                                                                                        \
    int g = op_group_of(a.offsets, a.groups, row0, lane), loaded = -1;

// The k-th of a group's vectors: eight values of a thread's piece j, kept in shared memory (registers are short)
template <int NV>
__device__ __forceinline__ void vec_put(float4* vecs, int width, int k, int j, const float (&v)[8]) {
    vecs[((k * NV + j) * 2) * width] = make_float4(v[0], v[1], v[2], v[3]);
    vecs[((k * NV + j) * 2 + 1) * width] = make_float4(v[4], v[5], v[6], v[7]);
}
template <int NV>
__device__ __forceinline__ void vec_get(const float4* vecs, int width, int k, int j, float (&v)[8]) {
    const float4 p = vecs[((k * NV + j) * 2) * width], q = vecs[((k * NV + j) * 2 + 1) * width];
    v[0] = p.x; v[1] = p.y; v[2] = p.z; v[3] = p.w; v[4] = q.x; v[5] = q.y; v[6] = q.z; v[7] = q.w;
}

__device__ __forceinline__ void wait_stage(int stages) {      // the oldest of `stages` rows in flight has arrived
    if (stages == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
}

// r and h of a row in one pass over x and b: two row arrays in, two out, the branch's sum and the stream's are the only
// exchanges between threads.  In 16-bit types no limit of the GPU is reached: 280 warp instructions per 256 columns with dropout, a
// quarter of them the mask, use half of the issue slots, and with a quarter of the warps resident the rest waits on the sums' barriers
// and shuffles and on shared memory; in float32 it is memory.  8192 x 4096 bf16, p = 0.1: 66 us (4.1 TB/s; without dropout 53 us,
// 5.1; without post norm and gate 54 us); float32 104 us (5.1 TB/s).
template <typename T, int NV, bool STAGED, bool LAYER, bool ASKEW, bool WARP, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB)
norm_forward_kernel(const __grid_constant__ NormDev P) {
    HOP_TEAM_SETUP(2 + (a.token_gate != nullptr), LAYER ? 4 : 2)
    RowIn<T, NV, ASKEW, STAGED> in_x, in_b, in_t;
    in_x.open(a.x, a.x_stride, row0, icol);
    in_b.open(a.b, a.b_stride, row0, icol);
    in_t.open(a.token_gate, a.token_gate_stride, row0, icol);
    RowOut<T, NV, ASKEW> out_r, out_h;
    out_r.open(a.b ? a.r : nullptr, a.r_stride, row0, wcol);
    out_h.open(a.pre_norm ? a.h : nullptr, a.h_stride, row0, wcol);
    auto fetch = [&]() {
        if constexpr (STAGED) {
            if (fetched++ < rows) {
                in_x.fetch(windows_at + to, wide, pcols, lane); in_b.fetch(windows_at + to + kArray, wide, pcols, lane); in_t.fetch(windows_at + to + 2 * kArray, wide, pcols, lane);
            }
            to += stage_size;
            if (to == ring) to = 0;
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    for (int i = 0; i + 1 < P.stages; ++i) fetch();
    // Vectors 0: scale * gate * w_post, 1: w_pre, 2: the shift scale * gate * c_post, 3: c_pre
    auto make = [&](int k, int j, float (&v)[8]) {
        if (k == 1) vec8(a.w_pre, a.w_pre_stride, g, col[j], n[j], 1.f, v);
        else if (k == 3) vec8(a.c_pre, a.c_pre_stride, g, col[j], n[j], 0.f, v);
        else {
            float t[8];
            vec8(a.gate, a.gate_stride, g, col[j], n[j], 1.f, t);
            if (k == 0) vec8(a.w_post, a.w_post_stride, g, col[j], n[j], 1.f, v);
            else vec8(a.c_post, a.c_post_stride, g, col[j], n[j], 0.f, v);
            HOP_FOR_8 v[i] *= a.scale * t[i];
        }
    };
    auto get = [&](int k, int j, float (&v)[8]) {
        if constexpr (STAGED) vec_get<NV>(vecs, width, k, j, v);
        else make(k, j, v);
    };
    const uint32_t first_row = (uint32_t)row0;
    int left = 0;               // rows of the group from here
    auto enter = [&](int i) {   // the group that row i belongs to: its vectors
        const int64_t row = row0 + i;
        int64_t end = a.rows;
        for (; g < a.groups && (end = a.offsets ? (int64_t)a.offsets[g + 1] : a.rows) <= row; ++g) end = a.rows;
        left = (int)min(end - row, (int64_t)rows + 1);
        if (g >= a.groups) return;
        loaded = g;
        if constexpr (STAGED) {
            for (int k = 0; k < (LAYER ? 4 : 2); ++k) {
                HOP_FOR_PIECES {
                    float v[8];
                    make(k, j, v);
                    vec_put<NV>(vecs, width, k, j, v);
                }
            }
        }
    };
    for (int i = 0; i < rows; ++i, --left) {
        fetch();
        if (left == 0) enter(i);
        float x[NV][8], b[NV][8], v[8];
        uint32_t o[NV][4];
        if (P.drop) HOP_FOR_PIECES drop_words(P.d, (uint32_t)(col[j] >> 3), first_row + i, o[j]);
        if constexpr (STAGED) wait_stage(P.stages);
        const unsigned char* win = windows + from;
        from += stage_size;
        if (from == ring) from = 0;
        if (g >= a.groups) {
            HOP_FOR_PIECES HOP_FOR_8 x[j][i] = 0.f;
            if (a.b) out_r.write(lane, pcols, n, wide, x, scratch);
            if (a.pre_norm) out_h.write(lane, pcols, n, wide, x, scratch);
        } else {
            float mean, inv;
            if (a.b) {
                in_b.read(win + kArray, lane, pcols, n, b);
                if (a.post_norm) {
                    row_stats<NV, LAYER, WARP>(b, n, icols, a.eps, buf, turn, mean, inv);
                    HOP_FOR_PIECES {
                        if (LAYER) HOP_FOR_8 b[j][i] -= mean;
                        scale8(b[j], b[j], inv);
                    }
                }
                in_x.read(win, lane, pcols, n, x);
                HOP_FOR_PIECES {
                    get(0, j, v);
                    mul8(b[j], b[j], v);
                    if (LAYER) { get(2, j, v); HOP_FOR_8 b[j][i] += v[i]; }
                }
                if (a.token_gate) {
                    float t[NV][8];
                    in_t.read(win + 2 * kArray, lane, pcols, n, t);
                    HOP_FOR_PIECES mul8(b[j], b[j], t[j]);
                }
                HOP_FOR_PIECES {
                    if (P.drop) drop8(P.d, o[j], b[j]);
                    fmas8(x[j], x[j], a.skip, b[j]);
                    if (LAYER) HOP_FOR_8 x[j][i] = i < n[j] ? x[j][i] : 0.f;      // (an RMS norm leaves the zeros there)
                }
                out_r.write(lane, pcols, n, wide, x, scratch);
            } else {
                in_x.read(win, lane, pcols, n, x);
            }
            if (a.pre_norm) {
                row_stats<NV, LAYER, WARP>(x, n, icols, a.eps, buf, turn, mean, inv);
                HOP_FOR_PIECES {
                    get(1, j, v);
                    if (LAYER) HOP_FOR_8 x[j][i] -= mean;
                    scale8(x[j], x[j], inv);
                    mul8(x[j], x[j], v);
                    if (LAYER) { get(3, j, v); HOP_FOR_8 x[j][i] += v[i]; }
                }
                out_h.write(lane, pcols, n, wide, x, scratch);
            }
        }
        in_x.here += in_x.stride; in_b.here += in_b.stride; in_t.here += in_t.stride; out_r.here += out_r.stride; out_h.here += out_h.stride;
        __syncwarp();           // the warp's window has been read: the next fetch may write it
    }
}

// Gradients.  Both rows' statistics are formed again from r and b (they are read anyway), so nothing is saved by the
// forward pass.  Column sums of a team's rows stay in registers; at a change of group and at the end they go to the
// team's own place [team + group] of the workspace (unique, since team and group only ever grow along the rows), and
// norm_sums_kernel adds the places of each group in order: no atomics, the same bits every time.
// 16384 x 2048 bf16 in 16 groups, p = 0.1: 105 us with the sums (3.9 TB/s); 480 instructions per 256 columns take 58 % of the issue
// slots at the 16 warps an SM that the column sums in registers allow, the rest waits on the row's two sums; float32 164 us (4.9
// TB/s); layer norms, with four column sums and three sums a row, 157 us in bf16 and 204 in float32.
//   acc 0: sum dh r_hat   1: sum q t b_hat   2: sum dh   3: sum q t     (t: the token gate; 2 and 3 with shifts only;
//   q without its factor `scale`, which norm_sums_kernel applies)
template <typename T, int NV, bool STAGED, bool LAYER, bool ASKEW, bool WARP, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB)
norm_backward_kernel(const __grid_constant__ NormDev P) {
    constexpr int NACC = LAYER ? 4 : 2;
    HOP_TEAM_SETUP(4 + (a.token_gate != nullptr), LAYER ? 3 : 2)
    RowIn<T, NV, ASKEW, STAGED> in_r, in_b, in_dr, in_dh, in_t;
    in_r.open(a.dh ? a.r : nullptr, a.r_stride, row0, icol);
    in_b.open(a.b, a.b_stride, row0, icol);
    in_dr.open(a.dr, a.dr_stride, row0, icol);
    in_dh.open(a.dh, a.dh_stride, row0, icol);
    in_t.open(a.token_gate, a.token_gate_stride, row0, icol);
    RowOut<T, NV, ASKEW> out_x, out_b, out_t;
    out_x.open(a.dx, a.dx_stride, row0, wcol);
    out_b.open(a.db, a.db_stride, row0, wcol);
    out_t.open(a.dtoken_gate, a.dtoken_gate_stride, row0, wcol);
    auto fetch = [&]() {
        if constexpr (STAGED) {
            if (fetched++ < rows) {
                in_r.fetch(windows_at + to, wide, pcols, lane); in_b.fetch(windows_at + to + kArray, wide, pcols, lane); in_dr.fetch(windows_at + to + 2 * kArray, wide, pcols, lane);
                in_dh.fetch(windows_at + to + 3 * kArray, wide, pcols, lane); in_t.fetch(windows_at + to + 4 * kArray, wide, pcols, lane);
            }
            to += stage_size;
            if (to == ring) to = 0;
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    for (int i = 0; i + 1 < P.stages; ++i) fetch();
    float acc[NACC][NV][8];
    // Vectors 0: scale * gate * w_post, 1: w_pre, 2: scale * c_post (for dtoken_gate)
    auto make = [&](int k, int j, float (&v)[8]) {
        if (k == 1) {
            vec8(a.w_pre, a.w_pre_stride, g, col[j], n[j], 1.f, v);
        } else if (k == 2) {
            vec8(a.c_post, a.c_post_stride, g, col[j], n[j], 0.f, v);
            HOP_FOR_8 v[i] *= a.scale;
        } else {
            float t[8];
            vec8(a.gate, a.gate_stride, g, col[j], n[j], 1.f, t);
            vec8(a.w_post, a.w_post_stride, g, col[j], n[j], 1.f, v);
            HOP_FOR_8 v[i] *= a.scale * t[i];
        }
    };
    auto get = [&](int k, int j, float (&v)[8]) {
        if constexpr (STAGED) vec_get<NV>(vecs, width, k, j, v);
        else make(k, j, v);
    };
    auto flush = [&]() {
        if (loaded < 0 || !P.partial) return;
        float* dst = P.partial + (team + loaded) * NACC * (int64_t)a.cols;
#pragma unroll
        for (int k = 0; k < NACC; ++k)
            HOP_FOR_PIECES {
                if (n[j] == 8 && (a.cols & 3) == 0) {
                    float4* q = reinterpret_cast<float4*>(dst + (int64_t)k * a.cols + col[j]);
                    q[0] = make_float4(acc[k][j][0], acc[k][j][1], acc[k][j][2], acc[k][j][3]);
                    q[1] = make_float4(acc[k][j][4], acc[k][j][5], acc[k][j][6], acc[k][j][7]);
                } else {
                    HOP_FOR_8 if (i < n[j]) dst[(int64_t)k * a.cols + col[j] + i] = acc[k][j][i];
                }
            }
    };
    const uint32_t first_row = (uint32_t)row0;
    int left = 0;               // rows of the group from here
    auto enter = [&](int i) {   // the group that row i belongs to: its vectors
        const int64_t row = row0 + i;
        int64_t end = a.rows;
        for (; g < a.groups && (end = a.offsets ? (int64_t)a.offsets[g + 1] : a.rows) <= row; ++g) end = a.rows;
        left = (int)min(end - row, (int64_t)rows + 1);
        if (g >= a.groups) return;
        flush();
        loaded = g;
#pragma unroll
        for (int k = 0; k < NACC; ++k) HOP_FOR_PIECES HOP_FOR_8 acc[k][j][i] = 0.f;
        if constexpr (STAGED) {
            for (int k = 0; k < (LAYER ? 3 : 2); ++k) {
                HOP_FOR_PIECES {
                    float v[8];
                    make(k, j, v);
                    vec_put<NV>(vecs, width, k, j, v);
                }
            }
        }
    };
    for (int i = 0; i < rows; ++i, --left) {
        fetch();
        if (left == 0) enter(i);
        float r[NV][8], b[NV][8], dh[NV][8], v[8];
        uint32_t o[NV][4];
        if (P.drop) HOP_FOR_PIECES drop_words(P.d, (uint32_t)(col[j] >> 3), first_row + i, o[j]);
        if constexpr (STAGED) wait_stage(P.stages);
        const unsigned char* win = windows + from;
        from += stage_size;
        if (from == ring) from = 0;
        if (g >= a.groups) {
            HOP_FOR_PIECES HOP_FOR_8 r[j][i] = 0.f;
            out_x.write(lane, pcols, n, wide, r, scratch);
            if (a.b) out_b.write(lane, pcols, n, wide, r, scratch);
            if (a.dtoken_gate) out_t.write(lane, pcols, n, wide, r, scratch);
        } else {
            // Sums over the row first; dr, which they do not need, is read behind them, and b twice: what is held across a
            // sum costs registers
            HOP_FOR_PIECES HOP_FOR_8 { r[j][i] = 0.f; b[j][i] = 0.f; dh[j][i] = 0.f; }
            float rmean = 0.f, gmean = 0.f, bmean = 0.f, binv = 1.f;
            float z[3] = {0.f, 0.f, 0.f};
            if (a.b && a.post_norm) in_b.read(win + kArray, lane, pcols, n, b);
            if (a.dh) {
                in_r.read(win, lane, pcols, n, r);
                in_dh.read(win + 3 * kArray, lane, pcols, n, dh);
            }
            if constexpr (LAYER) {
                float t[3] = {0.f, 0.f, 0.f};
                HOP_FOR_PIECES {
                    get(1, j, v);
                    HOP_FOR_8 { t[0] += r[j][i]; t[1] += b[j][i]; t[2] = fmaf(dh[j][i], v[i], t[2]); }
                }
                team_sum<3, WARP>(t, buf, turn);
                rmean = t[0] * icols; gmean = t[2] * icols; bmean = t[1] * icols;
                HOP_FOR_PIECES HOP_FOR_8 {
                    r[j][i] = i < n[j] ? r[j][i] - rmean : 0.f;
                    const float u = i < n[j] ? b[j][i] - bmean : 0.f;
                    z[1] = fmaf(u, u, z[1]);
                }
            } else {
                HOP_FOR_PIECES dot8(z[1], b[j], b[j]);
            }
            HOP_FOR_PIECES {
                get(1, j, v);
                dot8(z[0], r[j], r[j]);
                mul8(v, v, dh[j]);
                dot8(z[2], v, r[j]);
            }
            team_sum<3, WARP>(z, buf, turn);
            float (&q)[NV][8] = r;          // dr', then q, where r_hat was
            if (a.dh) {
                const float rinv = rsqrtf(fmaf(z[0], icols, a.eps)), k = -z[2] * icols * rinv;
                HOP_FOR_PIECES {
                    get(1, j, v);
                    scale8(r[j], r[j], rinv);
                    fma8(acc[0][j], dh[j], r[j], acc[0][j]);
                    mul8(v, v, dh[j]);
                    if constexpr (LAYER) {
                        HOP_FOR_8 { acc[2][j][i] += dh[j][i]; v[i] -= gmean; }
                    }
                    fmas8(q[j], r[j], k, v);
                    scale8(q[j], q[j], rinv);
                }
            }
            if (a.dr) {
                in_dr.read(win + 2 * kArray, lane, pcols, n, b);
                HOP_FOR_PIECES HOP_FOR_8 q[j][i] += b[j][i];
            }
            HOP_FOR_PIECES {
                if (LAYER) HOP_FOR_8 q[j][i] = i < n[j] ? q[j][i] : 0.f;      // (its mean lands behind the row's end too)
                scale8(b[j], q[j], a.skip);
            }
            out_x.write(lane, pcols, n, wide, b, scratch);
            if (a.b) {
                if (a.post_norm) binv = rsqrtf(fmaf(z[1], icols, a.eps));
                HOP_FOR_PIECES if (P.drop) drop8(P.d, o[j], q[j]);
                in_b.read(win + kArray, lane, pcols, n, b);
                HOP_FOR_PIECES {
                    if (LAYER) HOP_FOR_8 b[j][i] -= bmean;          // (behind the row's end q is 0)
                    scale8(b[j], b[j], binv);
                }
                if (a.token_gate) {
                    float t[NV][8];
                    if (a.dtoken_gate) {
                        HOP_FOR_PIECES {
                            get(0, j, v);
                            mul8(t[j], b[j], v);
                            if (LAYER) { get(2, j, v); HOP_FOR_8 t[j][i] += v[i]; }
                            mul8(t[j], t[j], q[j]);
                        }
                        out_t.write(lane, pcols, n, wide, t, scratch);
                    }
                    in_t.read(win + 4 * kArray, lane, pcols, n, t);
                    HOP_FOR_PIECES mul8(q[j], q[j], t[j]);
                }
                float e[2] = {0.f, 0.f};
                HOP_FOR_PIECES {
                    get(0, j, v);
                    fma8(acc[1][j], q[j], b[j], acc[1][j]);
                    if (LAYER) HOP_FOR_8 acc[3][j][i] += q[j][i];
                    mul8(q[j], q[j], v);
                    dot8(e[0], q[j], b[j]);
                    if (LAYER) HOP_FOR_8 e[1] += q[j][i];
                }
                if (a.post_norm) {
                    if constexpr (LAYER) {
                        team_sum<2, WARP>(e, buf, turn);
                    } else {
                        float e1[1] = {e[0]};
                        team_sum<1, WARP>(e1, buf, turn);
                        e[0] = e1[0];
                    }
                    e[0] *= -icols; e[1] *= icols;
                    HOP_FOR_PIECES {
                        fmas8(q[j], b[j], e[0], q[j]);
                        if (LAYER) HOP_FOR_8 q[j][i] -= e[1];
                        scale8(q[j], q[j], binv);
                    }
                }
                out_b.write(lane, pcols, n, wide, q, scratch);
            }
        }
        in_r.here += in_r.stride; in_b.here += in_b.stride; in_dr.here += in_dr.stride; in_dh.here += in_dh.stride; in_t.here += in_t.stride;
        out_x.here += out_x.stride; out_b.here += out_b.stride; out_t.here += out_t.stride;
        __syncwarp();           // the warp's window has been read: the next fetch may write it
    }
    flush();
}

template <auto Kernel>
cudaError_t norm_launch(const NormDev& P, const NormPlan& pl, cudaStream_t st) {
    if (pl.smem > 48 * 1024) {
        const cudaError_t e = hop_allow_max_smem<Kernel, kNormSmem>();
        if (e != cudaSuccess) return e;
    }
    return hop_launch_dependent(Kernel, dim3((pl.teams + pl.teams_per_block - 1) / pl.teams_per_block), pl.threads * pl.teams_per_block, pl.smem, st, P);
}
template <typename T, int NV, bool STAGED, bool LAYER, bool ASKEW, bool WARP, int MAXT, int BLOCKS>
cudaError_t norm_forward_launch(const NormDev& P, const NormPlan& pl, cudaStream_t st) { return norm_launch<norm_forward_kernel<T, NV, STAGED, LAYER, ASKEW, WARP, MAXT, BLOCKS>>(P, pl, st); }
template <typename T, int NV, bool STAGED, bool LAYER, bool ASKEW, bool WARP, int MAXT, int BLOCKS>
cudaError_t norm_backward_launch(const NormDev& P, const NormPlan& pl, cudaStream_t st) { return norm_launch<norm_backward_kernel<T, NV, STAGED, LAYER, ASKEW, WARP, MAXT, BLOCKS>>(P, pl, st); }

template <typename T, bool LAYER, bool ASKEW>
cudaError_t norm_sized(const NormDev& P, const NormPlan& pl, bool backward, cudaStream_t st) {
    const bool warp = pl.teams_per_block > 1, small = pl.threads <= 256;
    if (!backward) {
        if (!pl.stages) return norm_forward_launch<T, 2, false, LAYER, ASKEW, false, 1024, 1>(P, pl, st);
        if (warp && pl.nv == 1) return norm_forward_launch<T, 1, true, LAYER, ASKEW, true, 128, kWarpBlocks[0]>(P, pl, st);
        if (warp) return norm_forward_launch<T, 2, true, LAYER, ASKEW, true, 128, kWarpBlocks[0]>(P, pl, st);
        if (small) return norm_forward_launch<T, 2, true, LAYER, ASKEW, false, 256, kSmallBlocks[0]>(P, pl, st);
        return norm_forward_launch<T, 2, true, LAYER, ASKEW, false, 512, kLargeBlocks[0]>(P, pl, st);
    }
    if (!pl.stages && pl.nv == 2) return norm_backward_launch<T, 2, false, LAYER, ASKEW, false, 1024, 1>(P, pl, st);
    if (warp && pl.nv == 1) return norm_backward_launch<T, 1, true, LAYER, ASKEW, true, 128, kWarpBlocks[1]>(P, pl, st);
    if constexpr (LAYER) {
        if (pl.nv == 1 && small) return norm_backward_launch<T, 1, true, true, ASKEW, false, 256, kSmallBlocks[1]>(P, pl, st);
        if (pl.nv == 1) return norm_backward_launch<T, 1, true, true, ASKEW, false, 512, kLargeBlocks[1]>(P, pl, st);
    } else {
        if (warp) return norm_backward_launch<T, 2, true, false, ASKEW, true, 128, kWarpBlocks[1]>(P, pl, st);
        if (small) return norm_backward_launch<T, 2, true, false, ASKEW, false, 256, kSmallBlocks[1]>(P, pl, st);
    }
    return norm_backward_launch<T, 2, true, LAYER, ASKEW, false, 512, kLargeBlocks[1]>(P, pl, st);
}
template <typename T>
cudaError_t norm_typed(const NormDev& P, const NormPlan& pl, bool backward, bool askew, cudaStream_t st) {
    if (askew) return P.a.kind == HOP_NORM_LAYER ? norm_sized<T, true, true>(P, pl, backward, st) : norm_sized<T, false, true>(P, pl, backward, st);
    return P.a.kind == HOP_NORM_LAYER ? norm_sized<T, true, false>(P, pl, backward, st) : norm_sized<T, false, false>(P, pl, backward, st);
}

}  // namespace
