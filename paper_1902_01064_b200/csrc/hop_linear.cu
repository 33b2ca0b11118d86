// Grouped matrix products (hop_linear) on the 5th-generation tensor cores: y = x W_g^T, dx = dy W_g, dW_g = dy^T x over
// the rows of each group, with the groups' ends read on the device.
//
// One persistent kernel walks the result tiles of all groups (a tile never crosses a group).  A tile is 128 rows x BN
// columns per thread block; with CG = 2 two blocks of a cluster share one 256 x BN tile (cta_group::2), each holding its
// 128 rows and half of the B operand, so that a block fetches 32 KB per 64 terms instead of 48 KB: at full tensor rate
// 64 B per clock and SM, which the L2 can deliver (96 B it cannot).
//   warps 0, 3  producers: TMA loads of 64-term slices of A and of B into a ring of shared-memory stages (128-byte swizzle)
//   warp 1      MMA issue (one lane of the leading block): 4 x tcgen05.mma per slice into one of two accumulators
//   warp 2      weight gradients: zeroes the rows of a group's last slice that belong to the next group
//   warps 4-11  epilogue: accumulator -> registers -> global memory, a warp owns 32 rows and half of the columns
// Operands whose terms are contiguous (x and W forward, dy for dx) are K-major; the others (W for dx, dy and x for dW) are
// taken as they lie, MN-major, so nothing is ever transposed in memory.
//
// Accuracy: the tensor cores truncate at every accumulation step, always toward zero, so the error of a sum in them grows with
// its length: after 4096 / 65536 / 200 000 terms by 4.2e-6 / 6.6e-5 / 2.0e-4 of the result for terms of random sign, 2.4e-5 / 3.9e-4 /
// 1.3e-3 for terms of one sign.  For a float32 result the accumulator is therefore handed over every 768 terms and added in
// registers: 9e-7 for random signs and 4.4e-6 for one sign, at any length from there on (a plain float32 sum: 5e-7 to 3e-6 and 2e-7 to
// 1e-6); every 512 terms cost 8 % more clocks.  A 16-bit result is rounded as it leaves tensor memory while the truncation of
// the worst case, terms of one sign, stays below 1/18 of half a unit of the type: up to 4096 terms in half precision, 32768 in bfloat16.
// Longer ones, of which for dW only the rows of all groups together are known at the launch, take the float32 form and are rounded
// at the store: dW of 8192 rows of 4096 x 4096 in half precision 191 -> 201 us, 8 groups of 2048 rows of 4096 x 1024 no slower.
//
// What bounds it, measured on a B200 (bf16): tensor cores with groups of many rows -- 8192 x 4096 x 4096 forward 163 us
// (1680 TFLOP/s; 520 clocks a 64-term slice of a pair's tile, 512 at full rate), dx the same, dW 182 us to float32 and 164 us
// to bf16; weights' bytes with groups of few -- 64 groups of 8 rows of 2048 x 2048 101 us (5.3 TB/s); a kernel's length,
// 4.8 us from start to end, with little of either.  One block's 128 x 128 tile is bound by its shared memory (~625 clocks a
// slice, at half a pair's rate a block): it is for groups whose rows do not fill half of a pair's tile.
//
// All waits are bounded: one that runs out sets g_linear_error, the block lets its copies land, frees its tensor memory and
// returns.
#include <cuda.h>            // CUtensorMap and the cuTensorMapEncodeTiled prototype only; no libcuda link

#include "hop_internal.h"
#include "hop_ops.cuh"

namespace {

constexpr int kBK = 64;                     // terms per slice: 128 bytes, one swizzle row
constexpr int kStages = 6;
constexpr int kThreads = 12 * 32;
constexpr int kEpiWarps = 8;
constexpr int kPromote = 12;                // slices per accumulator hand-over: 768 terms
constexpr int kLongF16 = 4096, kLongBF16 = 32768;       // terms above which 16-bit results are handed over too
constexpr int kBand = 8;                    // row tiles that take their column tiles together (L2 reuse of both operands)
constexpr uint64_t kWaitNs = 10ull * 1000 * 1000 * 1000;

__device__ int32_t g_linear_error;

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mb_init(uint64_t* b, uint32_t c) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(s32(b)), "r"(c)); }
__device__ __forceinline__ uint32_t leader_addr(const void* p) {      // the same place in the cluster's first block
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(s32(p)));
    return r;
}
__device__ __forceinline__ void mb_expect(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(s32(b)), "r"(bytes) : "memory");
}
// RELEASE: what the thread wrote to shared memory is ordered before the arrival for the other block.  Without it the arrival
// says that tensor memory has been read, which the tcgen05 fence in front orders; a release at cluster scope would wait for
// the result's stores in flight (1000 clocks a tile).
template <int CG, bool RELEASE = true>
__device__ __forceinline__ void mb_arrive(uint64_t* b, uint32_t lead) {
    if constexpr (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(s32(b)) : "memory");
    else if constexpr (RELEASE) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(lead) : "memory");
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(lead) : "memory");
}
// One try, which may put the thread to sleep for up to 20 us
template <int CG>
__device__ __forceinline__ bool mb_try(uint64_t* b, uint32_t ph) {
    uint32_t ok;
    if constexpr (CG == 1)
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(s32(b)), "r"(ph), "r"(20000u) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(s32(b)), "r"(ph), "r"(20000u) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() { uint64_t t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
// Bounded: gives up after kWaitNs, or when another warp has.  (The longest a warp waits for another one's work is a 16-bit tile of
// kLongBF16 terms, a millisecond; the others are handed over in pieces.)
// PATIENT: between tries the thread sleeps (the epilogue's 256 threads, trying without a pause, slowed the tensor cores of
// their SM by a quarter: they share its shared-memory pipe).
template <int CG, bool PATIENT = false>
__device__ __forceinline__ bool mb_wait(uint64_t* b, uint32_t ph, volatile int* gave_up, uint64_t most_ns = kWaitNs) {
    if (mb_try<CG>(b, ph)) return true;
    const uint64_t start = now_ns();
    for (uint32_t it = 1;; ++it) {
        if constexpr (PATIENT) __nanosleep(100);
        if (mb_try<CG>(b, ph)) return true;
        if ((it & 63) == 0 && (*gave_up || now_ns() - start > most_ns)) return false;
    }
}
// The same for a whole warp, which goes on (or gives up) together
template <int CG>
__device__ __forceinline__ bool warp_wait(uint64_t* b, uint32_t ph, volatile int* gave_up, uint64_t most_ns = kWaitNs) {
    bool ok = true;
    if ((threadIdx.x & 31) == 0) ok = mb_wait<CG, true>(b, ph, gave_up, most_ns);
    ok = __all_sync(0xffffffffu, ok);
    return ok && __all_sync(0xffffffffu, mb_try<CG>(b, ph));      // (passed: at once; every lane then sees what the barrier ordered)
}
// TMA loads; PAIR: the bytes are counted at the leading block's barrier (bar is its address there)
template <bool PAIR>
__device__ __forceinline__ void tma2(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(m), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(m), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tma3(uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(m), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(m), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory matrix descriptor, 128-byte swizzle (layout type 2), descriptor version 1.  K-major: 8-row groups 1024 bytes
// apart (the leading offset is unused).  MN-major: 8-term groups 1024 bytes apart, 64-element pieces 8192 bytes apart.
template <bool MN>
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(MN ? 8192 >> 4 : 1) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {      // arrives at this place in every block of the pair
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(s32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(s32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
template <int CG>
__device__ __forceinline__ void sync_all() {
    if constexpr (CG == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}
__device__ __forceinline__ void tmem_ld32(uint32_t t, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
                   "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]),
                   "=r"(v[30]), "=r"(v[31]) : "r"(t) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t t, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(t) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
struct TcArgs {
    const int32_t* offsets;
    int64_t rows;
    int32_t groups, n, k, w_step;           // w_step 0: one weight matrix for all groups (its map has one plane)
    void* out;
    int64_t out_group_stride, out_stride;
    int32_t out_dtype, accumulate, vec;     // vec: every row of the result starts on a boundary of 16 or 4 bytes, else 0
    int32_t splits; int64_t part_stride;    // splits > 1: part p of a tile's terms goes to out + p * part_stride
    uint32_t idesc, deep;                   // deep: dW operands whose map has 64-column blocks as third dimension (bit 0 A, bit 1 B)
};

struct TcControl {
    uint64_t full[kStages], empty[kStages], tail[kStages], peer_tail[kStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int gave_up;
    int32_t row0[HOP_MAX_GROUPS + 2];       // first row of each group; [groups]: behind the last one; [groups + 1]: rows
    int32_t tile0[HOP_MAX_GROUPS + 2];      // first tile of each group
};

// How a result leaves the kernel: 16 bits, rounded as it leaves tensor memory; float32 sums; or 16 bits rounded once from float32
// sums, which are long or have what the result holds added first.
enum Result { kDirect, kFloat, kRounded };

__device__ __forceinline__ float2 widen2(uint32_t v, bool half) {
    return half ? __half22float2(*reinterpret_cast<const __half2*>(&v)) : __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v));
}
__device__ __forceinline__ uint32_t round2(float x, float y, bool half) {
    if (half) { const __half2 h = __floats2half2_rn(x, y); return *reinterpret_cast<const uint32_t*>(&h); }
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Writes up to 16 rows of 64 16-bit columns, `cols` of which exist, out of the warp's shared memory where rows lie off the
// 16-byte grid or the block over the last column: a lane takes two columns of each row.  Not inlined and rolled: inlined into
// every block of a tile this form took 14000 clocks a tile, nearly all of it instruction fetch.
__device__ __noinline__ void write_rows16(char* base, int64_t row_bytes, int rows, int cols, int vec, const unsigned char* scr, int lane) {
    const int c = lane * 2;
    const bool both = c + 2 <= cols;
    if (vec >= 4) {
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
            uint32_t v[8];
            char* p = base + (int64_t)r0 * row_bytes + lane * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const uint32_t*>(scr + (r0 + i) * 128 + (((lane >> 2) ^ ((r0 + i) & 7)) << 4) + (lane & 3) * 4);
#pragma unroll
            for (int i = 0; i < 8; ++i, p += row_bytes) {
                if (r0 + i < rows && both) *reinterpret_cast<uint32_t*>(p) = v[i];
                else if (r0 + i < rows && c < cols) *reinterpret_cast<uint16_t*>(p) = (uint16_t)v[i];
            }
        }
        return;
    }
    // odd rows: consecutive elements to consecutive lanes, so that every second store is not a hole
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 4) {
        uint16_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + (i >> 1), b = ((i & 1) * 32 + lane) * 2;
            v[i] = *reinterpret_cast<const uint16_t*>(scr + r * 128 + (((b >> 4) ^ (r & 7)) << 4) + (b & 15));
        }
        char* p = base + (int64_t)r0 * row_bytes + lane * 2;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + (i >> 1) < rows && (i & 1) * 32 + lane < cols) *reinterpret_cast<uint16_t*>(p + (i >> 1) * row_bytes + (i & 1) * 64) = v[i];
    }
}
// Writes a warp's block of the result, 32 rows (a lane holds one) of 128 bytes: through the warp's 2 KB of shared memory, 16
// rows at a time (16-byte units exchanged by row against bank conflicts), so that a store instruction covers whole 128-byte
// lines: with a lane storing its own row, 32 bytes at a time, the stores of float32 tiles held the tensor cores up (664
// clocks a slice, 551 without the stores).
template <int OUT>
__device__ __forceinline__ void put_block(const TcArgs& a, char* base, int64_t row_bytes, int rows, int cols, const uint32_t (&w)[32], unsigned char* scr, int lane) {
    if (rows <= 0 || cols <= 0) return;         // (the same for the whole warp)
    const bool half = a.out_dtype == HOP_DT_F16;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (h * 16 >= rows) break;
        if ((lane >> 4) == h) {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                *reinterpret_cast<uint4*>(scr + (lane & 15) * 128 + ((u ^ (lane & 7)) << 4)) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
        }
        __syncwarp();
        if (cols >= (OUT == kDirect ? 64 : 32) && a.vec >= 16) {
            char* p = base + (int64_t)(h * 16 + (lane >> 3)) * row_bytes + (lane & 7) * (OUT == kRounded ? 8 : 16);
            uint2 old[4];       // all four fetched before the first store, which the compiler may not move them over
            if constexpr (OUT == kRounded) {
#pragma unroll
                for (int i = 0; i < 4; ++i) old[i] = h * 16 + i * 4 + (lane >> 3) < rows ? *reinterpret_cast<const uint2*>(p + i * 4 * row_bytes) : make_uint2(0u, 0u);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i, p += 4 * row_bytes) {
                const int r = i * 4 + (lane >> 3);
                const uint4 q = *reinterpret_cast<const uint4*>(scr + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                if (h * 16 + r >= rows) continue;
                if constexpr (OUT == kDirect) {
                    *reinterpret_cast<uint4*>(p) = q;
                } else {
                    float4 f = make_float4(__uint_as_float(q.x), __uint_as_float(q.y), __uint_as_float(q.z), __uint_as_float(q.w));
                    if constexpr (OUT == kFloat) {
                        if (a.accumulate) { const float4 o = *reinterpret_cast<const float4*>(p); f.x += o.x; f.y += o.y; f.z += o.z; f.w += o.w; }
                        *reinterpret_cast<float4*>(p) = f;
                    } else {
                        const float2 x = widen2(old[i].x, half), y = widen2(old[i].y, half);
                        *reinterpret_cast<uint2*>(p) = make_uint2(round2(f.x + x.x, f.y + x.y, half), round2(f.z + y.x, f.w + y.y, half));
                    }
                }
            }
        } else if constexpr (OUT != kDirect) {  // a column a lane (inlined but rolled: a call would spill the tile's sums)
            constexpr int kSize = OUT == kFloat ? 4 : 2;
#pragma unroll 1
            for (int r0 = 0; r0 < 16 && h * 16 + r0 < rows; r0 += 4) {
                float v[4];
                char* p = base + (int64_t)(h * 16 + r0) * row_bytes + lane * kSize;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float*>(scr + (r0 + i) * 128 + (((lane >> 2) ^ ((r0 + i) & 7)) << 4) + (lane & 3) * 4);
                if (OUT == kRounded || a.accumulate) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (h * 16 + r0 + i >= rows || lane >= cols) continue;
                        if constexpr (OUT == kFloat) v[i] += *reinterpret_cast<const float*>(p + i * row_bytes);
                        else v[i] += widen2(*reinterpret_cast<const uint16_t*>(p + i * row_bytes), half).x;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i, p += row_bytes) {
                    if (h * 16 + r0 + i >= rows || lane >= cols) continue;
                    if constexpr (OUT == kFloat) *reinterpret_cast<float*>(p) = v[i];
                    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)round2(v[i], 0.f, half);
                }
            }
        } else {
            write_rows16(base + h * 16 * row_bytes, row_bytes, min(16, rows - h * 16), cols, a.vec, scr, lane);
        }
        __syncwarp();
    }
}

template <int CG, int BN, int WAY, int OUT>
__global__ void __launch_bounds__(kThreads, 1)
linear_tc_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ TcArgs a) {
    constexpr bool PROMOTE = OUT != kDirect;                // float32 sums in registers
    constexpr bool DW = WAY == HOP_LINEAR_DW, A_MN = DW, B_MN = WAY != HOP_LINEAR_FORWARD;
    constexpr int TM = 128 * CG;                            // rows of a tile
    constexpr int BNB = BN / CG;                            // columns whose operand this block fetches
    constexpr int kABytes = 128 * kBK * 2, kBBytes = BNB * kBK * 2, kStageBytes = kABytes + kBBytes;
    // Forward and dx of small groups fetch rows in boxes of 32: a group of a few rows reads a few rows
    constexpr int kABox = CG == 1 ? 32 : 128;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (s32(smem_raw) & 1023)) & 1023);
    TcControl* cb = reinterpret_cast<TcControl*>(smem + kStages * kStageBytes + kEpiWarps * 2048);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = CG == 1 ? 0u : (blockIdx.x & 1u);
    volatile int* gave_up = &cb->gave_up;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { mb_init(&cb->full[s], 1); mb_init(&cb->empty[s], 1); mb_init(&cb->tail[s], 1); mb_init(&cb->peer_tail[s], 1); }
        for (int b = 0; b < 2; ++b) { mb_init(&cb->acc_full[b], 1); mb_init(&cb->acc_empty[b], CG * kEpiWarps); }
        cb->gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 3 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapA) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapB) : "memory");
    }
    if (warp == 2) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(&cb->tmem)), "n"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(&cb->tmem)), "n"(2 * BN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    dependency_wait();      // what comes before touches nothing of the caller's
    // Group starts (clamped into [0, rows] and made non-decreasing, whatever offsets holds) and tile counts
    const int col_tiles = ((WAY == HOP_LINEAR_FORWARD ? a.n : a.k) + BN - 1) / BN;
    for (int i = tid; i <= a.groups + 1; i += kThreads) {
        int64_t o = i == 0 ? 0 : i > a.groups ? a.rows : !a.offsets ? a.rows : (int64_t)a.offsets[i];
        cb->row0[i] = (int32_t)min(max(o, (int64_t)0), a.rows);
    }
    __syncthreads();
    const int tiled_groups = DW ? a.groups : a.groups + 1;      // rows behind the last group form one that is only zeroed
    if (warp == 0) {
        int top = 0;
        for (int base = 0; base <= a.groups + 1; base += 32) {
            const int i = base + lane;
            int v = i <= a.groups + 1 ? cb->row0[i] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v = max(v, u); }
            v = max(v, top);
            top = __shfl_sync(0xffffffffu, v, 31);
            if (i <= a.groups + 1) cb->row0[i] = v;
        }
        __syncwarp();
        int sum = 0;
        for (int base = 0; base < tiled_groups; base += 32) {
            const int i = base + lane;
            int v = 0;
            if (i < tiled_groups) v = col_tiles * (DW ? (a.n + TM - 1) / TM : (cb->row0[i + 1] - cb->row0[i] + TM - 1) / TM);
            int inc = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += u; }
            if (i < tiled_groups) cb->tile0[i] = sum + inc - v;
            sum += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) cb->tile0[tiled_groups] = sum;
    }
    fence_before();
    sync_all<CG>();
    fence_after();
    if (a.splits > 1) launch_dependents();
    const uint32_t tmem = cb->tmem;
    const int tiles = cb->tile0[tiled_groups] * a.splits;
    const int step = gridDim.x / CG, first = blockIdx.x / CG;

    int g = 0;
    struct Tile { int64_t row; int rows_left, col, part; int t0, x0, len, slices; } t;
    // The group of a unit (unit numbers only grow, so it is found by walking on) and the terms it has; all the MMA warp needs
    auto depth = [&](int unit) {
        const int tile = a.splits > 1 ? unit / a.splits : unit;
        while (tile >= cb->tile0[g + 1]) ++g;
        t.t0 = cb->row0[g];
        t.len = DW ? cb->row0[g + 1] - t.t0 : g < a.groups ? (WAY == HOP_LINEAR_FORWARD ? a.k : a.n) : 0;
        t.slices = (t.len + kBK - 1) / kBK;
        t.part = t.x0 = 0;
        if (a.splits > 1) {             // this part's slices
            t.part = unit - tile * a.splits;
            const int per = (t.slices + a.splits - 1) / a.splits, c0 = min(t.part * per, t.slices);
            t.slices = min(per, t.slices - c0);
            t.x0 = c0 * kBK;
            t.len = min(t.len - t.x0, t.slices * kBK);
            if (DW) { t.t0 += t.x0; t.x0 = 0; }
        }
        return tile;
    };
    auto locate = [&](int unit) {
        const int at = depth(unit) - cb->tile0[g], r0 = cb->row0[g], r1 = cb->row0[g + 1];
        const int row_tiles = ((DW ? a.n : r1 - r0) + TM - 1) / TM;
        const int band = at / (kBand * col_tiles), in = at - band * kBand * col_tiles;
        const int wide = min(kBand, row_tiles - band * kBand), nt = in / wide;
        t.col = nt * BN;
        t.row = (DW ? 0 : r0) + (int64_t)(band * kBand + in - nt * wide) * TM;
        t.rows_left = (int)((DW ? a.n : r1) - t.row);
    };
    bool ok = true;
    int site = 0;

    if (warp == 0 || warp == 3) {
        // ------------------------------------------------ producers: warp 0 the A operand, warp 3 the B operand (a warp
        // issues a TMA load in ~90 clocks, so one alone is behind the tensor cores with four or five loads a slice)
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            for (int tile = first; tile < tiles && ok; tile += step) {
                locate(tile);
                // boxes of A rows this block fetches, and the bytes of a slice in all blocks of the pair: the leading block
                // alone announces them (a remote arrival per slice cost its thread ~1000 clocks; the peer's bytes may come
                // in before that, the count is signed and the phase still waits for the arrival)
                const int row = (int)t.row + (int)rank * 128, left = t.rows_left - (int)rank * 128;
                auto boxes_of = [&](int l) { return DW || l <= 0 ? 0 : min(128 / kABox, (l + kABox - 1) / kABox); };
                const int boxes = boxes_of(left);
                const uint32_t bytes = DW ? CG * kStageBytes : CG * kBBytes + (boxes + (CG == 2 ? boxes_of(left - 128) : 0)) * kABox * kBK * 2;
                const int wg = g * a.w_step, bcol = t.col + (int)rank * BNB;
                for (int c = 0; c < t.slices; ++c) {
                    if (!mb_wait<CG>(&cb->empty[s], ph ^ 1u, gave_up)) { ok = false; site = 1; break; }
                    const uint32_t sa = s32(smem) + s * kStageBytes, sb = sa + kABytes;
                    const int x = c * kBK;                      // (dx and forward: from the part's first term)
                    const bool tail = DW && t.len - x < kBK && (t.len & 15);      // other groups' rows follow: warp 2 sees them first
                    if (warp == 0) {
                        if (tail) mb_expect(&cb->tail[s], kStageBytes);
                        else if (rank == 0) mb_expect(&cb->full[s], bytes);
                    }
                    auto load = [&](auto pair, uint32_t bar) {
                        constexpr bool PAIR = decltype(pair)::value;
                        if (warp == 0) {
                            if constexpr (DW) {
                                if (a.deep & 1) tma3<PAIR>(sa, &mapA, 0, t.t0 + x, row / 64, bar);
                                else
#pragma unroll
                                    for (int i = 0; i < 2; ++i) tma2<PAIR>(sa + i * 8192, &mapA, row + i * 64, t.t0 + x, bar);
                            } else {
                                for (int i = 0; i < boxes; ++i) tma2<PAIR>(sa + i * kABox * kBK * 2, &mapA, t.x0 + x, row + i * kABox, bar);
                            }
                        } else if constexpr (DW) {
                            if (a.deep & 2) tma3<PAIR>(sb, &mapB, 0, t.t0 + x, bcol / 64, bar);
                            else
#pragma unroll
                                for (int i = 0; i < BNB / 64; ++i) tma2<PAIR>(sb + i * 8192, &mapB, bcol + i * 64, t.t0 + x, bar);
                        } else if constexpr (B_MN) {
#pragma unroll
                            for (int i = 0; i < BNB / 64; ++i) tma3<PAIR>(sb + i * 8192, &mapB, bcol + i * 64, t.x0 + x, wg, bar);
                        } else {
                            tma3<PAIR>(sb, &mapB, t.x0 + x, bcol, wg, bar);
                        }
                    };
                    if (tail) load(std::false_type{}, s32(&cb->tail[s]));
                    else load(std::integral_constant<bool, CG == 2>{}, CG == 1 ? s32(&cb->full[s]) : leader_addr(&cb->full[s]));
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issue
        if (lane == 0 && rank == 0) {
            // descriptors of stage 0; a 16-term step is 32 bytes along a K-major row, 16 rows of 128 bytes MN-major
            constexpr uint64_t kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;
            const uint64_t desc_a = smem_desc<A_MN>(s32(smem)), desc_b = smem_desc<B_MN>(s32(smem) + kABytes);
            int s = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            for (int tile = first; tile < tiles && ok; tile += step) {
                depth(tile);
                int c = 0;
                while (c < t.slices && ok) {
                    const int stop = PROMOTE ? min(t.slices, c + kPromote) : t.slices;
                    if (!mb_wait<CG>(&cb->acc_empty[buf], aph ^ 1u, gave_up)) { ok = false; site = 2; break; }
                    fence_after();
                    const uint32_t d = tmem + buf * BN;
                    uint32_t more = 0;                          // the first MMA of an accumulator overwrites it
                    for (int c1 = c; c1 < stop; ++c1) {
                        if (!mb_wait<CG>(&cb->full[s], ph, gave_up)) { ok = false; site = 3; break; }
                        fence_after();
                        const uint64_t da = desc_a + (uint64_t)(s * (kStageBytes >> 4)), db = desc_b + (uint64_t)(s * (kStageBytes >> 4));
                        const int left = t.len - c1 * kBK;
                        if (!DW || left >= kBK) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                mma<CG>(d, da + j * kStepA, db + j * kStepB, a.idesc, more);
                                more = 1;
                            }
                        } else {
                            for (int j = 0; j * 16 < left; ++j) {
                                mma<CG>(d, da + j * kStepA, db + j * kStepB, a.idesc, more);
                                more = 1;
                            }
                        }
                        mma_commit<CG>(&cb->empty[s]);
                        if (++s == kStages) { s = 0; ph ^= 1u; }
                    }
                    if (!ok) break;
                    mma_commit<CG>(&cb->acc_full[buf]);
                    c = stop;
                    if (++buf == 2) { buf = 0; aph ^= 1u; }
                }
            }
        }
    } else if (warp == 2) {
        // ------------------------------------------------ zeroes what a group's last slice holds of other rows: the rows
        // from the group's end to the end of the 16-term step that contains it (their values could be infinite or NaN, so
        // both operands are cleared; a row of a 64-element piece is 128 contiguous bytes whatever the swizzle)
        if constexpr (DW) {
            int at = 0;
            uint32_t tph = 0, pph = 0;
            for (int tile = first; tile < tiles && ok; tile += step) {
                depth(tile);
                if (t.slices && (t.len & 15)) {
                    const int s = (at + t.slices - 1) % kStages;
                    if (!warp_wait<1>(&cb->tail[s], (tph >> s) & 1u, gave_up)) { ok = false; site = 4; break; }
                    tph ^= 1u << s;         // (a barrier per stage: the producer may be several one-slice tiles ahead)
                    const int r0 = t.len - (t.slices - 1) * kBK, r1 = (r0 + 15) & ~15;
                    for (int i = lane; i < (r1 - r0) * (kStageBytes / 1024); i += 32) {
                        const int r = r0 + (i >> 3) % (r1 - r0), piece = (i >> 3) / (r1 - r0);
                        *reinterpret_cast<uint4*>(smem + s * kStageBytes + piece * 8192 + r * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if constexpr (CG == 2) {        // the leading block passes both blocks' slices on
                        if (rank == 1) { if (lane == 0) mb_arrive<2>(nullptr, leader_addr(&cb->peer_tail[s])); }
                        else if (!warp_wait<2>(&cb->peer_tail[s], (pph >> s) & 1u, gave_up)) { ok = false; site = 6; break; }
                        pph ^= 1u << s;
                    }
                    if (lane == 0 && rank == 0) mb_arrive<1>(&cb->full[s], 0u);
                }
                at = (at + t.slices) % kStages;
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ epilogue
        constexpr int HC = BN / 2;                              // columns of this warp
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        int buf = 0;
        uint32_t aph = 0;
        const uint32_t lead_empty[2] = {CG == 1 ? 0u : leader_addr(&cb->acc_empty[0]), CG == 1 ? 0u : leader_addr(&cb->acc_empty[1])};
        constexpr int kCols = OUT == kFloat ? 32 : 64, kSize = OUT == kFloat ? 4 : 2;
        unsigned char* scr = smem + kStages * kStageBytes + (warp - 4) * 2048;
        const int64_t row_bytes = a.out_stride * kSize;
        const bool f16 = a.out_dtype == HOP_DT_F16;
        for (int tile = first; tile < tiles && ok; tile += step) {
            locate(tile);
            const int in_tile = (int)rank * 128 + quarter * 32, live = min(32, t.rows_left - in_tile);
            const int col0 = t.col + half * HC, left = (WAY == HOP_LINEAR_FORWARD ? a.n : a.k) - col0;
            char* at = reinterpret_cast<char*>(a.out) + (t.part * a.part_stride + (DW ? (int64_t)g * a.out_group_stride : 0) + (t.row + in_tile) * a.out_stride + col0) * kSize;
            if (t.slices == 0) {
                if (!(DW && a.accumulate)) {
                    uint32_t z[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) z[i] = 0u;
#pragma unroll 1
                    for (int i = 0; i < HC; i += kCols) put_block<OUT == kFloat ? kFloat : kDirect>(a, at + i * kSize, row_bytes, live, left - i, z, scr, lane);
                }
                continue;
            }
            if constexpr (PROMOTE) {
                float acc[HC];
#pragma unroll
                for (int i = 0; i < HC; ++i) acc[i] = 0.f;
                for (int c = 0; c < t.slices; c += kPromote) {
                    if (!warp_wait<CG>(&cb->acc_full[buf], aph, gave_up)) { ok = false; site = 5; break; }
                    fence_after();
#pragma unroll
                    for (int i = 0; i < HC; i += 16) {
                        uint32_t v[16];
                        tmem_ld16(tmem + lanes + buf * BN + half * HC + i, v);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[i + e] += __uint_as_float(v[e]);
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mb_arrive<CG, false>(&cb->acc_empty[buf], lead_empty[buf]);
                    if (++buf == 2) { buf = 0; aph ^= 1u; }
                }
                if (!ok) break;
                if (OUT == kRounded && !a.accumulate) {
#pragma unroll
                    for (int i = 0; i < HC; i += 64) {
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) w[e] = round2(acc[i + 2 * e], acc[i + 2 * e + 1], f16);
                        put_block<kDirect>(a, at + i * 2, row_bytes, live, left - i, w, scr, lane);
                    }
                    continue;
                }
#pragma unroll
                for (int i = 0; i < HC; i += 32) {
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(acc[i + e]);
                    put_block<OUT>(a, at + i * kSize, row_bytes, live, left - i, w, scr, lane);
                }
            } else {
                if (!warp_wait<CG>(&cb->acc_full[buf], aph, gave_up)) { ok = false; site = 5; break; }
                fence_after();
#pragma unroll 1
                for (int i = 0; i < HC; i += 64) {
                    uint32_t w[32];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t v[32];
                        tmem_ld32(tmem + lanes + buf * BN + half * HC + i + k * 32, v);
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[k * 16 + e] = round2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]), f16);
                    }
                    if (i + 64 == HC) {                         // everything is in registers: the accumulator is free
                        fence_before();
                        __syncwarp();
                        if (lane == 0) mb_arrive<CG, false>(&cb->acc_empty[buf], lead_empty[buf]);
                    }
                    put_block<OUT>(a, at + i * 2, row_bytes, live, left - i, w, scr, lane);
                }
                if (++buf == 2) { buf = 0; aph ^= 1u; }
            }
        }
    }
    if (!ok) {      // a wait ran out: tell the host and the other warps, and let the copies in flight land
        atomicCAS(&g_linear_error, 0, (6 << 24) | site);
        cb->gave_up = 1;
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    __syncwarp();
    fence_before();
    sync_all<CG>();
    if (warp == 2) {
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * BN) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * BN) : "memory");
    }
}

// Self-test of the bounded wait: one warp waits on a barrier that nothing completes, gives up and records it.
constexpr int kSelftestSite = 0xffffff;
__global__ void __launch_bounds__(32)
linear_wait_selftest_kernel(uint64_t most_ns) {
    __shared__ uint64_t bar;
    __shared__ int gave_up;
    if (threadIdx.x == 0) {
        mb_init(&bar, 1);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (!warp_wait<1>(&bar, 0u, &gave_up, most_ns) && threadIdx.x == 0) atomicCAS(&g_linear_error, 0, (6 << 24) | kSelftestSite);
}

// Adds the parts of a split product in order and writes the result: four columns a thread.
template <typename O>
__global__ void __launch_bounds__(256)
linear_join_kernel(const float* part, int64_t part_stride, int splits, int64_t rows, int64_t rows_per_group, int cols, int padded, O* out,
                   int64_t group_stride, int64_t row_stride, int accumulate) {
    const int quads = padded / 4;
    dependency_wait();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * quads; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = i / quads;
        const int c = (int)(i - r * quads) * 4;
        const float* p = part + r * padded + c;
        float4 v = *reinterpret_cast<const float4*>(p);
#pragma unroll 4
        for (int s = 1; s < splits; ++s) {
            const float4 w = *reinterpret_cast<const float4*>(p + s * part_stride);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
        const int64_t g = rows_per_group ? r / rows_per_group : 0;
        O* o = out + g * group_stride + (r - g * rows_per_group) * row_stride + c;
        const float q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < cols) o[e] = op_t<O>(accumulate ? op_f(o[e]) + q[e] : q[e]);
    }
}

// Copies rows of 16-bit elements whose address or stride TMA cannot take into rows of whole 16-byte units (what pads them
// is never read as a term).  A warp takes a row, 256 columns and four such pieces at a time: whole units in, shifted into
// place, whole units out.
struct PackArgs { const uint16_t* src[2]; int64_t group_stride[2], row_stride[2], rows[2], all[2]; int cols[2], units[2]; uint4* dst[2]; const int32_t* offsets; };
__global__ void __launch_bounds__(256)
linear_pack_kernel(const __grid_constant__ PackArgs a) {
    constexpr int N = 4;
    const int lane = threadIdx.x & 31;
    const int64_t step = (int64_t)gridDim.x * 8;
    dependency_wait();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int units = a.units[k], cols = a.cols[k];
        int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
        if (row >= a.all[k]) continue;
        int64_t in = row % a.rows[k];
        int g = (int)(row / a.rows[k]);
        const uint16_t* src = a.src[k] + g * a.group_stride[k];
        for (; row < a.all[k]; row += step, in += step) {
            while (in >= a.rows[k]) { in -= a.rows[k]; src += a.group_stride[k]; ++g; }
            // weights of a group without rows are not read
            if (k == 1 && a.offsets && a.offsets[g + 1] <= (g ? a.offsets[g] : 0)) continue;
            const char* p0 = reinterpret_cast<const char*>(src + in * a.row_stride[k]);
            const uint32_t m = (uint32_t)(reinterpret_cast<uintptr_t>(p0) & 15);
            const uint4* q = reinterpret_cast<const uint4*>(p0 - m);        // (a unit with a byte of the row lies in the row's allocation)
            const int touched = ((int)m + cols * 2 + 15) / 16;
            uint4* out = a.dst[k] + row * units;
            for (int u0 = 0; u0 < units; u0 += 32 * N) {
                uint4 u[N], last[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int at = u0 + j * 32 + lane;
                    u[j] = last[j] = make_uint4(0u, 0u, 0u, 0u);
                    if (at < touched) u[j] = q[at];
                    if (lane == 31 && at + 1 < touched) last[j] = q[at + 1];
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (u0 + j * 32 >= units) break;
                    uint32_t w[8] = {u[j].x, u[j].y, u[j].z, u[j].w, 0u, 0u, 0u, 0u};
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[4 + e] = __shfl_down_sync(0xffffffffu, w[e], 1);
                    if (lane == 31) { w[4] = last[j].x; w[5] = last[j].y; w[6] = last[j].z; w[7] = last[j].w; }
                    op_shift_words(w, m);
                    if (u0 + j * 32 + lane < units) out[u0 + j * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
    }
    launch_dependents();
}

// ------------------------------------------------------------------------------------------------ host side
int linear_check(const hop_linear_args* a, char* eb, int64_t el) {
    const char* who = "hop_linear";
    if (!a) return hop_op_fail(eb, el, HOP_E_ARG, "%s: null arguments", who);
    if (a->way < HOP_LINEAR_FORWARD || a->way > HOP_LINEAR_DW) return hop_op_fail(eb, el, HOP_E_ARG, "%s: unknown way %d", who, a->way);
    if (!hop_op_dtype_ok(a->dtype) || !hop_op_dtype_ok(a->out_dtype)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: unknown dtype", who);
    if (a->dtype == HOP_DT_F32) return hop_op_fail(eb, el, HOP_E_UNSUPPORTED, "%s: operands are float16 or bfloat16", who);
    if (a->out_dtype != HOP_DT_F32 && a->out_dtype != a->dtype) return hop_op_fail(eb, el, HOP_E_UNSUPPORTED, "%s: the result is float32 or of the operands' type", who);
    if (a->accumulate && a->way != HOP_LINEAR_DW) return hop_op_fail(eb, el, HOP_E_UNSUPPORTED, "%s: only weight gradients accumulate", who);
    // (tiles of up to 256 rows and slices of 64 are counted in signed 32 bits, rounded up)
    if (a->rows < 0 || a->rows > (1ll << 31) - 256) return hop_op_fail(eb, el, HOP_E_ARG, "%s: %lld rows (0 .. 2^31-256)", who, (long long)a->rows);
    if (a->n < 1 || a->k < 1 || a->n > (1 << 29) || a->k > (1 << 29)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: n = %d, k = %d", who, a->n, a->k);
    if (a->groups < 1 || a->groups > HOP_MAX_GROUPS) return hop_op_fail(eb, el, HOP_E_ARG, "%s: %d groups (1 .. %d)", who, a->groups, HOP_MAX_GROUPS);
    if (!a->offsets && a->groups != 1) return hop_op_fail(eb, el, HOP_E_ARG, "%s: several groups need offsets", who);
    const int cols = a->way == HOP_LINEAR_FORWARD ? a->n : a->k;
    const double row_tiles = a->way == HOP_LINEAR_DW ? (double)a->groups * (a->n / 128 + 1) : (double)a->rows / 128 + a->groups + 1;
    if (row_tiles * (cols / 64 + 1) >= 2147483647.0) return hop_op_fail(eb, el, HOP_E_ARG, "%s: more than 2^31 tiles", who);
    return HOP_OK;
}

// An operand as the kernel takes it: [groups][rows][cols], in place when TMA can address it, else packed into the workspace.
struct Operand {
    const void* p; int64_t group_stride, stride, rows; int cols, groups;
    bool packed; int64_t at;                // offset in the workspace
    int64_t packed_bytes() const { return (int64_t)groups * rows * ((cols + 7) / 8) * 16; }
};
bool tma_can(const Operand& o) {
    if (((uintptr_t)o.p & 15) || o.stride * 2 % 16 || o.stride < o.cols || o.stride >= (1ll << 38)) return false;
    return o.groups == 1 || (o.group_stride * 2 % 16 == 0 && o.group_stride > 0 && o.group_stride < (1ll << 38));
}
// How a call is carried out: its operands, tile shape, parts, and where things lie in the workspace
struct Plan { Operand op[2]; bool pair; int bn, splits, padded; int64_t out_rows, part_at, bytes; };

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

Plan linear_plan(const hop_linear_args& a) {
    Plan p;
    const bool fwd = a.way == HOP_LINEAR_FORWARD, dw = a.way == HOP_LINEAR_DW;
    p.op[0] = {a.a, 0, a.a_stride, a.rows, fwd ? a.k : a.n, 1, false, 0};
    if (dw) p.op[1] = {a.b, 0, a.b_stride, a.rows, a.k, 1, false, 0};
    else p.op[1] = {a.w, a.w_group_stride, a.w_stride, a.n, a.k, a.w_group_stride == 0 ? 1 : a.groups, false, 0};
    int64_t at = 0;
    for (Operand& o : p.op) {
        o.packed = !tma_can(o);
        if (o.packed) { o.at = at; at += ceil_div(o.packed_bytes(), 256) * 256; }
    }
    // Pairs of blocks (256 x 256 tiles) where groups fill more than half of such a tile's rows and there are enough tiles for
    // the rounds to take no longer: a pair spends ~525 clocks a slice on a tile, one block ~625 on a quarter of it (its shared
    // memory is the limit).  What is known here of the groups is their number: half of them are taken to end inside a tile.
    const int cols = fwd ? a.n : a.k;
    const int64_t live = std::min<int64_t>(a.groups, a.rows);
    auto row_tiles = [&](int tm) { return dw ? a.groups * ceil_div(a.n, tm) : std::max<int64_t>(live, ceil_div(a.rows, tm) + live / 2); };
    const int64_t tp = row_tiles(256) * ceil_div(cols, 256), ts = row_tiles(128) * ceil_div(cols, 128);
    const int64_t cost_pair = ceil_div(tp, kHopSMs / 2) * 525, cost_one = ceil_div(ts, kHopSMs) * 625;
    p.pair = cols > 128 && (dw ? a.n > 128 : a.rows > 128 * live) && cost_pair <= cost_one;
    p.bn = p.pair ? 256 : 128;
    // Parts: few tiles with many terms are shared out along the terms, at least 8 slices to a part (a join follows)
    const int64_t tiles = p.pair ? tp : ts, room = (p.pair ? kHopSMs / 2 : kHopSMs) / std::max<int64_t>(1, tiles);
    const int64_t slices = ceil_div(dw ? a.rows / a.groups : fwd ? a.k : a.n, kBK);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({room, slices / 8, 16}));
    p.out_rows = dw ? (int64_t)a.groups * a.n : a.rows;
    p.padded = (cols + 3) / 4 * 4;
    p.part_at = at;
    if (p.splits > 1) at += p.splits * p.out_rows * p.padded * 4;
    p.bytes = at;
    return p;
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
cudaError_t encoder(EncodeFn* out) {
    static EncodeFn fn = nullptr;       // the same value whoever writes it first
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q);
        if (e != cudaSuccess) return e;
        if (!p || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
        fn = (EncodeFn)p;
    }
    *out = fn;
    return cudaSuccess;
}
// dims 2: [rows][cols]; 3: [groups][rows][cols]; 0: [cols / 64][rows][64], so that one load brings several 64-column pieces
cudaError_t make_map(EncodeFn enc, CUtensorMap* m, const Operand& o, int dims, int box_rows, int pieces = 1) {
    const bool deep = dims == 0;
    const cuuint64_t d[3] = {deep ? 64u : (cuuint64_t)o.cols, (cuuint64_t)o.rows, deep ? (cuuint64_t)o.cols / 64 : (cuuint64_t)o.groups};
    const cuuint64_t st[2] = {(cuuint64_t)o.stride * 2, deep ? 128u : (cuuint64_t)(o.groups > 1 ? o.group_stride : o.stride * o.rows) * 2};
    const cuuint32_t box[3] = {kBK, (cuuint32_t)box_rows, (cuuint32_t)pieces}, one[3] = {1, 1, 1};
    // The encoder is a driver call and fails in a thread whose first CUDA call it is (torch's backward threads): cudaSetDevice
    // then makes the device's context current and it is asked again.
    for (int again = 0; again < 2; ++again) {
        if (enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, deep ? 3u : (cuuint32_t)dims, const_cast<void*>(o.p), d, st, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
            return cudaSuccess;
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaSetDevice(dev);
        if (e != cudaSuccess) return e;
    }
    return cudaErrorInvalidValue;
}

template <auto Kernel>
cudaError_t launch_tc(int cg, int grid, size_t smem, cudaStream_t st, const CUtensorMap& ma, const CUtensorMap& mb, const TcArgs& t) {
    const cudaError_t e = hop_allow_max_smem<Kernel>();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    cfg.attrs = at;
    if (cg > 1) {
        at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        at[cfg.numAttrs].val.clusterDim.x = cg;
        at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
    return cudaLaunchKernelEx(&cfg, Kernel, ma, mb, t);
}
template <int CG, int BN, int OUT>
cudaError_t launch_way(int way, int grid, cudaStream_t st, const CUtensorMap& ma, const CUtensorMap& mb, const TcArgs& t) {
    constexpr size_t smem = (size_t)kStages * (128 + BN / CG) * kBK * 2 + kEpiWarps * 2048 + sizeof(TcControl) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory");
    if (way == HOP_LINEAR_FORWARD) return launch_tc<linear_tc_kernel<CG, BN, HOP_LINEAR_FORWARD, OUT>>(CG, grid, smem, st, ma, mb, t);
    if (way == HOP_LINEAR_DX) return launch_tc<linear_tc_kernel<CG, BN, HOP_LINEAR_DX, OUT>>(CG, grid, smem, st, ma, mb, t);
    return launch_tc<linear_tc_kernel<CG, BN, HOP_LINEAR_DW, OUT>>(CG, grid, smem, st, ma, mb, t);
}
template <int CG, int BN>
cudaError_t launch_result(int out, int way, int grid, cudaStream_t st, const CUtensorMap& ma, const CUtensorMap& mb, const TcArgs& t) {
    if (out == kFloat) return launch_way<CG, BN, kFloat>(way, grid, st, ma, mb, t);
    return out == kRounded ? launch_way<CG, BN, kRounded>(way, grid, st, ma, mb, t) : launch_way<CG, BN, kDirect>(way, grid, st, ma, mb, t);
}

cudaError_t linear_run(const hop_linear_args& a, cudaStream_t st) {
    const bool dw = a.way == HOP_LINEAR_DW;
    const int so = hop_op_size(a.out_dtype);
    cudaError_t e;
    if (a.rows == 0) {      // weight gradients of nothing
        if (a.accumulate) return cudaSuccess;
        for (int g = 0; g < a.groups; ++g) {
            e = cudaMemset2DAsync((char*)a.out + (int64_t)g * a.out_group_stride * so, (size_t)(a.n > 1 ? a.out_stride : a.k) * so, 0, (size_t)a.k * so, (size_t)a.n, st);
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
    }
    EncodeFn enc;
    if ((e = encoder(&enc)) != cudaSuccess) return e;
    Plan p = linear_plan(a);
    if (p.op[0].packed || p.op[1].packed) {
        PackArgs q = {};            // (an operand taken in place has no rows here)
        q.offsets = p.op[1].groups > 1 ? a.offsets : nullptr;
        for (int k = 0; k < 2; ++k) {
            Operand& o = p.op[k];
            if (!o.packed) continue;
            q.src[k] = (const uint16_t*)o.p; q.group_stride[k] = o.group_stride; q.row_stride[k] = o.stride; q.rows[k] = o.rows; q.cols[k] = o.cols;
            q.units[k] = (o.cols + 7) / 8;
            q.all[k] = (int64_t)o.groups * o.rows;
            q.dst[k] = (uint4*)((char*)a.workspace + o.at);
            o.p = q.dst[k]; o.stride = q.units[k] * 8; o.group_stride = o.rows * o.stride;
        }
        e = hop_launch_dependent(linear_pack_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(std::max(q.all[0], q.all[1]), 8), kHopSMs * 8)), 256, 0, st, q);
        if (e != cudaSuccess) return e;
    }
    const int cols = a.way == HOP_LINEAR_FORWARD ? a.n : a.k, cg = p.pair ? 2 : 1, bn = p.bn;
    const bool split = p.splits > 1;
    CUtensorMap ma, mb;
    // dW: a slice's 64-column pieces in one load where they are whole
    const uint32_t deep = dw ? (p.op[0].cols % 64 == 0 ? 1u : 0u) | (p.op[1].cols % 64 == 0 ? 2u : 0u) : 0u;
    e = make_map(enc, &ma, p.op[0], deep & 1 ? 0 : 2, dw ? kBK : cg == 1 ? 32 : 128, deep & 1 ? 2 : 1);
    if (e == cudaSuccess) e = make_map(enc, &mb, p.op[1], deep & 2 ? 0 : dw ? 2 : 3, a.way == HOP_LINEAR_FORWARD ? bn / cg : kBK, deep & 2 ? bn / cg / 64 : 1);
    if (e != cudaSuccess) return e;
    TcArgs t;
    t.deep = deep;
    t.offsets = a.offsets; t.rows = a.rows; t.groups = a.groups; t.n = a.n; t.k = a.k;
    t.w_step = p.op[1].groups > 1 ? 1 : 0;
    t.splits = p.splits; t.part_stride = split ? p.out_rows * p.padded : 0;
    float* parts = (float*)((char*)a.workspace + p.part_at);
    t.out = split ? parts : a.out;
    t.out_group_stride = split ? (int64_t)a.n * p.padded : a.out_group_stride;
    t.out_stride = split ? p.padded : a.out_stride;
    t.out_dtype = split ? HOP_DT_F32 : a.out_dtype;
    t.accumulate = split ? 0 : a.accumulate;
    const uintptr_t all = (uintptr_t)t.out | (uintptr_t)(t.out_stride * (split ? 4 : so)) | (uintptr_t)(dw && a.groups > 1 ? t.out_group_stride * (split ? 4 : so) : 0);
    t.vec = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 0;
    // instruction descriptor: D float32 (bit 4), A and B f16 (0) or bf16 (1) at bits 7 and 10, MN-major flags at bits 15 and 16,
    // N / 8 at bit 17, M / 16 at bit 24
    const uint32_t f = a.dtype == HOP_DT_BF16 ? 1u : 0u;
    t.idesc = (1u << 4) | (f << 7) | (f << 10) | ((dw ? 1u : 0u) << 15) | ((a.way == HOP_LINEAR_FORWARD ? 0u : 1u) << 16) | ((uint32_t)(bn / 8) << 17) | ((uint32_t)(128 * cg / 16) << 24);
    const int64_t row_tiles = dw ? (int64_t)a.groups * ceil_div(a.n, 128 * cg) : a.rows / (128 * cg) + a.groups + 1;
    const int grid = (int)std::min<int64_t>(row_tiles * ceil_div(cols, bn) * p.splits * cg, kHopSMs);
    // (of dW's sums only the rows of all groups together are known here)
    const bool far = (dw ? a.rows : a.way == HOP_LINEAR_FORWARD ? a.k : a.n) > (a.out_dtype == HOP_DT_F16 ? kLongF16 : kLongBF16);
    const int out = t.out_dtype == HOP_DT_F32 ? kFloat : t.accumulate || far ? kRounded : kDirect;
    e = p.pair ? launch_result<2, 256>(out, a.way, grid, st, ma, mb, t) : launch_result<1, 128>(out, a.way, grid, st, ma, mb, t);
    if (e != cudaSuccess || !split) return e;
    const int blocks = (int)std::min<int64_t>(ceil_div(p.out_rows * (p.padded / 4), 256), kHopSMs * 8);
    const int64_t per = dw ? a.n : 0;
#define HOP_JOIN(T) e = hop_launch_dependent(linear_join_kernel<T>, dim3(blocks), 256, 0, st, parts, t.part_stride, p.splits, p.out_rows, per, cols, p.padded, (T*)a.out, a.out_group_stride, a.out_stride, a.accumulate)
    if (a.out_dtype == HOP_DT_F32) HOP_JOIN(float);
    else if (a.out_dtype == HOP_DT_F16) HOP_JOIN(__half);
    else HOP_JOIN(__nv_bfloat16);
#undef HOP_JOIN
    return e;
}

}  // namespace

extern "C" int hop_linear_workspace(const hop_linear_args* args, int64_t* bytes, char* errbuf, int64_t errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!bytes) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_linear_workspace: null bytes");
    const int rc = linear_check(args, errbuf, errbuf_len);
    if (rc) return rc;
    *bytes = args->rows == 0 ? 0 : linear_plan(*args).bytes;
    return HOP_OK;
}

extern "C" int hop_linear(const hop_linear_args* args, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    const int rc = linear_check(args, errbuf, errbuf_len);
    if (rc) return rc;
    const hop_linear_args& a = *args;
    const bool dw = a.way == HOP_LINEAR_DW;
    if (a.rows == 0 && !dw) return HOP_OK;
    if (!a.out || (a.rows && (!a.a || (dw ? !a.b : !a.w)))) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_linear: null operand");
    const int so = hop_op_size(a.out_dtype);
    if ((uintptr_t)a.a % 2 || (uintptr_t)a.b % 2 || (uintptr_t)a.w % 2 || (uintptr_t)a.out % so || (uintptr_t)a.offsets % 4)
        return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_linear: a pointer is not aligned to its element");
    const int64_t need = a.rows == 0 ? 0 : linear_plan(a).bytes;
    if (need && (!a.workspace || a.workspace_bytes < need || ((uintptr_t)a.workspace & 255)))
        return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_linear: workspace of %lld bytes, 256-byte aligned, needed (got %lld)", (long long)need, (long long)a.workspace_bytes);
    return hop_op_cuda(errbuf, errbuf_len, "hop_linear", linear_run(a, (cudaStream_t)cuda_stream));
}

extern "C" int hop_linear_selftest_bounded_wait(int64_t nanoseconds, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (nanoseconds < 1 || nanoseconds > 1000000000) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_linear_selftest_bounded_wait: %lld ns (1 .. 10^9)", (long long)nanoseconds);
    linear_wait_selftest_kernel<<<1, 32, 0, (cudaStream_t)cuda_stream>>>((uint64_t)nanoseconds);
    return hop_op_cuda(errbuf, errbuf_len, "hop_linear_selftest_bounded_wait", cudaGetLastError());
}

extern "C" int hop_linear_status(int32_t* device_error_word, char* errbuf, int64_t errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!device_error_word) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_linear_status: null word");
    int32_t w = 0, zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&w, g_linear_error, sizeof(w));
    if (e == cudaSuccess && w) e = cudaMemcpyToSymbol(g_linear_error, &zero, sizeof(zero));
    if (e != cudaSuccess) return hop_op_cuda(errbuf, errbuf_len, "hop_linear_status", e);
    *device_error_word = w;
    return w ? hop_op_fail(errbuf, errbuf_len, HOP_E_DEVICE, "hop_linear: a wait inside a product kernel ran out (site %d)", w & 0xffffff) : HOP_OK;
}
