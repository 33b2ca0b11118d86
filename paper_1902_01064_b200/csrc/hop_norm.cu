// Dropout, and the fused end of a block: norm of the block's output, gate, dropout, residual scale and sum, norm for the
// next block (hop_dropout, hop_norm_forward, hop_norm_backward).
#include "hop_norm.cuh"

namespace {

DropRng drop_rng(double p, uint64_t seed, uint32_t step, uint32_t site) {
    DropRng r;
    r.thr = (uint32_t)(p * 65536.0 + 0.5);
    r.last = (r.thr << 16) - 1u;            // largest word whose upper half is dropped (p = 1: every word)
    r.step = step; r.site = site;
    r.scale = r.thr >= 65536u ? 0.f : (float)(65536.0 / (65536.0 - (double)r.thr));
    for (uint32_t i = 0; i < 10; ++i) { r.k0[i] = (uint32_t)seed + i * kPhiloxW0; r.k1[i] = (uint32_t)(seed >> 32) + i * kPhiloxW1; }
    return r;
}
// One read and one write of a row array; in 16-bit types the mask (40 of 140 instructions per eight columns, the wide
// multiplies on half of the multiply-add pipe) costs 15 us of 102 at 16384 x 8192, in float32 none (88 us, a copy's time).
// Rows on the 16-byte grid: one thread per eight columns, kDropPieces pieces in flight.  (row, block of columns) of a
// thread's next piece, and its addresses, come from additions: no division or multiplication in the loop.
// 16384 x 8192 bf16, p = 0.1: 102 us with 40 blocks an SM, 109 with 8, 117 with a block for every 512 pieces (a copy of the same
// bytes: 88); 4096 x 4096: 18.5 us with 8 blocks an SM, 22.6 with 40.  So: eight pieces a thread, 8 to 40 blocks an SM.
template <typename T> constexpr int kDropPieces = sizeof(T) == 4 ? 1 : 2;
struct DropSteps { uint32_t rows, blocks, dr, dc; int64_t dx, dy, wx, wy; };      // a step, and what a wrap into the next row adds (elements)
template <typename T>
__global__ void __launch_bounds__(256, 5)
dropout_kernel(const T* x, int64_t xs, T* y, int64_t ys, int64_t cols, const __grid_constant__ DropSteps t, const __grid_constant__ DropRng d) {
    constexpr int U = kUnits<T>, N = kDropPieces<T>;
    const uint64_t first = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    uint32_t row = (uint32_t)min(first / t.blocks, (uint64_t)0xffffffffu), c = (uint32_t)(first % t.blocks);
    const T* px = x + (int64_t)row * xs + (int64_t)c * 8;
    T* py = y + (int64_t)row * ys + (int64_t)c * 8;
    const uint32_t whole = (uint32_t)(cols / 8);            // blocks below this one have eight columns
    dependency_wait();
    while (row < t.rows) {
        uint32_t w[N][4 * U], r[N], b[N];
        const T* qx[N];
        T* qy[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            r[k] = row; b[k] = c; qx[k] = px; qy[k] = py;
            if (row < t.rows && c < whole) {
#pragma unroll
                for (int i = 0; i < U; ++i) { const uint4 u = reinterpret_cast<const uint4*>(px)[i]; w[k][4 * i] = u.x; w[k][4 * i + 1] = u.y; w[k][4 * i + 2] = u.z; w[k][4 * i + 3] = u.w; }
            }
            if (row < t.rows) {
                const uint32_t before = row;
                row += t.dr; c += t.dc; px += t.dx; py += t.dy;
                if (c >= t.blocks) { c -= t.blocks; ++row; px += t.wx; py += t.wy; }
                if (row < before) row = 0xffffffffu;        // (past the last of nearly 2^32 rows)
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (r[k] >= t.rows) break;
            float v[8];
            uint32_t o[4];
            if (d.thr) drop_words(d, b[k], r[k], o);
            if (b[k] < whole) {
                unpack8<T>(w[k], v);
                if (d.thr) drop8(d, o, v);
                pack8<T>(v, w[k]);
#pragma unroll
                for (int i = 0; i < U; ++i) reinterpret_cast<uint4*>(qy[k])[i] = make_uint4(w[k][4 * i], w[k][4 * i + 1], w[k][4 * i + 2], w[k][4 * i + 3]);
            } else {
                const int n = (int)(cols - (int64_t)b[k] * 8);
                op_load8<T, false>(qx[k], n, v);
                if (d.thr) drop8(d, o, v);
                op_store8<T, false>(qy[k], n, v);
            }
        }
    }
}
// Rows off the grid: a warp takes 256 columns of a row at a time; a lane gets the unit behind its own from its neighbour.
// 16384 x 8191 bf16, p = 0.1: 173 us (3.1 TB/s: the shifts, and element stores through shared memory, beside the mask); 16384 x 4001
// float32: 93 us (5.6 TB/s).
template <typename T>
__global__ void __launch_bounds__(256)
dropout_askew_kernel(const T* x, int64_t xs, T* y, int64_t ys, int64_t rows, int64_t cols, const __grid_constant__ DropRng d) {
    __shared__ __align__(16) unsigned char scratch[8][32 * kUnits<T> * 16];
    constexpr int U = kUnits<T>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t chunks = (cols + 255) / 256, stride = (int64_t)gridDim.x * 8;
    const int64_t first = (int64_t)blockIdx.x * 8 + warp;
    const int64_t dr = stride / chunks, dc = stride % chunks;
    dependency_wait();
    for (int64_t row = first / chunks, c = first % chunks; row < rows;) {
        const int wide = (int)min((int64_t)256, cols - c * 256), n = max(0, min(8, wide - lane * 8));
        const char* p = reinterpret_cast<const char*>(x + row * xs + c * 256);
        const uint32_t m = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15);
        const uint4* q = reinterpret_cast<const uint4*>(p - m);
        const int total = (int)m + wide * (int)sizeof(T);
        uint32_t w[4 * U + 4], o[4];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            uint4 u = make_uint4(0u, 0u, 0u, 0u);
            if ((lane * U + i) * 16 < total) u = q[lane * U + i];
            w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
        }
        uint4 last = make_uint4(0u, 0u, 0u, 0u);
        if (lane == 31 && 32 * U * 16 < total) last = q[32 * U];
        if (d.thr) drop_words(d, (uint32_t)(c * 32 + lane), (uint32_t)row, o);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * U + i] = __shfl_down_sync(0xffffffffu, w[i], 1);
        if (lane == 31) { w[4 * U] = last.x; w[4 * U + 1] = last.y; w[4 * U + 2] = last.z; w[4 * U + 3] = last.w; }
        op_shift_words(w, m);
        float v[8];
        unpack8<T>(w, v);
        if (d.thr) drop8(d, o, v);
        warp_store<T, true>(y + row * ys + c * 256, lane, n, wide, v, scratch[warp]);
        row += dr; c += dc;
        if (c >= chunks) { c -= chunks; ++row; }
    }
}

NormPlan norm_plan(const hop_norm_args& a, bool backward) {
    NormPlan p;
    // Two pieces of eight columns a thread: what a row costs a warp besides its columns (sums, copies, loop) is half of all
    // instructions with one
    const int pieces = (a.cols + 7) / 8;
    // (a layer norm's gradients with their four column sums would spill: one, up to 4096 columns)
    p.nv = a.cols <= 256 || (backward && a.kind == HOP_NORM_LAYER && a.cols <= 4096) ? 1 : 2;
    p.threads = (((pieces + p.nv - 1) / p.nv) + 31) / 32 * 32;
    p.teams_per_block = p.threads == 32 ? 4 : 1;
    // Blocks an SM holds by their registers, then rows in flight (two to four) by what shared memory is left to each; fewer
    // blocks where two rows do not fit; one row, or none at all (rows and vectors read straight from memory) where one block
    // is too wide for that
    const int arrays = (backward ? 4 : 2) + (a.token_gate != nullptr), warps = p.threads / 32 * p.teams_per_block;
    const int vectors = a.kind == HOP_NORM_RMS ? 2 : backward ? 3 : 4;
    const size_t window = (size_t)(32 * (hop_op_size(a.dtype) / 2) + 1) * 16, row = window * p.nv * warps * arrays, scratch = (window - 16) * warps;
    const size_t fixed = scratch + (size_t)warps * 1024 * p.nv * vectors;
    int per_sm = p.teams_per_block > 1 ? kWarpBlocks[backward] : p.threads <= 256 ? kSmallBlocks[backward] * (256 / p.threads) : kLargeBlocks[backward];
    auto fit = [&](int blocks) {                        // rows in flight with that many blocks an SM (2 KB of each: static and reserved)
        const size_t room = std::min<size_t>(kNormSmem, 227 * 1024 / blocks - 2048);
        return p.threads > 512 || fixed > room ? 0 : (int)std::min<size_t>(4, (room - fixed) / row);
    };
    while (per_sm > 1 && fit(per_sm) < 2) --per_sm;
    p.stages = fit(per_sm);
    p.smem = p.stages ? fixed + p.stages * row : scratch;
    const int64_t resident = (int64_t)kHopSMs * p.teams_per_block * per_sm;
    p.rows_per_team = (int)std::max<int64_t>(1, (a.rows + resident - 1) / resident);
    // (a team's offsets are 32 bits wide)
    int64_t far = 1;
    for (int64_t st : {a.x_stride, a.b_stride, a.token_gate_stride, a.r_stride, a.h_stride, a.dr_stride, a.dh_stride, a.dx_stride, a.db_stride, a.dtoken_gate_stride})
        far = std::max(far, st);
    p.rows_per_team = (int)std::max<int64_t>(1, std::min<int64_t>(p.rows_per_team, (1ll << 31) / (far * hop_op_size(a.dtype))));
    p.teams = (int)((a.rows + p.rows_per_team - 1) / p.rows_per_team);
    return p;
}

// Adds the teams' places of each group and forms the vectors' gradients.  Block: X * V columns, V a thread, and as many teams
// side by side as its threads allow; what takes time are the loads, so they are wide, four in flight, and spread over more
// blocks of fewer columns where a group has many places.  Whole backward passes in bf16 (RMS), us, with 4 / 16 / 64 teams side by side
// on 32 columns and 256 on 8: 16384 x 2048, places a group 11: 91.6 / 91.6 / 116 / 215, 38: 87.6 / 86.4 / 92.1 / 117, 75: 88.5 / 85.6 /
// 87.4 / 98.5, 588: 133 / 102 / 88.6 / 88.2; 65536 x 512, 445: 118 / 101 / 87.4 / 86.8, 1774: 213 / 144 / 98.4 / 92.9.  Widths that are
// no multiple of four, a column a thread, 4 / 16 side by side on 32 and 64 on 8: 16384 x 1001, 20 places 115 / 122 / 147, 1173: 189 /
// 132 / 122; 4099 x 1001, 207: 51 / 42 / 44.
template <int NACC, int V, int X>
__global__ void __launch_bounds__(512)
norm_sums_kernel(const __grid_constant__ NormDev P) {
    __shared__ float part[NACC * V][512];
    const hop_norm_args& a = P.a;
    const int cx = threadIdx.x % X, ty = threadIdx.x / X, lanes = blockDim.x / X, c = (blockIdx.x * X + cx) * V, g = blockIdx.y;
    dependency_wait();          // before anything is read: offsets too may come from a kernel just in front of the call
    int64_t lo = 0, hi = a.rows;
    if (a.offsets) {
        lo = min(max((int64_t)a.offsets[g], (int64_t)0), a.rows);
        hi = min(max((int64_t)a.offsets[g + 1], lo), a.rows);
        if (g == 0) lo = 0;
    }
    float s[NACC][V];
#pragma unroll
    for (int k = 0; k < NACC; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) s[k][v] = 0.f;
    if (hi > lo && c < a.cols) {
        const int t1 = (int)((hi - 1) / P.rows_per_team);
        const float* p = P.partial + (int64_t)g * NACC * a.cols + c;
#pragma unroll 4
        for (int t = (int)(lo / P.rows_per_team) + ty; t <= t1; t += lanes)
#pragma unroll
            for (int k = 0; k < NACC; ++k) {
                const float* q = p + ((int64_t)t * NACC + k) * a.cols;
                if constexpr (V == 4) {
                    const float4 f = *reinterpret_cast<const float4*>(q);
                    s[k][0] += f.x; s[k][1] += f.y; s[k][2] += f.z; s[k][3] += f.w;
                } else {
                    s[k][0] += *q;
                }
            }
    }
#pragma unroll
    for (int k = 0; k < NACC; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) part[k * V + v][threadIdx.x] = s[k][v];
    for (int half = lanes / 2; half > 0; half /= 2) {
        __syncthreads();
        if (ty < half)
#pragma unroll
            for (int k = 0; k < NACC * V; ++k) part[k][threadIdx.x] += part[k][threadIdx.x + half * X];
    }
    __syncthreads();
    // a thread a column
    if (threadIdx.x >= X * V) return;
    const int col = blockIdx.x * X * V + threadIdx.x;
    if (col >= a.cols) return;
    float z[NACC];
#pragma unroll
    for (int k = 0; k < NACC; ++k) z[k] = part[k * V + threadIdx.x % V][threadIdx.x / V];
    // (a group without rows: zeros, whatever its vectors hold)
    const bool any = hi > lo;
    const float gate = !any ? 0.f : a.scale * (a.gate ? a.gate[(int64_t)g * a.gate_stride + col] : 1.f);
    const float w = any && a.w_post ? a.w_post[(int64_t)g * a.w_post_stride + col] : 1.f;
    if (a.dw_pre) a.dw_pre[(int64_t)g * a.dw_pre_stride + col] = z[0];
    if (a.dw_post) a.dw_post[(int64_t)g * a.dw_post_stride + col] = gate * z[1];
    float dg = w * z[1];
    if constexpr (NACC == 4) {
        if (a.dc_pre) a.dc_pre[(int64_t)g * a.dc_pre_stride + col] = z[2];
        if (a.dc_post) a.dc_post[(int64_t)g * a.dc_post_stride + col] = gate * z[3];
        if (any && a.c_post) dg = fmaf(a.c_post[(int64_t)g * a.c_post_stride + col], z[3], dg);
    }
    if (a.dgate) a.dgate[(int64_t)g * a.dgate_stride + col] = a.scale * dg;
}
template <int NACC>
cudaError_t sums_launch(const NormDev& P, int teams, cudaStream_t st) {
    const int places = teams / P.a.groups + 2;              // of an average group
    const dim3 wide((P.a.cols + 31) / 32, P.a.groups), narrow((P.a.cols + 7) / 8, P.a.groups);
    if (P.a.cols % 4 == 0) {
        if (places > 256) return hop_launch_dependent(norm_sums_kernel<NACC, 4, 2>, narrow, 512, 0, st, P);
        return hop_launch_dependent(norm_sums_kernel<NACC, 4, 8>, wide, 8 * (places <= 16 ? 4 : places <= 64 ? 16 : 64), 0, st, P);
    }
    if (places > 64) return hop_launch_dependent(norm_sums_kernel<NACC, 1, 8>, narrow, 512, 0, st, P);
    return hop_launch_dependent(norm_sums_kernel<NACC, 1, 32>, wide, 32 * (places <= 16 ? 4 : 16), 0, st, P);
}

// ------------------------------------------------------------------------------------------------ host side
bool aligned16(const void* p, int64_t stride, int size) { return !p || (((uintptr_t)p | (uintptr_t)(stride * size)) & 15) == 0; }

int norm_check(const hop_norm_args* a, bool backward, char* eb, int64_t el) {
    const char* who = backward ? "hop_norm_backward" : "hop_norm_forward";
    if (!a) return hop_op_fail(eb, el, HOP_E_ARG, "%s: null arguments", who);
    if (!hop_op_dtype_ok(a->dtype)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: unknown dtype %d", who, a->dtype);
    if (a->kind != HOP_NORM_RMS && a->kind != HOP_NORM_LAYER) return hop_op_fail(eb, el, HOP_E_ARG, "%s: unknown norm kind %d", who, a->kind);
    if (a->rows < 0 || a->rows >= (1ll << 31)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: %lld rows (0 .. 2^31-1)", who, (long long)a->rows);
    if (a->cols < 1 || a->cols > HOP_NORM_MAX_COLS) return hop_op_fail(eb, el, HOP_E_ARG, "%s: %d columns (1 .. %d)", who, a->cols, HOP_NORM_MAX_COLS);
    if (a->groups < 1 || a->groups > HOP_MAX_GROUPS) return hop_op_fail(eb, el, HOP_E_ARG, "%s: %d groups (1 .. %d)", who, a->groups, HOP_MAX_GROUPS);
    if (!a->offsets && a->groups != 1) return hop_op_fail(eb, el, HOP_E_ARG, "%s: several groups need offsets", who);
    if (!(a->p >= 0.0 && a->p <= 1.0)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: dropout probability %g outside [0, 1]", who, a->p);
    if (!(a->eps >= 0.f)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: eps %g", who, (double)a->eps);
    if (a->kind == HOP_NORM_RMS && (a->c_post || a->c_pre)) return hop_op_fail(eb, el, HOP_E_UNSUPPORTED, "%s: an RMS norm has no shift", who);
    if (a->gate && a->token_gate) return hop_op_fail(eb, el, HOP_E_ARG, "%s: gate and token_gate exclude each other", who);
    if (!a->post_norm && (a->w_post || a->c_post)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: w_post / c_post without post_norm", who);
    if (!a->pre_norm && (a->w_pre || a->c_pre)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: w_pre / c_pre without pre_norm", who);
    if (a->rows == 0) return HOP_OK;
    if (!a->b && (a->post_norm || a->gate || a->token_gate || a->p != 0.0)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: post norm, gate and dropout need b", who);
    if (!a->b && !a->pre_norm) return hop_op_fail(eb, el, HOP_E_ARG, "%s: nothing to compute (neither b nor pre_norm)", who);
    return HOP_OK;
}

bool needs_sums(const hop_norm_args& a) { return a.dw_post || a.dc_post || a.dgate || a.dw_pre || a.dc_pre; }
int64_t norm_workspace(const hop_norm_args& a) {
    if (!needs_sums(a) || a.rows == 0) return 0;
    const NormPlan pl = norm_plan(a, true);
    return ((int64_t)pl.teams + a.groups) * (a.kind == HOP_NORM_LAYER ? 4 : 2) * a.cols * 4;
}

int norm_run(const hop_norm_args* a, bool backward, void* stream, char* eb, int64_t el) {
    const char* who = backward ? "hop_norm_backward" : "hop_norm_forward";
    if (eb && el > 0) eb[0] = 0;
    int rc = norm_check(a, backward, eb, el);
    if (rc) return rc;
    NormDev P;
    P.a = *a;
    hop_norm_args& q = P.a;
    if (!backward) {
        q.dr = q.dh = nullptr; q.dx = q.db = q.dtoken_gate = nullptr;
        q.dw_post = q.dc_post = q.dgate = q.dw_pre = q.dc_pre = nullptr;
        if (q.rows && (!q.x || (q.b && !q.r) || (q.pre_norm && !q.h))) return hop_op_fail(eb, el, HOP_E_ARG, "%s: null x, r or h", who);
        if (q.rows == 0) return HOP_OK;
        if (!q.pre_norm) q.h = nullptr;
        if (!q.b) q.r = nullptr;
    } else {
        q.x = nullptr; q.h = nullptr;
        if (!q.pre_norm) q.dh = nullptr;
        if (q.rows) {
            if (!q.dr && !q.dh) return hop_op_fail(eb, el, HOP_E_ARG, "%s: neither dr nor dh", who);
            if (!q.dx || (q.dh && !q.r) || (q.b && !q.db)) return hop_op_fail(eb, el, HOP_E_ARG, "%s: null r, dx or db", who);
        }
        if ((q.dw_pre || q.dc_pre) && !q.pre_norm) return hop_op_fail(eb, el, HOP_E_ARG, "%s: dw_pre / dc_pre without pre_norm", who);
        if ((q.dw_post || q.dc_post) && !q.post_norm) return hop_op_fail(eb, el, HOP_E_ARG, "%s: dw_post / dc_post without post_norm", who);
        if (q.kind == HOP_NORM_RMS && (q.dc_post || q.dc_pre)) return hop_op_fail(eb, el, HOP_E_UNSUPPORTED, "%s: an RMS norm has no shift", who);
        if (q.dtoken_gate && !q.token_gate) return hop_op_fail(eb, el, HOP_E_ARG, "%s: dtoken_gate without token_gate", who);
        if (q.dgate && (q.token_gate || (q.rows && !q.b))) return hop_op_fail(eb, el, HOP_E_ARG, "%s: dgate needs b and no token_gate", who);
        if (!q.b) { q.db = nullptr; q.skip = 1.f; }      // r was x itself
    }
    const int size = hop_op_size(q.dtype);
    const struct { const void* p; int64_t stride; } rows[] = {{q.x, q.x_stride}, {q.b, q.b_stride}, {q.token_gate, q.token_gate_stride}, {q.r, q.r_stride}, {q.h, q.h_stride},
        {q.dr, q.dr_stride}, {q.dh, q.dh_stride}, {q.dx, q.dx_stride}, {q.db, q.db_stride}, {q.dtoken_gate, q.dtoken_gate_stride}};
    for (const auto& row : rows) {
        if ((uintptr_t)row.p % size) return hop_op_fail(eb, el, HOP_E_ARG, "%s: a pointer is not aligned to its element", who);
        // (rows are addressed by unsigned 32-bit offsets from a team's first one)
        if (row.p && row.stride < 0) return hop_op_fail(eb, el, HOP_E_ARG, "%s: a row stride of %lld", who, (long long)row.stride);
    }
    for (const void* p : {(const void*)q.offsets, (const void*)q.w_post, (const void*)q.c_post, (const void*)q.gate, (const void*)q.w_pre, (const void*)q.c_pre,
                          (const void*)q.dw_post, (const void*)q.dc_post, (const void*)q.dgate, (const void*)q.dw_pre, (const void*)q.dc_pre})
        if ((uintptr_t)p % 4) return hop_op_fail(eb, el, HOP_E_ARG, "%s: offsets or a vector is not aligned to its element", who);
    const NormPlan pl = norm_plan(q, backward);
    P.d = drop_rng(q.p, q.seed, q.step, q.site);
    P.drop = P.d.thr != 0;
    P.rows_per_team = pl.rows_per_team;
    P.stages = pl.stages;
    P.partial = nullptr;
    if (backward && needs_sums(q) && q.rows) {
        const int64_t need = norm_workspace(q);
        if (!q.workspace || q.workspace_bytes < need || ((uintptr_t)q.workspace & 255))
            return hop_op_fail(eb, el, HOP_E_ARG, "%s: workspace of %lld bytes, 256-byte aligned, needed (got %lld)", who, (long long)need, (long long)q.workspace_bytes);
        P.partial = (float*)q.workspace;
    }
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    if (q.rows) {
        const bool askew = !(aligned16(q.x, q.x_stride, size) && aligned16(q.b, q.b_stride, size) && aligned16(q.token_gate, q.token_gate_stride, size) &&
                             aligned16(q.r, q.r_stride, size) && aligned16(q.h, q.h_stride, size) && aligned16(q.dr, q.dr_stride, size) &&
                             aligned16(q.dh, q.dh_stride, size) && aligned16(q.dx, q.dx_stride, size) && aligned16(q.db, q.db_stride, size) &&
                             aligned16(q.dtoken_gate, q.dtoken_gate_stride, size));
        if (q.dtype == HOP_DT_F32) e = hop_norm_launch_f32(P, pl, backward, askew, st);
        else if (q.dtype == HOP_DT_F16) e = hop_norm_launch_f16(P, pl, backward, askew, st);
        else e = hop_norm_launch_bf16(P, pl, backward, askew, st);
    }
    if (e == cudaSuccess && backward && needs_sums(q)) {
        e = q.kind == HOP_NORM_LAYER ? sums_launch<4>(P, pl.teams, st) : sums_launch<2>(P, pl.teams, st);
    }
    return hop_op_cuda(eb, el, who, e);
}

template <typename T>
cudaError_t dropout_typed(const void* x, int64_t xs, void* y, int64_t ys, int64_t rows, int64_t cols, const DropRng& d, cudaStream_t st) {
    if (aligned16(x, xs, sizeof(T)) && aligned16(y, ys, sizeof(T))) {
        const int64_t pieces = rows * ((cols + 7) / 8);
        const int grid = (int)std::min<int64_t>((pieces + 255) / 256, std::max<int64_t>(kHopSMs * 8, std::min<int64_t>(kHopSMs * 40, pieces / 2048)));
        DropSteps t;
        const int64_t blocks = (cols + 7) / 8, stride = (int64_t)grid * 256;
        t.rows = (uint32_t)rows; t.blocks = (uint32_t)blocks; t.dr = (uint32_t)(stride / blocks); t.dc = (uint32_t)(stride % blocks);
        t.dx = (int64_t)t.dr * xs + (int64_t)t.dc * 8; t.dy = (int64_t)t.dr * ys + (int64_t)t.dc * 8;
        t.wx = xs - blocks * 8; t.wy = ys - blocks * 8;
        return hop_launch_dependent(dropout_kernel<T>, dim3(grid), 256, 0, st, (const T*)x, xs, (T*)y, ys, cols, t, d);
    }
    const int64_t chunks = rows * ((cols + 255) / 256);
    return hop_launch_dependent(dropout_askew_kernel<T>, dim3((unsigned)std::min<int64_t>((chunks + 7) / 8, kHopSMs * 8)), 256, 0, st, (const T*)x, xs, (T*)y, ys, rows, cols, d);
}

}  // namespace

extern "C" int hop_norm_workspace(const hop_norm_args* args, int64_t* bytes, char* errbuf, int64_t errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!bytes) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_norm_workspace: null bytes");
    const int rc = norm_check(args, true, errbuf, errbuf_len);
    if (rc) return rc;
    *bytes = norm_workspace(*args);
    return HOP_OK;
}
extern "C" int hop_norm_forward(const hop_norm_args* args, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
    return norm_run(args, false, cuda_stream, errbuf, errbuf_len);
}
extern "C" int hop_norm_backward(const hop_norm_args* args, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
    return norm_run(args, true, cuda_stream, errbuf, errbuf_len);
}

extern "C" int hop_dropout(const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t rows, int64_t cols, int32_t dtype,
                           double p, uint64_t seed, uint32_t step, uint32_t site, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!hop_op_dtype_ok(dtype)) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_dropout: unknown dtype %d", dtype);
    if (rows < 0 || cols < 0 || rows > 0xffffffffll || cols > (1ll << 34))       // (a block of eight columns and a step from it fit 32 bits)
        return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_dropout: %lld x %lld (rows below 2^32, cols up to 2^34)", (long long)rows, (long long)cols);
    if (!(p >= 0.0 && p <= 1.0)) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_dropout: probability %g outside [0, 1]", p);
    if (rows == 0 || cols == 0) return HOP_OK;
    const int size = hop_op_size(dtype);
    if (!x || !y || (uintptr_t)x % size || (uintptr_t)y % size) return hop_op_fail(errbuf, errbuf_len, HOP_E_ARG, "hop_dropout: null or misaligned pointer");
    const DropRng d = drop_rng(p, seed, step, site);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (dtype == HOP_DT_F32) e = dropout_typed<float>(x, x_stride, y, y_stride, rows, cols, d, st);
    else if (dtype == HOP_DT_F16) e = dropout_typed<__half>(x, x_stride, y, y_stride, rows, cols, d, st);
    else e = dropout_typed<__nv_bfloat16>(x, x_stride, y, y_stride, rows, cols, d, st);
    return hop_op_cuda(errbuf, errbuf_len, "hop_dropout", e);
}
