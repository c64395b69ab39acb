// The norms after and before a block in one pass: the norm of the block's output B, its gate, the sum with the scaled residual
// stream X and the norm in front of the next block; and the backward pass with the reduction of the parameters' gradients.
//
//   xh1 = (B - mean1) rstd1,  U = xh1 w1 + b1,  Y = a X + gate U,  xh2 = (Y - mean2) rstd2,  N = xh2 w2 + b2
//   (statistics over the features of a token; RMS: means of 0; xh2 is that of Y before its rounding)
//   backward: g2 = dN w2,  dYt = dY + rstd2 (g2 - [mean g2] - xh2 mean(g2 xh2)),  dX = a dYt,  dgate = dYt U,
//   g1 = dYt gate w1,  dB = rstd1 (g1 - [mean g1] - xh1 mean(g1 xh1))
//   dw2 = sum_t dN xh2,  db2 = sum_t dN,  dw1 = sum_t dYt gate xh1,  db1 = sum_t dYt gate   (bracketed: layer norm only)
//
// The backward reads X and B and forms U and Y again, so nothing but the statistics is kept, and the gradients are those of the
// function without Y's rounding. HBM-bound: four rows of a token forward, six backward, one more each for a token's gate.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kThreads = 256;
constexpr int kStrips = 1024;  // workgroups of a backward launch at most, each with a row of partial sums per parameter

// Sums of two values over the THREADS threads that share a row (a wave, or the workgroup), in every one of them; `lds` of 8 floats
// is free again after the next barrier of the caller's (buffers in turn).
template <int THREADS = kThreads>
__device__ __forceinline__ void group_sum2(float &a, float &b, float *lds) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (THREADS == 64) return;
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x >> 6] = a;
        lds[4 + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        a += lds[i];
        b += lds[4 + i];
    }
}

template <int THREADS = kThreads>
__device__ __forceinline__ float group_sum(float a, float *lds) {
    a = wave_sum(a);
    if constexpr (THREADS == 64) return a;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// Piece c .. c + 7 of a row of C elements (zeros past its end); rows of whole eights by a buffer load, whose range check takes
// the place of a branch. `row` is the same for every lane of a wave; NULL reads as zeros.
template <bool TAIL, typename T>
__device__ __forceinline__ void load_piece(Raw8<T> &v, const void *base, int64_t at, int C, int c) {
    const T *row = static_cast<const T *>(base) + at;
    if constexpr (TAIL) {
        v.load(row + c, base ? C - c : 0);
    } else {
        const uint64_t p = (uint64_t)row;
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
        v.load_row(make_rsrc((const void *)((uint64_t)hi << 32 | lo), base ? (int64_t)C * (int64_t)sizeof(T) : 0), c);
    }
}

// A row is shared by THREADS threads (64: four rows per workgroup), NV vectors of 8 elements each: vector j of thread t starts at
// column (j THREADS + t) 8. The row is read once; U and Y stay in registers in fp32.
template <typename T, typename WT, int THREADS, int NV, bool TAIL>
__global__ void __launch_bounds__(kThreads) sandwich_fwd_kernel(SandwichArgs a) {
    __shared__ float lds[4][8];
    constexpr int kRows = kThreads / THREADS;
    const int t = threadIdx.x % THREADS, C = a.C;
    const int64_t row = a.first + (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS, at = row * C;
    if (row >= a.T) return;  // whole waves where rows share a workgroup; no barrier is used there
    Raw8<T> xr[NV], br[NV], gr[NV];
    Raw8<WT> w1[NV], b1[NV], gf[NV], w2[NV], b2[NV];
    const bool token = a.gate_kind == kGateToken, feature = a.gate_kind == kGateFeature;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
        load_piece<TAIL>(br[j], a.B, at, C, c);
        load_piece<TAIL>(xr[j], a.X, at, C, c);
        if (token) load_piece<TAIL>(gr[j], a.gate, at, C, c);
    }
    // the parameters are under way together with the row: a token alone waits for memory once
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
        load_piece<TAIL>(w1[j], a.w1, 0, C, c);
        load_piece<TAIL>(w2[j], a.w2, 0, C, c);
        if (feature) load_piece<TAIL>(gf[j], a.gate, 0, C, c);
        if (a.b1) load_piece<TAIL>(b1[j], a.b1, 0, C, c);
        if (a.b2) load_piece<TAIL>(b2[j], a.b2, 0, C, c);
    }
    const float inv_n = 1.0f / (float)C;
    float mean1 = 0.0f, mean2 = 0.0f, q = 0.0f;
    if (a.layer) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) s += br[j][e];
        mean1 = group_sum<THREADS>(s, lds[0]) * inv_n;
    }
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int n = C - (j * THREADS + t) * 8;  // elements of this vector that exist
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float d = e < n ? br[j][e] - mean1 : 0.0f;
            q = __builtin_fmaf(d, d, q);
        }
    }
    const float rstd1 = 1.0f / sqrtf(group_sum<THREADS>(q, lds[1]) * inv_n + a.eps);
    float y[NV][8], s = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; j++) {
#pragma unroll
        for (int e = 0; e < 8; e++) {  // columns past C have X, w1, b1 of 0
            const float u = __builtin_fmaf((br[j][e] - mean1) * rstd1, w1[j][e], a.b1 ? b1[j][e] : 0.0f);
            const float gate = token ? gr[j][e] : feature ? gf[j][e] : 1.0f;
            y[j][e] = __builtin_fmaf(a.scale, xr[j][e], gate * u);
            s += y[j][e];
        }
    }
    if (a.layer) mean2 = group_sum<THREADS>(s, lds[2]) * inv_n;
    q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int n = C - (j * THREADS + t) * 8;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float d = e < n ? y[j][e] - mean2 : 0.0f;
            q = __builtin_fmaf(d, d, q);
        }
    }
    const float rstd2 = 1.0f / sqrtf(group_sum<THREADS>(q, lds[3]) * inv_n + a.eps);
    T *const Y = static_cast<T *>(a.Y) + at, *const N = static_cast<T *>(a.N) + at;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
        if (c < C) {
            store8_n<TAIL>(Y + c, C - c, y[j]);
#pragma unroll
            for (int e = 0; e < 8; e++) y[j][e] = __builtin_fmaf((y[j][e] - mean2) * rstd2, w2[j][e], a.b2 ? b2[j][e] : 0.0f);
            store8_n<TAIL>(N + c, C - c, y[j]);
        }
    }
    if (t == 0 && a.stats) {
        a.stats[row] = rstd1;
        a.stats[a.T + row] = rstd2;
        if (a.layer) {
            a.stats[2 * a.T + row] = mean1;
            a.stats[3 * a.T + row] = mean2;
        }
    }
}

// A workgroup takes `rows` consecutive rows. The parameters lie in LDS in their own type (a row's worth of registers less; without
// a gate, a feature's gates of 1), the sums over the rows stay in registers and leave as one row of partial sums per
// workgroup (waves that take rows by themselves are added in order through LDS first). BIAS: the sums without xh too; TOKEN: gates
// of the tokens' own.
template <typename T, typename WT, int THREADS, int NV, bool BIAS, bool TOKEN, bool TAIL>
__global__ void __launch_bounds__(kThreads) sandwich_bwd_kernel(SandwichArgs a) {
    constexpr int kRows = kThreads / THREADS, kWidth = NV * THREADS * 8;  // rows under way in a workgroup; columns it covers
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ float lds[2][8];
    const int t = threadIdx.x % THREADS, sub = threadIdx.x / THREADS, C = a.C;
    WT *const lw1 = reinterpret_cast<WT *>(smem), *const lw2 = lw1 + kWidth, *const lgate = lw2 + kWidth,
             *const lb1 = lgate + (TOKEN ? 0 : kWidth);
    {
        auto fill = [&](WT *to, const void *from, float missing) {
            for (int c = threadIdx.x; c < kWidth; c += kThreads)
                store_one(to + c, from && c < C ? load_one(static_cast<const WT *>(from) + c) : missing);
        };
        fill(lw1, a.w1, 0.0f);
        fill(lw2, a.w2, 0.0f);
        if constexpr (!TOKEN) fill(lgate, a.gate, 1.0f);
        if constexpr (BIAS) fill(lb1, a.b1, 0.0f);
    }
    __syncthreads();
    auto param = [&](const WT *p, int j) {
        Raw8<WT> v;
        v.load(p + (j * THREADS + t) * 8, 8);
        return v;
    };
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int64_t last = first + a.rows < a.T ? first + a.rows : a.T;
    constexpr int kSums = BIAS ? 4 : 2;
    float sums[kSums][NV][8];
#pragma unroll
    for (int i = 0; i < kSums; i++)
#pragma unroll
        for (int j = 0; j < NV; j++) zero8(sums[i][j]);
    const float inv_n = 1.0f / (float)C;
    for (int64_t row = first + sub; row < last; row += kRows) {
        const int64_t at = row * C;
        const float rstd1 = a.stats[row], rstd2 = a.stats[a.T + row];
        const float mean1 = a.layer ? a.stats[2 * a.T + row] : 0.0f, mean2 = a.layer ? a.stats[3 * a.T + row] : 0.0f;
        Raw8<T> xr[NV], br[NV], nr[NV], yr[NV], gr[TOKEN ? NV : 1];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * THREADS + t) * 8;
            load_piece<TAIL>(br[j], a.B, at, C, c);
            load_piece<TAIL>(xr[j], a.X, at, C, c);
            if constexpr (TOKEN) load_piece<TAIL>(gr[j], a.gate, at, C, c);
            load_piece<TAIL>(nr[j], a.dN, at, C, c);
            load_piece<TAIL>(yr[j], a.dY, at, C, c);
        }
        // keeps the compiler from holding over the next sum what the packed rows and the LDS give again
        auto again = [&]() {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < NV; j++) {
                br[j].keep_packed(), nr[j].keep_packed(), yr[j].keep_packed();
                if constexpr (TOKEN) gr[j].keep_packed();
            }
        };
        // xh2 of the row, and the two means that the second norm's gradient takes
        float d[NV][8], sg = 0.0f, sgx = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            __builtin_amdgcn_sched_barrier(0);  // one vector's values in fp32 at a time
            const Raw8<WT> w1 = param(lw1, j), w2 = param(lw2, j), gf = TOKEN ? w1 : param(lgate, j), b1 = BIAS ? param(lb1, j) : w1;
#pragma unroll
            for (int e = 0; e < 8; e++) {  // columns past C have dN = 0
                const float u = __builtin_fmaf((br[j][e] - mean1) * rstd1, w1[e], BIAS ? b1[e] : 0.0f);
                const float gate = TOKEN ? gr[TOKEN ? j : 0][e] : gf[e];
                const float xh2 = (__builtin_fmaf(a.scale, xr[j][e], gate * u) - mean2) * rstd2;
                const float n = nr[j][e], g = n * w2[e];
                sums[0][j][e] = __builtin_fmaf(n, xh2, sums[0][j][e]);
                if constexpr (BIAS) sums[2][j][e] += n;
                sg += g;
                sgx = __builtin_fmaf(g, xh2, sgx);
                d[j][e] = xh2;
            }
        }
        group_sum2<THREADS>(sg, sgx, lds[0]);
        const float mg2 = a.layer ? sg * inv_n : 0.0f, mgx2 = sgx * inv_n;
        sg = sgx = 0.0f;
        again();
#pragma unroll
        for (int j = 0; j < NV; j++) {
            __builtin_amdgcn_sched_barrier(0);  // one vector's values in fp32 at a time
            const Raw8<WT> w1 = param(lw1, j), w2 = param(lw2, j), gf = TOKEN ? w1 : param(lgate, j);
#pragma unroll
            for (int e = 0; e < 8; e++) {  // columns past C have w1 = 0
                d[j][e] = __builtin_fmaf(rstd2, nr[j][e] * w2[e] - mg2 - d[j][e] * mgx2, yr[j][e]);
                const float xh1 = (br[j][e] - mean1) * rstd1;
                const float through = TOKEN ? d[j][e] * gr[TOKEN ? j : 0][e] : d[j][e];  // a feature's gate is applied to the sum
                sums[1][j][e] = __builtin_fmaf(through, xh1, sums[1][j][e]);
                if constexpr (BIAS) sums[3][j][e] += through;
                const float g = (TOKEN ? through : through * gf[e]) * w1[e];
                sg += g;
                sgx = __builtin_fmaf(g, xh1, sgx);
            }
        }
        group_sum2<THREADS>(sg, sgx, lds[1]);
        const float mg1 = a.layer ? sg * inv_n : 0.0f, mgx1 = sgx * inv_n;
        again();
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * THREADS + t) * 8;
            __builtin_amdgcn_sched_barrier(0);
            if (c < C) {
                const Raw8<WT> w1 = param(lw1, j), gf = TOKEN ? w1 : param(lgate, j), b1 = BIAS ? param(lb1, j) : w1;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = a.scale * d[j][e];
                store8_n<TAIL>(static_cast<T *>(a.dX) + at + c, C - c, v);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float xh1 = (br[j][e] - mean1) * rstd1;
                    const float g = d[j][e] * (TOKEN ? gr[TOKEN ? j : 0][e] : gf[e]) * w1[e];
                    v[e] = rstd1 * (g - mg1 - xh1 * mgx1);
                }
                store8_n<TAIL>(static_cast<T *>(a.dB) + at + c, C - c, v);
                if (TOKEN && a.dgate) {
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        v[e] = d[j][e] * __builtin_fmaf((br[j][e] - mean1) * rstd1, w1[e], BIAS ? b1[e] : 0.0f);
                    store8_n<TAIL>(static_cast<T *>(a.dgate) + at + c, C - c, v);
                }
            }
        }
    }
    float *const join = reinterpret_cast<float *>(smem);  // kWidth floats, over the parameters
#pragma unroll
    for (int i = 0; i < kSums; i++) {
        if constexpr (THREADS == 64) {
            for (int s = 1; s < kRows; s++) {
                __syncthreads();
                if (sub == s)
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) join[(j * 8 + e) * 64 + t] = sums[i][j][e];
                __syncthreads();
                if (sub == 0)
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) sums[i][j][e] += join[(j * 8 + e) * 64 + t];
            }
        }
        if (sub == 0) {
            float *const part = a.part + ((int64_t)i * gridDim.x + blockIdx.x) * C;
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (j * THREADS + t) * 8;
                if (c < C) store8_n<TAIL>(part + c, C - c, sums[i][j]);
            }
        }
    }
}

// One element of a row: the residual stream's value, and what it is made of
template <typename T>
struct Element {
    float xh1, u, gate, y;
    __device__ __forceinline__ Element(const SandwichArgs &a, int64_t row, int c, float mean1, float rstd1) {
        const int64_t i = row * a.C + c;
        const float w1 = load_param(a.w1, a.w_dtype, c), b1 = a.b1 ? load_param(a.b1, a.w_dtype, c) : 0.0f;
        gate = a.gate_kind == kGateNone ? 1.0f
               : a.gate_kind == kGateFeature ? load_param(a.gate, a.w_dtype, c) : load_one(static_cast<const T *>(a.gate) + i);
        xh1 = (load_one(static_cast<const T *>(a.B) + i) - mean1) * rstd1;
        u = __builtin_fmaf(xh1, w1, b1);
        y = __builtin_fmaf(a.scale, load_one(static_cast<const T *>(a.X) + i), gate * u);
    }
};

// A workgroup per row, which it reads once for each sum and once for the outputs, element by element.
template <typename T>
__global__ void __launch_bounds__(kThreads) sandwich_fwd_long_kernel(SandwichArgs a) {
    __shared__ float lds[2][8];
    const int64_t row = a.first + blockIdx.x;
    const int C = a.C;
    const float n = (float)C;
    const T *b = static_cast<const T *>(a.B) + row * C;
    float mean1 = 0.0f, mean2 = 0.0f, q = 0.0f;
    if (a.layer) {
        float s = 0.0f;
        for (int c = threadIdx.x; c < C; c += kThreads) s += load_one(b + c);
        mean1 = group_sum(s, lds[0]) / n;
    }
    for (int c = threadIdx.x; c < C; c += kThreads) {
        const float d = load_one(b + c) - mean1;
        q = __builtin_fmaf(d, d, q);
    }
    const float rstd1 = 1.0f / sqrtf(group_sum(q, lds[1]) / n + a.eps);
    if (a.layer) {
        float s = 0.0f;
        for (int c = threadIdx.x; c < C; c += kThreads) s += Element<T>(a, row, c, mean1, rstd1).y;
        mean2 = group_sum(s, lds[0]) / n;
    }
    q = 0.0f;
    for (int c = threadIdx.x; c < C; c += kThreads) {
        const float d = Element<T>(a, row, c, mean1, rstd1).y - mean2;
        q = __builtin_fmaf(d, d, q);
    }
    __syncthreads();  // the second buffer's readers are done
    const float rstd2 = 1.0f / sqrtf(group_sum(q, lds[1]) / n + a.eps);
    for (int c = threadIdx.x; c < C; c += kThreads) {
        const float y = Element<T>(a, row, c, mean1, rstd1).y;
        const float b2 = a.b2 ? load_param(a.b2, a.w_dtype, c) : 0.0f;
        store_one(static_cast<T *>(a.Y) + row * C + c, y);
        store_one(static_cast<T *>(a.N) + row * C + c, __builtin_fmaf((y - mean2) * rstd2, load_param(a.w2, a.w_dtype, c), b2));
    }
    if (threadIdx.x == 0 && a.stats) {
        a.stats[row] = rstd1;
        a.stats[a.T + row] = rstd2;
        if (a.layer) {
            a.stats[2 * a.T + row] = mean1;
            a.stats[3 * a.T + row] = mean2;
        }
    }
}

// A workgroup takes `rows` rows one after the other; the sums over them are added up in its row of the partial sums.
template <typename T>
__global__ void __launch_bounds__(kThreads) sandwich_bwd_long_kernel(SandwichArgs a) {
    __shared__ float lds[2][8];
    const int C = a.C;
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int64_t last = first + a.rows < a.T ? first + a.rows : a.T;
    const int64_t strip = (int64_t)gridDim.x * C;
    float *const part = a.part + (int64_t)blockIdx.x * C;
    for (int64_t row = first; row < last; row++) {
        const float rstd1 = a.stats[row], rstd2 = a.stats[a.T + row];
        const float mean1 = a.layer ? a.stats[2 * a.T + row] : 0.0f, mean2 = a.layer ? a.stats[3 * a.T + row] : 0.0f;
        const T *dn = static_cast<const T *>(a.dN) + row * C;
        const T *dy = a.dY ? static_cast<const T *>(a.dY) + row * C : nullptr;
        float sg = 0.0f, sgx = 0.0f;
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float g = load_one(dn + c) * load_param(a.w2, a.w_dtype, c);
            sg += g;
            sgx = __builtin_fmaf(g, (Element<T>(a, row, c, mean1, rstd1).y - mean2) * rstd2, sgx);
        }
        group_sum2(sg, sgx, lds[0]);
        const float mg2 = a.layer ? sg / (float)C : 0.0f, mgx2 = sgx / (float)C;
        auto grad_y = [&](const Element<T> &e, int c) {
            const float g = load_one(dn + c) * load_param(a.w2, a.w_dtype, c), xh2 = (e.y - mean2) * rstd2;
            return __builtin_fmaf(rstd2, g - mg2 - xh2 * mgx2, dy ? load_one(dy + c) : 0.0f);
        };
        sg = sgx = 0.0f;
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const Element<T> e(a, row, c, mean1, rstd1);
            const float d = grad_y(e, c), dn1 = load_one(dn + c);
            const float g = d * e.gate * load_param(a.w1, a.w_dtype, c);
            sg += g;
            sgx = __builtin_fmaf(g, e.xh1, sgx);
            const float through = a.gate_kind == kGateToken ? d * e.gate : d;  // a feature's gate is applied to the sum
            float v[4] = {dn1 * ((e.y - mean2) * rstd2), through * e.xh1, dn1, through};
            for (int i = 0; i < a.sums; i++) {
                float *const at = part + i * strip + c;
                *at = row == first ? v[i] : *at + v[i];
            }
        }
        group_sum2(sg, sgx, lds[1]);
        const float mg1 = a.layer ? sg / (float)C : 0.0f, mgx1 = sgx / (float)C;
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const Element<T> e(a, row, c, mean1, rstd1);
            const float d = grad_y(e, c), g = d * e.gate * load_param(a.w1, a.w_dtype, c);
            const int64_t i = row * C + c;
            store_one(static_cast<T *>(a.dX) + i, a.scale * d);
            store_one(static_cast<T *>(a.dB) + i, rstd1 * (g - mg1 - e.xh1 * mgx1));
            if (a.gate_kind == kGateToken && a.dgate) store_one(static_cast<T *>(a.dgate) + i, d * e.u);
        }
    }
}

// Sums of the partial rows in order and in fp64: 16 columns x 16 row groups per sum of a workgroup, 8 loads in flight. A feature's
// gate is applied here: with S = sum_t dYt xh1 and R = sum_t dYt, dw1 = gate S, db1 = gate R, dgate = w1 S + b1 R.
__global__ void __launch_bounds__(1024) sandwich_finish_kernel(SandwichArgs a, int parts) {
    __shared__ double lds[4][16][17];
    const int col = threadIdx.x & 15, grp = (threadIdx.x >> 4) & 15, k = threadIdx.x >> 8, c = blockIdx.x * 16 + col, C = a.C;
    const int per = (parts + 15) / 16, r0 = grp * per, r1 = r0 + per < parts ? r0 + per : parts;
    const float *part = a.part + (int64_t)k * parts * C;
    double s = 0.0;
    if (c < C) {
        int r = r0;
        for (; r + 8 <= r1; r += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = part[(int64_t)(r + i) * C + c];
#pragma unroll
            for (int i = 0; i < 8; i++) s += (double)v[i];
        }
        for (; r < r1; r++) s += (double)part[(int64_t)r * C + c];
    }
    lds[k][grp][col] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= C) return;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    for (int q = 0; q < a.sums; q++)
        for (int i = 0; i < 16; i++) v[q] += lds[q][i][col];
    const bool feature = a.gate_kind == kGateFeature;
    const double gate = feature ? (double)load_param(a.gate, a.w_dtype, c) : 1.0;
    a.dw2[c] = (float)v[0];
    a.dw1[c] = (float)(gate * v[1]);
    if (a.db2) a.db2[c] = (float)v[2];
    if (a.db1) a.db1[c] = (float)(gate * v[3]);
    if (feature && a.dgate) {
        const double b1 = a.b1 ? (double)load_param(a.b1, a.w_dtype, c) : 0.0;
        static_cast<float *>(a.dgate)[c] = (float)((double)load_param(a.w1, a.w_dtype, c) * v[1] + b1 * v[3]);
    }
}

int64_t bwd_parts(int64_t T) {
    const int64_t rows = std::max<int64_t>(4, (T + kStrips - 1) / kStrips);
    return (T + rows - 1) / rows;
}

template <int... Vs, typename F>
bool pick_nv(int64_t need, F &&f) {
    bool done = false;
    ((!done && need <= Vs ? (f(std::integral_constant<int, Vs>{}), done = true) : false), ...);
    return done;
}

// Threads per row and vectors per thread: a wave per row up to 1,024 features, a workgroup up to 8,192 (32 elements per
// thread), false beyond that. f(threads, vectors, whether a row has a piece of fewer than 8)
template <typename F>
bool sandwich_shape(int64_t C, F &&f) {
    const int64_t vecs = (C + 7) / 8;
    auto tail = [&](auto threads, auto nv) { C % 8 ? f(threads, nv, std::true_type{}) : f(threads, nv, std::false_type{}); };
    if (vecs <= 64 * 2) return pick_nv<1, 2>((vecs + 63) / 64, [&](auto nv) { tail(std::integral_constant<int, 64>{}, nv); });
    return pick_nv<2, 4>((vecs + 255) / 256, [&](auto nv) { tail(std::integral_constant<int, 256>{}, nv); });
}

template <typename T, typename WT>
hipError_t sandwich_fwd(SandwichArgs a, hipStream_t st) {
    constexpr int64_t kRows = (int64_t(1) << 24) - 4;  // a launch's work-items (256 per row at most) stay below 2^32; whole workgroups
    for (a.first = 0; a.first < a.T; a.first += kRows) {
        const int64_t rows = std::min(kRows, a.T - a.first);
        const bool done = sandwich_shape(a.C, [&](auto threads, auto nv, auto tail) {
            constexpr int TH = decltype(threads)::value, per = kThreads / TH;
            sandwich_fwd_kernel<T, WT, TH, decltype(nv)::value, decltype(tail)::value>
                <<<(unsigned)((rows + per - 1) / per), kThreads, 0, st>>>(a);
        });
        if (!done) sandwich_fwd_long_kernel<T><<<(unsigned)rows, kThreads, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, typename WT>
hipError_t sandwich_bwd(const SandwichArgs &a, unsigned parts, hipStream_t st) {
    const bool done = sandwich_shape(a.C, [&](auto threads, auto nv, auto tail) {
        constexpr int TH = decltype(threads)::value, NV = decltype(nv)::value;
        constexpr size_t width = (size_t)NV * TH * 8;
        const bool token = a.gate_kind == kGateToken;
        const size_t params = (2 + !token + (a.sums == 4)) * width * sizeof(WT);
        const size_t lds = TH == 64 ? std::max(params, width * sizeof(float)) : params;
        auto go = [&](auto bias, auto of_token) {
            auto *const kernel = sandwich_bwd_kernel<T, WT, TH, NV, decltype(bias)::value, decltype(of_token)::value, decltype(tail)::value>;
            if (lds > 64 * 1024)
                (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            kernel<<<parts, kThreads, lds, st>>>(a);
        };
        if (a.sums == 4) token ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
        else token ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    });
    if (!done) sandwich_bwd_long_kernel<T><<<parts, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t sandwich_bwd_ws(int64_t T, int64_t C) {
    // the most strips that any number of tokens up to T takes, four sums
    return kWsHeader + (size_t)std::min<int64_t>((T + 3) / 4, kStrips) * (size_t)C * 4 * sizeof(float);
}

hipError_t launch_sandwich_fwd(int dtype, SandwichArgs a, hipStream_t st) {
    if (dtype == kBF16) return a.w_dtype == kBF16 ? sandwich_fwd<uint16_t, uint16_t>(a, st) : sandwich_fwd<uint16_t, float>(a, st);
    return a.w_dtype == kBF16 ? sandwich_fwd<float, uint16_t>(a, st) : sandwich_fwd<float, float>(a, st);
}

hipError_t launch_sandwich_bwd(int dtype, SandwichArgs a, void *ws, hipStream_t st) {
    const int64_t parts = bwd_parts(a.T);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader);
    a.rows = (a.T + parts - 1) / parts;
    a.sums = a.b1 || a.db1 || a.db2 ? 4 : 2;
    hipError_t e;
    if (dtype == kBF16) e = a.w_dtype == kBF16 ? sandwich_bwd<uint16_t, uint16_t>(a, (unsigned)parts, st) : sandwich_bwd<uint16_t, float>(a, (unsigned)parts, st);
    else e = a.w_dtype == kBF16 ? sandwich_bwd<float, uint16_t>(a, (unsigned)parts, st) : sandwich_bwd<float, float>(a, (unsigned)parts, st);
    if (e != hipSuccess) return e;
    sandwich_finish_kernel<<<(unsigned)((a.C + 15) / 16), 256 * a.sums, 0, st>>>(a, (int)parts);
    return hipGetLastError();
}

}  // namespace focus
