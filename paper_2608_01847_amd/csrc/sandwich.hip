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

constexpr int kThreads = 256;  // of a workgroup whose waves take rows by themselves, and of the kernels for long rows
constexpr int kMostThreads = 1024;
constexpr int kChunk = 64;     // rows whose gradients of a parameter are added up one by one in fp32, as a rule
constexpr int kStrips = 1024;  // workgroups of a backward launch at most, each with a row of partial sums per parameter

// Sums of two values over the threads that share a row, in every one of them: a wave (WAVE), or the workgroup of up to 16 waves.
// `lds` of 32 floats is free again after the next barrier of the caller's (buffers in turn).
template <bool WAVE = false>
__device__ __forceinline__ void group_sum2(float &a, float &b, float *lds) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (WAVE) return;
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x >> 6] = a;
        lds[16 + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll 4  // four reads under way: one by one, 16 waves take 0.7 us a row
    for (unsigned i = 0; i < blockDim.x / 64; i++) {
        a += lds[i];
        b += lds[16 + i];
    }
}

template <bool WAVE = false>
__device__ __forceinline__ float group_sum(float a, float *lds) {
    a = wave_sum(a);
    if constexpr (WAVE) return a;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = 0.0f;
    for (unsigned i = 0; i < blockDim.x / 64; i++) a += lds[i];
    return a;
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

// The parameters as the kernels use them, 8 at a time in fp32, 0 past the last feature: the gain and the shift after the block
// (times the gate, where a feature has one) and those before the next. `Params` keeps them in LDS, over the columns that a row's
// threads cover.
template <bool BIAS, bool TOKEN>
__device__ __forceinline__ void load_params(const SandwichArgs &a, int c, float (&w1)[8], float (&b1)[8], float (&w2)[8], float (&b2)[8]) {
    const int n = a.C - c;
    load8_param(a.w1, a.w_dtype, c, n, w1);
    load8_param(a.w2, a.w_dtype, c, n, w2);
    if constexpr (BIAS) {
        load8_param(a.b1, a.w_dtype, c, a.b1 ? n : 0, b1);
        load8_param(a.b2, a.w_dtype, c, a.b2 ? n : 0, b2);
    }
    if (!TOKEN && a.gate_kind == kGateFeature) {
        float g[8];
        load8_param(a.gate, a.w_dtype, c, n, g);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            w1[e] *= g[e];
            if constexpr (BIAS) b1[e] *= g[e];
        }
    }
}

template <bool BIAS, bool TOKEN>
struct Params {
    float *w1, *w2, *b1, *b2;
    __device__ __forceinline__ Params(const SandwichArgs &a, float *lds, int width) {
        w1 = lds, w2 = lds + width, b1 = lds + 2 * width, b2 = lds + 3 * width;
        const int c = threadIdx.x * 8;  // at least as many threads as vectors
        if (c >= width) return;
        float v[4][8];
        load_params<BIAS, TOKEN>(a, c, v[0], v[2], v[1], v[3]);
#pragma unroll
        for (int i = 0; i < (BIAS ? 4 : 2); i++)
#pragma unroll
            for (int h = 0; h < 2; h++)
                reinterpret_cast<float4 *>(lds + i * width + c)[h] = make_float4(v[i][4 * h], v[i][4 * h + 1], v[i][4 * h + 2], v[i][4 * h + 3]);
    }
    static size_t bytes(size_t width) { return (BIAS ? 4 : 2) * width * sizeof(float); }
};

__device__ __forceinline__ void lds8(const float *p, float (&v)[8]) {
    const float4 x = reinterpret_cast<const float4 *>(p)[0], y = reinterpret_cast<const float4 *>(p)[1];
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
}

// A row is shared by a wave (WAVE: four rows in a workgroup) or by the workgroup, NV vectors of 8 elements per thread: with n threads
// vector j of thread t starts at column (j n + t) 8. A row is read once, and U and Y stay in registers in fp32. Waves take one row each,
// with the parameters from the caches; a workgroup takes `rows` consecutive rows, with the parameters in LDS, and asks for the next
// row's pieces as soon as their registers are free. BIAS: with shifts; TOKEN: with gates of the tokens' own.
// Bound by memory: 65,536 x 2,560 bf16 268 us, 5.0 TB/s, bytes 1.00 times the tensors' (with 256 threads of two vectors and no row asked
// for ahead 313); 8,192 x 8,192 with token gates 129 us, 5.2 TB/s; a wave per row at 131,072 x 1,024 191 to 197 us, 5.5 TB/s. One row is four
// dependent trips to memory and LDS: 1 x 8,192 5.3 us.
template <typename T, bool WAVE, int NV, bool BIAS, bool TOKEN, bool TAIL>
__global__ void __launch_bounds__(WAVE ? kThreads : kMostThreads) sandwich_fwd_kernel(SandwichArgs a) {
    extern __shared__ __attribute__((aligned(16))) float smem[];
    __shared__ float lds[4][32];
    const int n_row = WAVE ? 64 : (int)blockDim.x;  // threads of a row
    const int t = WAVE ? threadIdx.x % 64 : threadIdx.x, sub = WAVE ? threadIdx.x / 64 : 0, C = a.C;
    const int64_t first = a.first + (int64_t)blockIdx.x * a.rows, last = first + a.rows < a.T ? first + a.rows : a.T;
    Raw8<T> xr[NV], br[NV], gr[TOKEN ? NV : 1];
    auto fetch = [&](Raw8<T> *to, const void *from, int64_t row) {
        const int n = row < last ? C : 0;
#pragma unroll
        for (int j = 0; j < NV; j++) load_piece<TAIL>(to[j], from, row * C, n, (j * n_row + t) * 8);
    };
    fetch(br, a.B, first + sub);
    fetch(xr, a.X, first + sub);
    if constexpr (TOKEN) fetch(gr, a.gate, first + sub);
    float *const p[4] = {smem, smem + NV * n_row * 8, smem + 2 * NV * n_row * 8, smem + 3 * NV * n_row * 8};
    if constexpr (!WAVE) {
        Params<BIAS, TOKEN>(a, smem, NV * n_row * 8);
        __syncthreads();
    }
    const float inv_n = 1.0f / (float)C;
    for (int64_t row = first + sub; row < last; row += WAVE ? 4 : 1) {
        const int64_t at = row * C;
        float mean1 = 0.0f, mean2 = 0.0f, q = 0.0f, y[NV][8], s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) y[j][e] = br[j][e];
        if (a.layer) {
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) s += y[j][e];
            mean1 = group_sum<WAVE>(s, lds[0]) * inv_n;
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int n = C - (j * n_row + t) * 8;  // elements of this vector that exist
#pragma unroll
                for (int e = 0; e < 8; e++) y[j][e] = e < n ? y[j][e] - mean1 : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) q = __builtin_fmaf(y[j][e], y[j][e], q);
        if constexpr (!WAVE) fetch(br, a.B, row + 1);
        const float rstd1 = 1.0f / sqrtf(group_sum<WAVE>(q, lds[1]) * inv_n + a.eps);
        s = 0.0f;
        float w2[WAVE ? NV : 1][8], b2[WAVE ? NV : 1][8];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * n_row + t) * 8;
            float w[8], b[8];
            if constexpr (WAVE) {
                load_params<BIAS, TOKEN>(a, c, w, b, w2[j], b2[j]);
            } else {
                lds8(p[0] + c, w);
                if constexpr (BIAS) lds8(p[2] + c, b);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {  // columns past C are 0
                const float xh = y[j][e] * rstd1;
                float u = BIAS ? __builtin_fmaf(xh, w[e], b[e]) : xh * w[e];
                if constexpr (TOKEN) u *= gr[TOKEN ? j : 0][e];
                y[j][e] = __builtin_fmaf(a.scale, xr[j][e], u);
                s += y[j][e];
            }
        }
        if constexpr (!WAVE) {
            fetch(xr, a.X, row + 1);
            if constexpr (TOKEN) fetch(gr, a.gate, row + 1);
        }
        if (a.layer) mean2 = group_sum<WAVE>(s, lds[2]) * inv_n;
        q = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int n = C - (j * n_row + t) * 8;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = !a.layer ? y[j][e] : e < n ? y[j][e] - mean2 : 0.0f;
                q = __builtin_fmaf(d, d, q);
            }
        }
        const float rstd2 = 1.0f / sqrtf(group_sum<WAVE>(q, lds[3]) * inv_n + a.eps);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * n_row + t) * 8;
            if (c < C) {
                float w[8], b[8];
                if constexpr (WAVE) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        w[e] = w2[j][e];
                        if constexpr (BIAS) b[e] = b2[j][e];
                    }
                } else {
                    lds8(p[1] + c, w);
                    if constexpr (BIAS) lds8(p[3] + c, b);
                }
                store8_n<TAIL>(static_cast<T *>(a.Y) + at + c, C - c, y[j]);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float xh = (y[j][e] - mean2) * rstd2;
                    y[j][e] = BIAS ? __builtin_fmaf(xh, w[e], b[e]) : xh * w[e];
                }
                store8_n<TAIL>(static_cast<T *>(a.N) + at + c, C - c, y[j]);
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
}

// Rows, threads and the next row's pieces as in the forward; the sums over the rows stay in registers, for `chunk` of them (64 as a
// rule, so that no chain of fp32 additions is as long as a workgroup's rows), and are then added to its row of partial sums (waves
// that take rows by themselves are added in order through LDS first). BIAS: the sums without xh too.
// Memory and its latency bound rows of whole eights: 65,536 x 2,560 bf16 458 us, 4.4 TB/s, bytes 1.00 times the tensors', without a
// gradient of Y 408; 8,192 x 8,192 with token gates 213 us, 5.0 TB/s; 16,384 x 8,192 fp32 632 us, 5.1 TB/s. The next row's B and gates have
// registers of their own where there are as many (bf16, whole eights), since the present ones are needed to the row's end: fetched there
// 65,536 x 2,560 took 6% longer; dN and dY the same way 2 and 8%. Before, a workgroup of 256 threads with two vectors each took 8% longer
// than one of five waves, that without the next row under way 20% and with the parameters converted anew for each row 6%. A wave per row:
// 131,072 x 1,024 339 us, 4.8 TB/s; 262,144 x 512 with token gates 458.
// Rows that are no whole eights take more registers (addresses, the last piece's branches) than the 128 that 1,024 threads leave each: in
// fp32 33 of them go to memory with shifts and token gates, 17 with shifts, 12 with token gates, 1 otherwise, in bf16 8 with both (2 in
// fp32 rows of whole eights with both, none elsewhere). Layer norm, token gates and shifts, 32,768 x 2,561 fp32 896 us, 3.0 TB/s, x 2,560
// 564, 4.8; bf16 444 and 325; 8,192 x 5,001 fp32 487, 2.7 TB/s.
template <typename T, bool WAVE, int NV, bool BIAS, bool TOKEN, bool TAIL>
__global__ void __launch_bounds__(WAVE ? kThreads : kMostThreads) sandwich_bwd_kernel(SandwichArgs a) {
    constexpr int kRows = WAVE ? 4 : 1;
    extern __shared__ __attribute__((aligned(16))) float smem[];
    __shared__ float lds[2][32];
    const int n_row = WAVE ? 64 : (int)blockDim.x;
    const int t = WAVE ? threadIdx.x % 64 : threadIdx.x, sub = WAVE ? threadIdx.x / 64 : 0, C = a.C;
    const int64_t first = (int64_t)blockIdx.x * a.rows, last = first + a.rows < a.T ? first + a.rows : a.T;
    constexpr int kSums = BIAS ? 4 : 2;
    float sums[kSums][NV][8];
#pragma unroll
    for (int i = 0; i < kSums; i++)
#pragma unroll
        for (int j = 0; j < NV; j++) zero8(sums[i][j]);
    const float inv_n = 1.0f / (float)C;
    Raw8<T> xr[NV], br[NV], nr[NV], yr[NV], gr[TOKEN ? NV : 1];
    // B and a token's gate are needed to the row's end: the next row's have registers of their own, where there are as many
    constexpr bool kAhead = !WAVE && !TAIL && sizeof(T) == 2;
    Raw8<T> bn[kAhead ? NV : 1], gn[kAhead && TOKEN ? NV : 1];
    auto fetch = [&](Raw8<T> *to, const void *from, int64_t row) {
        const int n = WAVE || row < last ? C : 0;  // waves ask for the rows that they take alone
#pragma unroll
        for (int j = 0; j < NV; j++) load_piece<TAIL>(to[j], from, row * C, n, (j * n_row + t) * 8);
    };
    float stat[4];
    auto fetch_stats = [&](int64_t row) {
        row = WAVE || row < last ? row : first;
#pragma unroll
        for (int i = 0; i < 4; i++) stat[i] = i < 2 || a.layer ? a.stats[i * a.T + row] : 0.0f;
    };
    auto fetch_all = [&](int64_t row) {
        fetch(br, a.B, row);
        fetch(xr, a.X, row);
        if constexpr (TOKEN) fetch(gr, a.gate, row);
        fetch(nr, a.dN, row);
        fetch(yr, a.dY, row);
        fetch_stats(row);
    };
    if constexpr (!WAVE) fetch_all(first);
    const Params<BIAS, TOKEN> p(a, smem, NV * n_row * 8);
    __syncthreads();
    const int rows = (int)(last - first);
    for (int start = 0; start < rows; start += a.chunk * kRows) {
        const int end = rows - start < a.chunk * kRows ? rows : start + a.chunk * kRows;
        for (int i = start + sub; i < end; i += kRows) {
            const int64_t row = first + i, at = row * C;
            if constexpr (WAVE) fetch_all(row);
            // xh = h rstd - mean rstd in one operation: what the product is off by is as little as the mean itself may be
            const float rstd1 = stat[0], rstd2 = stat[1], off1 = -stat[2] * rstd1, off2 = -stat[3] * rstd2;
            if constexpr (!WAVE) fetch_stats(row + 1);
            if constexpr (kAhead) {
                fetch(bn, a.B, row + 1);
                if constexpr (TOKEN) fetch(gn, a.gate, row + 1);
            }
            // keeps the compiler from holding over the next sum what the packed rows and the LDS give again
            auto again = [&]() {
                asm volatile("" ::: "memory");
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    br[j].keep_packed();
                    if constexpr (WAVE) nr[j].keep_packed(), yr[j].keep_packed();
                    if constexpr (TOKEN) gr[j].keep_packed();
                }
            };
            // xh2 of the row, and the two means that the second norm's gradient takes
            float d[NV][8], sg = 0.0f, sgx = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; j++) {
                __builtin_amdgcn_sched_barrier(0);  // one vector's values in fp32 at a time
                const int c = (j * n_row + t) * 8;
                float w1[8], w2[8], b1[8];
                lds8(p.w1 + c, w1);
                lds8(p.w2 + c, w2);
                if constexpr (BIAS) lds8(p.b1 + c, b1);
#pragma unroll
                for (int e = 0; e < 8; e++) {  // columns past C have dN = 0
                    const float xh1 = __builtin_fmaf(br[j][e], rstd1, off1);
                    float u = BIAS ? __builtin_fmaf(xh1, w1[e], b1[e]) : xh1 * w1[e];
                    if constexpr (TOKEN) u *= gr[TOKEN ? j : 0][e];
                    const float xh2 = __builtin_fmaf(__builtin_fmaf(a.scale, xr[j][e], u), rstd2, off2);
                    const float n = nr[j][e], g = n * w2[e];
                    sums[0][j][e] = __builtin_fmaf(n, xh2, sums[0][j][e]);
                    if constexpr (BIAS) sums[2][j][e] += n;
                    sg += g;
                    sgx = __builtin_fmaf(g, xh2, sgx);
                    d[j][e] = xh2;
                }
            }
            if constexpr (!WAVE) fetch(xr, a.X, row + 1);
            group_sum2<WAVE>(sg, sgx, lds[0]);
            const float mg2 = a.layer ? sg * inv_n : 0.0f, mgx2 = sgx * inv_n;
            sg = sgx = 0.0f;
            again();
#pragma unroll
            for (int j = 0; j < NV; j++) {
                __builtin_amdgcn_sched_barrier(0);
                const int c = (j * n_row + t) * 8;
                float w1[8], w2[8];
                lds8(p.w1 + c, w1);
                lds8(p.w2 + c, w2);
#pragma unroll
                for (int e = 0; e < 8; e++) {  // columns past C have w1 = 0
                    const float g2 = __builtin_fmaf(-d[j][e], mgx2, __builtin_fmaf(nr[j][e], w2[e], -mg2));
                    d[j][e] = __builtin_fmaf(rstd2, g2, yr[j][e]);
                    const float xh1 = __builtin_fmaf(br[j][e], rstd1, off1);
                    const float through = TOKEN ? d[j][e] * gr[TOKEN ? j : 0][e] : d[j][e];  // a feature's gate is applied to the sum
                    sums[1][j][e] = __builtin_fmaf(through, xh1, sums[1][j][e]);
                    if constexpr (BIAS) sums[3][j][e] += through;
                    const float g = through * w1[e];
                    sg += g;
                    sgx = __builtin_fmaf(g, xh1, sgx);
                }
            }
            if constexpr (!WAVE) {
                fetch(nr, a.dN, row + 1);
                fetch(yr, a.dY, row + 1);
            }
            group_sum2<WAVE>(sg, sgx, lds[1]);
            const float mg1 = a.layer ? sg * inv_n : 0.0f, mgx1 = sgx * inv_n;
            again();
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (j * n_row + t) * 8;
                __builtin_amdgcn_sched_barrier(0);
                if (c < C) {
                    float v[8], w1[8], b1[8];
                    lds8(p.w1 + c, w1);
                    if constexpr (BIAS) lds8(p.b1 + c, b1);
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = a.scale * d[j][e];
                    store8_n<TAIL>(static_cast<T *>(a.dX) + at + c, C - c, v);
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float xh1 = __builtin_fmaf(br[j][e], rstd1, off1);
                        const float g = (TOKEN ? d[j][e] * gr[TOKEN ? j : 0][e] : d[j][e]) * w1[e];
                        v[e] = rstd1 * __builtin_fmaf(-xh1, mgx1, g - mg1);
                    }
                    store8_n<TAIL>(static_cast<T *>(a.dB) + at + c, C - c, v);
                    if (TOKEN && a.dgate) {
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            const float xh1 = __builtin_fmaf(br[j][e], rstd1, off1);
                            v[e] = d[j][e] * (BIAS ? __builtin_fmaf(xh1, w1[e], b1[e]) : xh1 * w1[e]);
                        }
                        store8_n<TAIL>(static_cast<T *>(a.dgate) + at + c, C - c, v);
                    }
                }
            }
            if constexpr (kAhead) {
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    br[j] = bn[j];
                    if constexpr (TOKEN) gr[j] = gn[j];
                }
            } else if constexpr (!WAVE) {
                fetch(br, a.B, row + 1);
                if constexpr (TOKEN) fetch(gr, a.gate, row + 1);
            }
        }
        int lane = t;
        asm volatile("" : "+v"(lane));  // addresses formed here: formed before the rows, they would hold registers over them
        float *const join = smem + (BIAS ? 4 : 2) * NV * n_row * 8;  // of waves that take rows by themselves: a row's width behind the parameters
#pragma unroll
        for (int i = 0; i < kSums; i++) {
            if constexpr (WAVE) {
                for (int s = 1; s < kRows; s++) {
                    __syncthreads();
                    if (sub == s)
#pragma unroll
                        for (int j = 0; j < NV; j++)
#pragma unroll
                            for (int e = 0; e < 8; e++) join[(j * 8 + e) * 64 + lane] = sums[i][j][e];
                    __syncthreads();
                    if (sub == 0)
#pragma unroll
                        for (int j = 0; j < NV; j++)
#pragma unroll
                            for (int e = 0; e < 8; e++) sums[i][j][e] += join[(j * 8 + e) * 64 + lane];
                }
            }
            if (sub == 0) {
                float *const part = a.part + ((int64_t)i * gridDim.x + blockIdx.x) * C;
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    const int c = (j * n_row + lane) * 8;
                    if (c < C) {
                        if (start) {
                            float v[8];
                            load8_n(part + c, TAIL ? C - c : 8, v);
#pragma unroll
                            for (int e = 0; e < 8; e++) sums[i][j][e] += v[e];
                        }
                        store8_n<TAIL>(part + c, C - c, sums[i][j]);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < NV; j++) zero8(sums[i][j]);
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

// Rows of more than 8,192 features, which registers and LDS do not hold: a workgroup per row, which it reads once for each sum and once
// for the outputs, element by element. Not tuned: 2,048 x 8,200 bf16 79 us, backward 517 (x 8,192 25 and 44).
template <typename T>
__global__ void __launch_bounds__(kThreads) sandwich_fwd_long_kernel(SandwichArgs a) {
    __shared__ float lds[2][32];
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

// A workgroup takes `rows` rows, kLongRows at a time: first their means, row by row, then their gradients and the sums over them, column
// by column, which are added to its row of the partial sums, so that no chain of fp32 additions is as long as its rows.
constexpr int kLongRows = kChunk;
template <typename T>
__global__ void __launch_bounds__(kThreads) sandwich_bwd_long_kernel(SandwichArgs a) {
    __shared__ float lds[2][32];
    __shared__ float4 means[kLongRows];  // of g2, g2 xh2, g1 and g1 xh1
    const int C = a.C;
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int64_t last = first + a.rows < a.T ? first + a.rows : a.T;
    const int64_t strip = (int64_t)gridDim.x * C;
    float *const part = a.part + (int64_t)blockIdx.x * C;
    struct Row {
        const T *dn, *dy;
        float rstd1, rstd2, mean1, mean2;
    };
    auto row_of = [&](int64_t row) {
        return Row{static_cast<const T *>(a.dN) + row * C, a.dY ? static_cast<const T *>(a.dY) + row * C : nullptr, a.stats[row],
                   a.stats[a.T + row], a.layer ? a.stats[2 * a.T + row] : 0.0f, a.layer ? a.stats[3 * a.T + row] : 0.0f};
    };
    auto grad_y = [&](const Row &r, const Element<T> &e, int c, float mg2, float mgx2) {
        const float g = load_one(r.dn + c) * load_param(a.w2, a.w_dtype, c), xh2 = (e.y - r.mean2) * r.rstd2;
        return __builtin_fmaf(r.rstd2, g - mg2 - xh2 * mgx2, r.dy ? load_one(r.dy + c) : 0.0f);
    };
    for (int64_t start = first; start < last; start += kLongRows) {
        const int n = (int)(last - start < kLongRows ? last - start : kLongRows);
        for (int i = 0; i < n; i++) {
            const Row r = row_of(start + i);
            float sg = 0.0f, sgx = 0.0f;
            for (int c = threadIdx.x; c < C; c += kThreads) {
                const float g = load_one(r.dn + c) * load_param(a.w2, a.w_dtype, c);
                sg += g;
                sgx = __builtin_fmaf(g, (Element<T>(a, start + i, c, r.mean1, r.rstd1).y - r.mean2) * r.rstd2, sgx);
            }
            group_sum2(sg, sgx, lds[0]);
            const float mg2 = a.layer ? sg / (float)C : 0.0f, mgx2 = sgx / (float)C;
            sg = sgx = 0.0f;
            for (int c = threadIdx.x; c < C; c += kThreads) {
                const Element<T> e(a, start + i, c, r.mean1, r.rstd1);
                const float g = grad_y(r, e, c, mg2, mgx2) * e.gate * load_param(a.w1, a.w_dtype, c);
                sg += g;
                sgx = __builtin_fmaf(g, e.xh1, sgx);
            }
            group_sum2(sg, sgx, lds[1]);
            if (threadIdx.x == 0) means[i] = make_float4(mg2, mgx2, a.layer ? sg / (float)C : 0.0f, sgx / (float)C);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += kThreads) {
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int i = 0; i < n; i++) {
                const Row r = row_of(start + i);
                const float4 m = means[i];
                const Element<T> e(a, start + i, c, r.mean1, r.rstd1);
                const float dn = load_one(r.dn + c), d = grad_y(r, e, c, m.x, m.y), g = d * e.gate * load_param(a.w1, a.w_dtype, c);
                const float through = a.gate_kind == kGateToken ? d * e.gate : d;  // a feature's gate is applied to the sum
                v[0] += dn * ((e.y - r.mean2) * r.rstd2);
                v[1] += through * e.xh1;
                v[2] += dn;
                v[3] += through;
                const int64_t at = (start + i) * C + c;
                store_one(static_cast<T *>(a.dX) + at, a.scale * d);
                store_one(static_cast<T *>(a.dB) + at, r.rstd1 * (g - m.z - e.xh1 * m.w));
                if (a.gate_kind == kGateToken && a.dgate) store_one(static_cast<T *>(a.dgate) + at, d * e.u);
            }
            for (int i = 0; i < a.sums; i++) {
                float *const at = part + i * strip + c;
                *at = start == first ? v[i] : *at + v[i];
            }
        }
        __syncthreads();  // the means are read
    }
}

// Sums of the partial rows in order and in fp64: 16 columns x 16 row groups per sum of a workgroup, 8 loads in flight. Bound by the
// loads' latency, 8 rounds of them at 1,024 rows: 9 us for 1,001 features and 4 sums, 10.5 for 2,560 and 2. 64 row groups of 16 threads
// for all sums took 15 (16 MB in 64-byte pieces, and twice the LDS steps). A feature's gate is applied here: with S = sum_t dYt xh1 and R = sum_t dYt, dw1 = gate S, db1 = gate R, dgate = w1 S + b1 R.
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

// Who shares a row: a wave up to 1,024 features, beyond that a workgroup of as many waves as its vectors of 8 take; false past
// 8,192. f(wave, vectors per thread, whether a row has a piece of fewer than 8, threads)
template <typename F>
bool sandwich_shape(int64_t C, F &&f) {
    const int64_t vecs = (C + 7) / 8;
    auto tail = [&](auto wave, auto nv, int64_t n) {
        C % 8 ? f(wave, nv, std::true_type{}, (unsigned)n) : f(wave, nv, std::false_type{}, (unsigned)n);
    };
    if (vecs > kMostThreads) return false;
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 2> two{};
    if (vecs <= 64) tail(std::true_type{}, one, kThreads);
    else if (vecs <= 128) tail(std::true_type{}, two, kThreads);
    else tail(std::false_type{}, one, (vecs + 63) / 64 * 64);
    return true;
}

// Workgroups of a launch that keeps the parameters in LDS: as many as are resident at once with four waves per SIMD (a second round
// of workgroups would take as long as the first), each with `least` rows at least.
int64_t sandwich_parts(int64_t T, int64_t C, int64_t least) {
    const int64_t waves = C <= 1024 ? 4 : std::min<int64_t>(16, (C + 511) / 512);
    const int64_t strips = std::min<int64_t>(kStrips, 256 * (16 / waves)), rows = std::max<int64_t>(least, (T + strips - 1) / strips);
    return (T + rows - 1) / rows;
}

// Launches kernel(bias, token) with the parameters' LDS
template <typename F>
void sandwich_go(const SandwichArgs &a, bool bias, bool wave, int nv, unsigned threads, unsigned parts, hipStream_t st, F &&kernel) {
    const size_t width = (size_t)nv * (wave ? 64 : threads) * 8;
    auto go = [&](auto with_bias, auto of_token) {
        auto *const k = kernel(with_bias, of_token);
        // the parameters, 128 KB at most, and where waves take rows by themselves what joins their sums
        const size_t lds = Params<decltype(with_bias)::value, decltype(of_token)::value>::bytes(width) + (wave ? width * sizeof(float) : 0);
        if (lds > 64 * 1024)
            (void)hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        k<<<parts, threads, lds, st>>>(a);
    };
    const bool token = a.gate_kind == kGateToken;
    if (bias) token ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    else token ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
}

template <typename T>
hipError_t sandwich_fwd(SandwichArgs a, hipStream_t st) {
    // A launch's work-items stay below 2^32. Up to 1,024 features a workgroup is four rows; up to 8,192 there are as many as are
    // resident; beyond that one per row.
    const int64_t most = a.C <= 1024 ? int64_t(1) << 25 : a.C <= 8 * kMostThreads ? a.T : (int64_t(1) << 24) - 1;
    for (a.first = 0; a.first < a.T; a.first += most) {
        const int64_t rows = std::min(most, a.T - a.first);
        const int64_t parts = a.C <= 1024 ? (rows + 3) / 4 : a.C <= 8 * kMostThreads ? sandwich_parts(rows, a.C, 1) : rows;
        a.rows = (rows + parts - 1) / parts;
        if (a.C <= 1024) a.rows = 4;
        const bool done = sandwich_shape(a.C, [&](auto wave, auto nv, auto tail, unsigned threads) {
            sandwich_go(a, a.b1 || a.b2, wave.value, nv.value, threads, (unsigned)parts, st, [](auto bias, auto token) {
                return &sandwich_fwd_kernel<T, decltype(wave)::value, decltype(nv)::value, decltype(bias)::value,
                                            decltype(token)::value, decltype(tail)::value>;
            });
        });
        if (!done) sandwich_fwd_long_kernel<T><<<(unsigned)parts, kThreads, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t sandwich_bwd(const SandwichArgs &a, unsigned parts, hipStream_t st) {
    const bool done = sandwich_shape(a.C, [&](auto wave, auto nv, auto tail, unsigned threads) {
        sandwich_go(a, a.sums == 4, wave.value, nv.value, threads, parts, st, [](auto bias, auto token) {
            return &sandwich_bwd_kernel<T, decltype(wave)::value, decltype(nv)::value, decltype(bias)::value, decltype(token)::value,
                                        decltype(tail)::value>;
        });
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
    return dtype == kBF16 ? sandwich_fwd<uint16_t>(a, st) : sandwich_fwd<float>(a, st);
}

hipError_t launch_sandwich_bwd(int dtype, SandwichArgs a, void *ws, hipStream_t st) {
    const int64_t parts = sandwich_parts(a.T, a.C, 4);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader);
    a.rows = (a.T + parts - 1) / parts;
    // rows of a chain of fp32 additions: 64, and where there are more than 64 such chains (a wave has a quarter of the rows up to 1,024
    // features) the root of their number
    const int64_t of_one = a.C <= 1024 ? (a.rows + 3) / 4 : a.rows;
    a.chunk = kChunk;
    while ((int64_t)a.chunk * a.chunk < of_one) a.chunk++;
    a.sums = a.b1 || a.db1 || a.db2 ? 4 : 2;
    const hipError_t e = dtype == kBF16 ? sandwich_bwd<uint16_t>(a, (unsigned)parts, st) : sandwich_bwd<float>(a, (unsigned)parts, st);
    if (e != hipSuccess) return e;
    sandwich_finish_kernel<<<(unsigned)((a.C + 15) / 16), 256 * a.sums, 0, st>>>(a, (int)parts);
    return hipGetLastError();
}

}  // namespace focus
