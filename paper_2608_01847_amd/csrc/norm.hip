// Layer norm and RMS norm over the features of a token, with the residual sum in front, and their backward
// pass with the reduction of the gain's and the shift's gradients over the tokens.
//
//   H = X + R (rounded to the tensors' type),  mean = (1/C) sum H (layer) or 0 (RMS),
//   rstd = 1 / sqrt((1/C) sum (H - mean)^2 + eps),  xh = (H - mean) rstd,  Y = xh w + b
//   g = dY w:  dX = rstd (g - [mean g] - xh mean(g xh)) + dR,  dw = sum_t dY xh,  db = sum_t dY
//   (the bracketed term is the layer norm's only)
//
// HBM-bound: a row is read once and stays in registers between the sums and the outputs, in fp32. The
// variance is the sum of squared differences from the mean, so a large mean costs no digits.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormStrips = 1024;  // workgroups of a backward launch, each with one row of partial sums

// Sum over the THREADS threads that share a row: a wave, or a workgroup through `lds`, which is free again after the
// next barrier of its caller's loop (two buffers in turn).
template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float *lds) {
    v = wave_sum(v);
    if constexpr (THREADS > 64) {
        constexpr int W = THREADS / 64;
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < W; i++) v += lds[i];
    }
    return v;
}

template <int THREADS>
__device__ __forceinline__ void row_sum2(float &a, float &b, float *lds) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (THREADS > 64) {
        constexpr int W = THREADS / 64;
        if ((threadIdx.x & 63) == 0) {
            lds[threadIdx.x >> 6] = a;
            lds[W + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < W; i++) {
            a += lds[i];
            b += lds[W + i];
        }
    }
}

// Piece c .. c + 7 of a row of C elements (zeros past its end). Rows of whole eights go through the range check of a buffer
// load instead of a branch around each piece, over which the compiler holds the unpacked values. The row's address is the same
// for every lane of a wave.
template <bool TAIL, typename T>
__device__ __forceinline__ void load_piece(Raw8<T> &v, const T *row, int C, int c) {
    if constexpr (TAIL) {
        v.load(row + c, C - c);
    } else {
        const uint64_t p = (uint64_t)row;
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
        v.load_row(make_rsrc((const void *)((uint64_t)hi << 32 | lo), (int64_t)C * (int64_t)sizeof(T)), c);
    }
}

struct NormFwdArgs {
    const void *X, *R, *w, *b;
    void *H, *Y;
    float *mean, *rstd;
    int64_t T;
    int C, w_dtype, layer;
    float eps;
};

// A row is shared by THREADS threads (64: four rows per workgroup), NV vectors of 8 elements each: vector j of
// thread t starts at column (j THREADS + t) 8. HBM-bound: 65,536 x 2,560 bf16 with the residual, 1.34 GB, 226 us (5.9 TB/s;
// a copy reaches 4.8). One row of 8,192 takes 5 us, four trips to memory and back.
template <typename T, int THREADS, int NV, bool TAIL>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_kernel(NormFwdArgs a) {
    __shared__ float lds[2][2 * (kNormThreads / 64)];
    constexpr int kRows = kNormThreads / THREADS;
    const int t = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
    if (row >= a.T) return;  // whole waves where rows share a workgroup; no barrier is used there
    const int C = a.C;
    const T *x = static_cast<const T *>(a.X) + row * C;
    float h[NV][8];
    Raw8<T> xr[NV], rr[NV];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
        load_piece<TAIL>(xr[j], x, C, c);
        if (a.R) load_piece<TAIL>(rr[j], static_cast<const T *>(a.R) + row * C, C, c);
    }
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
#pragma unroll
        for (int e = 0; e < 8; e++) h[j][e] = xr[j][e];
        if (a.R && c < C) {
            float rv[8];
#pragma unroll
            for (int e = 0; e < 8; e++) rv[e] = rr[j][e];
            add_rounded<T>(h[j], rv);
            store8_n<TAIL>(static_cast<T *>(a.H) + row * C + c, C - c, h[j]);
        }
    }
    float mean = 0.0f;
    if (a.layer) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) s += h[j][e];
        mean = row_sum<THREADS>(s, lds[0]) / (float)C;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int n = C - (j * THREADS + t) * 8;  // elements of this vector that exist
#pragma unroll
        for (int e = 0; e < 8; e++) {
            h[j][e] = e < n ? h[j][e] - mean : 0.0f;
            q = __builtin_fmaf(h[j][e], h[j][e], q);
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<THREADS>(q, lds[1]) / (float)C + a.eps);
    T *y = static_cast<T *>(a.Y) + row * C;
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
        if (c < C) {
            float wv[8], bv[8];
            load8_param(a.w, a.w_dtype, c, C - c, wv);
            if (a.b) load8_param(a.b, a.w_dtype, c, C - c, bv);
            else zero8(bv);
#pragma unroll
            for (int e = 0; e < 8; e++) h[j][e] = __builtin_fmaf(h[j][e] * rstd, wv[e], bv[e]);
            store8_n<TAIL>(y + c, C - c, h[j]);
        }
    }
    if (t == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

// Rows too long for the registers: the row is read three times (layer: sum, squares, output), element by element.
template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_long_kernel(NormFwdArgs a) {
    __shared__ float lds[2][2 * (kNormThreads / 64)];
    const int64_t row = blockIdx.x;
    const int C = a.C;
    const T *h = static_cast<const T *>(a.X) + row * C;
    if (a.R) {
        const T *x = h, *r = static_cast<const T *>(a.R) + row * C;
        T *hout = static_cast<T *>(a.H) + row * C;
        for (int c = threadIdx.x; c < C; c += kNormThreads) store_one(hout + c, load_one(x + c) + load_one(r + c));
        h = hout;  // each thread reads back its own elements only
    }
    float mean = 0.0f;
    if (a.layer) {
        float s = 0.0f;
        for (int c = threadIdx.x; c < C; c += kNormThreads) s += load_one(h + c);
        mean = row_sum<kNormThreads>(s, lds[0]) / (float)C;
    }
    float q = 0.0f;
    for (int c = threadIdx.x; c < C; c += kNormThreads) {
        const float d = load_one(h + c) - mean;
        q = __builtin_fmaf(d, d, q);
    }
    const float rstd = 1.0f / sqrtf(row_sum<kNormThreads>(q, lds[1]) / (float)C + a.eps);
    T *y = static_cast<T *>(a.Y) + row * C;
    for (int c = threadIdx.x; c < C; c += kNormThreads) {
        const float bv = a.b ? load_param(a.b, a.w_dtype, c) : 0.0f;
        store_one(y + c, __builtin_fmaf((load_one(h + c) - mean) * rstd, load_param(a.w, a.w_dtype, c), bv));
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

struct NormBwdArgs {
    const void *dY, *H, *w, *dR;
    const float *mean, *rstd;
    void *dX;
    float *part_w, *part_b;  // [gridDim.x][C]; part_b NULL where no shift's gradient is asked for
    int64_t T, rows;         // rows per workgroup
    int C, w_dtype, layer;
};

// A workgroup takes `rows` consecutive rows; the sums over them of dY xh and dY stay in registers and leave as one row
// of partial sums per workgroup (waves that take rows by themselves are added in order through LDS first).
// HBM-bound: 65,536 x 2,560 bf16 with the residual's gradient, 1.34 GB, 280 us (4.8 TB/s); 1,024 workgroups are four per CU, all
// resident, so the sums leave once. 2,037 x 1,001 fp32, 24 MB: 10 us, of which two rows' latency per wave is most.
template <typename T, int THREADS, int NV, bool BIAS, bool TAIL>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(NormBwdArgs a) {
    constexpr int kRows = kNormThreads / THREADS;  // rows under way in a workgroup
    __shared__ float lds[2][2 * (kNormThreads / 64)];
    __shared__ float join[THREADS == 64 ? NV * 8 * 64 : 1];
    __shared__ float gain[THREADS == 64 ? NV * 8 * 64 : 1];
    const int t = threadIdx.x % THREADS, sub = threadIdx.x / THREADS, C = a.C;
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int64_t last = first + a.rows < a.T ? first + a.rows : a.T;
    float wv[THREADS == 64 ? 1 : NV][8], dw[NV][8], db[BIAS ? NV : 1][8];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * THREADS + t) * 8;
        zero8(dw[j]);
        if constexpr (BIAS) zero8(db[j]);
        if constexpr (THREADS != 64) {
            zero8(wv[j]);
            if (c < C) load8_param(a.w, a.w_dtype, c, C - c, wv[j]);
        }
    }
    // the four waves of a workgroup share the gain in LDS
    if constexpr (THREADS == 64) {
        for (int c = threadIdx.x; c < NV * 8 * 64; c += kNormThreads) gain[c] = c < C ? load_param(a.w, a.w_dtype, c) : 0.0f;
        __syncthreads();
    }
    auto weights = [&](int j, float (&w)[8]) {
        if constexpr (THREADS == 64) {
            const float4 *p = reinterpret_cast<const float4 *>(&gain[(j * 64 + t) * 8]);
            const float4 x = p[0], y = p[1];
            w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w, w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) w[e] = wv[j][e];
        }
    };
    const float inv_c = 1.0f / (float)C;
    int turn = 0;
    for (int64_t row = first + sub; row < last; row += kRows) {
        const T *dy = static_cast<const T *>(a.dY) + row * C, *h = static_cast<const T *>(a.H) + row * C;
        const T *dr = a.dR ? static_cast<const T *>(a.dR) + row * C : nullptr;
        const float rstd = a.rstd[row], mean = a.layer ? a.mean[row] : 0.0f;
        // the row as it lies, unpacked once for the sums and once for the result: half the registers of bf16 rows in
        // fp32, and twice the waves
        Raw8<T> gr[NV], hr[NV], rr[NV];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * THREADS + t) * 8;
            load_piece<TAIL>(gr[j], dy, C, c);
            load_piece<TAIL>(hr[j], h, C, c);
            load_piece<TAIL>(rr[j], dr, dr ? C : 0, c);
        }
        float sg = 0.0f, sgx = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            float w[8];
            weights(j, w);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float g = gr[j][e], xh = (hr[j][e] - mean) * rstd;  // columns past C hold g = 0
                dw[j][e] = __builtin_fmaf(g, xh, dw[j][e]);
                if constexpr (BIAS) db[j][e] += g;
                const float gw = g * w[e];
                sg += gw;
                sgx = __builtin_fmaf(gw, xh, sgx);
            }
        }
        row_sum2<THREADS>(sg, sgx, lds[turn]);
        turn ^= 1;
        const float mg = a.layer ? sg * inv_c : 0.0f, mgx = sgx * inv_c;
        T *dx = static_cast<T *>(a.dX) + row * C;
        asm volatile("" ::: "memory");  // the gain is read from LDS again rather than held
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * THREADS + t) * 8;
            gr[j].keep_packed();
            hr[j].keep_packed();
            if (c < C) {
                float w[8], x[8];
                weights(j, w);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float xh = (hr[j][e] - mean) * rstd;
                    x[e] = __builtin_fmaf(rstd, gr[j][e] * w[e] - mg - xh * mgx, rr[j][e]);
                }
                store8_n<TAIL>(dx + c, C - c, x);
            }
        }
    }
    auto put = [&](float (&v)[NV][8], float *part) {
        if constexpr (THREADS == 64) {
            for (int s = 1; s < kRows; s++) {
                __syncthreads();
                if (sub == s)
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) join[(j * 8 + e) * 64 + t] = v[j][e];
                __syncthreads();
                if (sub == 0)
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) v[j][e] += join[(j * 8 + e) * 64 + t];
            }
        }
        if (sub == 0) {
            float *const row = part + (int64_t)blockIdx.x * C;
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (j * THREADS + t) * 8;
                if (c < C) store8_n<TAIL>(row + c, C - c, v[j]);
            }
        }
    };
    put(dw, a.part_w);
    if constexpr (BIAS) put(db, a.part_b);
}

// Rows too long for the registers: dX row by row, then the columns' sums over the workgroup's rows, both re-reading.
template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_long_kernel(NormBwdArgs a) {
    __shared__ float lds[2][2 * (kNormThreads / 64)];
    const int C = a.C;
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int64_t last = first + a.rows < a.T ? first + a.rows : a.T;
    const T *dY = static_cast<const T *>(a.dY), *H = static_cast<const T *>(a.H);
    for (int c = threadIdx.x; c < C; c += kNormThreads) {  // before dX, which may stand in dY's place
        float dw = 0.0f, db = 0.0f;
        for (int64_t row = first; row < last; row++) {
            const float g = load_one(dY + row * C + c);
            dw = __builtin_fmaf(g, (load_one(H + row * C + c) - (a.layer ? a.mean[row] : 0.0f)) * a.rstd[row], dw);
            db += g;
        }
        a.part_w[(int64_t)blockIdx.x * C + c] = dw;
        if (a.part_b) a.part_b[(int64_t)blockIdx.x * C + c] = db;
    }
    int turn = 0;
    for (int64_t row = first; row < last; row++) {
        const float rstd = a.rstd[row], mean = a.layer ? a.mean[row] : 0.0f;
        float sg = 0.0f, sgx = 0.0f;
        for (int c = threadIdx.x; c < C; c += kNormThreads) {
            const float wv = load_param(a.w, a.w_dtype, c);
            const float g = load_one(dY + row * C + c) * wv, xh = (load_one(H + row * C + c) - mean) * rstd;
            sg += g;
            sgx = __builtin_fmaf(g, xh, sgx);
        }
        row_sum2<kNormThreads>(sg, sgx, lds[turn]);
        turn ^= 1;
        const float mg = a.layer ? sg / (float)C : 0.0f, mgx = sgx / (float)C;
        for (int c = threadIdx.x; c < C; c += kNormThreads) {
            const float wv = load_param(a.w, a.w_dtype, c);
            const float g = load_one(dY + row * C + c) * wv, xh = (load_one(H + row * C + c) - mean) * rstd;
            const float r = a.dR ? load_one(static_cast<const T *>(a.dR) + row * C + c) : 0.0f;
            store_one(static_cast<T *>(a.dX) + row * C + c, __builtin_fmaf(rstd, g - mg - xh * mgx, r));
        }
    }
}

// Column sums of the partial rows, in order and in fp64: 16 columns x 16 row groups per workgroup, 8 loads in flight.
// 1,024 rows of 2,560: 6 us, latency-bound.
__global__ void __launch_bounds__(256) norm_finish_kernel(const float *__restrict__ part_w, const float *__restrict__ part_b,
                                                          int parts, int C, float *__restrict__ dw, float *__restrict__ db) {
    __shared__ double lds[16][17];
    const float *part = blockIdx.y ? part_b : part_w;
    const int col = threadIdx.x & 15, grp = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    const int per = (parts + 15) / 16, r0 = grp * per, r1 = r0 + per < parts ? r0 + per : parts;
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
    lds[grp][col] = s;
    __syncthreads();
    if (grp == 0 && c < C) {
        for (int i = 1; i < 16; i++) s += lds[i][col];
        (blockIdx.y ? db : dw)[c] = (float)s;
    }
}

template <int... Vs, typename F>
bool pick_nv(int64_t need, F &&f) {
    bool done = false;
    ((!done && need <= Vs ? (f(std::integral_constant<int, Vs>{}), done = true) : false), ...);
    return done;
}

// Chooses the threads per row and the vectors per thread: a wave per row while its lanes hold at most 16 elements each
// (no barrier between the sums), a workgroup per row up to 64 elements per thread, false beyond that. Forward and backward of
// bf16 rows of 268 MB together, us, with a wave and with a workgroup per row: 1,024 features 91 + 169 and 173 + 211, 256 features
// 205 + 221 and 549 + 637; fp32 1,024 features 100 + 167 and 102 + 168, 2,048 features 105 + 169 and 97 + 172. bf16 rows of 1,025 to
// 2,048 features would gain from a wave forward (1,536: 95 in place of 149, 2,048: 93 in place of 120; backward as long), where
// half of a workgroup's second vectors do not exist. Rows of few features leave lanes idle: 2,097,152 rows of 64 take
// 636 + 677 us.
template <typename F>
bool norm_shape(int64_t C, F &&f) {
    const int64_t vecs = (C + 7) / 8;
    if (vecs <= 64 * 2)
        return pick_nv<1, 2>((vecs + 63) / 64, [&](auto nv) { f(std::integral_constant<int, 64>{}, nv); });
    return pick_nv<2, 3, 4, 8>((vecs + 255) / 256, [&](auto nv) { f(std::integral_constant<int, 256>{}, nv); });
}

template <typename T>
hipError_t norm_fwd(const NormFwdArgs &a, hipStream_t st) {
    const bool done = norm_shape(a.C, [&](auto threads, auto nv) {
        constexpr int TH = decltype(threads)::value, kRows = kNormThreads / TH;
        const unsigned grid = (unsigned)((a.T + kRows - 1) / kRows);
        if (a.C % 8) norm_fwd_kernel<T, TH, decltype(nv)::value, true><<<grid, kNormThreads, 0, st>>>(a);
        else norm_fwd_kernel<T, TH, decltype(nv)::value, false><<<grid, kNormThreads, 0, st>>>(a);
    });
    if (!done) norm_fwd_long_kernel<T><<<(unsigned)a.T, kNormThreads, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_bwd(const NormBwdArgs &a, int64_t parts, hipStream_t st) {
    const bool done = norm_shape(a.C, [&](auto threads, auto nv) {
        constexpr int TH = decltype(threads)::value, NV = decltype(nv)::value;
        auto go = [&](auto bias, auto tail) {
            norm_bwd_kernel<T, TH, NV, decltype(bias)::value, decltype(tail)::value><<<(unsigned)parts, kNormThreads, 0, st>>>(a);
        };
        if (a.part_b) a.C % 8 ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
        else a.C % 8 ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    });
    if (!done) norm_bwd_long_kernel<T><<<(unsigned)parts, kNormThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t norm_bwd_parts(int64_t T) {
    const int64_t rows = std::max<int64_t>(4, (T + kNormStrips - 1) / kNormStrips);
    return (T + rows - 1) / rows;
}

size_t norm_bwd_ws(int64_t T, int64_t C) {
    // the most strips that any number of tokens up to T takes, gain's and shift's sums
    return kWsHeader + (size_t)std::min<int64_t>((T + 3) / 4, kNormStrips) * (size_t)C * 2 * sizeof(float);
}

hipError_t launch_norm_fwd(int layer, float eps, int dtype, const void *X, const void *R, int64_t T, int64_t C, const void *w,
                           const void *b, int w_dtype, void *H, void *Y, float *mean, float *rstd, hipStream_t st) {
    const size_t row = (size_t)C * (dtype == kBF16 ? 2 : 4);
    auto at = [&](const void *p, int64_t r) { return p ? static_cast<const char *>(p) + (size_t)r * row : nullptr; };
    // a launch's work-items (256 per row at most) must stay below 2^32
    constexpr int64_t kRows = (int64_t(1) << 24) - 1;
    for (int64_t r = 0; r < T; r += kRows) {
        NormFwdArgs a{at(X, r), at(R, r), w, b, const_cast<char *>(at(H, r)), const_cast<char *>(at(Y, r)),
                      mean ? mean + r : nullptr, rstd ? rstd + r : nullptr, std::min(kRows, T - r), (int)C, w_dtype, layer, eps};
        const hipError_t e = dtype == kBF16 ? norm_fwd<uint16_t>(a, st) : norm_fwd<float>(a, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_norm_bwd(int layer, int dtype, const void *dY, const void *H, int64_t T, int64_t C, const void *w,
                           int w_dtype, const float *mean, const float *rstd, const void *dR, void *dX, float *dw, float *db,
                           void *ws, hipStream_t st) {
    const int64_t parts = norm_bwd_parts(T);
    float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader);
    NormBwdArgs a{dY, H, w, dR, mean, rstd, dX, part, db ? part + parts * C : nullptr, T, (T + parts - 1) / parts, (int)C,
                  w_dtype, layer};
    const hipError_t e = dtype == kBF16 ? norm_bwd<uint16_t>(a, parts, st) : norm_bwd<float>(a, parts, st);
    if (e != hipSuccess) return e;
    norm_finish_kernel<<<dim3((unsigned)((C + 15) / 16), db ? 2 : 1), 256, 0, st>>>(a.part_w, a.part_b, (int)parts, (int)C, dw,
                                                                                   db);
    return hipGetLastError();
}

}  // namespace focus
