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

// Sums of two values over a workgroup, in every thread; `lds` of 8 floats is free again after the next barrier of the caller's
// (buffers in turn).
__device__ __forceinline__ void group_sum2(float &a, float &b, float *lds) {
    a = wave_sum(a);
    b = wave_sum(b);
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

__device__ __forceinline__ float group_sum(float a, float *lds) {
    float b = 0.0f;
    group_sum2(a, b, lds);
    return a;
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

// Sums of the partial rows in order and in fp64: 16 columns x 16 row groups per workgroup, 8 loads in flight; blockIdx.y is the
// sum. A feature's gate is applied here: with S = sum_t dYt xh1 and R = sum_t dYt, dw1 = gate S, db1 = gate R, dgate = w1 S + b1 R.
__global__ void __launch_bounds__(256) sandwich_finish_kernel(SandwichArgs a, int parts) {
    __shared__ double lds[4][16][17];
    const int col = threadIdx.x & 15, grp = threadIdx.x >> 4, c = blockIdx.x * 16 + col, C = a.C;
    const int per = (parts + 15) / 16, r0 = grp * per, r1 = r0 + per < parts ? r0 + per : parts;
    for (int k = 0; k < a.sums; k++) {
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
    }
    __syncthreads();
    if (grp != 0 || c >= C) return;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    for (int k = 0; k < a.sums; k++)
        for (int i = 0; i < 16; i++) v[k] += lds[k][i][col];
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

}  // namespace

size_t sandwich_bwd_ws(int64_t T, int64_t C) {
    // the most strips that any number of tokens up to T takes, four sums
    return kWsHeader + (size_t)std::min<int64_t>((T + 3) / 4, kStrips) * (size_t)C * 4 * sizeof(float);
}

hipError_t launch_sandwich_fwd(int dtype, SandwichArgs a, hipStream_t st) {
    constexpr int64_t kRows = (int64_t(1) << 24) - 1;  // a launch's work-items stay below 2^32
    for (a.first = 0; a.first < a.T; a.first += kRows) {
        const unsigned grid = (unsigned)std::min(kRows, a.T - a.first);
        if (dtype == kBF16) sandwich_fwd_long_kernel<uint16_t><<<grid, kThreads, 0, st>>>(a);
        else sandwich_fwd_long_kernel<float><<<grid, kThreads, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_sandwich_bwd(int dtype, SandwichArgs a, void *ws, hipStream_t st) {
    const int64_t parts = bwd_parts(a.T);
    a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader);
    a.rows = (a.T + parts - 1) / parts;
    a.sums = a.b1 || a.db1 || a.db2 ? 4 : 2;
    if (dtype == kBF16) sandwich_bwd_long_kernel<uint16_t><<<(unsigned)parts, kThreads, 0, st>>>(a);
    else sandwich_bwd_long_kernel<float><<<(unsigned)parts, kThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    sandwich_finish_kernel<<<(unsigned)((a.C + 15) / 16), 256, 0, st>>>(a, (int)parts);
    return hipGetLastError();
}

}  // namespace focus
