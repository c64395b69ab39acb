// Softmax cross entropy of an output layer over its vocabulary, without the logits: log probabilities of given tokens from
// hidden states X [T][K] and weights W [V][K], and the gradients of both.
//
//   z[t][v] = sum_k X[t][k] W[v][k],  lse[t] = log sum_v exp z[t][v],  logp[t] = z[t][target] - lse[t]
//   D[t][v] = g ([v == target] - p) + h p,  p = exp(z - lse),  g = d_logp[t] (0 where left out),  h = d_lse[t]
//   dX = D W,  dW = D^T X
//
// Forward: a tile of logits is reduced at once to each token's maximum and sum of exponentials over the tile's part of the
// vocabulary; a second kernel joins the parts. Backward: the vocabulary goes in pieces; of each the logits are formed again
// and D, which both products read, is what lies in memory.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kTileV = 64, kTileT = 64;  // logits of a tile
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;  // a launch's work-items (256 per workgroup) stay below 2^32

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct CeArgs {
    const void *X, *W;
    const int64_t *target;
    float *lse, *logp;       // [T]; logp NULL where no targets are given
    const float *g, *h;      // gradients of logp and lse, NULL: 0
    float2 *part;            // [tiles][T] maximum and sum of a tile's exponentials
    float *zt;               // [T] logit of the target
    float *D;                // [T][pitch] of the piece
    int64_t T, V, K, pitch, v0, t0;  // first token and first vocabulary entry of the launch
    int tiles_v;
};

// 64 tokens x 64 vocabulary entries of the logits in fp32, 4 x 4 per thread: acc[i][j] is that of token t0 + 4 (thread / 16)
// + i and entry v0 + 4 (thread % 16) + j. For rows of K that the matrix-instruction kernels do not take; bound by LDS reads
// (two of 16 bytes per 16 products).
template <int DT>
__device__ __forceinline__ void logits_tile(const CeArgs &a, int64_t t0, int64_t v0, float (&acc)[4][4]) {
    __shared__ float As[16][68];
    __shared__ float Bs[16][68];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = 0.0f;
    for (int64_t k0 = 0; k0 < a.K; k0 += 16) {
        for (int i = threadIdx.x; i < 64 * 16; i += 256) {
            const int r = i / 16, kk = i % 16;
            const int64_t k = k0 + kk;
            As[kk][r] = t0 + r < a.T && k < a.K ? load1(a.X, DT, (t0 + r) * a.K + k) : 0.0f;
            Bs[kk][r] = v0 + r < a.V && k < a.K ? load1(a.W, DT, (v0 + r) * a.K + k) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 16; kk++) {
            float x[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[i] = As[kk][ty * 4 + i];
                w[i] = Bs[kk][tx * 4 + i];
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = __builtin_fmaf(x[i], w[j], acc[i][j]);
        }
        __syncthreads();
    }
}

template <int DT>
__global__ void __launch_bounds__(256) ce_stats_kernel(CeArgs a) {
    const int tile = (int)(blockIdx.x % (unsigned)a.tiles_v);
    const int64_t t0 = a.t0 + (int64_t)(blockIdx.x / (unsigned)a.tiles_v) * kTileT, v0 = (int64_t)tile * kTileV;
    float acc[4][4];
    logits_tile<DT>(a, t0, v0, acc);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const float kNone = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t t = t0 + ty * 4 + i;
        const int64_t want = a.target && t < a.T ? a.target[t] : -1;
        float m = kNone;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int64_t v = v0 + tx * 4 + j;
            if (v >= a.V) acc[i][j] = kNone;
            else if (v == want) a.zt[t] = acc[i][j];
            m = fmaxf(m, acc[i][j]);
        }
        for (int s = 8; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; j++) sum += expf(acc[i][j] - m);  // a NaN stays one
        for (int s = 8; s >= 1; s >>= 1) sum += __shfl_xor(sum, s, 64);
        if (tx == 0 && t < a.T) a.part[(int64_t)tile * a.T + t] = make_float2(m, sum);
    }
}

// Joins the parts of a token: m = max m_i, s = sum s_i exp(m_i - m), in a fixed order. `per` lanes (a power of two up to 64)
// share a token, each taking every per-th part.
__global__ void __launch_bounds__(256) ce_join_kernel(CeArgs a, int tiles, int per, uint32_t *flag) {
    const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / per;
    const int lane = threadIdx.x % per;
    float m = -__builtin_inff(), s = 0.0f;
    if (t < a.T) {
        for (int i = lane; i < tiles; i += per) m = fmaxf(m, a.part[(int64_t)i * a.T + t].x);
        for (int d = per / 2; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        for (int i = lane; i < tiles; i += per) {
            const float2 p = a.part[(int64_t)i * a.T + t];
            s += p.y * expf(p.x - m);
        }
        for (int d = per / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    }
    if (t >= a.T || lane != 0) return;
    const float ls = logf(s);
    a.lse[t] = m + ls;
    bool bad = !(s < __builtin_inff()) || !(__builtin_fabsf(m) < __builtin_inff());
    if (a.logp) {
        const int64_t want = a.target[t];
        const bool there = want >= 0 && want < a.V;
        bad = bad || want >= a.V;
        a.logp[t] = there ? (a.zt[t] - m) - ls : 0.0f;
    }
    if (bad) raise_domain_flag(flag);
}

// D of the piece's tile, in fp32
template <int DT>
__global__ void __launch_bounds__(256) ce_grad_kernel(CeArgs a, uint32_t *flag) {
    const int tile = (int)(blockIdx.x % (unsigned)a.tiles_v);
    const int64_t t0 = a.t0 + (int64_t)(blockIdx.x / (unsigned)a.tiles_v) * kTileT, v0 = a.v0 + (int64_t)tile * kTileV;
    float acc[4][4];
    logits_tile<DT>(a, t0, v0, acc);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t t = t0 + ty * 4 + i;
        if (t >= a.T) continue;
        const int64_t want = a.target ? a.target[t] : -1;
        const bool there = want >= 0 && want < a.V;
        const float g = a.g && there ? a.g[t] : 0.0f, h = a.h ? a.h[t] : 0.0f, lse = a.lse[t];
        bad = bad || want >= a.V || ((g != 0.0f || h != 0.0f) && !(__builtin_fabsf(lse) <= 65536.0f));
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int64_t v = v0 + tx * 4 + j;
            if (v - a.v0 >= a.pitch) continue;
            const float p = expf(acc[i][j] - lse);
            a.D[t * a.pitch + (v - a.v0)] = v < a.V ? (v == want ? g : 0.0f) + (h - g) * p : 0.0f;
        }
    }
    if (bad) raise_domain_flag(flag);
}

// C[m][n] = before[m][n] + sum_r A(m, r) B[r][n] in fp32, 64 x 64 per workgroup, A(m, r) at A[m am + r ar]; written to
// `sums` in fp32, or to `out` in its type.
struct CeProduct {
    const float *A, *before;
    const void *B;
    float *sums;
    void *out;
    int64_t am, ar, M, N, R, m0;
    int b_dtype, out_dtype, tiles_n;
};
__global__ void __launch_bounds__(256) ce_product_kernel(CeProduct a) {
    __shared__ float As[16][68];
    __shared__ float Bs[16][68];
    const int64_t m0 = a.m0 + (int64_t)(blockIdx.x / (unsigned)a.tiles_n) * 64, n0 = (int64_t)(blockIdx.x % (unsigned)a.tiles_n) * 64;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int64_t r0 = 0; r0 < a.R; r0 += 16) {
        for (int i = threadIdx.x; i < 64 * 16; i += 256) {
            const bool along_m = a.am == 1;
            const int m = along_m ? i % 64 : i / 16, ra = along_m ? i / 64 : i % 16, n = i % 64, rb = i / 64;
            As[ra][m] = m0 + m < a.M && r0 + ra < a.R ? a.A[(m0 + m) * a.am + (r0 + ra) * a.ar] : 0.0f;
            Bs[rb][n] = n0 + n < a.N && r0 + rb < a.R ? load1(a.B, a.b_dtype, (r0 + rb) * a.N + n0 + n) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int rr = 0; rr < 16; rr++) {
            float x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[i] = As[rr][ty * 4 + i];
                y[i] = Bs[rr][tx * 4 + i];
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = __builtin_fmaf(x[i], y[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t m = m0 + ty * 4 + i;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int64_t n = n0 + tx * 4 + j;
            if (m >= a.M || n >= a.N) continue;
            const float v = acc[i][j] + (a.before ? a.before[m * a.N + n] : 0.0f);
            if (a.sums) a.sums[m * a.N + n] = v;
            else store1(a.out, a.out_dtype, m * a.N + n, v);
        }
    }
}

// Runs of row tiles whose launches stay within the grid's limit: f(first row tile, row tiles)
template <typename F>
hipError_t in_runs(int64_t tiles_m, int64_t tiles_n, F &&f) {
    const int64_t most = std::max<int64_t>(1, kMaxGrid / tiles_n);
    for (int64_t m = 0; m < tiles_m; m += most) {
        f(m, std::min(most, tiles_m - m));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t product(CeProduct p, hipStream_t st) {
    p.tiles_n = (int)cdiv(p.N, 64);
    return in_runs(cdiv(p.M, 64), p.tiles_n, [&](int64_t first, int64_t count) {
        p.m0 = first * 64;
        ce_product_kernel<<<(unsigned)(count * p.tiles_n), 256, 0, st>>>(p);
    });
}

size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// Vocabulary entries of a piece: D of a piece takes 1 GiB at most, as far as 256 entries allow
constexpr int64_t kPieceBytes = int64_t(1) << 30;
int64_t piece(int64_t T, int64_t V) {
    const int64_t fit = kPieceBytes / (T * (int64_t)sizeof(float)) / 256 * 256;
    return std::min(std::max<int64_t>(fit, 256), cdiv(V, 256) * 256);
}

}  // namespace

size_t linear_ce_fwd_ws(int64_t T, int64_t V) {
    return kWsHeader + round256((size_t)T * sizeof(float)) + (size_t)cdiv(V, kTileV) * (size_t)T * sizeof(float2);
}

size_t linear_ce_bwd_ws(int64_t T, int64_t V, int64_t K) {
    if (T == 0) return kWsHeader;
    // D's piece for T tokens, or for fewer, whose pieces may be up to the limit
    const size_t most = std::max<size_t>((size_t)T * 256 * sizeof(float), std::min<size_t>((size_t)T * (size_t)(cdiv(V, 256) * 256) * sizeof(float), kPieceBytes));
    return kWsHeader + round256((size_t)T * (size_t)K * sizeof(float)) + most;
}

hipError_t launch_linear_ce_fwd(int dtype, const void *X, const void *W, int64_t T, int64_t V, int64_t K, const int64_t *target,
                                float *logp, float *lse, uint32_t *flag, void *ws, hipStream_t st) {
    char *const base = static_cast<char *>(ws) + kWsHeader;
    CeArgs a{};
    a.X = X, a.W = W, a.target = target, a.lse = lse, a.logp = logp, a.T = T, a.V = V, a.K = K;
    a.zt = reinterpret_cast<float *>(base);
    a.part = reinterpret_cast<float2 *>(base + round256((size_t)T * sizeof(float)));
    a.tiles_v = (int)cdiv(V, kTileV);
    hipError_t e = in_runs(cdiv(T, kTileT), a.tiles_v, [&](int64_t first, int64_t count) {
        a.t0 = first * kTileT;
        if (dtype == kBF16) ce_stats_kernel<kBF16><<<(unsigned)(count * a.tiles_v), 256, 0, st>>>(a);
        else ce_stats_kernel<kF32><<<(unsigned)(count * a.tiles_v), 256, 0, st>>>(a);
    });
    if (e != hipSuccess) return e;
    const int per = T >= 4096 ? 8 : 64;
    ce_join_kernel<<<(unsigned)cdiv(T * per, 256), 256, 0, st>>>(a, a.tiles_v, per, flag);
    return hipGetLastError();
}

hipError_t launch_linear_ce_bwd(int dtype, const void *X, const void *W, int64_t T, int64_t V, int64_t K, const int64_t *target,
                                const float *lse, const float *g, const float *h, void *dX, void *dW, int dw_dtype,
                                uint32_t *flag, void *ws, hipStream_t st) {
    char *const base = static_cast<char *>(ws) + kWsHeader;
    float *const sums = reinterpret_cast<float *>(base);
    CeArgs a{};
    a.X = X, a.W = W, a.target = target, a.lse = const_cast<float *>(lse), a.g = g, a.h = h, a.T = T, a.V = V, a.K = K;
    a.D = reinterpret_cast<float *>(base + round256((size_t)T * (size_t)K * sizeof(float)));
    const int64_t width = piece(T, V);
    const size_t esz = dtype == kBF16 ? 2 : 4, dsz = dw_dtype == kBF16 ? 2 : 4;
    for (int64_t v0 = 0; v0 < V; v0 += width) {
        const int64_t n = std::min(width, V - v0);
        a.v0 = v0, a.pitch = n;
        a.tiles_v = (int)cdiv(n, kTileV);
        hipError_t e = in_runs(cdiv(T, kTileT), a.tiles_v, [&](int64_t first, int64_t count) {
            a.t0 = first * kTileT;
            if (dtype == kBF16) ce_grad_kernel<kBF16><<<(unsigned)(count * a.tiles_v), 256, 0, st>>>(a, flag);
            else ce_grad_kernel<kF32><<<(unsigned)(count * a.tiles_v), 256, 0, st>>>(a, flag);
        });
        if (e != hipSuccess) return e;
        const bool last = v0 + n == V;
        if (dX) {
            CeProduct p{};
            p.A = a.D, p.am = n, p.ar = 1, p.M = T, p.N = K, p.R = n, p.b_dtype = dtype, p.out_dtype = dtype;
            p.B = static_cast<const char *>(W) + (size_t)v0 * (size_t)K * esz;
            p.before = v0 ? sums : nullptr;
            p.sums = last ? nullptr : sums;
            p.out = dX;
            e = product(p, st);
            if (e != hipSuccess) return e;
        }
        if (dW) {
            CeProduct p{};
            p.A = a.D, p.am = 1, p.ar = n, p.M = n, p.N = K, p.R = T, p.b_dtype = dtype, p.out_dtype = dw_dtype;
            p.B = X;
            p.out = static_cast<char *>(dW) + (size_t)v0 * (size_t)K * dsz;
            e = product(p, st);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace focus
