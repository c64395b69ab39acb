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
//
// bf16 operands with K a multiple of 16 go to the matrix instructions (linear_ce_mfma.hip), D in bf16 relative to a token's scale
// r = max(|g|, |h|):
//   D = r D',  dX[t] = r[t] (D' W)[t],  dW = G D'^T X',  X'[t] = X[t] r[t] / G  (rounded),  G = max r
// so that the tokens' weights are rounded into X' where they differ, and nowhere where they are those of a mean (X' is X then).
// fp32 with K a multiple of 16 goes to the fp32 matrix instructions (gemm_f32.hip); other shapes take the kernels below.
#include "linear_ce.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kTileV = 64, kTileT = 64;  // logits of a tile
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;  // a launch's work-items (256 per workgroup) stay below 2^32

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

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

// Joins the parts of a token: m = max m_i, s = sum s_i exp(m_i - m), in a fixed order. A workgroup takes `tokens` (a power of two)
// neighbours, so that its loads run along part's rows; the 256 / tokens threads of one take every so many-th part, eight at a time
// under way, each with a running maximum. Bound by latency: 8,192 tokens of 594 parts (39 MB) 20 us, with a wave per token, whose loads
// lie a row apart, 62; one token of 1,187 parts 5 us.
__global__ void __launch_bounds__(256) ce_join_kernel(CeArgs a, int tiles, int tokens, uint32_t *flag) {
    __shared__ float2 lds[256];
    const float kNone = -__builtin_inff();
    const int per = 256 / tokens, lane = threadIdx.x / tokens;
    const int64_t t = (int64_t)blockIdx.x * tokens + threadIdx.x % tokens;
    auto join = [&](float &m, float &s, float2 p) {  // an empty part is (-inf, 0)
        const float top = fmaxf(m, p.x);
        s = (m == top ? s : s * expf(m - top)) + (p.x == top ? p.y : p.y * expf(p.x - top));
        m = top;
    };
    float m = kNone, s = 0.0f;
    if (t < a.T) {
        for (int i = lane; i < tiles; i += 8 * per) {
            float2 p[8];
#pragma unroll
            for (int u = 0; u < 8; u++) p[u] = i + u * per < tiles ? a.part[(int64_t)(i + u * per) * a.T + t] : make_float2(kNone, 0.0f);
#pragma unroll
            for (int u = 0; u < 8; u++) join(m, s, p[u]);
        }
    }
    lds[threadIdx.x] = make_float2(m, s);
    __syncthreads();
    for (int w = per / 2; w >= 1; w >>= 1) {
        if (lane < w) {
            join(m, s, lds[threadIdx.x + w * tokens]);
            lds[threadIdx.x] = make_float2(m, s);
        }
        __syncthreads();
    }
    if (t >= a.T || lane != 0) return;
    const float ls = logf(s);
    a.lse[t] = m + ls;
    const int64_t want = a.target ? a.target[t] : 0;  // a token left out raises nothing
    bool bad = want >= 0 && (!(s < __builtin_inff()) || !(__builtin_fabsf(m) < kCeMostLogit));
    if (a.logp) {
        const bool there = want >= 0 && want < a.V;
        bad = bad || want >= a.V;
        a.logp[t] = there ? (a.zt[t] - m) - ls : 0.0f;
    }
    if (bad) raise_domain_flag(flag);
}

// D of the piece's tile, in fp32. This and the product below are for rows of K that no matrix-instruction kernel takes, and not tuned:
// 301 x 5,003 x 1,001 195 us forward and 1.29 ms backward, with K = 1,008 47 and 139 in fp32, 17 and 60 in bf16.
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
        const bool none = g == 0.0f && h == 0.0f;
        bad = bad || want >= a.V || ((g != 0.0f || h != 0.0f) && !(__builtin_fabsf(lse) <= 65536.0f));
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int64_t v = v0 + tx * 4 + j;
            if (v - a.v0 >= a.pitch) continue;
            const float p = expf(acc[i][j] - lse);
            static_cast<float *>(a.D)[t * a.pitch + (v - a.v0)] = v < a.V && !none ? (v == want ? g : 0.0f) + (h - g) * p : 0.0f;
        }
    }
    if (bad) raise_domain_flag(flag);
}

// C[m][n] = before[m][n] + sum_r A(m, r) B[r][n] in fp32, 64 x 64 per workgroup, A(m, r) at A[m am + r ar]; written to
// `sums` in fp32, or to `out` in its type. rows: row r of B is token r's, zeros where that has no gradient.
struct CeProduct {
    const float *A, *before, *g, *h;
    const int64_t *target;
    const void *B;
    float *sums;
    void *out;
    int64_t am, ar, M, N, R, m0, V;
    int b_dtype, out_dtype, tiles_n, rows;
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
            const bool real = n0 + n < a.N && r0 + rb < a.R && (!a.rows || ce_takes_part(a.target, a.g, a.h, a.V, r0 + rb));
            Bs[rb][n] = real ? load1(a.B, a.b_dtype, (r0 + rb) * a.N + n0 + n) : 0.0f;
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

// ---- around the matrix-instruction kernels ------------------------------------------------------
// r[t] = max(|g|, |h|) of the tokens (g: 0 where left out) and G, their maximum, by one workgroup: 4,096 tokens 6 us, 8,192 9. (As
// part of the next kernel, every workgroup of which forms G then, no faster: 1,500 x 3,001 x 512 backward 69 us, so 72.)
__global__ void __launch_bounds__(1024) ce_scales_kernel(const int64_t *__restrict__ target, const float *__restrict__ g,
                                                         const float *__restrict__ h, int64_t T, int64_t V, float *__restrict__ r,
                                                         float *__restrict__ most) {
    __shared__ float lds[16];
    float m = 0.0f;
    for (int64_t t = threadIdx.x; t < T; t += 1024) {
        const bool kept = g && target[t] >= 0 && target[t] < V;
        const float a = kept ? __builtin_fabsf(g[t]) : 0.0f, b = h ? __builtin_fabsf(h[t]) : 0.0f;
        const float v = a > b || a != a ? a : b;  // a NaN stays one
        r[t] = v;
        m = v > m || v != v ? v : m;
    }
    for (int d = 32; d >= 1; d >>= 1) {
        const float o = __shfl_xor(m, d, 64);
        m = o > m || o != o ? o : m;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 0; i < 16; i++) m = lds[i] > m || lds[i] != lds[i] ? lds[i] : m;
    *most = m;
}

// X' = X r / G, rounded to bf16; 8 elements per thread (K is a multiple of 16). A token whose gradient is 0 has a row of zeros. Bound
// by memory: 8,192 x 2,560 15 us, 5.6 TB/s.
__global__ void __launch_bounds__(256) ce_scale_x_kernel(const uint16_t *__restrict__ X, const float *__restrict__ r,
                                                         const float *__restrict__ most, int64_t first, int64_t n, int64_t K,
                                                         uint16_t *__restrict__ out) {
    const int64_t i = first + ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    const float s = r[i / K], f = s == 0.0f ? 0.0f : s / *most;
    float v[8];
    load8_n(X + i, 8, v);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = f == 0.0f ? 0.0f : v[e] * f;
    store8_n(out + i, 8, v);
}

// total = before + the splits' sums in order; to `sums` in fp32, or times the row's (or everything's, or no) factor to `out`. Bound by
// memory: three splits of 8,192 x 2,560, the sum so far and the new one 63 us, 6.6 TB/s (the splits partly from the caches); many splits
// of little by their latency, hence eight under way (63 of 64 x 512: 9 us, one at a time 16)
__global__ void __launch_bounds__(256) ce_sums_kernel(const float *__restrict__ part, int64_t splits, const float *__restrict__ before,
                                                      const float *__restrict__ factor, int per_row, int64_t first, int64_t n, int64_t K,
                                                      float *__restrict__ sums, void *__restrict__ out, int out_dtype) {
    const int64_t i = first + ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    float s[8], v[8];
    load8_n(part + i, 8, s);
    int64_t z = 1;
    for (; z + 8 <= splits; z += 8) {  // eight under way
        float u[8][8];
#pragma unroll
        for (int k = 0; k < 8; k++) load8_n(part + (z + k) * n + i, 8, u[k]);
#pragma unroll
        for (int k = 0; k < 8; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) s[e] += u[k][e];
    }
    for (; z < splits; z++) {
        load8_n(part + z * n + i, 8, v);
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] += v[e];
    }
    if (before) {
        load8_n(before + i, 8, v);
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] += v[e];
    }
    if (sums) {
        store8_n(sums + i, 8, s);
        return;
    }
    if (factor) {
        const float f = per_row ? factor[i / K] : *factor;
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] *= f;
    }
    if (out_dtype == kBF16) store8_n(static_cast<uint16_t *>(out) + i, 8, s);
    else store8_n(static_cast<float *>(out) + i, 8, s);
}

// f(first element, workgroups) in launches whose work-items stay below 2^32, 2,048 elements per workgroup
template <typename F>
hipError_t in_elements(int64_t n, F &&f) {
    for (int64_t i = 0; i < n; i += kMaxGrid * 2048) {
        f(i, (unsigned)cdiv(std::min(n - i, kMaxGrid * 2048), 2048));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

bool on_mfma(int dtype, int64_t K) { return dtype == kBF16 && K % 16 == 0; }

// Pieces of the vocabulary, of D takes 512 MiB each at most (in fp32, whose products are slower against what a piece costs, 128 MiB; a
// tile's 256 entries each at least); the last one is what is left. 8,192 tokens, vocabulary 151,936, both
// ways: 22.0 ms, with 1 GiB 22.1.
constexpr int64_t piece_most(int64_t esz) { return int64_t(1) << (esz == 2 ? 29 : 27); }
int64_t piece_width(int64_t T, int64_t V, int64_t esz) {
    const int64_t fit = std::max<int64_t>(1, std::min(piece_most(esz) / (T * esz), kCeMostWidth) / 256);
    return std::min(fit, cdiv(V, 256)) * 256;
}
// bytes of D for T tokens or fewer
size_t piece_bytes(int64_t T, int64_t V, int64_t esz) {
    return std::max<size_t>((size_t)(T * 256 * esz), (size_t)std::min(T * cdiv(V, 256) * 256 * esz, piece_most(esz)));
}

constexpr int64_t kMostSplits = 64;

// Splits of a product [M][N] over its reduction R, as the input gradient of a linear has them: whole rounds of 256 x 256 tiles, one
// per CU, in units of a step of 32 (0.9 us), 8 of them for a tile's end; the fp32 sums written and read (about 4 MB in a unit)
struct Splits {
    int64_t count, chunk;
};
Splits mfma_splits(int64_t R, int64_t M, int64_t N) {
    const int64_t tiles = cdiv(M, kCeTile) * cdiv(N, kCeTile), steps = cdiv(R, 32);
    const int64_t most = tiles >= 4 * 256 ? 1 : std::min<int64_t>(std::min<int64_t>(kMostSplits, steps / 8), kDxSums / (M * N));
    int64_t best = -1, count = 1;
    for (int64_t s = 1; s <= std::max<int64_t>(1, most); s++) {
        const int64_t cost = cdiv(tiles * s, 256) * (cdiv(steps, s) + 8) + (s > 1 ? s * M * N * 8 / 4000000 + 4 : 0);
        if (best < 0 || cost < best) best = cost, count = s;
    }
    const int64_t chunk = cdiv(steps, count) * 32;
    return {cdiv(R, chunk), chunk};
}

// fp32 sums of the splits: one of dX, or as many of dX or dW as kDxSums holds
size_t sums_bytes(int64_t T, int64_t V, int64_t K) {
    const int64_t rows = std::max(T, std::min(cdiv(V, 256) * 256, kCeMostWidth));
    const int64_t many = rows > kDxSums / K / kMostSplits ? kDxSums : kMostSplits * rows * K;
    return round256((size_t)std::max(T * K, many) * sizeof(float));
}

struct MfmaSpace {
    float *r, *most, *sums, *part;
    uint16_t *x, *D;
};
size_t mfma_space(int64_t T, int64_t V, int64_t K, char *base, MfmaSpace *s) {
    size_t at = kWsHeader;
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += round256(bytes);
        return p;
    };
    char *const most = take(sizeof(float)), *const r = take((size_t)T * sizeof(float)), *const x = take((size_t)T * (size_t)K * 2);
    char *const sums = take((size_t)T * (size_t)K * sizeof(float)), *const part = take(sums_bytes(T, V, K));
    char *const D = take(piece_bytes(T, V, 2));
    if (s)
        *s = MfmaSpace{reinterpret_cast<float *>(r), reinterpret_cast<float *>(most), reinterpret_cast<float *>(sums),
                       reinterpret_cast<float *>(part), reinterpret_cast<uint16_t *>(x), reinterpret_cast<uint16_t *>(D)};
    return at;
}

// ---- fp32 ---------------------------------------------------------------------------------------
// Splits of a product's reduction over R into tiles of 64 x 64, in ns: the tiles that a CU has take a step of 32 rows in turn, 0.69 us
// where it has one, 0.56 of two and 0.51 of three, which is how many run at once, 1.5 us for their start and end; the sums' launch, and
// what it and the tiles move. dX of 1,024 x 10,000 x 1,024 (256 tiles) 217 us unsplit, 175 in two and 162 in three, of 301 x 5,003 x 1,008
// (80 tiles) 48 in three and 41 in six, of 100 x 8,000 x 2,048 (64) 48 in four and 40 in eight.
Splits f32_splits(int64_t R, int64_t N, int64_t K) {
    const int64_t tiles = cdiv(N, 64) * cdiv(K, 64), steps = cdiv(R, 32), cus = 256;
    const int64_t most = tiles >= 16 * cus ? 1 : std::min<int64_t>(std::min<int64_t>(kMostSplits, steps), kDxSums / (N * K));
    int64_t best = -1, count = 1;
    for (int64_t s = 1; s <= std::max<int64_t>(1, most); s++) {
        const int64_t on_cu = cdiv(tiles * s, cus), step = on_cu == 1 ? 690 : on_cu == 2 ? 560 : 510;
        const int64_t cost = on_cu * cdiv(steps, s) * step + cdiv(on_cu, 3) * 1500 + (s > 1 ? 5000 + s * N * K / 560 : 0);
        if (best < 0 || cost < best) best = cost, count = s;
    }
    const int64_t chunk = cdiv(steps, count) * 32;
    return {cdiv(R, chunk), chunk};
}

struct F32Space {
    float *sums, *part, *x, *D, *Dt;
};
size_t f32_space(int64_t T, int64_t V, int64_t K, char *base, F32Space *s) {
    const size_t x = round256((size_t)T * (size_t)K * sizeof(float)), part = sums_bytes(T, V, K);
    const size_t D = round256(piece_bytes((T + 3) / 4 * 4, V, sizeof(float)));  // transposed too, its rows of whole fours
    size_t at = kWsHeader;
    auto take = [&](size_t bytes) {
        float *p = reinterpret_cast<float *>(base + at);
        at += bytes;
        return p;
    };
    float *const sums = take(x), *const parts = take(part), *const rows = take(x), *const d = take(D), *const dt = take(D);
    if (s) *s = F32Space{sums, parts, rows, d, dt};
    return at;
}

hipError_t bwd_f32(CeArgs a, float *dX, float *dW, uint32_t *flag, char *ws, hipStream_t st) {
    F32Space s;
    f32_space(a.T, a.V, a.K, ws, &s);
    const int64_t T = a.T, V = a.V, K = a.K, width = piece_width((T + 3) / 4 * 4, V, sizeof(float)), pitch_t = (T + 3) / 4 * 4;
    a.D = s.D;
    auto finish = [&](int64_t splits, const float *before, int64_t n, float *sums, float *out) {
        return in_elements(n, [&](int64_t first, unsigned grid) {
            ce_sums_kernel<<<grid, 256, 0, st>>>(s.part, splits, before, nullptr, 0, first, n, K, sums, out, kF32);
        });
    };
    for (int64_t v0 = 0; v0 < V; v0 += width) {
        const int64_t n = std::min(width, V - v0), edge = ce_f32_tile(T, n);
        a.v0 = v0, a.pitch = (n + 3) / 4 * 4, a.tiles_v = (int)cdiv(n, edge);
        hipError_t e = in_runs(cdiv(T, edge), a.tiles_v, [&](int64_t first, int64_t count) {
            a.t0 = first * edge;
            launch_ce_grad_f32(a, edge, count * edge, s.Dt, pitch_t, dW && v0 == 0 ? s.x : nullptr, flag, st);
        });
        if (e != hipSuccess) return e;
        if (dX) {
            const Splits p = f32_splits(n, T, K);
            const bool alone = p.count == 1 && n == V;
            e = launch_dw_f32(s.Dt, static_cast<const float *>(a.W) + v0 * K, n, T, pitch_t, K, p.chunk, p.count, alone ? dX : s.part, st);
            if (e == hipSuccess && !alone) e = finish(p.count, v0 ? s.sums : nullptr, T * K, v0 + n == V ? nullptr : s.sums, dX);
            if (e != hipSuccess) return e;
        }
        if (dW) {
            const Splits p = f32_splits(T, n, K);
            float *const out = dW + v0 * K;
            e = launch_dw_f32(s.D, s.x, T, n, a.pitch, K, p.chunk, p.count, p.count == 1 ? out : s.part, st);
            if (e == hipSuccess && p.count > 1) e = finish(p.count, nullptr, n * K, nullptr, out);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

hipError_t bwd_mfma(CeArgs a, void *dX, void *dW, int dw_dtype, uint32_t *flag, char *ws, hipStream_t st) {
    MfmaSpace s;
    mfma_space(a.T, a.V, a.K, ws, &s);
    const int64_t T = a.T, V = a.V, K = a.K;
    ce_scales_kernel<<<1, 1024, 0, st>>>(a.target, a.g, a.h, T, V, s.r, s.most);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.scale = s.r, a.D = s.D;
    if (dW) {
        e = in_elements(T * K, [&](int64_t first, unsigned grid) {
            ce_scale_x_kernel<<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(a.X), s.r, s.most, first, T * K, K, s.x);
        });
        if (e != hipSuccess) return e;
    }
    const int64_t width = piece_width(T, V, 2);
    a.pitch = width;
    for (int64_t v0 = 0; v0 < V; v0 += width) {
        const int64_t n = std::min(width, V - v0), edge = ce_mfma_tile(T, n);
        a.v0 = v0;
        a.tiles_v = (int)(cdiv(n, kCeTile) * kCeTile / edge);  // whole tiles of the products that read D
        e = in_runs(cdiv(T, edge), a.tiles_v, [&](int64_t first, int64_t count) {
            a.t0 = first * edge;
            launch_ce_grad_mfma(a, edge, count * edge, flag, st);
        });
        if (e != hipSuccess) return e;
        const char *const W = static_cast<const char *>(a.W) + (size_t)v0 * (size_t)K * 2;
        if (dX) {
            const Splits p = mfma_splits(n, T, K);
            e = launch_dx_sums(s.D, W, T, n, width, K, p.chunk, p.count, s.part, st);
            if (e != hipSuccess) return e;
            const bool last = v0 + n == V;
            e = in_elements(T * K, [&](int64_t first, unsigned grid) {
                ce_sums_kernel<<<grid, 256, 0, st>>>(s.part, p.count, v0 ? s.sums : nullptr, s.r, 1, first, T * K, K,
                                                     last ? nullptr : s.sums, dX, kBF16);
            });
            if (e != hipSuccess) return e;
        }
        if (dW) {
            char *const out = static_cast<char *>(dW) + (size_t)v0 * (size_t)K * (dw_dtype == kBF16 ? 2 : 4);
            const Splits p = mfma_splits(T, n, K);
            e = launch_dw_mfma(s.D, s.x, T, n, width, K, p.chunk, p.count, s.most, out, dw_dtype, s.part, st);
            if (e != hipSuccess) return e;
            if (p.count > 1)
                e = in_elements(n * K, [&](int64_t first, unsigned grid) {
                    ce_sums_kernel<<<grid, 256, 0, st>>>(s.part, p.count, nullptr, s.most, 0, first, n * K, K, nullptr, out, dw_dtype);
                });
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace

size_t linear_ce_fwd_ws(int64_t T, int64_t V) {
    // parts of 64 vocabulary entries, or of 32 in fp32 where there are fewer than 256 tiles of 64 x 64
    const int64_t parts = std::max(cdiv(V, kTileV) * T, std::min(cdiv(V, 32) * T, int64_t(2) * 256 * 64));
    return kWsHeader + round256((size_t)T * sizeof(float)) + (size_t)parts * sizeof(float2);
}

size_t linear_ce_bwd_ws(int64_t T, int64_t V, int64_t K) {
    if (T == 0) return kWsHeader;
    const size_t simple = kWsHeader + round256((size_t)T * (size_t)K * sizeof(float)) + piece_bytes(T, V, sizeof(float));
    return std::max(simple, std::max(mfma_space(T, V, K, nullptr, nullptr), f32_space(T, V, K, nullptr, nullptr)));
}

hipError_t launch_linear_ce_fwd(int dtype, const void *X, const void *W, int64_t T, int64_t V, int64_t K, const int64_t *target,
                                float *logp, float *lse, uint32_t *flag, void *ws, hipStream_t st) {
    char *const base = static_cast<char *>(ws) + kWsHeader;
    CeArgs a{};
    a.X = X, a.W = W, a.target = target, a.lse = lse, a.logp = logp, a.T = T, a.V = V, a.K = K;
    a.zt = reinterpret_cast<float *>(base);
    a.part = reinterpret_cast<float2 *>(base + round256((size_t)T * sizeof(float)));
    const bool mfma = on_mfma(dtype, K), few = mfma && T <= kCeFew, f32 = dtype == kF32 && ce_f32_supported(T, V, K);
    const int64_t rows = mfma ? ce_mfma_tile(T, V) : f32 ? ce_f32_tile(T, V) : kTileT;
    a.tiles_v = (int)cdiv(V, few ? kCeFewV : rows);
    hipError_t e = hipSuccess;
    if (few) {
        launch_ce_stats_few(a, st);
        e = hipGetLastError();
    } else {
        e = in_runs(cdiv(T, rows), a.tiles_v, [&](int64_t first, int64_t count) {
            a.t0 = first * rows;
            if (mfma) launch_ce_stats_mfma(a, rows, count * rows, st);
            else if (f32) launch_ce_stats_f32(a, rows, count * rows, st);
            else if (dtype == kBF16) ce_stats_kernel<kBF16><<<(unsigned)(count * a.tiles_v), 256, 0, st>>>(a);
            else ce_stats_kernel<kF32><<<(unsigned)(count * a.tiles_v), 256, 0, st>>>(a);
        });
    }
    if (e != hipSuccess) return e;
    const int tokens = T >= 1024 ? 32 : T >= 32 ? 8 : 1;
    ce_join_kernel<<<(unsigned)cdiv(T, tokens), 256, 0, st>>>(a, a.tiles_v, tokens, flag);
    return hipGetLastError();
}

hipError_t launch_linear_ce_bwd(int dtype, const void *X, const void *W, int64_t T, int64_t V, int64_t K, const int64_t *target,
                                const float *lse, const float *g, const float *h, void *dX, void *dW, int dw_dtype,
                                uint32_t *flag, void *ws, hipStream_t st) {
    char *const base = static_cast<char *>(ws) + kWsHeader;
    float *const sums = reinterpret_cast<float *>(base);
    CeArgs a{};
    a.X = X, a.W = W, a.target = target, a.lse = const_cast<float *>(lse), a.g = g, a.h = h, a.T = T, a.V = V, a.K = K;
    if (dtype == kF32 && ce_f32_supported(T, V, K))
        return bwd_f32(a, static_cast<float *>(dX), static_cast<float *>(dW), flag, static_cast<char *>(ws), st);
    if (on_mfma(dtype, K)) return bwd_mfma(a, dX, dW, dw_dtype, flag, static_cast<char *>(ws), st);
    a.D = base + round256((size_t)T * (size_t)K * sizeof(float));
    const int64_t width = piece_width(T, V, sizeof(float));
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
            p.A = static_cast<const float *>(a.D), p.am = n, p.ar = 1, p.M = T, p.N = K, p.R = n, p.b_dtype = dtype, p.out_dtype = dtype;
            p.B = static_cast<const char *>(W) + (size_t)v0 * (size_t)K * esz;
            p.before = v0 ? sums : nullptr;
            p.sums = last ? nullptr : sums;
            p.out = dX;
            e = product(p, st);
            if (e != hipSuccess) return e;
        }
        if (dW) {
            CeProduct p{};
            p.A = static_cast<const float *>(a.D), p.am = 1, p.ar = n, p.M = n, p.N = K, p.R = T, p.b_dtype = dtype, p.out_dtype = dw_dtype;
            p.B = X, p.rows = 1, p.target = target, p.g = g, p.h = h, p.V = V;
            p.out = static_cast<char *>(dW) + (size_t)v0 * (size_t)K * dsz;
            e = product(p, st);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace focus
