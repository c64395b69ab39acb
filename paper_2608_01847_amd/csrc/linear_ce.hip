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
// bf16 operands go to the matrix instructions (linear_ce_mfma.hip), D in bf16 relative to a token's scale r, the power of two at or
// below max(|g|, |h|):
//   D = r D',  dX[t] = r[t] (D' W)[t],  dW = G D'^T X',  X'[t] = X[t] r[t] / G,  G = max r
// Scaling by powers of two rounds nothing. Rounding D' would cost the gradients as many digits as their own rounding does, nearly all of
// them in one entry per token, the target's, which is most of a token's D and shared by all of its row: what that entry's rounding
// leaves, e[t], goes into both gradients by itself,
//   dX[t] += r[t] e[t] W[target[t]],  dW[target[t]] += G e[t] X'[t].
// fp32 goes to the fp32 matrix instructions (gemm_f32.hip). Rows of another K than a multiple of 16 are padded with zeros first.
#include "linear_ce.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;  // a launch's work-items (256 per workgroup) stay below 2^32

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

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

size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// ---- around the matrix-instruction kernels ------------------------------------------------------
// The power of two at or below a number that is not negative (0, infinity and NaN stay)
__device__ __forceinline__ float power_below(float v) {
    const uint32_t b = __float_as_uint(v);
    if (b >= 0x7F800000u || b == 0) return v;
    return __uint_as_float(b >= 0x00800000u ? b & 0x7F800000u : 0x80000000u >> __builtin_clz(b));
}

// r[t] of max(|g|, |h|) of the tokens (g: 0 where left out), their targets' places in the vocabulary (-1: none, or no gradient) and G, the
// largest r, by one workgroup: 4,096 tokens 7 us, 8,192 12. (As part of the next kernel, every workgroup of which forms G then, no faster:
// 1,500 x 3,001 x 512 backward 3 us longer.)
__global__ void __launch_bounds__(1024) ce_scales_kernel(const int64_t *__restrict__ target, const float *__restrict__ g,
                                                         const float *__restrict__ h, int64_t T, int64_t V, float *__restrict__ r,
                                                         int32_t *__restrict__ place, float *__restrict__ most) {
    __shared__ float lds[16];
    float m = 0.0f;
    for (int64_t t = threadIdx.x; t < T; t += 1024) {
        const bool kept = g && target[t] >= 0 && target[t] < V;
        const float a = kept ? __builtin_fabsf(g[t]) : 0.0f, b = h ? __builtin_fabsf(h[t]) : 0.0f;
        const float v = power_below(a > b || a != a ? a : b);  // a NaN stays one
        r[t] = v;
        place[t] = kept && v != 0.0f ? (int32_t)target[t] : -1;
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

// X' = X r / G, exact in bf16; 8 elements per thread (K is a multiple of 16). A token whose gradient is 0 has a row of zeros. Bound
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

// total = before + the splits' sums in order; to `sums` in fp32, or, with rest[t] W[place[t]] where `place` is given, times the row's (or
// everything's, or no) factor to `out`. Bound by memory: three splits of 8,192 x 2,560, the sum so far and the new one 63 us, 6.6 TB/s (the
// splits partly from the caches), of 4,096 x 2,560 with `rest` 27 us, without 23; many splits of little by their latency, hence eight under
// way (63 of 64 x 512: 9 us, one at a time 16)
__global__ void __launch_bounds__(256) ce_sums_kernel(const float *__restrict__ part, int64_t splits, const float *__restrict__ before,
                                                      const float *__restrict__ factor, int per_row, const int32_t *__restrict__ place,
                                                      const float *__restrict__ rest, const uint16_t *__restrict__ W, int64_t first,
                                                      int64_t n, int64_t K, float *__restrict__ sums, void *__restrict__ out,
                                                      int out_dtype) {
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
    const int64_t row = per_row ? i / K : 0;
    if (place && place[row] >= 0) {
        const float e = rest[row];
        load8_n(W + place[row] * K + (i - row * K), 8, v);
#pragma unroll
        for (int u = 0; u < 8; u++) s[u] = __builtin_fmaf(e, v[u], s[u]);
    }
    if (factor) {
        const float f = factor[row];
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

// ---- rows of another K than a multiple of 16 ------------------------------------------------------
int64_t padded(int64_t K) { return (K + 15) / 16 * 16; }

// out [rows][to] = in [rows][from] with zeros behind, or without what is behind; a wave per row, element by element (rows start
// anywhere), eight under way. Bound by memory: 32,000 x 2,561 bf16 64 us, 5.1 TB/s. 4,096 tokens x 32,000 x 2,561 take 745 us forward and
// 2.24 ms backward with it, with 2,560 features 650 and 1.85.
template <typename T>
__global__ void __launch_bounds__(256) ce_pad_kernel(const T *__restrict__ in, int64_t first, int64_t rows, int64_t from, int64_t to,
                                                     T *__restrict__ out) {
    const int64_t row = first + (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (row >= rows) return;
    in += row * from, out += row * to;
    for (int64_t c0 = threadIdx.x % 64; c0 < to; c0 += 64 * 8) {
        T v[8];
#pragma unroll
        for (int u = 0; u < 8; u++) v[u] = c0 + 64 * u < from && c0 + 64 * u < to ? in[c0 + 64 * u] : T(0);
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (c0 + 64 * u < to) out[c0 + 64 * u] = v[u];
    }
}
hipError_t copy_rows(int dtype, const void *in, int64_t rows, int64_t from, int64_t to, void *out, hipStream_t st) {
    for (int64_t i = 0; i < rows; i += kMaxGrid * 4) {
        const unsigned grid = (unsigned)cdiv(std::min(rows - i, kMaxGrid * 4), 4);
        if (dtype == kBF16) ce_pad_kernel<<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(in), i, rows, from, to, static_cast<uint16_t *>(out));
        else ce_pad_kernel<<<grid, 256, 0, st>>>(static_cast<const float *>(in), i, rows, from, to, static_cast<float *>(out));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// bytes of a padded copy, of fp32 elements
size_t pad_bytes(int64_t rows, int64_t K) { return K % 16 ? round256((size_t)rows * (size_t)padded(K) * sizeof(float)) : 0; }

// Pieces of the vocabulary, of which D takes 512 MiB each at most (in fp32, whose products are slower against what a piece costs, 128 MiB; a
// tile's 256 entries each at least); the last one is what is left. With 1 GiB 8,192 tokens, vocabulary 151,936, both ways, take 0.5% longer.
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
// of a reduction over R: eight steps of 32 each at least, in fp32 one
int64_t mfma_most_splits(int64_t R) { return std::min<int64_t>(kMostSplits, cdiv(R, 32) / 8); }
int64_t f32_most_splits(int64_t R) { return std::min<int64_t>(kMostSplits, cdiv(R, 32)); }

struct Splits {
    int64_t count, chunk;
};
// Splits of a product [M][N] over its reduction R, as the input gradient of a linear has them, whose sums have `room`: whole rounds of
// 256 x 256 tiles, one per CU, in units of a step of 32 (0.9 us), 8 of them for a tile's end; the fp32 sums written and read (about 4 MB in
// a unit)
Splits mfma_splits(int64_t R, int64_t M, int64_t N, int64_t room) {
    const int64_t tiles = cdiv(M, kCeTile) * cdiv(N, kCeTile), steps = cdiv(R, 32);
    const int64_t most = tiles >= 4 * 256 ? 1 : std::min(mfma_most_splits(R), std::min(room, kDxSums) / (M * N));
    int64_t best = -1, count = 1;
    for (int64_t s = 1; s <= std::max<int64_t>(1, most); s++) {
        const int64_t cost = cdiv(tiles * s, 256) * (cdiv(steps, s) + 8) + (s > 1 ? s * M * N * 8 / 4000000 + 4 : 0);
        if (best < 0 || cost < best) best = cost, count = s;
    }
    const int64_t chunk = cdiv(steps, count) * 32;
    return {cdiv(R, chunk), chunk};
}

// Room for the fp32 sums of the splits, in elements: one of dX, or of dX and of the widest piece's dW as many as the rules below may take.
// Splitting saves less than the time of a reduction's steps in one tile, which the sums' own must stay below: `worth` elements of them a
// step. It grows with T: a workspace serves fewer tokens too.
int64_t sums_room(int64_t T, int64_t V, int64_t K, int64_t (*splits)(int64_t), int64_t worth) {
    const int64_t rows = std::min(cdiv(V, 256) * 256, kCeMostWidth);
    auto many = [&](int64_t R, int64_t n) {
        const int64_t count = splits(R), most = std::min(kDxSums, worth * (cdiv(R, 32) + 8));
        return count <= 1 ? 0 : n > most / K / count ? most : count * n * K;
    };
    return std::max(T * K, std::max(many(V, T), many(T, rows)));
}
int64_t mfma_room(int64_t T, int64_t V, int64_t K) { return sums_room(T, V, K, mfma_most_splits, 500000); }
int64_t f32_room(int64_t T, int64_t V, int64_t K) { return sums_room(T, V, K, f32_most_splits, 690 * 560); }

struct MfmaSpace {
    float *r, *rest, *most, *sums, *part;
    int32_t *place;
    uint16_t *x, *D;
};
size_t mfma_space(int64_t T, int64_t V, int64_t K, char *base, MfmaSpace *s) {
    size_t at = kWsHeader;
    auto take = [&](size_t bytes) {
        char *p = base + at;
        at += round256(bytes);
        return p;
    };
    char *const most = take(sizeof(float)), *const r = take((size_t)T * sizeof(float)), *const rest = take((size_t)T * sizeof(float));
    char *const place = take((size_t)T * sizeof(int32_t)), *const x = take((size_t)T * (size_t)K * 2);
    char *const sums = take((size_t)T * (size_t)K * sizeof(float)), *const part = take((size_t)mfma_room(T, V, K) * sizeof(float));
    char *const D = take(piece_bytes(T, V, 2));
    if (s)
        *s = MfmaSpace{reinterpret_cast<float *>(r),    reinterpret_cast<float *>(rest), reinterpret_cast<float *>(most),
                       reinterpret_cast<float *>(sums), reinterpret_cast<float *>(part), reinterpret_cast<int32_t *>(place),
                       reinterpret_cast<uint16_t *>(x), reinterpret_cast<uint16_t *>(D)};
    return at;
}

// ---- fp32 ---------------------------------------------------------------------------------------
// Splits of a product's reduction over R into tiles of 64 x 64, in ns: the tiles that a CU has take a step of 32 rows in turn, 0.69 us
// where it has one, 0.56 of two and 0.51 of three, which is how many run at once, 1.5 us for their start and end; the sums' launch, and
// what it and the tiles move. dX of 1,024 x 10,000 x 1,024 (256 tiles) 217 us unsplit, 175 in two and 162 in three, of 301 x 5,003 x 1,008
// (80 tiles) 48 in three and 41 in six, of 100 x 8,000 x 2,048 (64) 48 in four and 40 in eight.
Splits f32_splits(int64_t R, int64_t N, int64_t K, int64_t room) {
    const int64_t tiles = cdiv(N, 64) * cdiv(K, 64), steps = cdiv(R, 32), cus = 256;
    const int64_t most = tiles >= 16 * cus ? 1 : std::min(f32_most_splits(R), std::min(room, kDxSums) / (N * K));
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
    const size_t x = round256((size_t)T * (size_t)K * sizeof(float)), part = round256((size_t)f32_room(T, V, K) * sizeof(float));
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
    const int64_t room = f32_room(T, V, K);
    a.D = s.D;
    auto finish = [&](int64_t splits, const float *before, int64_t n, float *sums, float *out) {
        return in_elements(n, [&](int64_t first, unsigned grid) {
            ce_sums_kernel<<<grid, 256, 0, st>>>(s.part, splits, before, nullptr, 0, nullptr, nullptr, nullptr, first, n, K, sums, out, kF32);
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
            const Splits p = f32_splits(n, T, K, room);
            const bool alone = p.count == 1 && n == V;
            e = launch_dw_f32(s.Dt, static_cast<const float *>(a.W) + v0 * K, n, T, pitch_t, K, p.chunk, p.count, alone ? dX : s.part, st);
            if (e == hipSuccess && !alone) e = finish(p.count, v0 ? s.sums : nullptr, T * K, v0 + n == V ? nullptr : s.sums, dX);
            if (e != hipSuccess) return e;
        }
        if (dW) {
            const Splits p = f32_splits(T, n, K, room);
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
    const int64_t T = a.T, V = a.V, K = a.K, room = mfma_room(T, V, K);
    ce_scales_kernel<<<1, 1024, 0, st>>>(a.target, a.g, a.h, T, V, s.r, s.place, s.most);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.scale = s.r, a.rest = s.rest, a.D = s.D;
    const int32_t *const place = a.g ? s.place : nullptr;  // nothing is at a target's place without its gradient
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
            const Splits p = mfma_splits(n, T, K, room);
            e = launch_dx_sums(s.D, W, T, n, width, K, p.chunk, p.count, s.part, st);
            if (e != hipSuccess) return e;
            const bool last = v0 + n == V;
            e = in_elements(T * K, [&](int64_t first, unsigned grid) {
                ce_sums_kernel<<<grid, 256, 0, st>>>(s.part, p.count, v0 ? s.sums : nullptr, s.r, 1, place, s.rest,
                                                     static_cast<const uint16_t *>(a.W), first, T * K, K, last ? nullptr : s.sums, dX, kBF16);
            });
            if (e != hipSuccess) return e;
        }
        if (dW) {
            char *const out = static_cast<char *>(dW) + (size_t)v0 * (size_t)K * (dw_dtype == kBF16 ? 2 : 4);
            const Splits p = mfma_splits(T, n, K, room);
            e = launch_dw_mfma(s.D, s.x, T, n, width, K, p.chunk, p.count, s.most, place, s.rest, v0, out, dw_dtype, s.part, st);
            if (e != hipSuccess) return e;
            if (p.count > 1)
                e = in_elements(n * K, [&](int64_t first, unsigned grid) {
                    ce_sums_kernel<<<grid, 256, 0, st>>>(s.part, p.count, nullptr, s.most, 0, nullptr, nullptr, nullptr, first, n * K, K,
                                                         nullptr, out, dw_dtype);
                });
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

hipError_t fwd(int dtype, CeArgs a, uint32_t *flag, char *base, hipStream_t st) {
    a.zt = reinterpret_cast<float *>(base);
    a.part = reinterpret_cast<float2 *>(base + round256((size_t)a.T * sizeof(float)));
    const bool mfma = dtype == kBF16, few = mfma && a.T <= kCeFew;
    const int64_t T = a.T, edge = mfma ? ce_mfma_tile(T, a.V) : ce_f32_tile(T, a.V);
    a.tiles_v = (int)cdiv(a.V, few ? kCeFewV : edge);
    hipError_t e = hipSuccess;
    if (few) {
        launch_ce_stats_few(a, st);
        e = hipGetLastError();
    } else {
        e = in_runs(cdiv(T, edge), a.tiles_v, [&](int64_t first, int64_t count) {
            a.t0 = first * edge;
            if (mfma) launch_ce_stats_mfma(a, edge, count * edge, st);
            else launch_ce_stats_f32(a, edge, count * edge, st);
        });
    }
    if (e != hipSuccess) return e;
    const int tokens = T >= 1024 ? 32 : T >= 32 ? 8 : 1;
    ce_join_kernel<<<(unsigned)cdiv(T, tokens), 256, 0, st>>>(a, a.tiles_v, tokens, flag);
    return hipGetLastError();
}

hipError_t bwd(int dtype, const CeArgs &a, void *dX, void *dW, int dw_dtype, uint32_t *flag, char *ws, hipStream_t st) {
    return dtype == kBF16 ? bwd_mfma(a, dX, dW, dw_dtype, flag, ws, st)
                          : bwd_f32(a, static_cast<float *>(dX), static_cast<float *>(dW), flag, ws, st);
}

// The workspace of rows that are multiples of 16
size_t fwd_space(int64_t T, int64_t V) {
    // parts of 64 vocabulary entries, or of 32 in fp32 where there are fewer than 256 tiles of 64 x 64
    const int64_t parts = std::max(cdiv(V, 64) * T, std::min(cdiv(V, 32) * T, int64_t(2) * 256 * 64));
    return kWsHeader + round256(round256((size_t)T * sizeof(float)) + (size_t)parts * sizeof(float2));
}
size_t bwd_space(int64_t T, int64_t V, int64_t K) {
    return round256(std::max(mfma_space(T, V, K, nullptr, nullptr), f32_space(T, V, K, nullptr, nullptr)));
}

}  // namespace

size_t linear_ce_fwd_ws(int64_t T, int64_t V, int64_t K) { return fwd_space(T, V) + pad_bytes(T, K) + pad_bytes(V, K); }

size_t linear_ce_bwd_ws(int64_t T, int64_t V, int64_t K) {
    return T == 0 ? kWsHeader : bwd_space(T, V, padded(K)) + 2 * (pad_bytes(T, K) + pad_bytes(V, K));
}

hipError_t launch_linear_ce_fwd(int dtype, const void *X, const void *W, int64_t T, int64_t V, int64_t K, const int64_t *target,
                                float *logp, float *lse, uint32_t *flag, void *ws, hipStream_t st) {
    char *const base = static_cast<char *>(ws);
    CeArgs a{};
    a.X = X, a.W = W, a.target = target, a.lse = lse, a.logp = logp, a.T = T, a.V = V, a.K = padded(K);
    if (K % 16) {
        char *const x = base + fwd_space(T, V), *const w = x + pad_bytes(T, K);
        hipError_t e = copy_rows(dtype, X, T, K, a.K, x, st);
        if (e == hipSuccess) e = copy_rows(dtype, W, V, K, a.K, w, st);
        if (e != hipSuccess) return e;
        a.X = x, a.W = w;
    }
    return fwd(dtype, a, flag, base + kWsHeader, st);
}

hipError_t launch_linear_ce_bwd(int dtype, const void *X, const void *W, int64_t T, int64_t V, int64_t K, const int64_t *target,
                                const float *lse, const float *g, const float *h, void *dX, void *dW, int dw_dtype,
                                uint32_t *flag, void *ws, hipStream_t st) {
    char *const base = static_cast<char *>(ws);
    CeArgs a{};
    a.X = X, a.W = W, a.target = target, a.lse = const_cast<float *>(lse), a.g = g, a.h = h, a.T = T, a.V = V, a.K = padded(K);
    if (K % 16 == 0) return bwd(dtype, a, dX, dW, dw_dtype, flag, base, st);
    char *const x = base + bwd_space(T, V, padded(K)), *const w = x + pad_bytes(T, K), *const dx = w + pad_bytes(V, K), *const dw = dx + pad_bytes(T, K);
    hipError_t e = copy_rows(dtype, X, T, K, a.K, x, st);
    if (e == hipSuccess) e = copy_rows(dtype, W, V, K, a.K, w, st);
    if (e != hipSuccess) return e;
    a.X = x, a.W = w;
    e = bwd(dtype, a, dX ? dx : nullptr, dW ? dw : nullptr, dw_dtype, flag, base, st);
    if (e == hipSuccess && dX) e = copy_rows(dtype, dx, T, a.K, K, dX, st);
    if (e == hipSuccess && dW) e = copy_rows(dw_dtype, dw, V, a.K, K, dW, st);
    return e;
}

}  // namespace focus
