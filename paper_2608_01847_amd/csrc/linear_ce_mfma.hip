// Logit tiles of the linear cross entropy on the bf16 matrix instructions (v_mfma_f32_32x32x16_bf16, fp32 sums).
//
// A workgroup of four waves forms 256 vocabulary entries x 256 tokens of W X^T, so that a lane holds one token's logits: rows =
// vocabulary, columns = tokens. The maximum and the sum of exponentials over the tile's vocabulary are then sums over a lane's
// registers, its partner's and another wave's, and no logit leaves the chip (forward); or the tile turns into that of D (backward),
// which goes to memory in bf16, through LDS. Operands are K-contiguous and go straight into a ring of LDS stages, several steps ahead
// of the matrix instructions, as in the reconstruction GEMM's forward. Few tiles: 128 x 128, two workgroups per CU.
//
// Bound by the matrix units at the clock that they leave the card: 8,192 x 151,936 x 2,560 forward 5.1-5.4 ms, 1.18-1.25 PFLOP/s (a
// library product of the shape, logits written, 1.40), matrix units busy 68% of a CU's cycles at 1.75 GHz, no LDS bank conflicts. The
// edge is 256 because an operand byte read from LDS then feeds 128 products; 8 waves of 128 x 64 would read half as much again.
// A cycle saved beside the products brings little: with what a token's D takes asked for before the products, eight trips to memory less
// of about 120,000 cycles a tile, the backward of that size became 0.8% faster (17.0 ms now).
//
// Up to 16 tokens the products are too few to hide the weights' way from memory, 2 K bytes per logit row: waves read 32 vocabulary
// rows each straight into the matrix instructions' registers.
#include "linear_ce.h"
#include "mfma_common.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kThreads = 256;
constexpr int kStep = 32;  // k per step
// E: the tile's edge. A stage holds 32 k of E rows of each operand; 160 KB of LDS, or two workgroups' 64 KB
template <int E>
struct Geometry {
    static constexpr int kStages = E == 256 ? 5 : 4, kOpBytes = E * 64, kStageBytes = 2 * kOpBytes, kLds = kStages * kStageBytes;
    static constexpr int kFrags = E / 64;   // of 32 rows, of a wave's half of an operand
    static constexpr int kLoads = E / 32;   // per thread and stage
};
constexpr float kLog2e = 1.44269504088896341f;

// e^(z - m) = 2^(z log2e - c) 2^-r with c = fl(m log2e) and r what that rounding lost: one operation per exponent, and no digit lost
// to the size of m
struct Exponent {
    float c, factor;
    __device__ __forceinline__ Exponent(float at, float f) : c(at), factor(f) {}
    __device__ __forceinline__ explicit Exponent(float m) {
        c = m * kLog2e;
        factor = exp2_raw(-__builtin_fmaf(m, kLog2e, -c));
    }
    __device__ __forceinline__ float operator()(float z) const { return exp2_raw(__builtin_fmaf(z, kLog2e, -c)); }
};

template <int E>
struct TileFrags {
    bf16x8_t a[E / 64], b[E / 64];
};

// acc[i][j][r] = logit of vocabulary entry v0 + E / 2 wm + 32 i + 8 (r / 4) + 4 (lane / 32) + r % 4 and token t0 + E / 2 wn + 32 j +
// lane % 32; entries past V and tokens past T have rows of zeros. All LDS may be used again afterwards.
template <int E>
__device__ __forceinline__ void logits_tile(const CeArgs &a, int64_t v0, int64_t t0, char *smem, f32x16_t (&acc)[E / 64][E / 64]) {
    using G = Geometry<E>;
    constexpr int S = G::kStages, N = G::kFrags, L = G::kLoads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    const int lr = lane & 31, lh = lane >> 5;
    const f32x16_t zero = {};
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
        for (int j = 0; j < N; j++) acc[i][j] = zero;
    lds_char *const lsm = (lds_char *)smem;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const int64_t pitch = a.K * 2;
    FwdDma<L / 2> dma;
    dma.init(pitch, wave_u, lane);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(static_cast<const char *>(a.W) + v0 * pitch, (a.V - v0) * pitch);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(static_cast<const char *>(a.X) + t0 * pitch, (a.T - t0) * pitch);
    const int64_t nk = (a.K + kStep - 1) / kStep;
    // Load i of step j into its stage: first the rows of W, then those of X. Past the rows' end a load brings zeros without going
    // to memory, so that every step is the same number of loads, which is what the waits count.
    auto issue = [&](int64_t j, int stage, int i) {
        const uint32_t base = (uint32_t)j * 64u, bad = dma.step_bad(pitch, base);
        lds_char *const st = lsm + stage * G::kStageBytes;
        if (i < L / 2) dma.issue_one(ra, base, bad, st, wave_u, i);
        else dma.issue_one(rb, base, bad, st + G::kOpBytes, wave_u, i - L / 2);
    };
#pragma unroll
    for (int s = 0; s < S - 1; s++)
#pragma unroll
        for (int i = 0; i < L; i++) issue(s, s, i);
    auto frags = [&](TileFrags<E> &f, const char *st, int ks) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            f.a[i] = *reinterpret_cast<const bf16x8_t *>(st + fwd_off(wm * (E / 2) + i * 32 + lr, ks * 2 + lh));
            f.b[i] = *reinterpret_cast<const bf16x8_t *>(st + G::kOpBytes + fwd_off(wn * (E / 2) + i * 32 + lr, ks * 2 + lh));
        }
    };
    // Before the barrier of step kt this thread's loads of steps up to kt + 1 have landed, after it everyone's have: the fragments
    // of step kt + 1 are read while step kt is multiplied, in three sets that rotate, and stage (kt - 1) % S, last read in step
    // kt - 2, takes step kt + S - 1.
    FOCUS_WAIT_VMCNT(L * (S - 3));
    asm volatile("s_barrier" ::: "memory");
    TileFrags<E> f, g, h;
    frags(f, smem, 0);
    frags(g, smem, 1);
    int sc = 0;  // kt % S
    auto step = [&](int64_t kt, TileFrags<E> &P, TileFrags<E> &Q, TileFrags<E> &R) {
        FOCUS_WAIT_VMCNT(L * (S - 3));
        asm volatile("s_barrier" ::: "memory");
        const int next = sc == S - 1 ? 0 : sc + 1, free = sc == 0 ? S - 1 : sc - 1;
        const char *const st = smem + next * G::kStageBytes;
        // the loads spread over the matrix instructions: closer together they fill the load queue, on which a wave then waits
        auto issue_at = [&](int i) {
            __builtin_amdgcn_sched_barrier(0);
            issue(kt + S - 1, free, i);
            __builtin_amdgcn_sched_barrier(0);
        };
        constexpr int every = N * N * 2 / L;
        frags(R, st, 0);
        static_for<N * N>([&](auto idx) {
            constexpr int i = idx / N, jj = idx % N;
            acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(P.a[i], P.b[jj], acc[i][jj], 0, 0, 0);
            if constexpr (idx % every == 1) issue_at(idx / every);
        });
        frags(P, st, 1);
        static_for<N * N>([&](auto idx) {
            constexpr int i = idx / N, jj = idx % N;
            acc[i][jj] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Q.a[i], Q.b[jj], acc[i][jj], 0, 0, 0);
            if constexpr (idx % every == 1) issue_at(L / 2 + idx / every);
        });
        sc = next;
    };
    int64_t kt = 0;
    for (; kt + 3 <= nk; kt += 3) {
        step(kt, f, g, h);
        step(kt + 1, h, f, g);
        step(kt + 2, g, h, f);
    }
    if (kt < nk) step(kt, f, g, h);
    if (kt + 1 < nk) step(kt + 1, h, f, g);
    FOCUS_WAIT_VMCNT(0);  // the loads past the end write zeros
    __syncthreads();
}

// Place (in the vocabulary) of register r of row block i of this lane, from the tile's first entry
template <int E>
__device__ __forceinline__ int entry_of(int i, int r) {
    const int lane = threadIdx.x & 63, wm = threadIdx.x >> 7;
    return E / 2 * wm + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
}

// Place in the tile from v0 on of a target, or -1
template <int E>
__device__ __forceinline__ int place_of(int64_t want, int64_t v0) {
    const int64_t d = want - v0;
    return d >= 0 && d < E ? (int)d : -1;
}

// Whether a lane's place lies in its wave's half of the tile, for any lane of the wave
template <int E>
__device__ __forceinline__ bool near_any(int at) {
    const int half = (threadIdx.x >> 7) * (E / 2);
    return __any(at >= half && at < half + E / 2);
}

}  // namespace

// Maximum and sum of exponentials of every token of the tile over its vocabulary entries, and the logit of a target there: for a
// wave 256 exponentials a lane, about 10,000 cycles beside the products' 82,000 at 2,560 features.
template <int E>
__global__ void __launch_bounds__(kThreads, E == 256 ? 1 : 2) ce_stats_mfma_kernel(CeArgs a) {
    __shared__ __attribute__((aligned(16))) char smem[Geometry<E>::kLds];
    constexpr int N = Geometry<E>::kFrags;
    uint32_t tv, tt;
    grouped_tile(xcd_tile(blockIdx.x, gridDim.x), (uint32_t)a.tiles_v, gridDim.x / (uint32_t)a.tiles_v, tv, tt);
    const int64_t v0 = (int64_t)tv * E, t0 = a.t0 + (int64_t)tt * E;
    // asked for before the products, each thread one token's: behind them, four trips to memory one after the other
    const int64_t own = t0 + threadIdx.x;
    const int place = a.target && threadIdx.x < E && own < a.T ? place_of<E>(a.target[own], v0) : -1;
    f32x16_t acc[N][N];
    logits_tile<E>(a, v0, t0, smem, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, lr = lane & 31, lh = lane >> 5;
    float2 *const red = reinterpret_cast<float2 *>(smem);  // [2 waves along the vocabulary][E tokens]
    int *const places = reinterpret_cast<int *>(smem + 2 * E * sizeof(float2));
    if (threadIdx.x < E) places[threadIdx.x] = place;
    __syncthreads();
    const int here = (int)std::min<int64_t>(E, a.V - v0);  // entries that exist
    auto reduce = [&](auto whole, auto j) {
        const int64_t t = t0 + E / 2 * wn + 32 * j + lr;
        const int at = places[E / 2 * wn + 32 * j + lr];
        if (near_any<E>(at)) {
            static_for<N>([&](auto i) {
                static_for<16>([&](auto r) {
                    if (at == entry_of<E>(i, r)) a.zt[t] = acc[i][j][(int)r];
                });
            });
        }
        if constexpr (!whole) {
            static_for<N>([&](auto i) {
                static_for<16>([&](auto r) { acc[i][j][(int)r] = entry_of<E>(i, r) < here ? acc[i][j][(int)r] : -__builtin_inff(); });
            });
        }
        float m = -__builtin_inff();
        static_for<N>([&](auto i) { static_for<16>([&](auto r) { m = fmaxf(m, acc[i][j][(int)r]); }); });
        m = fmaxf(m, __shfl_xor(m, 32, 64));
        const Exponent e(m);
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // a NaN stays one
        static_for<N>([&](auto i) { static_for<16>([&](auto r) { s[r % 4] += e(acc[i][j][(int)r]); }); });
        float sum = ((s[0] + s[1]) + (s[2] + s[3])) * e.factor;
        if (m == -__builtin_inff()) {  // no entry here exists, or none is a number
            sum = 0.0f;
            static_for<N>([&](auto i) {
                static_for<16>([&](auto r) { sum += acc[i][j][(int)r] == m ? 0.0f : __builtin_nanf(""); });
            });
        }
        sum += __shfl_xor(sum, 32, 64);
        if (lh == 0) red[wm * E + E / 2 * wn + 32 * j + lr] = make_float2(m, sum);
    };
    if (here == E) static_for<N>([&](auto j) { reduce(std::true_type{}, j); });
    else static_for<N>([&](auto j) { reduce(std::false_type{}, j); });
    __syncthreads();
    if (threadIdx.x >= E || own >= a.T) return;
    const float2 x = red[threadIdx.x], y = red[E + threadIdx.x];
    const float m = fmaxf(x.x, y.x);
    a.part[(int64_t)tv * a.T + own] = make_float2(m, (x.x == m ? x.y : x.y * expf(x.x - m)) + (y.x == m ? y.y : y.y * expf(y.x - m)));
}

// The tile of D: D[t][v] = (h - g) p + g [v == target] relative to the token's scale, p = exp(z - lse), rounded to bf16; what that
// leaves of a target's entry, the largest of most tokens, goes to `rest`. Entries past V are zeros.
template <int E>
__global__ void __launch_bounds__(kThreads, E == 256 ? 1 : 2) ce_grad_mfma_kernel(CeArgs a, uint32_t *flag) {
    __shared__ __attribute__((aligned(16))) char smem[Geometry<E>::kLds];
    constexpr int N = Geometry<E>::kFrags;
    uint32_t tv, tt;
    grouped_tile(xcd_tile(blockIdx.x, gridDim.x), (uint32_t)a.tiles_v, gridDim.x / (uint32_t)a.tiles_v, tv, tt);
    const int64_t c0 = (int64_t)tv * E, v0 = a.v0 + c0, t0 = a.t0 + (int64_t)tt * E;
    // what a token's D takes, as in the forward: the factor of the exponentials, what a target's entry adds, lse log2e, its place
    float4 own = make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));
    bool bad = false;
    if (threadIdx.x < E && t0 + threadIdx.x < a.T) {
        const int64_t t = t0 + threadIdx.x, want = a.target ? a.target[t] : -1;
        const float g = a.g && want >= 0 && want < a.V ? a.g[t] : 0.0f, h = a.h ? a.h[t] : 0.0f, lse = a.lse[t], scale = a.scale[t];
        bad = want >= a.V || ((g != 0.0f || h != 0.0f) && !(__builtin_fabsf(lse) <= 65536.0f));
        const Exponent e(lse);
        // quotients: the inverse of a tiny scale would overflow
        if (scale != 0.0f) own = make_float4((h - g) / scale * e.factor, g / scale, e.c, __int_as_float(place_of<E>(want, v0)));
    }
    f32x16_t acc[N][N];
    logits_tile<E>(a, v0, t0, smem, acc);
    float4 *const tokens = reinterpret_cast<float4 *>(smem + 2 * E * E);  // behind the tile
    if (threadIdx.x < E) tokens[threadIdx.x] = own;
    __syncthreads();
    const int lane = threadIdx.x & 63, wn = threadIdx.x >> 6 & 1, lr = lane & 31;
    static_for<N>([&](auto j) {
        const float4 of = tokens[E / 2 * wn + 32 * j + lr];
        const Exponent e{of.z, 1.0f};
        static_for<N>([&](auto i) { static_for<16>([&](auto r) { acc[i][j][(int)r] = of.x * e(acc[i][j][(int)r]); }); });
        const int at = __float_as_int(of.w);
        if (near_any<E>(at)) {
            float *const rest = a.rest + t0 + E / 2 * wn + 32 * j + lr;
            static_for<N>([&](auto i) {
                static_for<16>([&](auto r) {
                    if (at == entry_of<E>(i, r)) {
                        const float full = acc[i][j][(int)r] += of.y;
                        *rest = full - __uint_as_float(cvt_pk_bf16(full, 0.0f) << 16);
                    }
                });
            });
        }
        const bool none = of.x == 0.0f && of.y == 0.0f;  // no gradient (or no token), whatever X and lse hold
        if (__any(none)) {
            static_for<N>([&](auto i) {
                static_for<16>([&](auto r) { acc[i][j][(int)r] = none ? 0.0f : acc[i][j][(int)r]; });
            });
        }
    });
    if (v0 + E > a.V) {
        static_for<N * N>([&](auto ij) {
            static_for<16>([&](auto r) {
                if (v0 + entry_of<E>(ij / N, r) >= a.V) acc[ij / N][ij % N][(int)r] = 0.0f;
            });
        });
    }
    store_tile_bf16<E>(acc, smem, static_cast<uint16_t *>(a.D) + t0 * a.pitch, a.T - t0, a.pitch, (uint32_t)c0);
    if (bad) raise_domain_flag(flag);
}

// Up to 16 tokens: a wave takes 32 vocabulary entries, whose rows it reads straight into the operand registers (v_mfma_f32_16x16x32:
// a load instruction takes 64 bytes each of 16 rows), kAhead steps of 32 k under way; the tokens' rows come from the caches. Bound
// by the weights' way from memory: 1 x 151,936 x 2,560 162 us, 4.8 TB/s; 16 tokens 200. With 32 x 32 tiles, which read 32 bytes of
// a row at a time, 218; the waves of a workgroup on every fourth step of the same 32 entries, added up through LDS, 162 and 208, and
// 139 for 117 at 4 x 32,000 x 8,192 (14 to 6.5 at 8 x 3,000 x 1,024, where 24 workgroups leave most CUs without work). From 17 tokens on
// the tiles above take less (208 us for 253).
typedef float f32x4_t __attribute__((ext_vector_type(4)));
constexpr int kAhead = 8;
__global__ void __launch_bounds__(kThreads) ce_stats_few_kernel(CeArgs a) {
    __shared__ float2 red[4][kCeFew];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, quad = lane >> 4;
    const int64_t v0 = (int64_t)blockIdx.x * kCeFewV + wave * 32;
    const uint32_t pitch = (uint32_t)a.K * 2u;
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(static_cast<const char *>(a.W) + v0 * pitch, (a.V - v0) * (int64_t)pitch);
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.X, a.T * (int64_t)pitch);
    const uint32_t off = (uint32_t)l16 * pitch + (uint32_t)quad * 16u;
    auto load = [&](__amdgpu_buffer_rsrc_t rs, uint32_t k, int group) {  // k: bytes; past the row's end zeros
        const uint32_t past = (uint32_t)(k + quad * 16u >= pitch) << 31;
        return __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)((off + 16u * group * pitch + k) | past), 0, 0));
    };
    f32x4_t part[4][2] = {}, acc[2];  // four chains of roundings: a logit is off by 0.4 times as much as with one
    bf16x8_t w[kAhead][2], x[kAhead];
    auto fetch = [&](int i, uint32_t k) {
#pragma unroll
        for (int g = 0; g < 2; g++) w[i][g] = load(rw, k, g);
        x[i] = load(rx, k, 0);
    };
#pragma unroll
    for (int i = 0; i < kAhead; i++) fetch(i, 64u * i);
    for (uint32_t k = 0; k < pitch; k += 64u * kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
#pragma unroll
            for (int g = 0; g < 2; g++) part[i % 4][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[i][g], x[i], part[i % 4][g], 0, 0, 0);
            fetch(i, k + 64u * (kAhead + i));
        }
    }
#pragma unroll
    for (int g = 0; g < 2; g++) acc[g] = (part[0][g] + part[1][g]) + (part[2][g] + part[3][g]);
    // lane: token l16, entries v0 + 16 g + 4 quad + r
    const int64_t want = a.target && l16 < a.T ? a.target[l16] : -1;
    float m = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int g = 0; g < 2; g++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int64_t v = v0 + 16 * g + 4 * quad + r;
            if (v >= a.V) acc[g][r] = -__builtin_inff();
            else if (v == want) a.zt[l16] = acc[g][r];
            m = fmaxf(m, acc[g][r]);
        }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
#pragma unroll
    for (int g = 0; g < 2; g++)
#pragma unroll
        for (int r = 0; r < 4; r++) sum += acc[g][r] == -__builtin_inff() ? 0.0f : expf(acc[g][r] - m);  // a NaN stays one
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (quad == 0) red[wave][l16] = make_float2(m, sum);
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= kCeFew || t >= a.T) return;
    m = fmaxf(fmaxf(red[0][t].x, red[1][t].x), fmaxf(red[2][t].x, red[3][t].x));
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) sum += red[i][t].x == m ? red[i][t].y : red[i][t].y * expf(red[i][t].x - m);
    a.part[(int64_t)blockIdx.x * a.T + t] = make_float2(m, sum);
}

// 128 x 128 tiles where their rounds, 512 tiles each, are no longer than those of 256 x 256 tiles, 256 each: a round of the former
// takes 0.9 of one of the latter. Scores, us, with small and with large tiles: 100 tokens, vocabulary 10,000, 2,560 features (79
// small tiles) 35 and 59, 1,000 x 8,000 x 2,048 (504) 46 and 58, 2,048 x 4,000 x 2,560 (512) 58 and 64, 64 x 151,936 x 2,560
// (1,187) 185 and 216; 512 x 32,000 x 1,024 (1,000) 49 and 44.
int64_t ce_mfma_tile(int64_t T, int64_t n) {
    auto rounds = [&](int64_t edge, int64_t at_once) { return ((T + edge - 1) / edge * ((n + edge - 1) / edge) + at_once - 1) / at_once; };
    return 9 * rounds(kCeTile / 2, 2 * kMfmaConcurrentWgs) <= 10 * rounds(kCeTile, kMfmaConcurrentWgs) ? kCeTile / 2 : kCeTile;
}

void launch_ce_stats_mfma(const CeArgs &a, int64_t edge, int64_t tokens, hipStream_t st) {
    const unsigned grid = (unsigned)((tokens + edge - 1) / edge) * (unsigned)a.tiles_v;
    if (edge == kCeTile) ce_stats_mfma_kernel<kCeTile><<<grid, kThreads, 0, st>>>(a);
    else ce_stats_mfma_kernel<kCeTile / 2><<<grid, kThreads, 0, st>>>(a);
}

void launch_ce_grad_mfma(const CeArgs &a, int64_t edge, int64_t tokens, uint32_t *flag, hipStream_t st) {
    const unsigned grid = (unsigned)((tokens + edge - 1) / edge) * (unsigned)a.tiles_v;
    if (edge == kCeTile) ce_grad_mfma_kernel<kCeTile><<<grid, kThreads, 0, st>>>(a, flag);
    else ce_grad_mfma_kernel<kCeTile / 2><<<grid, kThreads, 0, st>>>(a, flag);
}

void launch_ce_stats_few(const CeArgs &a, hipStream_t st) { ce_stats_few_kernel<<<(unsigned)a.tiles_v, kThreads, 0, st>>>(a); }

}  // namespace focus
