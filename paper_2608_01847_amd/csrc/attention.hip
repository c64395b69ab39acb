// Attention over whole prompts in fp32 (v_mfma_f32_32x32x2_f32), forward and backward, and the choice between it and the
// bf16 kernels.
//
//   S = scale q k^T (causal: keys past the query's own place hidden, the last query at the last key),
//   P = softmax(S), O = P v, lse = log sum exp S
//   dv = P^T dO, dP = dO v^T, dS = P (dP - rowsum(dO O)) scale, dq = dS k, dk = dS^T q
//
// A workgroup takes 32 queries (forward, dq) or 32 keys (dk, dv) of one head; its four waves take alternate tiles of 32
// of the other side, each with its own running maximum and sum, and are joined through LDS in a fixed order. The
// scores are formed transposed (keys down the accumulator's rows, one query per lane), so that the softmax runs within
// a lane and its partner, and a register of probabilities is at once the B operand of the next product: register r
// holds the keys acc_row(r) (lanes 0-31) and acc_row(r) + 4 (lanes 32-63), the two that one instruction contracts.
// Operands come straight from global memory: one instruction takes 64 cycles for 512 bytes of operands, and a wave's loads of a
// tile are under way together. Bound by the latency of those loads, one wave per SIMD having no other to hide it: 4 x 2,048
// tokens, 16 heads of 64, full: forward 0.75 ms, 92 TFLOP/s of the 142 that an fp32 product of 4,096^3 reaches, backward 3.7 ms
// (65 TFLOP/s of its seven products); 794 tokens in six sequences, 8 heads of 64: forward 16 us, dq 23, dk and dv 35. The keys of few
// queries are not split: one query of 32/8 heads of 128 on 8,192 keys is 32 workgroups, 512 us.
#include "attn_common.h"

namespace focus {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 32;

__device__ __forceinline__ void load4(const float *p, float (&v)[4]) {
    const float4 w = *reinterpret_cast<const float4 *>(p);
    v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
}

// Loads are not branched around: what does not exist is loaded from a place that does and replaced by zeros, so that all of
// a tile's loads are under way together (`row` is a row that exists in every function here).

// One row's part of a lane: features 8 j + 4 (lane / 32) .. + 3 for every j (zeros where !ok or past D).
template <int DT>
__device__ __forceinline__ void load_row(const float *row, bool ok, int D, int half, float (&v)[4 * DT][4]) {
#pragma unroll
    for (int j = 0; j < 4 * DT; j++) {
        const int d = 8 * j + 4 * half;
        const bool in = ok && d < D;
        load4(row + (in ? d : 0), v[j]);
#pragma unroll
        for (int e = 0; e < 4; e++) v[j][e] = in ? v[j][e] : 0.0f;
    }
}

// 32 x 32 products of the 32 rows in a (rows of the result) with those in b (columns)
template <int DT>
__device__ __forceinline__ f32x16_t row_products(const float (&a)[4 * DT][4], const float (&b)[4 * DT][4]) {
    f32x16_t acc = {};
#pragma unroll
    for (int j = 0; j < 4 * DT; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j][e], b[j][e], acc, 0, 0, 0);
    return acc;
}

// A lane's features d = 32 t + lane % 32 of the 32 rows of an accumulator's registers; row i exists for i < n
template <int DT>
__device__ __forceinline__ void load_columns(const float *X, int64_t stride, int n, int D, int lane, float (&x)[16][DT]) {
    const int half = lane >> 5, col = lane & 31;
#pragma unroll
    for (int r = 0; r < 16; r++) {
        const int row = acc_row(r) + 4 * half;
#pragma unroll
        for (int t = 0; t < DT; t++) {
            const int d = 32 * t + col;
            x[r][t] = X[(row < n ? row : 0) * stride + (d < D ? d : 0)];
            x[r][t] = row < n && d < D ? x[r][t] : 0.0f;
        }
    }
}

// out^T[d][column] += sum over 32 rows of x[row][d] w[row][column], w in accumulator layout
template <int DT>
__device__ __forceinline__ void add_products(f32x16_t (&out)[DT], const float (&x)[16][DT], const float (&w)[16]) {
#pragma unroll
    for (int r = 0; r < 16; r++)
#pragma unroll
        for (int t = 0; t < DT; t++) out[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[r][t], w[r], out[t], 0, 0, 0);
}

// Everything loaded for a tile is under way before the first product, which the compiler would otherwise put off load by load
__device__ __forceinline__ void loads_first() { __builtin_amdgcn_sched_barrier(0); }

// Adds the four waves' accumulators in wave 0: (0 + 2) + (1 + 3).
template <int DT>
__device__ __forceinline__ void join(f32x16_t (&acc)[DT], float *lds, int wave, int lane) {
#pragma unroll
    for (int step = 2; step >= 1; step >>= 1) {
        __syncthreads();
        if (wave >= step && wave < 2 * step) {
#pragma unroll
            for (int t = 0; t < DT; t++)
#pragma unroll
                for (int r = 0; r < 16; r++) lds[(((wave - step) * DT + t) * 16 + r) * 64 + lane] = acc[t][r];
        }
        __syncthreads();
        if (wave < step) {
#pragma unroll
            for (int t = 0; t < DT; t++)
#pragma unroll
                for (int r = 0; r < 16; r++) acc[t][r] += lds[((wave * DT + t) * 16 + r) * 64 + lane];
        }
    }
}

// out^T of one lane's column to its row, times `f`
template <int DT>
__device__ __forceinline__ void store_column(float *row, int D, int half, const f32x16_t (&acc)[DT], float f) {
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const int d = 32 * t + 8 * g + 4 * half;
            if (d < D) {
                const float v[4] = {acc[t][4 * g] * f, acc[t][4 * g + 1] * f, acc[t][4 * g + 2] * f, acc[t][4 * g + 3] * f};
                store4(row + d, v);
            }
        }
}

template <int DT>
__global__ void __launch_bounds__(kThreads, 1) attn_fwd_kernel(AttnArgs a) {
    __shared__ float lds[2 * DT * 16 * 64];
    __shared__ float stat[2][kWaves][32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    SeqRange r;
    const int tile = slot_range<false>(a, kTile, (int)blockIdx.x, 1, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kTile, r.lq)) return;
    const int h = blockIdx.y, hk = h / (a.Hq / a.Hkv), D = a.D;
    const int q = tile * kTile + col, shift = r.lk - r.lq;
    const bool q_ok = q < r.lq;
    const float *K = static_cast<const float *>(a.k) + r.k0 * a.k_stride + (int64_t)hk * D;
    const float *V = static_cast<const float *>(a.v) + r.k0 * a.v_stride + (int64_t)hk * D;
    float qv[4 * DT][4];
    load_row<DT>(static_cast<const float *>(a.q) + (r.q0 + (q_ok ? q : 0)) * a.q_stride + (int64_t)h * D, q_ok, D, half, qv);
    const float c = a.scale * kLog2e;
    const int q_end = tile * kTile + kTile < r.lq ? tile * kTile + kTile : r.lq;
    const int k_end = a.causal ? (q_end + shift < r.lk ? q_end + shift : r.lk) : r.lk;
    const int seen = a.causal ? (q + shift < r.lk ? q + shift : r.lk - 1) : r.lk - 1;  // last key of this lane's query
    f32x16_t o[DT] = {};
    float m = -__builtin_inff(), l = 0.0f;
    for (int k0 = wave * kTile; k0 < k_end; k0 += kWaves * kTile) {
        const bool k_ok = k0 + col < r.lk;
        float kv[4 * DT][4], vx[16][DT];
        load_row<DT>(K + (k_ok ? k0 + col : 0) * a.k_stride, k_ok, D, half, kv);
        load_columns<DT>(V + k0 * a.v_stride, a.v_stride, r.lk - k0, D, lane, vx);
        loads_first();
        const f32x16_t acc = row_products<DT>(kv, qv);
        float p[16], top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < 16; i++) {
            p[i] = k0 + acc_row(i) + 4 * half <= seen ? acc[i] * c : -__builtin_inff();
            top = fmaxf(top, p[i]);
        }
        top = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), m);
        const float base = top == -__builtin_inff() ? 0.0f : top;
        const float alpha = exp2_raw(m - base);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            p[i] = exp2_raw(p[i] - base);
            sum += p[i];
        }
        m = top;
        l = l * alpha + sum;
#pragma unroll
        for (int t = 0; t < DT; t++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[t][i] *= alpha;
        add_products<DT>(o, vx, p);
    }
    l += __shfl_xor(l, 32, 64);
    if (half == 0) {
        stat[0][wave][col] = m;
        stat[1][wave][col] = l;
    }
    __syncthreads();
    float top = -__builtin_inff(), total = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; w++) top = fmaxf(top, stat[0][w][col]);
    const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < kWaves; w++) total += stat[1][w][col] * exp2_raw(stat[0][w][col] - base);
    const float mine = exp2_raw(m - base);
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[t][i] *= mine;
    join<DT>(o, lds, wave, lane);
    if (wave != 0 || !q_ok) return;
    const float inv = total > 0.0f ? 1.0f / total : (total == 0.0f ? 0.0f : total);
    store_column<DT>(static_cast<float *>(a.O) + ((r.q0 + q) * a.Hq + h) * D, D, half, o, inv);
    if (a.lse && half == 0) a.lse[(int64_t)h * a.Tq + r.q0 + q] = total == 0.0f ? -__builtin_inff() : (top + log2f(total)) * kLn2;
}

// dq of 32 queries, and delta = rowsum(dO O) for the keys' pass
template <int DT>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_q_kernel(AttnArgs a) {
    __shared__ float lds[2 * DT * 16 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    SeqRange r;
    const int tile = slot_range<false>(a, kTile, (int)blockIdx.x, 1, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kTile, r.lq)) return;
    const int h = blockIdx.y, hk = h / (a.Hq / a.Hkv), D = a.D;
    const int q = tile * kTile + col, shift = r.lk - r.lq;
    const bool q_ok = q < r.lq;
    const float *K = static_cast<const float *>(a.k) + r.k0 * a.k_stride + (int64_t)hk * D;
    const float *V = static_cast<const float *>(a.v) + r.k0 * a.v_stride + (int64_t)hk * D;
    float qv[4 * DT][4], gv[4 * DT][4];
    const int64_t oq = ((r.q0 + (q_ok ? q : 0)) * a.Hq + h) * D;
    float delta = 0.0f;
    load_row<DT>(static_cast<const float *>(a.O) + oq, q_ok, D, half, qv);
    load_row<DT>(static_cast<const float *>(a.dO) + oq, q_ok, D, half, gv);
#pragma unroll
    for (int j = 0; j < 4 * DT; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) delta = __builtin_fmaf(qv[j][e], gv[j][e], delta);
    delta += __shfl_xor(delta, 32, 64);
    if (wave == 0 && half == 0 && q_ok) a.delta[(int64_t)h * a.Tq + r.q0 + q] = delta;
    load_row<DT>(static_cast<const float *>(a.q) + (r.q0 + (q_ok ? q : 0)) * a.q_stride + (int64_t)h * D, q_ok, D, half, qv);
    const float c = a.scale * kLog2e;
    const float lse2 = q_ok ? a.lse[(int64_t)h * a.Tq + r.q0 + q] * kLog2e : 0.0f;
    const int q_end = tile * kTile + kTile < r.lq ? tile * kTile + kTile : r.lq;
    const int k_end = a.causal ? (q_end + shift < r.lk ? q_end + shift : r.lk) : r.lk;
    const int seen = a.causal ? (q + shift < r.lk ? q + shift : r.lk - 1) : r.lk - 1;
    f32x16_t dq[DT] = {};
    for (int k0 = wave * kTile; k0 < k_end; k0 += kWaves * kTile) {
        const bool k_ok = k0 + col < r.lk;
        float kv[4 * DT][4], vv[4 * DT][4], kx[16][DT];
        load_row<DT>(K + (k_ok ? k0 + col : 0) * a.k_stride, k_ok, D, half, kv);
        load_row<DT>(V + (k_ok ? k0 + col : 0) * a.v_stride, k_ok, D, half, vv);
        load_columns<DT>(K + k0 * a.k_stride, a.k_stride, r.lk - k0, D, lane, kx);
        loads_first();
        const f32x16_t sc = row_products<DT>(kv, qv);
        const f32x16_t dp = row_products<DT>(vv, gv);
        float ds[16];
#pragma unroll
        for (int i = 0; i < 16; i++)
            ds[i] = k0 + acc_row(i) + 4 * half <= seen ? exp2_raw(__builtin_fmaf(sc[i], c, -lse2)) * (dp[i] - delta) : 0.0f;
        add_products<DT>(dq, kx, ds);
    }
    join<DT>(dq, lds, wave, lane);
    if (wave != 0 || !q_ok) return;
    store_column<DT>(static_cast<float *>(a.dq) + (r.q0 + q) * a.dq_stride + (int64_t)h * D, D, half, dq, a.scale);
}

// dk and dv of 32 keys of one key-value head, summed over the query heads that share it
template <int DT>
__global__ void __launch_bounds__(kThreads, 1) attn_bwd_kv_kernel(AttnArgs a) {
    __shared__ float lds[2 * DT * 16 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    SeqRange r;
    const int tile = slot_range<true>(a, kTile, (int)blockIdx.x, 1, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kTile, r.lk)) return;
    const int hk = blockIdx.y, group = a.Hq / a.Hkv, D = a.D;
    const int k = tile * kTile + col, shift = r.lk - r.lq;
    const bool k_ok = k < r.lk;
    float kv[4 * DT][4], vv[4 * DT][4];
    load_row<DT>(static_cast<const float *>(a.k) + (r.k0 + (k_ok ? k : 0)) * a.k_stride + (int64_t)hk * D, k_ok, D, half, kv);
    load_row<DT>(static_cast<const float *>(a.v) + (r.k0 + (k_ok ? k : 0)) * a.v_stride + (int64_t)hk * D, k_ok, D, half, vv);
    const float c = a.scale * kLog2e;
    // first query that sees this tile's first key, and this lane's key
    const int q_first = a.causal && tile * kTile - shift > 0 ? (tile * kTile - shift) / kTile * kTile : 0;
    const int q_sees = a.causal ? k - shift : 0;
    const int q_tiles = r.lq > q_first ? (r.lq - q_first + kTile - 1) / kTile : 0;
    f32x16_t dk[DT] = {}, dv[DT] = {};
    for (int it = wave; it < q_tiles * group; it += kWaves) {
        const int h = hk * group + it / q_tiles, q0 = q_first + it % q_tiles * kTile;
        const float *Q = static_cast<const float *>(a.q) + (r.q0 + q0) * a.q_stride + (int64_t)h * D;
        const float *G = static_cast<const float *>(a.dO) + ((r.q0 + q0) * a.Hq + h) * D;
        const int64_t g_stride = (int64_t)a.Hq * D, at = (int64_t)h * a.Tq + r.q0 + q0;
        const int n = r.lq - q0;
        float x[16][DT], y[16][DT], ls[16], de[16];
        f32x16_t sc, dp;
        {
            float qv[4 * DT][4], gv[4 * DT][4];
            load_row<DT>(Q + (col < n ? col : 0) * a.q_stride, col < n, D, half, qv);
            load_row<DT>(G + (col < n ? col : 0) * g_stride, col < n, D, half, gv);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int row = acc_row(i) + 4 * half;
                ls[i] = a.lse[at + (row < n ? row : 0)];
                de[i] = a.delta[at + (row < n ? row : 0)];
            }
            if constexpr (DT <= 2) {  // more do not fit the registers
                load_columns<DT>(G, g_stride, n, D, lane, x);
                load_columns<DT>(Q, a.q_stride, n, D, lane, y);
            }
            loads_first();
            sc = row_products<DT>(qv, kv);
            dp = row_products<DT>(gv, vv);
        }
        if constexpr (DT > 2) {
            load_columns<DT>(G, g_stride, n, D, lane, x);
            loads_first();
        }
        float p[16], ds[16];
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int row = acc_row(i) + 4 * half;
            const bool ok = k_ok && row < n && q0 + row >= q_sees;
            p[i] = ok ? exp2_raw(__builtin_fmaf(sc[i], c, -ls[i] * kLog2e)) : 0.0f;
            ds[i] = ok ? p[i] * (dp[i] - de[i]) : 0.0f;
        }
        add_products<DT>(dv, x, p);
        if constexpr (DT > 2) {
            load_columns<DT>(Q, a.q_stride, n, D, lane, y);
            loads_first();
        }
        add_products<DT>(dk, y, ds);
    }
    join<DT>(dk, lds, wave, lane);
    join<DT>(dv, lds, wave, lane);
    if (wave != 0 || !k_ok) return;
    store_column<DT>(static_cast<float *>(a.dk) + (r.k0 + k) * a.dk_stride + (int64_t)hk * D, D, half, dk, a.scale);
    store_column<DT>(static_cast<float *>(a.dv) + (r.k0 + k) * a.dv_stride + (int64_t)hk * D, D, half, dv, 1.0f);
}

int64_t slots(int64_t T, int64_t n_seq, int rows) { return T / rows + n_seq; }

template <typename F>
void pick_dt(int D, F &&f) {
    if (D <= 32) f(std::integral_constant<int, 1>{});
    else if (D <= 64) f(std::integral_constant<int, 2>{});
    else if (D <= 96) f(std::integral_constant<int, 3>{});
    else f(std::integral_constant<int, 4>{});
}

hipError_t fwd(const AttnArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)slots(a.Tq, a.n_seq, kTile), (unsigned)a.Hq);
    pick_dt(a.D, [&](auto dt) { attn_fwd_kernel<decltype(dt)::value><<<grid, kThreads, 0, st>>>(a); });
    return hipGetLastError();
}

hipError_t bwd(const AttnArgs &a, hipStream_t st) {
    const dim3 gq((unsigned)slots(a.Tq, a.n_seq, kTile), (unsigned)a.Hq), gk((unsigned)slots(a.Tk, a.n_seq, kTile), (unsigned)a.Hkv);
    pick_dt(a.D, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (a.Tq > 0) attn_bwd_q_kernel<DT><<<gq, kThreads, 0, st>>>(a);
        if (a.Tk > 0) attn_bwd_kv_kernel<DT><<<gk, kThreads, 0, st>>>(a);
    });
    return hipGetLastError();
}

}  // namespace

size_t attn_fwd_ws(int dtype, int64_t Tq, int64_t Tk, int Hq, int Hkv, int D, int64_t n_seq) {
    const int splits = dtype == kBF16 ? attn_splits_bf16(Tq, Tk, Hq, Hkv, n_seq) : 1;  // the fp32 kernels have no parts
    if (splits == 1) return kWsHeader;
    return kWsHeader + attn_part_stats(splits, Tq * Hq) + (size_t)splits * (size_t)(Tq * Hq) * (size_t)D * sizeof(float);
}

static size_t delta_bytes(int64_t Tq, int Hq) { return ((size_t)Tq * (size_t)Hq * sizeof(float) + 255) / 256 * 256; }

size_t attn_bwd_ws(int dtype, int64_t Tq, int64_t Tk, int Hq, int Hkv, int D, int64_t n_seq) {
    const AttnBwdPlan p = dtype == kBF16 ? plan_attn_bwd_bf16(Tq, Tk, Hq, Hkv, n_seq) : AttnBwdPlan{1, 1};
    const size_t dq = p.q_splits > 1 ? (size_t)p.q_splits * (size_t)Tq * (size_t)Hq : 0;
    const size_t dkv = p.k_splits > 1 ? (size_t)p.k_splits * (size_t)Tk * (size_t)Hkv * 2 : 0;
    return kWsHeader + delta_bytes(Tq, Hq) + ((size_t)attn_rest_floats(p.q_splits, Tq * Hq) + (dq + dkv) * (size_t)D) * sizeof(float);
}

hipError_t launch_attn_fwd(int dtype, const AttnArgs &a, void *ws, hipStream_t st) {
    return dtype == kBF16 ? launch_attn_fwd_bf16(a, ws, st) : fwd(a, st);
}

hipError_t launch_attn_bwd(int dtype, AttnArgs a, void *ws, hipStream_t st) {
    a.delta = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader);
    if (dtype != kBF16) return bwd(a, st);
    return launch_attn_bwd_bf16(a, reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader + delta_bytes(a.Tq, a.Hq)), st);
}

}  // namespace focus
