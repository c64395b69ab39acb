// Attention over whole prompts in bf16 on the matrix instructions (v_mfma_f32_32x32x16_bf16).
//
// A key-value head's query rows are the pairs (query, head of its group), the heads of a query one after the other: a
// workgroup takes 128 rows of them, 32 per wave, so that grouped heads share the keys and values that it stages and a
// causal tile's ragged edge is as narrow as it can be. The scores are formed transposed (keys down the accumulator's
// rows, one query row per lane): the softmax runs within a lane and its partner 32 lanes on, and a register of probabilities
// is already the B operand of the second product, whose contraction may take the keys in any order: step t of a 64-key
// tile contracts, for lanes 0-31 (32-63), keys 16 t + {0-3, 8-11} (+ 4), the order in which the accumulator holds them;
// the transposing LDS reads of V follow the same order.
//
// Keys and values go through LDS in tiles of 64, two stages each, loaded into registers half a tile's work before they are
// written. Range-checked buffer loads read rows past a sequence and features past head_dim as zeros.
#include "attn_common.h"

namespace focus {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kKeys = 64;   // rows of a staged tile
constexpr float kNone = -__builtin_inff();

// Geometry of a staged tile of 64 rows: DT x 32 features, a row of 128 (DT <= 2) or 256 bytes. 16-byte chunk c of row r
// lies at chunk c ^ key(r): 8 consecutive rows of one chunk (a fragment read), and 4 rows of two neighbouring chunks (half a
// transposing read), then lie in different banks.
template <int DT>
struct Tile {
    static constexpr int kChunks = DT <= 2 ? 8 : 16;
    static constexpr int kPitch = kChunks * 16;
    static constexpr int kBytes = kKeys * kPitch;
    static constexpr int kLoads = kKeys * kChunks / kThreads;  // 16-byte loads per thread
    static constexpr int kRowStep = kThreads / kChunks;        // rows between a thread's loads
    __device__ static __forceinline__ uint32_t key(uint32_t r) {
        if constexpr (kChunks == 16) return ((r & 7u) << 1) | ((r >> 3) & 1u);
        return (((r >> 1) & 3u) << 1) | ((r >> 3) & 1u);
    }
};

// A thread's part of the tiles of one operand
template <int DT>
struct Stager {
    using G = Tile<DT>;
    uint32_t off[G::kLoads];  // byte offsets in a tile of the tensor, bit 31 set past head_dim
    uint32_t lds;
    u32x4_t v[G::kLoads];
    __device__ __forceinline__ void init(int64_t stride, int D) {
        const uint32_t c = threadIdx.x % G::kChunks, r = threadIdx.x / G::kChunks;
        const uint32_t past = (int)c * 8 < D ? 0u : 0x80000000u;
#pragma unroll
        for (int i = 0; i < G::kLoads; i++) off[i] = ((r + i * G::kRowStep) * (uint32_t)(stride * 2) + c * 16u) | past;
        lds = r * G::kPitch + ((c ^ G::key(r)) << 4);
    }
    // rows `row` .. of a sequence of n rows that starts at base
    __device__ __forceinline__ void load(const uint16_t *base, int64_t stride, int row, int n, int D) {
        const int left = n - row < kKeys ? n - row : kKeys;
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(base + row * stride, left > 0 ? ((left - 1) * stride + D) * 2 : 0);
#pragma unroll
        for (int i = 0; i < G::kLoads; i++) v[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off[i], 0, 0);
    }
    __device__ __forceinline__ void store(char *tile) const {
#pragma unroll
        for (int i = 0; i < G::kLoads; i++)
            *(lds_u32x4 *)(uintptr_t)(lds_addr(tile) + lds + i * (G::kRowStep * G::kPitch)) = v[i];
    }
    __device__ static __forceinline__ uint32_t lds_addr(const char *p) {
        return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
    }
};

// A lane's LDS offsets of the fragments of a tile
template <int DT>
struct Frags {
    using G = Tile<DT>;
    uint32_t row;       // straight reads: row lane % 32, chunk lane / 32; chunk 2 s + that of step s at ^ 32 s
    uint32_t tr[2][DT];  // transposing reads: rows 8 e + 4 (lane / 32) .. + 3, features 32 t + 16 (lane / 16 % 2) .. + 15
    __device__ __forceinline__ void init(int lane) {
        const uint32_t r = lane & 31, h = lane >> 5;
        row = r * G::kPitch + ((h ^ G::key(r)) << 4);
        const uint32_t j = lane & 15, g = (lane >> 4) & 1;
#pragma unroll
        for (uint32_t e = 0; e < 2; e++) {
            const uint32_t tr_row = 8 * e + 4 * h + j / 4;
#pragma unroll
            for (uint32_t t = 0; t < DT; t++)
                tr[e][t] = tr_row * G::kPitch + (((4 * t + 2 * g + (j % 4) / 2) ^ G::key(tr_row)) << 4) + 8 * (j % 2);
        }
    }
    // A operand: 32 rows from row 32 b on, features 16 s .. 16 s + 15
    __device__ __forceinline__ bf16x8_t straight(uint32_t tile, int b, int s) const {
        return *(lds_bf16x8 *)(uintptr_t)((row ^ (uint32_t)(32 * s)) + tile + b * 32 * G::kPitch);
    }
    // A operand: features 32 t .. 32 t + 31, the 16 rows from 16 s on in accumulator order
    __device__ __forceinline__ bf16x8_t transposed(uint32_t tile, int s, int t) const {
        const i16x4_t v[2] = {
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(uintptr_t)(tr[0][t] + tile + s * 16 * G::kPitch)),
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(uintptr_t)(tr[1][t] + tile + s * 16 * G::kPitch))};
        return __builtin_bit_cast(bf16x8_t, v);
    }
};

__device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// the lane 32 on
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 8 accumulator registers from 8 s on as a B operand
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t &p, int s) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; e++) w[e] = pack_bf16(p[8 * s + 2 * e], p[8 * s + 2 * e + 1]);
    return __builtin_bit_cast(bf16x8_t, w);
}

// A wave's 32 query rows: this lane's row, and the key ranges that the wave sees
struct Rows {
    bool ok;
    int q, g;       // this lane's query and head of the group
    int seen;       // last key that it sees
    int all_seen;   // last key that every row of the wave sees
    int any_seen;   // last key that some row sees (-1: none)
};

template <int DT>
__device__ __forceinline__ void load_row(const uint16_t *row, bool ok, int D, int half, bf16x8_t (&v)[2 * DT]) {
#pragma unroll
    for (int s = 0; s < 2 * DT; s++) {
        const int d = 16 * s + 8 * half;
        u32x4_t w = {0u, 0u, 0u, 0u};
        if (ok && d < D) w = *reinterpret_cast<const u32x4_t *>(row + d);
        v[s] = __builtin_bit_cast(bf16x8_t, w);
    }
}

// out^T, a lane's query row down its registers, times f, to the row in memory: the halves of a lane pair exchange 4
// features each, so that both write 16 bytes at a time
template <int DT>
__device__ __forceinline__ void store_row(uint16_t *row, bool ok, int D, int half, const f32x16_t (&acc)[DT], float f) {
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            // registers 4 g + e: features 32 t + 8 g + 4 half + e; registers 4 (g + 1) + e: 8 more
            const uint32_t a0 = pack_bf16(acc[t][4 * g] * f, acc[t][4 * g + 1] * f), a1 = pack_bf16(acc[t][4 * g + 2] * f, acc[t][4 * g + 3] * f);
            const uint32_t b0 = pack_bf16(acc[t][4 * g + 4] * f, acc[t][4 * g + 5] * f), b1 = pack_bf16(acc[t][4 * g + 6] * f, acc[t][4 * g + 7] * f);
            const auto x = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            // lanes 0-31: features 8 g .. 8 g + 7, lanes 32-63: 8 (g + 1) .. + 7
            const int d = 32 * t + 8 * (g + half);
            if (ok && d < D) *reinterpret_cast<u32x4_t *>(row + d) = u32x4_t{x[0], y[0], x[1], y[1]};
        }
}

template <int DT>
__global__ void __launch_bounds__(kThreads, 2) attn_fwd_bf16_kernel(AttnArgs a) {
    using G = Tile<DT>;
    __shared__ __attribute__((aligned(16))) char smem[4 * G::kBytes];  // K, K, V, V
    constexpr int kRows = 32 * kWaves;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int hk = blockIdx.x % a.Hkv, group = a.Hq / a.Hkv, D = a.D;
    int tile;
    const int s = slot_sequence(a.cu_q, a.n_seq, kRows, (int)(gridDim.x / a.Hkv - 1 - blockIdx.x / a.Hkv), group, tile);
    SeqRange r;
    seq_range(a, s, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kRows, (int64_t)r.lq * group)) return;
    const int shift = r.lk - r.lq;
    const int64_t rows = (int64_t)r.lq * group, first = (int64_t)tile * kRows;
    const int64_t last = first + kRows < rows ? first + kRows - 1 : rows - 1;
    auto sees = [&](int64_t row) {
        const int k = a.causal ? (int)(row / group) + shift : r.lk - 1;
        return k < r.lk ? k : r.lk - 1;
    };
    const int k_end = sees(last) + 1;
    const int nk = k_end > 0 ? (k_end + kKeys - 1) / kKeys : 0;
    const int64_t w_first = first + 32 * wave, w_last = w_first + 31 < last ? w_first + 31 : last;
    const int any_seen = w_first <= last ? sees(w_last) : -1, all_seen = sees(w_first);
    const int64_t row = w_first + col;
    const bool ok = row <= last;
    const int q = (int)(row / group), h = hk * group + (int)(row - (int64_t)q * group);
    const int seen = ok ? sees(row) : r.lk - 1;

    bf16x8_t qv[2 * DT];
    load_row<DT>(static_cast<const uint16_t *>(a.q) + (r.q0 + q) * a.q_stride + (int64_t)h * D, ok, D, half, qv);
    if (a.scale < 0.0f) {  // the maximum is taken before the scale: move its sign to the queries
#pragma unroll
        for (int i = 0; i < 2 * DT; i++) qv[i] = -qv[i];
    }
    // a scale of 0 keeps hidden keys at -inf
    const float c = fmaxf(__builtin_fabsf(a.scale) * kLog2e, 1e-30f);

    const uint16_t *K = static_cast<const uint16_t *>(a.k) + r.k0 * a.k_stride + (int64_t)hk * D;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + r.k0 * a.v_stride + (int64_t)hk * D;
    Stager<DT> ks, vs;
    ks.init(a.k_stride, D);
    vs.init(a.v_stride, D);
    Frags<DT> f;
    f.init(lane);
    const uint32_t base = Stager<DT>::lds_addr(smem);

    f32x16_t o[DT] = {};
    float m = kNone, l = 0.0f;
    if (nk > 0) {
        ks.load(K, a.k_stride, 0, r.lk, D);
        vs.load(V, a.v_stride, 0, r.lk, D);
        ks.store(smem);
        vs.store(smem + 2 * G::kBytes);
    }
    __syncthreads();
    for (int j = 0; j < nk; j++) {
        const int st = j & 1, k0 = j * kKeys;
        const uint32_t kt = base + st * G::kBytes, vt = base + (2 + st) * G::kBytes;
        const bool more = j + 1 < nk, active = k0 <= any_seen;
        if (more) ks.load(K, a.k_stride, k0 + kKeys, r.lk, D);
        bf16x8_t p[4];
        if (active) {
            f32x16_t sc[2] = {};
#pragma unroll
            for (int i = 0; i < 2 * DT; i++)
#pragma unroll
                for (int b = 0; b < 2; b++) sc[b] = mfma(f.straight(kt, b, i), qv[i], sc[b]);
            if (k0 + kKeys - 1 > all_seen) {
#pragma unroll
                for (int b = 0; b < 2; b++)
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        if (k0 + 32 * b + acc_row(i) + 4 * half > seen) sc[b][i] = kNone;
            }
            float top = sc[0][0];
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
                for (int i = 0; i < 16; i++) top = fmaxf(top, sc[b][i]);
            top = max_halves(top) * c;
            // The reference that the exponents are taken from follows the maximum only where it is passed by more than
            // 8: probabilities stay below 2^8, and most tiles need no rescaling.
            if (__any(top > m + 8.0f)) {
                const float now = fmaxf(m, top);
                const float alpha = now == kNone ? 1.0f : exp2_raw(m - now);
                m = now;
                l *= alpha;
#pragma unroll
                for (int t = 0; t < DT; t++)
#pragma unroll
                    for (int i = 0; i < 16; i++) o[t][i] *= alpha;
            }
            const float from = m == kNone ? 0.0f : m;
            float sum = 0.0f;
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    sc[b][i] = exp2_raw(__builtin_fmaf(sc[b][i], c, -from));
                    sum += sc[b][i];
                }
            l += sum;
#pragma unroll
            for (int i = 0; i < 4; i++) p[i] = pack8(sc[i >> 1], i & 1);
        }
        if (more) {
            ks.store(smem + (st ^ 1) * G::kBytes);
            vs.load(V, a.v_stride, k0 + kKeys, r.lk, D);
        }
        if (active) {
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int t = 0; t < DT; t++) o[t] = mfma(f.transposed(vt, i, t), p[i], o[t]);
        }
        if (more) vs.store(smem + (2 + (st ^ 1)) * G::kBytes);
        __syncthreads();
    }
    l = sum_halves(l);
    // no key seen: zeros and -inf; a NaN among the scores stays one
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store_row<DT>(static_cast<uint16_t *>(a.O) + ((r.q0 + q) * a.Hq + h) * D, ok, D, half, o, inv);
    if (a.lse && ok && half == 0) a.lse[(int64_t)h * a.Tq + r.q0 + q] = l == 0.0f ? kNone : (m + log2f(l)) * kLn2;
}

template <typename F>
void pick_dt(int D, F &&f) {
    if (D <= 64) f(std::integral_constant<int, 2>{});
    else if (D <= 96) f(std::integral_constant<int, 3>{});
    else f(std::integral_constant<int, 4>{});
}

}  // namespace

hipError_t launch_attn_fwd_bf16(const AttnArgs &a, hipStream_t st) {
    const int64_t slots = a.Tq * (a.Hq / a.Hkv) / (32 * kWaves) + a.n_seq;
    pick_dt(a.D, [&](auto dt) { attn_fwd_bf16_kernel<decltype(dt)::value><<<(unsigned)(slots * a.Hkv), kThreads, 0, st>>>(a); });
    return hipGetLastError();
}

}  // namespace focus
