// Attention over whole prompts in bf16 on the matrix instructions (v_mfma_f32_32x32x16_bf16).
//
// A key-value head's query rows are the pairs (query, head of its group), the heads of a query one after the other: a
// workgroup takes 128 rows of them, 32 per wave, so that grouped heads share the keys and values that it stages and a
// causal tile's ragged edge is as narrow as it can be. The scores are formed transposed (keys down the accumulator's
// rows, one query row per lane): the softmax runs within a lane and its partner 32 lanes on, and a register of probabilities
// is already the B operand of the second product (rounded to bf16, the type that the instruction takes: 2^-9 of each, random
// over the keys, which makes O's error 1.35 to 1.41 times that of rounding O), whose contraction may take the keys in any order:
// step t of a 64-key tile contracts, for lanes 0-31 (32-63), keys 16 t + {0-3, 8-11} (+ 4), the order in which the accumulator
// holds them; the transposing LDS reads of V follow the same order.
//
// Keys and values go through LDS in tiles of 64, two stages each, by direct-to-LDS loads a tile ahead, whose range check reads
// rows past a sequence and features past head_dim as zeros.
#include "attn_common.h"

namespace focus {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kKeys = 64;   // rows of a staged tile
constexpr int kFewTiles = 4;  // of keys, at most: row tiles that the queries' backward goes through twice
constexpr float kNone = -__builtin_inff();

// Geometry of a staged tile of ROWS rows: DT x 32 features, a row of 128 (DT <= 2) or 256 bytes. 16-byte chunk c of row r
// lies at chunk c ^ key(r): 16 consecutive rows of one chunk (a fragment read) then fill the 256 bytes of a pass over the
// banks, and so do 4 rows of four neighbouring chunks (half a transposing read; keys that put two of the rows in one
// 64-byte quarter made those reads take twice as long).
template <int DT, int ROWS = kKeys>
struct Tile {
    static constexpr int kChunks = DT <= 2 ? 8 : 16;
    static constexpr int kPitch = kChunks * 16;
    static constexpr int kBytes = ROWS * kPitch;
    static constexpr int kLoads = ROWS * kChunks / kThreads;  // 16-byte loads per thread
    // linear in the bits of r (exclusive or), and of its low four alone
    __host__ __device__ static constexpr uint32_t key(uint32_t r) {
        return kChunks == 16 ? (r & 3u) << 2 | ((r >> 2) & 3u) : (r & 2u) << 1 | ((r >> 2) & 3u);
    }
};

__device__ __forceinline__ uint32_t lds_addr(const char *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

__device__ __forceinline__ uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// Direct-to-LDS loads of one operand's tiles: lane L of a wave's instruction i writes 16 bytes at 16 L from the
// instruction's place, 1 KB of whole rows, and so reads the chunk of its row that belongs there.
//
// The instructions are written out: to the compiler's builtin every LDS read may alias the loads under way, and it would
// wait for all of them before the first fragment of the tile at hand. They have no result in registers, and `landed` waits
// for them before the barrier that hands the tile over. A scalar register that holds part of the descriptor may have been
// written by a vector instruction just before, and M0 by a scalar one: the waits the hardware asks for stand in the block.
template <int DT, int ROWS = kKeys>
struct Dma {
    using G = Tile<DT, ROWS>;
    static constexpr uint32_t kRowsEach = 1024 / G::kPitch;
    uint32_t row, chunk;  // byte offsets of this lane's row and chunk of the first load
    __device__ __forceinline__ void init(int64_t stride, int wave, int lane) {
        const uint32_t r = (uint32_t)wave * (G::kLoads * kRowsEach) + (uint32_t)lane / G::kChunks;
        row = r * (uint32_t)(stride * 2);
        chunk = (((uint32_t)lane % G::kChunks) ^ G::key(r)) << 4;
    }
    // (the key's linearity needs rows that differ by whole kRowsEach to differ in bits that a lane's row does not use)
    static_assert(G::kLoads * kRowsEach >= 8 && (kRowsEach & (kRowsEach - 1)) == 0, "rows of a wave's loads");
    // offset of load i: past head_dim, and for the `lead` rows of the tile that lie before the base, with bit 31 set (read
    // as zeros)
    __device__ __forceinline__ uint32_t off(uint32_t i, int64_t stride, int D, int lead) const {
        const uint32_t c = chunk ^ (G::key(i * kRowsEach) << 4);
        return (row + i * kRowsEach * (uint32_t)(stride * 2) - (uint32_t)lead * (uint32_t)(stride * 2) + c) |
               ((int)c < 2 * D ? 0u : 0x80000000u);
    }
    // rows `row` .. of a sequence of n rows that starts at base, into the tile at LDS address `tile`, behind `lead` rows of
    // zeros
    __device__ __forceinline__ void load(const uint16_t *base, int64_t stride, int row, int n, int D, uint32_t tile, int wave,
                                         int lead = 0) const {
        const int left = n - row < ROWS - lead ? n - row : ROWS - lead;
        const uint64_t p = (uint64_t)(base + row * stride);
        const u32x4_t rs = {scalar((uint32_t)p), scalar((uint32_t)(p >> 32) & 0xFFFFu),
                            scalar(left > 0 ? (uint32_t)(((left - 1) * stride + D) * 2) : 0u), (uint32_t)kRsrcWord3};
        const uint32_t at = scalar(tile + (uint32_t)wave * (G::kLoads * 1024u));
        if constexpr (G::kLoads == 4) {
            asm volatile(
                "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                "s_add_u32 m0, %0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
                "s_add_u32 m0, %0, 0x800\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen lds\n\t"
                "s_add_u32 m0, %0, 0xc00\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds"
                :
                : "s"(at), "v"(off(0, stride, D, lead)), "v"(off(1, stride, D, lead)), "v"(off(2, stride, D, lead)), "v"(off(3, stride, D, lead)), "s"(rs)
                : "memory", "scc");
        } else {
            static_assert(G::kLoads == 2, "two or four loads per wave");
            asm volatile(
                "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                "s_add_u32 m0, %0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
                :
                : "s"(at), "v"(off(0, stride, D, lead)), "v"(off(1, stride, D, lead)), "s"(rs)
                : "memory", "scc");
        }
    }
};

// Every load of this wave has landed and every LDS read of it is done; then the same holds for the workgroup.
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A lane's LDS offsets of the fragments of a tile
template <int DT>
struct Frags {
    using G = Tile<DT>;
    uint32_t row;    // straight reads: row lane % 32, chunk lane / 32; chunk 2 s + that of step s at ^ 32 s
    uint32_t tr[2];  // transposing reads: rows 8 e + 4 (lane / 32) .. + 3, features 16 (lane / 16 % 2) .. + 15; 32 t more at ^ 64 t
    // `base`: LDS address of the tiles, a multiple of 256
    __device__ __forceinline__ void init(int lane, uint32_t base) {
        const uint32_t r = lane & 31, h = lane >> 5;
        row = base + r * G::kPitch + ((h ^ G::key(r)) << 4);
        const uint32_t j = lane & 15, g = (lane >> 4) & 1;
#pragma unroll
        for (uint32_t e = 0; e < 2; e++) {
            const uint32_t tr_row = 8 * e + 4 * h + j / 4;
            tr[e] = base + tr_row * G::kPitch + (((2 * g + (j % 4) / 2) ^ G::key(tr_row)) << 4) + 8 * (j % 2);
        }
    }
    // Keeps the compiler from holding every step's address in a register of its own over a loop: one operation forms
    // each, and the registers are short.
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(row), "+v"(tr[0]), "+v"(tr[1])); }
    // A operand: 32 rows from row 32 b of the tile at byte TILE on, features 16 s .. 16 s + 15
    template <uint32_t TILE>
    __device__ __forceinline__ bf16x8_t straight(int b, int s) const {
        return *(lds_bf16x8 *)(uintptr_t)((row ^ (uint32_t)(32 * s)) + (TILE + b * 32 * G::kPitch));
    }
    // A operand: features 32 t .. 32 t + 31, the 16 rows from 16 s on in accumulator order
    template <uint32_t TILE>
    __device__ __forceinline__ bf16x8_t transposed(int s, int t) const {
        const i16x4_t v[2] = {
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(uintptr_t)((tr[0] ^ (uint32_t)(64 * t)) + (TILE + s * 16 * G::kPitch))),
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(uintptr_t)((tr[1] ^ (uint32_t)(64 * t)) + (TILE + s * 16 * G::kPitch)))};
        return __builtin_bit_cast(bf16x8_t, v);
    }
};

// The same with every address in a register of its own: no operation per read.
template <int DT>
struct Addresses {
    using G = Tile<DT>;
    uint32_t row[2 * DT], tr[2][DT];
    __device__ __forceinline__ void init(int lane, uint32_t base) {
        Frags<DT> f;
        f.init(lane, base);
#pragma unroll
        for (int s = 0; s < 2 * DT; s++) row[s] = f.row ^ (uint32_t)(32 * s);
#pragma unroll
        for (int t = 0; t < DT; t++)
#pragma unroll
            for (int e = 0; e < 2; e++) tr[e][t] = f.tr[e] ^ (uint32_t)(64 * t);
        // from here on they are what they are, not something to be formed again
#pragma unroll
        for (int s = 0; s < 2 * DT; s++) asm volatile("" : "+v"(row[s]));
#pragma unroll
        for (int t = 0; t < DT; t++) asm volatile("" : "+v"(tr[0][t]), "+v"(tr[1][t]));
    }
    template <uint32_t TILE>
    __device__ __forceinline__ bf16x8_t straight(int b, int s) const {
        return *(lds_bf16x8 *)(uintptr_t)(row[s] + (TILE + b * 32 * G::kPitch));
    }
    template <uint32_t TILE>
    __device__ __forceinline__ bf16x8_t transposed(int s, int t) const {
        const i16x4_t v[2] = {
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(uintptr_t)(tr[0][t] + (TILE + s * 16 * G::kPitch))),
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(uintptr_t)(tr[1][t] + (TILE + s * 16 * G::kPitch)))};
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

// N groups of matrix instructions, each on up to F fragments that are read from LDS while the groups before run: R sets of
// registers in turn, R - 1 groups ahead. Left to itself the compiler reads each fragment just before its use, into the same
// few registers, and every pair of instructions waits out the LDS latency.
template <int N, int F = 4, int R = 2, typename Load, typename Run>
__device__ __forceinline__ void pipelined(Load &&load, Run &&run) {
    bf16x8_t x[R][F];
    static_for<R - 1>([&](auto g) {
        if constexpr (g < N) load(g, x[g]);
    });
    static_for<N>([&](auto g) {
        if constexpr (g + R - 1 < N) load(std::integral_constant<int, g + R - 1>{}, x[(g + R - 1) % R]);
        __builtin_amdgcn_sched_barrier(0);
        run(g, x[g % R]);
        __builtin_amdgcn_sched_barrier(0);
    });
}

// The lane's number formed again where it is needed, for kernels that have no register to keep it in
__device__ __forceinline__ int lane_again() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t & 63;
}

// 8 accumulator registers from 8 s on as a B operand
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t &p, int s) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; e++) w[e] = pack_bf16(p[8 * s + 2 * e], p[8 * s + 2 * e + 1]);
    return __builtin_bit_cast(bf16x8_t, w);
}

// What rounding those 8 to `high` left, rounded likewise: high + low has 16 bits
__device__ __forceinline__ bf16x8_t pack8_rest(const f32x16_t &p, int s, bf16x8_t high) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; e++)
        w[e] = pack_bf16(p[8 * s + 2 * e] - (float)high[2 * e], p[8 * s + 2 * e + 1] - (float)high[2 * e + 1]);
    return __builtin_bit_cast(bf16x8_t, w);
}

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

// The same unscaled and in fp32, into a part of a split sum
template <int DT>
__device__ __forceinline__ void store_part(float *row, bool ok, int D, int half, const f32x16_t (&acc)[DT]) {
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const int d = 32 * t + 8 * g + 4 * half;
            if (ok && d < D) *reinterpret_cast<f32x4_t *>(row + d) = f32x4_t{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
        }
}

// What a wave's lane does in the kernels whose columns are query rows: its row, and the keys that it, its wave and its
// workgroup see.
struct RowTile {
    bool ok;
    int q, h;       // this lane's query (in its sequence) and head
    int seen;       // last key that it sees
    int all_seen;   // last key that every row of the wave sees
    int any_seen;   // last key that some row of the wave sees (-1: none)
    int nk;         // tiles of 64 keys that the workgroup goes through
    __device__ __forceinline__ void init(const AttnArgs &a, const SeqRange &r, int tile, int hk, int wave, int col) {
        constexpr uint32_t kRows = 32 * kWaves;
        const uint32_t group = (uint32_t)(a.Hq / a.Hkv);
        const int shift = r.lk - r.lq;
        // rows of a key-value head are below 2^31 (checked on the host)
        const uint32_t rows = (uint32_t)r.lq * group, first = (uint32_t)tile * kRows;
        const uint32_t last = first + kRows < rows ? first + kRows - 1 : rows - 1;
        auto sees = [&](uint32_t query) {
            const int k = a.causal ? (int)query + shift : r.lk - 1;
            return k < r.lk ? k : r.lk - 1;
        };
        const int k_end = sees(last / group) + 1;
        nk = k_end > 0 ? (k_end + kKeys - 1) / kKeys : 0;
        const uint32_t w_first = first + 32 * (uint32_t)wave, w_last = w_first + 31 < last ? w_first + 31 : last;
        any_seen = w_first <= last ? sees(w_last / group) : -1;
        all_seen = sees(w_first / group);
        const uint32_t row = w_first + (uint32_t)col;
        ok = row <= last;
        q = (int)(row / group);
        h = hk * (int)group + (int)(row - (uint32_t)q * group);
        seen = ok ? sees((uint32_t)q) : r.lk - 1;
    }
};

// Forward of 128 query rows. Bound: two products of 4 D flops a visible pair on the matrix instructions, and an exponential
// per pair, a quarter-rate instruction: 256 of about 500 vector cycles beside 512 of the matrix unit for a wave's 32 x 32 pairs
// and 128 features. Two waves per SIMD (210 registers, 64 KB of LDS twice) overlap the two. Measured with 32/8 heads of 128,
// causal: 16,384 tokens 2.09 ms, 1.05 PFLOP/s (a bf16 product of 8,192^3 reaches 1.38), matrix units busy 53% of the cycles; 32 x
// 2,048 tokens 1.31-1.40 ms, 0.79-0.84, busy 42%: a workgroup's start and end, about 7 of its 41 us there, are hidden only
// by the other one on its CU. No LDS bank conflicts.
// SPLIT: the tiles of keys are dealt to gridDim.y workgroups, each leaving its unnormalised output, reference and sum in
// fp32 for attn_join_kernel. One query of 32/8 heads over 8,192 keys: 10 us and the join's 6, of 33 MB at 3.2 TB/s; latency.
template <int DT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 2) attn_fwd_bf16_kernel(AttnArgs a, AttnParts parts) {
    using G = Tile<DT>;
    __shared__ __attribute__((aligned(1024))) char smem[4 * G::kBytes];  // K, K, V, V
    constexpr int kRows = 32 * kWaves;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const Place at_work = place<SPLIT>(a.Hkv);
    const int hk = at_work.hk, part = at_work.part, group = a.Hq / a.Hkv, D = a.D;
    SeqRange r;
    const int tile = slot_range<false>(a, kRows, at_work.slot, group, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kRows, (int64_t)r.lq * group)) return;
    RowTile w;
    w.init(a, r, tile, hk, wave, col);
    const int per = SPLIT ? (w.nk + (int)gridDim.y - 1) / (int)gridDim.y : w.nk;
    const int j0 = SPLIT ? part * per : 0, nk = SPLIT && j0 + per < w.nk ? j0 + per : w.nk;  // tiles j0 .. nk - 1
    const int seen = w.seen, all_seen = w.all_seen, any_seen = w.any_seen, q = w.q, h = w.h;
    const bool ok = w.ok;

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
    Dma<DT> ks, vs;
    ks.init(a.k_stride, wave, lane);
    vs.init(a.v_stride, wave, lane);
    const uint32_t base = lds_addr(smem);
    Addresses<DT> f;
    f.init(lane, base);

    f32x16_t o[DT] = {};
    float m = kNone, l = 0.0f;
    // The scores of 32 keys are formed a step ahead: the exponentials of a step, as much work as its products, go between
    // the matrix instructions that form the next step's scores and the first half of this one's output, and the next step's
    // maximum between those of the second half.
    f32x16_t sa, sb;  // steps of the first and the second half of a tile
    float top;
    constexpr int kS = (2 * DT + 3) / 4;  // groups of four 16-feature steps
    auto load_keys = [&](auto stage, int b, auto g, bf16x8_t (&x)[4]) {
        constexpr uint32_t kTile = decltype(stage)::value * G::kBytes;
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (4 * g + i < 2 * DT) x[i] = f.template straight<kTile>(b, 4 * g + i);
    };
    auto hide = [&](f32x16_t &x, int k0) {  // keys that a row does not see, in the steps where there are any
        if (k0 + 31 > all_seen) {
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (k0 + acc_row(i) + 4 * half > seen) x[i] = kNone;
        }
    };
    // Tile j of the values is 32 rows behind tile j of the keys: what an iteration reads of either is then one tile.
    constexpr std::integral_constant<int, 0> s0{};
    constexpr std::integral_constant<int, 1> s1{};
    auto fetch = [&](int j, uint32_t stage) {
        if (j < nk) ks.load(K, a.k_stride, j * kKeys, r.lk, D, base + stage * G::kBytes, wave);
        if (j <= nk) vs.load(V, a.v_stride, j > 0 ? j * kKeys - 32 : 0, r.lk, D, base + (2 + stage) * G::kBytes, wave, j > 0 ? 0 : 32);
    };
    if (j0 < nk) fetch(j0, 0u);
    landed();
    const int last = any_seen < 0 ? -1 : any_seen / 32 < 2 * nk ? any_seen / 32 : 2 * nk - 1;  // this wave's last step
    if (2 * j0 <= last) {
        sa = f32x16_t{};
        pipelined<kS>([&](auto g, bf16x8_t (&x)[4]) { load_keys(s0, 0, g, x); },
                      [&](auto g, bf16x8_t (&x)[4]) {
#pragma unroll
                          for (int i = 0; i < 4; i++)
                              if (4 * g + i < 2 * DT) sa = mfma(x[i], qv[4 * g + i], sa);
                      });
        hide(sa, j0 * kKeys);
        top = sa[0];
#pragma unroll
        for (int i = 1; i < 16; i++) top = fmaxf(top, sa[i]);
    }
    // Step u of 32 keys with scores sc, its values the rows 32 b .. 32 b + 31 of the staged ones; the next step's scores into
    // sn from the keys 32 b .. (after the last step: whatever the stage holds, which nothing reads).
    auto step = [&](int u, auto stage, auto b, f32x16_t &sc, f32x16_t &sn) {
        constexpr uint32_t kValues = (2 + decltype(stage)::value) * G::kBytes;
        bf16x8_t p[2];
        float sum[2] = {0.0f, 0.0f};
        top = max_halves(top) * c;
        // The reference that the exponents are taken from follows the maximum only where it is passed by more than 8:
        // probabilities stay below 2^8, and most steps need no rescaling.
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
        // part n of `of` of the eight exponentials of half h of the accumulator; packed when they are complete
        auto exponentials = [&](int h, int n, int of) {
#pragma unroll
            for (int e = 8 * n / of; e < 8 * (n + 1) / of; e++) {
                const float x = exp2_raw(__builtin_fmaf(sc[8 * h + e], c, -from));
                sc[8 * h + e] = x;
                sum[e & 1] += x;
            }
            if (n == of - 1) p[h] = pack8(sc, h);
        };
        sn = f32x16_t{};
        pipelined<kS + 2>(
            [&](auto g, bf16x8_t (&x)[4]) {
                if constexpr (g < kS) {
                    load_keys(stage, b, g, x);
                } else {
#pragma unroll
                    for (int t = 0; t < DT; t++) x[t] = f.template transposed<kValues>(2 * b + g - kS, t);
                }
            },
            [&](auto g, bf16x8_t (&x)[4]) {
                if constexpr (g < kS) {
                    static_for<4>([&](auto i) {
                        if constexpr (4 * g + i < 2 * DT) {
                            sn = mfma(x[i], qv[4 * g + i], sn);
                            exponentials(0, 4 * g + i, 2 * DT);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    });
                    if constexpr (g == kS - 1) hide(sn, 32 * u + 32);
                } else if constexpr (g == kS) {
                    static_for<DT>([&](auto t) {
                        o[t] = mfma(x[t], p[0], o[t]);
                        exponentials(1, t, DT);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                } else {
                    top = sn[0];
#pragma unroll
                    for (int t = 0; t < DT; t++) o[t] = mfma(x[t], p[1], o[t]);
#pragma unroll
                    for (int i = 1; i < 16; i++) top = fmaxf(top, sn[i]);
                }
            });
        l += sum[0] + sum[1];
    };
    // iteration j: the second half of tile j - 1 and the first of tile j
    auto iteration = [&](int j, auto stage) {
        fetch(j + 1, decltype(stage)::value ^ 1u);
        if (j > j0 && 2 * j - 1 <= last) step(2 * j - 1, stage, s0, sb, sa);
        if (2 * j <= last) step(2 * j, stage, s1, sa, sb);
        landed();
    };
    if (j0 < nk) {
        for (int j = j0; j <= nk; j += 2) {
            iteration(j, s0);
            if (j < nk) iteration(j + 1, s1);
        }
    }
    l = sum_halves(l);
    if constexpr (SPLIT) {
        const int64_t at = ((int64_t)part * a.Hq + h) * a.Tq + r.q0 + q;
        if (ok && half == 0) {
            parts.m[at] = m;
            parts.l[at] = l;
        }
        if (l == 0.0f) return;  // the join does not look at this part's output
        store_part<DT>(parts.o + at * D, ok, D, half, o);
        return;
    }
    // no key seen: zeros and -inf; a NaN among the scores stays one
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store_row<DT>(static_cast<uint16_t *>(a.O) + ((r.q0 + q) * a.Hq + h) * D, ok, D, half, o, inv);
    if (a.lse && ok && half == 0) a.lse[(int64_t)h * a.Tq + r.q0 + q] = l == 0.0f ? kNone : (m + log2f(l)) * kLn2;
}

// Joins the parts of a split forward, a workgroup per row, two features per lane: each wave adds a run of the parts in
// order, eight loads under way, and the waves' sums are added in order. Latency-bound: two trips to memory, 6 us.
__global__ void __launch_bounds__(kThreads) attn_join_kernel(AttnArgs a, AttnParts parts, int splits) {
    __shared__ float2 lds[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = (int64_t)a.Hq * a.Tq, row = blockIdx.x;
    const int h = (int)(row / a.Tq);
    const int64_t q = row - (int64_t)h * a.Tq;
    if (a.cu_q && (q < a.cu_q[0] || q >= a.cu_q[a.n_seq])) return;  // a row of no sequence
    const float m = lane < splits ? parts.m[lane * rows + row] : kNone, l = lane < splits ? parts.l[lane * rows + row] : 0.0f;
    const float top = wave_max(m);
    const float w = top == kNone ? 1.0f : exp2_raw(m - top);
    const float total = wave_sum(l * w);
    const int per = (splits + kWaves - 1) / kWaves, s1 = (wave + 1) * per < splits ? (wave + 1) * per : splits;
    float x = 0.0f, y = 0.0f;
    for (int s0 = wave * per; s0 < s1; s0 += 8) {
        float2 v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int s = s0 + i < s1 ? s0 + i : s0;
            v[i] = {0.0f, 0.0f};
            // a part that saw no key has left no output
            if (s0 + i < s1 && __shfl(l, s, 64) != 0.0f && 2 * lane < a.D)
                v[i] = *reinterpret_cast<const float2 *>(parts.o + (s * rows + row) * a.D + 2 * lane);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float ws = __shfl(w, s0 + i < s1 ? s0 + i : s0, 64);
            x = __builtin_fmaf(v[i].x, ws, x);
            y = __builtin_fmaf(v[i].y, ws, y);
        }
    }
    lds[wave][lane] = {x, y};
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 1; i < kWaves; i++) {
        x += lds[i][lane].x;
        y += lds[i][lane].y;
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    if (2 * lane < a.D)
        *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(a.O) + (q * a.Hq + h) * a.D + 2 * lane) = pack_bf16(x * inv, y * inv);
    if (a.lse && lane == 0) a.lse[row] = total == 0.0f ? kNone : (top + log2f(total)) * kLn2;
}

// dq of 128 query rows, and delta = rowsum(dO O) for the keys' pass. Both score-shaped products are transposed as in the
// forward, so dS is the B operand of dq^T = k^T dS^T as it stands.
// Bound: four products of 2 D flops a visible pair (dS counts twice) and an exponential. 32 x 2,048 tokens, 32/8 heads of 128,
// causal: 2.13 ms, 1.03 PFLOP/s, matrix units busy 56%. Two waves per SIMD, 256 registers, in which the fragments' addresses are
// formed for each read. With one product of dS (1.72 ms) and delta as O gives it dq was off by 1.5 times its rounding.
// dS goes into its product in two parts, rounded to bf16 and what that left, so that 16 of its bits count. delta from the O that the
// forward rounded is off by that rounding, which all of a row's dS share: their sum over the row's keys, 0 from the exact delta,
// is what it is off by, and is added to it for the keys' pass. dq has it averaged over the row's keys; row tiles of few keys, whose dq
// it would spoil most, are gone through twice, the first time for the sum alone. Error of dq against 64 bits, in that of rounding
// it (rounded dS and this delta in brackets): 64 tokens 1.00 (1.71), 300 1.19 (1.58), 2,048 1.06 (1.54).
// SPLIT: the tiles of keys are dealt to gridDim.y workgroups, whose sums attn_grad_join_kernel adds.
template <int DT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 2) attn_bwd_q_bf16_kernel(AttnArgs a, AttnGradParts parts) {
    using G = Tile<DT>;
    __shared__ __attribute__((aligned(1024))) char smem[4 * G::kBytes];  // K, K, V, V
    constexpr int kRows = 32 * kWaves;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const Place at_work = place<SPLIT>(a.Hkv);
    const int hk = at_work.hk, part = at_work.part, group = a.Hq / a.Hkv, D = a.D;
    SeqRange r;
    const int tile = slot_range<false>(a, kRows, at_work.slot, group, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kRows, (int64_t)r.lq * group)) return;
    RowTile w;
    w.init(a, r, tile, hk, wave, col);

    bf16x8_t qv[2 * DT], gv[2 * DT];
    const int64_t at = ((r.q0 + w.q) * a.Hq + w.h) * D, stat = (int64_t)w.h * a.Tq + r.q0 + w.q;
    load_row<DT>(static_cast<const uint16_t *>(a.O) + at, w.ok, D, half, qv);
    load_row<DT>(static_cast<const uint16_t *>(a.dO) + at, w.ok, D, half, gv);
    float delta = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * DT; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) delta = __builtin_fmaf((float)qv[i][e], (float)gv[i][e], delta);
    delta = sum_halves(delta);
    load_row<DT>(static_cast<const uint16_t *>(a.q) + (r.q0 + w.q) * a.q_stride + (int64_t)w.h * D, w.ok, D, half, qv);
    const float c = a.scale * kLog2e;
    const float lse2 = w.ok ? a.lse[stat] * kLog2e : 0.0f;

    const uint16_t *K = static_cast<const uint16_t *>(a.k) + r.k0 * a.k_stride + (int64_t)hk * D;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + r.k0 * a.v_stride + (int64_t)hk * D;
    Dma<DT> ks, vs;
    ks.init(a.k_stride, wave, lane);
    vs.init(a.v_stride, wave, lane);
    const uint32_t base = lds_addr(smem);
    Frags<DT> f;
    f.init(lane, base);
    f32x16_t dq[DT] = {};
    const bool twice = w.nk <= kFewTiles;  // all of them in the first part then, which has the row's whole sum
    const int per = SPLIT && !twice ? (w.nk + (int)gridDim.y - 1) / (int)gridDim.y : w.nk;
    const int j0 = SPLIT ? part * per : 0, nk = SPLIT && j0 + per < w.nk ? j0 + per : w.nk;  // tiles j0 .. nk - 1
    float rest;  // sum of dS over this lane's half of the row
    auto iteration = [&](int j, auto stage, auto sum_only) {
        constexpr int st = decltype(stage)::value;
        constexpr bool SUM = decltype(sum_only)::value;
        constexpr uint32_t kt = st * G::kBytes, vt = (2 + st) * G::kBytes;
        f.hold();
        const int k0 = j * kKeys;
        const bool more = j + 1 < nk, active = k0 <= w.any_seen;
        if (more) {
            ks.load(K, a.k_stride, k0 + kKeys, r.lk, D, base + (st ^ 1) * G::kBytes, wave);
            vs.load(V, a.v_stride, k0 + kKeys, r.lk, D, base + (2 + (st ^ 1)) * G::kBytes, wave);
        }
        if (active) {
            f32x16_t sc, dp;
            bf16x8_t ds[2], low[2];
            // for each 32 keys: groups of S, then of dP (four steps of 16 features each) with the exponentials between their
            // instructions, then two of dq
            constexpr int kS = (2 * DT + 3) / 4, kAll = 2 * kS + (SUM ? 0 : 2);
            auto dscore = [&](int h) {  // half h of dS = P (dP - delta)
#pragma unroll
                for (int i = 8 * h; i < 8 * h + 8; i++) {
                    sc[i] *= dp[i];
                    rest += sc[i];
                }
                asm volatile("" : "+v"(rest));  // summed here: put off, the sum would hold its terms' registers
                if constexpr (!SUM) ds[h] = pack8(sc, h);
            };
            pipelined<2 * kAll>(
                [&](auto g, bf16x8_t (&x)[4]) {
                    constexpr int b = g / kAll, n = g % kAll;
                    if constexpr (n < 2 * kS) {
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (4 * (n % kS) + i < 2 * DT) x[i] = f.template straight<n < kS ? kt : vt>(b, 4 * (n % kS) + i);
                    } else {
#pragma unroll
                        for (int t = 0; t < DT; t++) x[t] = f.template transposed<kt>(2 * b + n - 2 * kS, t);
                    }
                },
                [&](auto g, bf16x8_t (&x)[4]) {
                    constexpr int b = g / kAll, n = g % kAll;
                    if constexpr (n == 0) sc = f32x16_t{};
                    if constexpr (n < kS) {
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (4 * n + i < 2 * DT) sc = mfma(x[i], qv[4 * n + i], sc);
                        if constexpr (n == kS - 1) {  // dP - delta
#pragma unroll
                            for (int i = 0; i < 16; i++) dp[i] = -delta;
                        }
                    } else if constexpr (n < 2 * kS) {
                        static_for<4>([&](auto i) {
                            constexpr int step = 4 * (n - kS) + i;
                            if constexpr (step < 2 * DT) {
                                dp = mfma(x[i], gv[step], dp);
#pragma unroll
                                for (int e = 16 * step / (2 * DT); e < 16 * (step + 1) / (2 * DT); e++)
                                    sc[e] = exp2_raw(__builtin_fmaf(sc[e], c, -lse2));
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        });
                    } else {
                        constexpr int m = n - 2 * kS;
                        static_for<DT>([&](auto t) {
                            dq[t] = mfma(x[t], ds[m], dq[t]);
                            if constexpr (t == 0) low[m] = pack8_rest(sc, m, ds[m]);
                            __builtin_amdgcn_sched_barrier(0);
                        });
                        static_for<DT>([&](auto t) {
                            dq[t] = mfma(x[t], low[m], dq[t]);
                            if constexpr (m == 0 && t == 0) dscore(1);
                            __builtin_amdgcn_sched_barrier(0);
                        });
                    }
                    if constexpr (n == 2 * kS - 1) {
                        if (k0 + 32 * b + 31 > w.all_seen) {
#pragma unroll
                            for (int i = 0; i < 16; i++)
                                if (k0 + 32 * b + acc_row(i) + 4 * half > w.seen) sc[i] = dp[i] = 0.0f;
                        }
                        dscore(0);
                        if constexpr (SUM) dscore(1);
                    }
                });
        }
        landed();
    };
    auto through = [&](auto sum_only) {
        rest = 0.0f;
        if (j0 < nk) {
            ks.load(K, a.k_stride, j0 * kKeys, r.lk, D, base, wave);
            vs.load(V, a.v_stride, j0 * kKeys, r.lk, D, base + 2 * G::kBytes, wave);
        }
        landed();
        for (int j = j0; j < nk; j += 2) {
            iteration(j, std::integral_constant<int, 0>{}, sum_only);
            if (j + 1 < nk) iteration(j + 1, std::integral_constant<int, 1>{}, sum_only);
        }
        rest = sum_halves(rest);
        if (!SPLIT || twice) delta += rest;
    };
    if (twice) through(std::true_type{});
    through(std::false_type{});
    if (w.ok && half == 0) {
        if (part == 0) a.delta[stat] = delta;
        if (SPLIT) parts.rest[(int64_t)part * a.Hq * a.Tq + stat] = twice ? 0.0f : rest;
    }
    if constexpr (SPLIT) {
        store_part<DT>(parts.dq + (((int64_t)part * a.Tq + r.q0 + w.q) * a.Hq + w.h) * D, w.ok, D, half, dq);
        return;
    }
    store_row<DT>(static_cast<uint16_t *>(a.dq) + (r.q0 + w.q) * a.dq_stride + (int64_t)w.h * D, w.ok, D, half, dq, a.scale);
}

// dk and dv of 128 keys of one key-value head, 32 per wave, over the queries of every head that shares it: tiles of queries
// from the last to the first that sees a key, the heads of each in turn, so that the workgroups of a sequence, which end at
// different queries, run through the same tiles at the same time (from the first on and head by head took as long where L2
// holds a sequence's: 4.56 ms both ways at 32 x 2,048 tokens).
// Here a lane's column is a key and the queries run down the accumulators (S = q k^T as it is written): P and dS are the
// B operands of dv^T = dO^T P and dk^T = q^T dS. Queries and their gradients go through LDS in tiles with their lse and delta,
// from which the accumulators start; a query that does not exist, or sees nothing, has probability 0.
// Bound: four products of 2 D flops a visible pair and an exponential. 32 x 2,048 tokens, 32/8 heads of 128, causal: 2.1 ms,
// 1.05 PFLOP/s, matrix units busy 55%, no bank conflicts. P and dS are rounded to bf16 as in the other kernels.
// Two waves per SIMD, whose 256 registers hold the sums (64 per gradient and 128 features) and k: from 65 features on, v is read
// from LDS each time and the tiles have 32 queries rather than 64.
// SPLIT: the tiles of queries, all heads together, are dealt to gridDim.y workgroups, whose sums attn_grad_join_kernel adds.
template <int DT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 2) attn_bwd_kv_bf16_kernel(AttnArgs a, AttnGradParts parts) {
    constexpr bool kWide = DT > 2;
    constexpr int kQ = kWide ? 32 : 64;  // queries of a tile
    using G = Tile<DT, kQ>;
    using GV = Tile<DT>;  // half of the workgroup's 128 keys
    constexpr int kRows = 32 * kWaves;
    __shared__ __attribute__((aligned(1024))) char smem[4 * G::kBytes + (kWide ? 2 * GV::kBytes : 0)];  // q, q, dO, dO, v
    __shared__ __attribute__((aligned(16))) float stats[2][2][kQ];  // [stage][-lse / scale, -delta]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const Place at_work = place<SPLIT>(a.Hkv);
    const int hk = at_work.hk, part = at_work.part, group = a.Hq / a.Hkv, D = a.D;
    SeqRange r;
    const int tile = slot_range<true>(a, kRows, at_work.slot, 1, r);
    check_ends<kThreads>(a);
    if (!tile_in(tile, kRows, r.lk)) return;
    const int shift = r.lk - r.lq, w_first = tile * kRows + 32 * wave, k = w_first + col;
    const bool ok = k < r.lk;
    // the first query that sees a key: of the workgroup's tile (where the loop starts), of the wave's first and last
    // key, of this lane's
    auto seen_from = [&](int key) { return a.causal && key > shift ? key - shift : 0; };
    const int q_first = seen_from(tile * kRows) / kQ * kQ;
    const int any_from = seen_from(w_first), all_from = seen_from(w_first + 31);
    const int per_head = r.lq > q_first ? (r.lq - q_first + kQ - 1) / kQ : 0;
    const int all_items = per_head * group;
    const int per = SPLIT ? (all_items + (int)gridDim.y - 1) / (int)gridDim.y : all_items, i0 = SPLIT ? part * per : 0;
    const int items = i0 + per < all_items ? per : all_items - i0;  // this workgroup's, none or fewer possibly
    const int head0 = i0 % group, q_start = q_first + (per_head - 1 - i0 / group) * kQ;

    // The accumulators of S and dP start from -lse / scale and -delta: exp2(c S') is the probability and P dP' is dS. A
    // scale too small to divide by does as well as the smallest that is not.
    const float scale = __builtin_fabsf(a.scale) < 1e-20f ? 1e-20f : a.scale, c = scale * kLog2e;
    const float nothing = __builtin_copysignf(3e38f, -scale);  // of a query that does not exist or sees nothing: c times it is far below -126
    const int64_t g_stride = (int64_t)a.Hq * D;
    const uint16_t *Q = static_cast<const uint16_t *>(a.q) + r.q0 * a.q_stride + (int64_t)hk * group * D;
    const uint16_t *dO = static_cast<const uint16_t *>(a.dO) + r.q0 * g_stride + (int64_t)hk * group * D;
    const uint16_t *V = static_cast<const uint16_t *>(a.v) + r.k0 * a.v_stride + (int64_t)hk * D;
    const int64_t stat = (int64_t)hk * group * a.Tq + r.q0;
    Dma<DT, kQ> qs, gs;
    qs.init(a.q_stride, wave, lane);
    gs.init(g_stride, wave, lane);
    const uint32_t base = lds_addr(smem);
    constexpr uint32_t kV = 4 * G::kBytes;
    Frags<DT> f;
    f.init(lane, base);
    // lse and delta of a tile's queries: loaded by every wave, without a branch (the values of two paths would be joined, and
    // so waited for, at once), looked at and written by the first when the tile's work is done
    constexpr int kStats = 2 * kQ / 64;
    float sv[kStats];
    auto load_stats = [&](int head, int q0) {
#pragma unroll
        for (int i = 0; i < kStats; i++) {
            const int v = lane + 64 * i, row = q0 + v % kQ;
            const float *from_stat = (v < kQ ? a.lse : a.delta) + stat + (int64_t)head * a.Tq;
            sv[i] = from_stat[row < r.lq ? row : r.lq - 1];
        }
    };
    auto store_stats = [&](int stage, int q0) {
        if (wave != 0) return;
#pragma unroll
        for (int i = 0; i < kStats; i++) {
            const int v = lane + 64 * i;
            const bool in = q0 + v % kQ < r.lq;
            (&stats[stage][0][0])[v] = v >= kQ ? (in ? -sv[i] : 0.0f) : in && sv[i] != kNone ? -sv[i] / scale : nothing;
        }
    };
    bf16x8_t kv[2 * DT], vv[kWide ? 1 : 2 * DT];
    load_row<DT>(static_cast<const uint16_t *>(a.k) + (r.k0 + k) * a.k_stride + (int64_t)hk * D, ok, D, half, kv);
    if constexpr (!kWide) load_row<DT>(V + k * a.v_stride, ok, D, half, vv);
    f32x16_t dk[DT] = {}, dv[DT] = {};
    if (items > 0) {
        load_stats(head0, q_start);
        qs.load(Q + (int64_t)head0 * D, a.q_stride, q_start, r.lq, D, base, wave);
        gs.load(dO + (int64_t)head0 * D, g_stride, q_start, r.lq, D, base + 2 * G::kBytes, wave);
        if constexpr (kWide) {
            Dma<DT> vs;
            vs.init(a.v_stride, wave, lane);
            vs.load(V, a.v_stride, tile * kRows, r.lk, D, base + kV, wave);
            vs.load(V, a.v_stride, tile * kRows + kKeys, r.lk, D, base + kV + GV::kBytes, wave);
        }
        store_stats(0, q_start);
    }
    landed();
    int head = head0, q0 = q_start;
    auto iteration = [&](int it, auto stage) {
        constexpr int st = decltype(stage)::value;
        constexpr uint32_t qt = st * G::kBytes, gt = (2 + st) * G::kBytes;
        const bool more = it + 1 < items, active = q0 + kQ > any_from;
        int next_head = head + 1, next_q0 = q0;
        if (next_head == group) {
            next_head = 0;
            next_q0 -= kQ;
        }
        load_stats(more ? next_head : head, more ? next_q0 : q0);
        if (more) {
            qs.load(Q + (int64_t)next_head * D, a.q_stride, next_q0, r.lq, D, base + (st ^ 1) * G::kBytes, wave);
            gs.load(dO + (int64_t)next_head * D, g_stride, next_q0, r.lq, D, base + (2 + (st ^ 1)) * G::kBytes, wave);
        }
        if (active) {
            f32x16_t sc, dp;
            bf16x8_t p[2], ds[2];
            // for each 32 queries: groups of S (two steps of 16 features), of dP (one step where v comes from LDS too),
            // then dv and dk of 16 queries each (two blocks of 32 features at a time)
            constexpr int kP = kWide ? 2 * DT : DT, kT = (DT + 1) / 2, kAll = DT + kP + 4 * kT;
            pipelined<kQ / 32 * kAll, 2, 3>(
                [&](auto g, bf16x8_t (&x)[2]) {
                    constexpr int b = g / kAll, n = g % kAll;
                    if constexpr (n == 0) f.hold();
                    if constexpr (n < DT) {
#pragma unroll
                        for (int i = 0; i < 2; i++) x[i] = f.template straight<qt>(b, 2 * n + i);
                    } else if constexpr (n < DT + kP) {
                        constexpr int m = n - DT;
                        if constexpr (kWide) {
                            x[0] = f.template straight<gt>(b, m);
                            x[1] = f.template straight<kV>(wave, m);
                        } else {
#pragma unroll
                            for (int i = 0; i < 2; i++) x[i] = f.template straight<gt>(b, 2 * m + i);
                        }
                    } else {
                        constexpr int m = (n - DT - kP) / kT, t0 = 2 * ((n - DT - kP) % kT);
#pragma unroll
                        for (int i = 0; i < 2; i++)
                            if (t0 + i < DT) x[i] = f.template transposed<m >= 2 ? qt : gt>(2 * b + (m & 1), t0 + i);
                    }
                },
                [&](auto g, bf16x8_t (&x)[2]) {
                    constexpr int b = g / kAll, n = g % kAll;
                    // an accumulator's start from its rows' statistics
                    auto start = [&](f32x16_t &acc, int which) {
                        const int half = lane_again() >> 5;
#pragma unroll
                        for (int q = 0; q < 4; q++) {
                            const f32x4_t v = *reinterpret_cast<const f32x4_t *>(&stats[st][which][32 * b + 8 * q + 4 * half]);
#pragma unroll
                            for (int e = 0; e < 4; e++) acc[4 * q + e] = v[e];
                        }
                    };
                    if constexpr (n == 0) start(sc, 0);
                    if constexpr (n == DT - 1) start(dp, 1);
                    if constexpr (n < DT) {
#pragma unroll
                        for (int i = 0; i < 2; i++) sc = mfma(x[i], kv[2 * n + i], sc);
                    } else if constexpr (n < DT + kP) {
                        // the probabilities, 16 / kP after each group
                        constexpr int m = n - DT;
                        if constexpr (kWide) {
                            dp = mfma(x[0], x[1], dp);
                        } else {
#pragma unroll
                            for (int i = 0; i < 2; i++) dp = mfma(x[i], vv[2 * m + i], dp);
                        }
#pragma unroll
                        for (int e = 16 * m / kP; e < 16 * (m + 1) / kP; e++) sc[e] = exp2_raw(sc[e] * c);
                    } else {
                        // dS between the instructions of dv, 8 at a time
                        constexpr int m = (n - DT - kP) / kT, t0 = 2 * ((n - DT - kP) % kT);
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            if (t0 + i >= DT) continue;
                            if constexpr (m >= 2) dk[t0 + i] = mfma(x[i], ds[m & 1], dk[t0 + i]);
                            else dv[t0 + i] = mfma(x[i], p[m & 1], dv[t0 + i]);
                        }
                        if constexpr (m < 2 && t0 == 0) {
#pragma unroll
                            for (int e = 8 * m; e < 8 * m + 8; e++) dp[e] *= sc[e];
                            ds[m & 1] = pack8(dp, m & 1);
                        }
                    }
                    if constexpr (n == DT + kP - 1) {
                        if (q0 + 32 * b < all_from) {
                            const int l = lane_again(), from = seen_from(w_first + (l & 31)), half = l >> 5;
#pragma unroll
                            for (int i = 0; i < 16; i++)
                                if (q0 + 32 * b + acc_row(i) + 4 * half < from) sc[i] = dp[i] = 0.0f;
                        }
#pragma unroll
                        for (int i = 0; i < 2; i++) p[i] = pack8(sc, i);
                    }
                });
        }
        if (more) store_stats(st ^ 1, next_q0);
        head = next_head;
        q0 = next_q0;
        landed();
    };
    for (int it = 0; it < items; it += 2) {
        iteration(it, std::integral_constant<int, 0>{});
        if (it + 1 < items) iteration(it + 1, std::integral_constant<int, 1>{});
    }
    if constexpr (SPLIT) {
        const int64_t at = (((int64_t)part * a.Tk + r.k0 + k) * a.Hkv + hk) * D;
        store_part<DT>(parts.dk + at, ok, D, half, dk);
        store_part<DT>(parts.dv + at, ok, D, half, dv);
        return;
    }
    store_row<DT>(static_cast<uint16_t *>(a.dk) + (r.k0 + k) * a.dk_stride + (int64_t)hk * D, ok, D, half, dk, a.scale);
    store_row<DT>(static_cast<uint16_t *>(a.dv) + (r.k0 + k) * a.dv_stride + (int64_t)hk * D, ok, D, half, dv, 1.0f);
}

// Adds the parts of a gradient [tokens][heads][D] in order, four features per thread, and rounds the sum times `scale`;
// dq's (`rest` given) also the parts of the rows' sums of dS, to delta.
// HBM-bound: three parts of 8,192 tokens with 8 heads of 128, 117 MB, 21 us (5.6 TB/s).
// cu: ends of the sequences, whose tokens alone have parts
__global__ void __launch_bounds__(256) attn_grad_join_kernel(const float *part, int splits, int64_t tokens, int heads, int D,
                                                             const int32_t *cu, int n_seq, uint16_t *out, int64_t stride,
                                                             float scale, const float *rest, float *delta) {
    const int64_t row = (int64_t)heads * D, all = tokens * row;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= all) return;
    const int64_t token = at / row;
    if (cu && (token < cu[0] || token >= cu[n_seq])) return;
    if (rest && at % D == 0) {
        const int64_t stat = (at - token * row) / D * tokens + token;
        float d = delta[stat];
        for (int s = 0; s < splits; s++) d += rest[s * heads * tokens + stat];
        delta[stat] = d;
    }
    f32x4_t sum = {};
    for (int s0 = 0; s0 < splits; s0 += 4) {
        f32x4_t v[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            v[i] = s0 + i < splits ? *reinterpret_cast<const f32x4_t *>(part + (s0 + i) * all + at) : f32x4_t{};
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += v[i][e];
    }
    *reinterpret_cast<uint2 *>(out + token * stride + (at - token * row)) =
        make_uint2(pack_bf16(sum[0] * scale, sum[1] * scale), pack_bf16(sum[2] * scale, sum[3] * scale));
}

template <typename F>
void pick_dt(int D, F &&f) {
    if (D <= 64) f(std::integral_constant<int, 2>{});
    else if (D <= 96) f(std::integral_constant<int, 3>{});
    else f(std::integral_constant<int, 4>{});
}

}  // namespace

// Parts that a forward's keys are split into: where the row tiles leave workgroups idle (two per CU), up to as many as fill
// them with 128 keys each at least (by the mean length; lengths are not known on the host) and a wave's lanes. Of these the
// number that gains most, none where none does: a tile of keys that a workgroup does not go through saves 1.15 us, and the parts
// cost 5 us and per row 1.2 ns and 0.15 for each of them (written, read and joined, a workgroup per row). In one part and in
// the parts taken here, us, heads of 128: one query of 32/8 heads on 8,192 keys 158 and 17 (64 parts), on 300 keys 15 and (in
// two) 17; causal prompts: 2,048 with 2/1 heads 42 and 26, 4,096 with 2/1 78 and 39, but 512 with 32/8 16 and (in three) 42, 1,024
// with 8/8 25 and (in seven) 33, four of 507 with 4/4 16 and (in three) 26. Lengths that differ widely lose by the mean: 2,000,
// 10, 10, 10 with 4/4 heads 42 and (in three) 35.
int attn_splits_bf16(int64_t Tq, int64_t Tk, int Hq, int Hkv, int64_t n_seq) {
    if (n_seq < 1) return 1;
    const int64_t wgs = (Tq * (Hq / Hkv) / (32 * kWaves) + n_seq) * Hkv, rows = Tq * Hq;
    const int64_t keys = Tk / n_seq, tiles = (keys + kKeys - 1) / kKeys;
    const int64_t most = std::min({int64_t(64), keys / (2 * kKeys), 2 * kMfmaConcurrentWgs / wgs});
    int64_t best = 1, gain = 0;  // ns
    for (int64_t s = 2; s <= most; s++) {
        const int64_t g = (tiles - (tiles + s - 1) / s) * 1150 - 5000 - rows * (24 + 3 * s) / 20;
        if (g > gain) gain = g, best = s;
    }
    return (int)best;
}

hipError_t launch_attn_fwd_bf16(const AttnArgs &a, void *ws, hipStream_t st) {
    const int64_t slots = a.Tq * (a.Hq / a.Hkv) / (32 * kWaves) + a.n_seq;
    const int splits = attn_splits_bf16(a.Tq, a.Tk, a.Hq, a.Hkv, a.n_seq);
    const int64_t rows = a.Tq * a.Hq;
    AttnParts p{};
    p.m = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader);
    p.l = p.m + splits * rows;
    p.o = reinterpret_cast<float *>(static_cast<char *>(ws) + kWsHeader + attn_part_stats(splits, rows));
    const dim3 grid((unsigned)(slots * a.Hkv), (unsigned)splits);
    pick_dt(a.D, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (splits > 1) attn_fwd_bf16_kernel<DT, true><<<grid, kThreads, 0, st>>>(a, p);
        else attn_fwd_bf16_kernel<DT, false><<<grid, kThreads, 0, st>>>(a, p);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    attn_join_kernel<<<(unsigned)rows, kThreads, 0, st>>>(a, p, splits);
    return hipGetLastError();
}

// Parts of a backward's sums. Where workgroups are few, one's run through all queries (keys) of a long sequence is the whole
// call's time: they are split until two per CU are busy, with 4 tiles each at least by the mean length. The keys' pass, whose
// runs over a causal sequence are from one to all of its queries long, is split on until there are four times as many with 64
// tiles each, so that long and short ones even out (backward of four sequences of 2,048 with 64/8 heads 1.10 ms, 1.16 without
// these parts and 1.18 with twice as many; of one of 8,192 3.76, 4.61 and 3.82). A part
// costs 64 KB of fp32 sums per 128 rows and gradient, written and read again: splitting both passes up to 2,048 workgroups
// with 8 tiles each made two sequences of 2,500 with 16/8 heads take 355 us in place of 246.
//
// The keys' parts also have to save more than their two joins cost: 8 us, and per key and head 0.2 ns and 0.25 for each part, at
// 1 us for a tile of 32 queries that a workgroup does not go through. In one part and in those, us, heads of 128: 64 queries of
// 32/8 heads on 2,048 keys 41 and (two) 54, 512 of 4/4 on 4,096 57 and (three) 66, four of 507 with 4/4 45 and (three) 52; but
// 256 with 32/8 60 and (eight) 47, 1,024 with 8/8 73 and (seven) 65, 4,096 with 2/1 313 and (fifteen) 92. Lengths that differ
// widely lose by the mean here too: 2,000, 10, 10, 10 with 4/4 heads 131 and (three) 110.
AttnBwdPlan plan_attn_bwd_bf16(int64_t Tq, int64_t Tk, int Hq, int Hkv, int64_t n_seq) {
    const int64_t kRows = 32 * kWaves, kBusy = 2 * kMfmaConcurrentWgs, kMost = 16;
    if (n_seq < 1) return {1, 1};
    const int64_t group = Hq / Hkv, q_wgs = (Tq * group / kRows + n_seq) * Hkv, k_wgs = (Tk / kRows + n_seq) * Hkv;
    const int64_t q_tiles = Tk / n_seq / kKeys, k_tiles = Tq / n_seq * group / 32;
    const int64_t q = std::min(kBusy / q_wgs, q_tiles / 4);
    const int64_t k = std::max(std::min(kBusy / k_wgs, k_tiles / 4), std::min(4 * kBusy / k_wgs, k_tiles / 64));
    auto clip = [&](int64_t s) { return (int)std::max<int64_t>(1, std::min(kMost, s)); };
    const int64_t parts = clip(k), saved = k_tiles - (k_tiles + parts - 1) / parts;
    const bool pays = saved * 1000 > 8000 + Tk * Hkv * (4 + 5 * parts) / 20;  // ns
    return {clip(q), pays ? (int)parts : 1};
}

hipError_t launch_attn_bwd_bf16(const AttnArgs &a, float *parts, hipStream_t st) {
    constexpr int kRows = 32 * kWaves;
    const int64_t q_slots = a.Tq * (a.Hq / a.Hkv) / kRows + a.n_seq, k_slots = a.Tk / kRows + a.n_seq;
    const AttnBwdPlan p = plan_attn_bwd_bf16(a.Tq, a.Tk, a.Hq, a.Hkv, a.n_seq);
    const int64_t dq_size = a.Tq * a.Hq * a.D, dk_size = a.Tk * a.Hkv * a.D;
    AttnGradParts g{};
    g.rest = parts;
    g.dq = parts + attn_rest_floats(p.q_splits, a.Tq * a.Hq);
    g.dk = g.dq + (p.q_splits > 1 ? p.q_splits * dq_size : 0);
    g.dv = g.dk + p.k_splits * dk_size;
    const dim3 q_grid((unsigned)(q_slots * a.Hkv), (unsigned)p.q_splits), k_grid((unsigned)(k_slots * a.Hkv), (unsigned)p.k_splits);
    auto add = [&](const float *part, int splits, int64_t tokens, int heads, const int32_t *cu, void *out, int64_t stride, float scale,
                   const float *rest) {
        const int64_t threads = tokens * heads * a.D / 4;
        attn_grad_join_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(part, splits, tokens, heads, a.D, cu, a.n_seq,
                                                                                static_cast<uint16_t *>(out), stride, scale, rest, a.delta);
    };
    pick_dt(a.D, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (a.Tq > 0 && p.q_splits > 1) attn_bwd_q_bf16_kernel<DT, true><<<q_grid, kThreads, 0, st>>>(a, g);
        else if (a.Tq > 0) attn_bwd_q_bf16_kernel<DT, false><<<q_grid, kThreads, 0, st>>>(a, g);
        if (a.Tq > 0 && p.q_splits > 1) add(g.dq, p.q_splits, a.Tq, a.Hq, a.cu_q, a.dq, a.dq_stride, a.scale, g.rest);  // and delta
        if (a.Tk > 0 && p.k_splits > 1) attn_bwd_kv_bf16_kernel<DT, true><<<k_grid, kThreads, 0, st>>>(a, g);
        else if (a.Tk > 0) attn_bwd_kv_bf16_kernel<DT, false><<<k_grid, kThreads, 0, st>>>(a, g);
    });
    if (a.Tk > 0 && p.k_splits > 1) {
        add(g.dk, p.k_splits, a.Tk, a.Hkv, a.cu_k, a.dk, a.dk_stride, a.scale, nullptr);
        add(g.dv, p.k_splits, a.Tk, a.Hkv, a.cu_k, a.dv, a.dv_stride, 1.0f, nullptr);
    }
    return hipGetLastError();
}

}  // namespace focus
