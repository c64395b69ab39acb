// Log probabilities of given tokens, entropy and the largest alternatives of rows of logits, and the gradient of both
// with respect to the logits.
//
//   lse = log sum_i exp z_i,  logp = z_target - lse,  entropy = -sum_i p_i log p_i,  p_i = exp(z_i - lse)
//   dz_i = g ([i = target] - p_i) - h p_i (log p_i + entropy),  g = d/dlogp, h = d/dentropy
//
// HBM-bound, one pass over the logits each way. Every thread keeps its own running maximum m, s = sum 2^d and
// w = sum d 2^d with d = (z - m) log2 e, joined over the workgroup at the end of the row: entropy = ln s - ln 2 w / s,
// sums of terms of one sign, in place of the difference of lse and sum p z. The difference z - m is taken first, so that
// the largest logit's d is exactly 0 and logits near the type's lowest value stay finite.
//
// The alternatives: logits are ordered by (value, lower index first), as 64-bit keys. Of the threads' largest logits,
// which the pass has anyway, follows a value that at least `top` logits of the row reach; the few threads that have such
// logits have theirs read a second time (from the caches), by all threads, and those that reach it are ranked in LDS. The LDS
// additions count and hand out places; no result depends on their order, keys being distinct.
//
// Measured, bf16: 8,192 rows of 151,936 with 5 alternatives, 2.49 GB, 436 us (5.7 TB/s); 4,096 rows of 32,000 forward 69 us
// (3.8 TB/s), gradient 90 us (5.8 TB/s both ways); one row of 151,936 with 20 alternatives 10 us and the join's 8, latency. Short
// rows are bound by what a row costs beside its logits, the join of 512 threads' sums: 16,384 rows of 1,000 114 us, of 16,384 146.
// Vectors of 8 logits, four per thread and step, are enough loads under way: fetching a step ahead (94 registers in place of 60)
// made 8,192 rows take 490 us.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kThreads = 512;
constexpr int kWavesL = kThreads / 64;
constexpr int kVecs = 4;                        // vectors of 8 logits per thread and step
constexpr int kStep = kThreads * kVecs * 8;     // logits per step
constexpr int kRoom = 1024;                     // collected keys
constexpr int kMaxSplits = 64;
constexpr int kMaxParts = 512;                  // parts of a split launch, at most: two workgroups per CU
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;

// the order of the values as unsigned integers (equal zeros equal); every number, -inf too, is above 0
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
    return ((uint64_t)order_of(v) << 32) | (0xFFFFFFFFu - index);
}
struct Stat {
    float m, s, w;  // the largest logit; s, w relative to it (m = -inf: nothing seen)
};
__device__ __forceinline__ Stat merge(const Stat &a, const Stat &b) {
    const float top = fmaxf(a.m, b.m), base = top == -__builtin_inff() ? 0.0f : top;
    // a part that has seen nothing has s = w = 0, as one far below the other will have: its shift must stay finite
    const float da = fmaxf((a.m - base) * kLog2e, -200.0f), db = fmaxf((b.m - base) * kLog2e, -200.0f);
    const float fa = exp2_raw(da), fb = exp2_raw(db);
    Stat r;
    r.m = top;
    r.s = a.s * fa + b.s * fb;
    r.w = fa * __builtin_fmaf(a.s, da, a.w) + fb * __builtin_fmaf(b.s, db, b.w);
    return r;
}
__device__ __forceinline__ Stat wave_merge(Stat v) {
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
        Stat o;
        o.m = __shfl_xor(v.m, x, 64);
        o.s = __shfl_xor(v.s, x, 64);
        o.w = __shfl_xor(v.w, x, 64);
        v = (threadIdx.x & x) ? merge(o, v) : merge(v, o);  // the same order in both lanes
    }
    return v;
}

struct TopLds {
    uint64_t list[kRoom];
    uint64_t cut[kMaxTop];
    uint32_t group[64];
    int hist[256];
    int flagged[kThreads];
    int n_flagged, pos;
};

// Ranks the `top` largest keys of a workgroup's elements, called by all threads: on return l.list holds them, largest
// first; returns their number (fewer than `top` where there are fewer elements). Thread t's elements are the vectors of eight
// t, t + kThreads, .. (nvec of them); load(i, k) gives the keys of vector i (0 for elements that do not exist), `best` is the
// largest order_of among the thread's own (0: none).
template <typename Load>
__device__ __forceinline__ int select_top(TopLds &l, int top, uint32_t best, int nvec, Load &&load) {
    // tau: the top-th of the largest values of 64 groups of threads, which `top` elements reach at least
    uint32_t group = best;
#pragma unroll
    for (int x = 1; x < kThreads / 64; x <<= 1) {
        const uint32_t o = __shfl_xor(group, x, 64);
        group = o > group ? o : group;
    }
    if (threadIdx.x % (kThreads / 64) == 0) l.group[threadIdx.x / (kThreads / 64)] = group;
    if (threadIdx.x == 0) l.n_flagged = l.pos = 0;
    __syncthreads();
    const int me = threadIdx.x & 63;
    const uint32_t g = l.group[me];
    int rank = 0;
#pragma unroll 16
    for (int j = 0; j < 64; j++) {
        const uint32_t o = __builtin_amdgcn_readlane(g, j);
        rank += o > g || (o == g && j < me) ? 1 : 0;
    }
    const uint32_t kth = __shfl(g, __builtin_ctzll(__ballot(rank == top - 1)), 64);
    uint64_t tau = (uint64_t)kth << 32;
    // the few threads that have any, whose vectors are then shared out among all
    if (best != 0 && best >= kth) l.flagged[atomicAdd(&l.n_flagged, 1)] = threadIdx.x;
    __syncthreads();
    const int flagged = l.n_flagged, items = flagged * nvec;
    auto scan = [&](auto &&f) {
        for (int i = threadIdx.x; i < items; i += kThreads) {
            uint64_t k[8];
            const int j = i / flagged;
            load(j * kThreads + l.flagged[i - j * flagged], k);
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (k[e] != 0) f(k[e]);
        }
    };
    auto collect = [&]() {
        scan([&](uint64_t k) {
            if (k >= tau) {
                const int at = atomicAdd(&l.pos, 1);
                if (at < kRoom) l.list[at] = k;
            }
        });
        __syncthreads();
        const int r = l.pos;
        __syncthreads();  // before it is cleared
        return r;
    };
    int n = collect();
    if (n > kRoom) {
        // Equal values, or few threads that hold most of the largest: tau rises byte by byte to what `top` keys reach, until
        // the list holds those that do. Keys are distinct, so the last byte ends it.
        uint64_t prefix = 0;
        int need = top, shift = 56;  // the need-th largest of the keys that begin with prefix is wanted
        for (;; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += kThreads) l.hist[i] = 0;
            if (threadIdx.x == 0) l.pos = 0;
            __syncthreads();
            scan([&](uint64_t k) {
                if (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&l.hist[(int)(k >> shift) & 255], 1);
            });
            __syncthreads();
            int bin = 255, above = 0;
            for (; bin > 0 && above + l.hist[bin] < need; bin--) above += l.hist[bin];
            const int reach = top - need + above + l.hist[bin];
            prefix |= (uint64_t)bin << shift;
            need -= above;
            __syncthreads();  // before the histogram is cleared again
            if (reach <= kRoom || shift == 0) break;
        }
        tau = prefix;
        n = collect();
        n = n < kRoom ? n : kRoom;
    }
    // ranks among what is left
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t k = l.list[i];
        int r = 0;
#pragma unroll 4
        for (int j = 0; j < n; j++) r += l.list[j] > k ? 1 : 0;
        if (r < top) l.cut[r] = k;
    }
    __syncthreads();
    const int kept = n < top ? n : top;
    if ((int)threadIdx.x < kept) l.list[threadIdx.x] = l.cut[threadIdx.x];
    __syncthreads();
    return kept;
}

// Eight consecutive logits as they lie in memory, missing ones -inf
template <typename T>
struct Logits8;
template <>
struct Logits8<uint16_t> {
    u32x4_any_t w;
    __device__ __forceinline__ void load(const uint16_t *p, int64_t left) {
        if (left >= 8) {
            w = *reinterpret_cast<const u32x4_any_t *>(p);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                w[e] = (2 * e < left ? p[2 * e] : 0xFF80u) | (uint32_t)(2 * e + 1 < left ? p[2 * e + 1] : 0xFF80u) << 16;
        }
    }
    __device__ __forceinline__ float operator[](int e) const {
        return __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
};
template <>
struct Logits8<float> {
    f32x4_any_t w[2];
    __device__ __forceinline__ void load(const float *p, int64_t left) {
        if (left >= 8) {
            w[0] = reinterpret_cast<const f32x4_any_t *>(p)[0];
            w[1] = reinterpret_cast<const f32x4_any_t *>(p)[1];
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) w[e >> 2][e & 3] = e < left ? p[e] : -__builtin_inff();
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return w[e >> 2][e & 3]; }
};

struct LogprobArgs {
    const void *Z;
    const int64_t *target;
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_index;
    uint32_t *flag;
    Stat *part;      // [T][splits]
    uint64_t *keys;  // [T][splits][top]
    int64_t T, V, per;  // logits per part
    int top, splits;
};

// One row's results from its statistics and the ranked list (by the threads of a workgroup, all in fp32)
__device__ __forceinline__ void finish_row(const LogprobArgs &a, int64_t row, const Stat &t, const uint64_t *list, int n,
                                           float target_logit, int64_t target) {
    const bool none = t.m == -__builtin_inff();  // every logit is -inf
    // A log probability is the logit's distance from the largest less log s: taken from lse it would have lse's digits only,
    // and a row of the type's lowest value probability 1 for every token.
    const float log_s = kLn2 * log2f(t.s), lse = none ? -__builtin_inff() : t.m + log_s;
    if (threadIdx.x == 0) {
        a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = none ? 0.0f : kLn2 * (log2f(t.s) - t.w / t.s);
        if (a.logp) a.logp[row] = target < 0 || target >= a.V ? 0.0f : none ? -__builtin_inff() : target_logit - t.m - log_s;
        if (t.s != t.s || target >= a.V) *a.flag = 1u;  // a NaN or +inf among the logits, or no such token
    }
    for (int i = threadIdx.x; i < a.top; i += kThreads) {
        const bool in = i < n;
        const uint64_t k = in ? list[i] : 0;
        const float v = value_of((uint32_t)(k >> 32));
        a.top_index[row * a.top + i] = in ? (int32_t)(0xFFFFFFFFu - (uint32_t)k) : -1;
        a.top_logp[row * a.top + i] = !in || none ? -__builtin_inff() : v - t.m - log_s;
    }
}

// A workgroup takes a row, or one of its parts where rows are few (a whole row would leave CUs idle).
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(LogprobArgs a) {
    __shared__ TopLds lds_top;
    __shared__ Stat lds_stat[kWavesL];
    const int64_t row = blockIdx.x / (unsigned)a.splits;
    const int split = (int)(blockIdx.x % (unsigned)a.splits);
    const int64_t v0 = split * a.per, v1 = v0 + a.per < a.V ? v0 + a.per : a.V;
    const T *z = static_cast<const T *>(a.Z) + row * a.V;
    const int64_t target = a.target && a.splits == 1 ? a.target[row] : -1;  // under way while the row streams
    const float zt = target >= 0 && target < a.V ? load_one(z + target) : 0.0f;
    Stat t = {-__builtin_inff(), 0.0f, 0.0f};
    for (int64_t c0 = v0; c0 < v1; c0 += kStep) {
        Logits8<T> v[kVecs];
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < kVecs; j++) {
            const int64_t c = c0 + (j * kThreads + (int)threadIdx.x) * 8;
            v[j].load(z + c, v1 - c);
        }
#pragma unroll
        for (int j = 0; j < kVecs; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) top = fmaxf(top, v[j][e]);
        const float m = fmaxf(t.m, top), base = m == -__builtin_inff() ? 0.0f : m;
        float s = 0.0f, w = 0.0f;
        auto add = [&](float d) {
            const float x = exp2_raw(d);
            s += x;
            w = __builtin_fmaf(x, d, w);
        };
        if (c0 + kStep <= v1) {
#pragma unroll
            for (int j = 0; j < kVecs; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) add((v[j][e] - base) * kLog2e);
        } else {  // the last step: no exponentials of vectors that do not exist, terms of 0 for what one of them lacks
#pragma unroll
            for (int j = 0; j < kVecs; j++) {
                const int64_t left = v1 - c0 - (j * kThreads + (int)threadIdx.x) * 8;
                if (left <= 0) break;
#pragma unroll
                for (int e = 0; e < 8; e++) add(e < left ? (v[j][e] - base) * kLog2e : -200.0f);
            }
        }
        if (w != w) {  // a masked logit, -inf, among them (0 times -inf), or a NaN, which s keeps
            w = 0.0f;
#pragma unroll
            for (int j = 0; j < kVecs; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float d = (v[j][e] - base) * kLog2e, x = exp2_raw(d);
                    w += x == 0.0f ? 0.0f : x * d;
                }
        }
        t = merge(t, Stat{m, s, w});
    }
    const uint32_t best = v0 + (int64_t)threadIdx.x * 8 < v1 ? order_of(t.m) : 0u;  // of this thread's own logits
    t = wave_merge(t);
    if ((threadIdx.x & 63) == 0) lds_stat[threadIdx.x >> 6] = t;
    __syncthreads();
    t = lds_stat[0];
#pragma unroll
    for (int i = 1; i < kWavesL; i++) t = merge(t, lds_stat[i]);
    int kept = 0;
    if constexpr (TOP)
        kept = select_top(lds_top, a.top, best, (int)((v1 - v0 + kThreads * 8 - 1) / (kThreads * 8)), [&](int i, uint64_t (&k)[8]) {
            const int64_t c = v0 + (int64_t)i * 8;
            Logits8<T> x;
            x.load(z + c, v1 - c);
#pragma unroll
            for (int e = 0; e < 8; e++) k[e] = c + e < v1 ? key_of(x[e], (uint32_t)(c + e)) : (uint64_t)0;
        });
    if (a.splits == 1) {
        finish_row(a, row, t, lds_top.list, kept, zt, target);
    } else {
        if (threadIdx.x == 0) a.part[blockIdx.x] = t;
        if constexpr (TOP)
            for (int i = threadIdx.x; i < a.top; i += kThreads)
                a.keys[(int64_t)blockIdx.x * a.top + i] = i < kept ? lds_top.list[i] : 0;
    }
}

// Joins the parts of a row, in order.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_join_kernel(LogprobArgs a) {
    __shared__ TopLds lds_top;
    const int64_t row = blockIdx.x;
    int kept = 0;
    Stat t = {-__builtin_inff(), 0.0f, 0.0f};
    if ((int)(threadIdx.x & 63) < a.splits) t = a.part[row * a.splits + (threadIdx.x & 63)];
    t = wave_merge(t);
    if constexpr (TOP) {
        static_assert(kMaxSplits * kMaxTop == 8 * kThreads, "eight keys per thread hold every part's");
        const int n = a.splits * a.top;
        auto load = [&](int i, uint64_t (&k)[8]) {
#pragma unroll
            for (int e = 0; e < 8; e++) k[e] = e * kThreads + i < n ? a.keys[row * n + e * kThreads + i] : 0;
        };
        uint64_t k[8];
        uint32_t best = 0;
        load(threadIdx.x, k);
#pragma unroll
        for (int e = 0; e < 8; e++) best = (uint32_t)(k[e] >> 32) > best ? (uint32_t)(k[e] >> 32) : best;
        kept = select_top(lds_top, a.top, best, 1, load);
    }
    const int64_t target = a.target ? a.target[row] : -1;
    const float zt = target >= 0 && target < a.V ? load_one(static_cast<const T *>(a.Z) + row * a.V + target) : 0.0f;
    finish_row(a, row, t, lds_top.list, kept, zt, target);
}

constexpr int kBwdThreads = 256;
constexpr int kBwdVecs = 4;
constexpr int kBwdChunk = kBwdThreads * kBwdVecs * 8;  // logits per workgroup

struct LogprobBwdArgs {
    const void *Z;
    const int64_t *target;
    const float *lse, *entropy, *d_logp, *d_entropy;
    void *dZ;
    uint32_t *flag;
    int64_t V;
    unsigned chunks;  // workgroups per row
};

// From here on the rounding of lse, 2^-24 of it, is more of a probability than rounding it to bf16 is (2^-9)
constexpr float kMostLse = 65536.0f;

// The gradient, element by element from the row's statistics: one read and one write of the logits.
template <typename T>
__global__ void __launch_bounds__(kBwdThreads) logprobs_bwd_kernel(LogprobBwdArgs a) {
    const int64_t row = blockIdx.x / a.chunks, c0 = (int64_t)(blockIdx.x % a.chunks) * kBwdChunk;
    const T *z = static_cast<const T *>(a.Z) + row * a.V;
    T *dz = static_cast<T *>(a.dZ) + row * a.V;
    const int64_t target = a.target ? a.target[row] : -1;
    const bool used = target >= 0 && target < a.V;
    const float lse = a.lse[row];
    const bool none = lse == -__builtin_inff();  // every logit is -inf: no gradient
    const float g = used && a.d_logp && !none ? a.d_logp[row] : 0.0f, h = a.d_entropy && !none ? a.d_entropy[row] : 0.0f;
    const float entropy = h != 0.0f ? a.entropy[row] : 0.0f;
    const float base = none ? 0.0f : lse;
    if ((g != 0.0f || h != 0.0f) && !(__builtin_fabsf(lse) <= kMostLse) && c0 == 0 && threadIdx.x == 0) *a.flag = 1u;
    float v[kBwdVecs][8];
#pragma unroll
    for (int j = 0; j < kBwdVecs; j++) {
        const int64_t c = c0 + (j * kBwdThreads + (int)threadIdx.x) * 8, left = a.V - c;
        if (left > 0) load8_n(z + c, left >= 8 ? 8 : (int)left, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kBwdVecs; j++) {
        const int64_t c = c0 + (j * kBwdThreads + (int)threadIdx.x) * 8, left = a.V - c;
        if (left <= 0) break;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float lp = fmaxf(v[j][e] - base, -200.0f);  // p is 0 from -88 on
            const float p = exp2_raw(lp * kLog2e);
            const float k = __builtin_fmaf(h, lp + entropy, g);
            v[j][e] = (c + e == target ? g : 0.0f) - p * k;
        }
        store8_n(dz + c, left >= 8 ? 8 : (int)left, v[j]);
    }
}

// Parts of a row: up to two workgroups per CU, and no more than the row has steps (so that a part is a step or little less at
// least), where that takes off enough of a row's steps to pay for the join and the rows do not keep the memory busy as they are. In
// parts and in one, us, 5 alternatives: one row of 100,000 (7 steps) 17.7 and 15.3, of 151,936 (10) 17.4 and 18.2, 16 rows of these
// 17.8 and 18.4, 32 rows 19.4 and 18.5, 63 rows 21.2 and 18.5; 64 rows of 300,000 (19) 24 and 31, 128 rows 29 and 31, 255 rows 40
// and 33.
int plan_splits(int64_t T, int64_t V) {
    const int64_t steps = (V + kStep - 1) / kStep;
    if (T > 128 || steps <= (T < 32 ? 7 : 16)) return 1;
    return (int)std::min<int64_t>({kMaxParts / T, steps, kMaxSplits});
}

template <typename T>
hipError_t fwd(const LogprobArgs &a, hipStream_t st) {
    const unsigned grid = (unsigned)(a.T * a.splits);
    if (a.top > 0) logprobs_kernel<T, true><<<grid, kThreads, 0, st>>>(a);
    else logprobs_kernel<T, false><<<grid, kThreads, 0, st>>>(a);
    if (a.splits > 1) {
        if (a.top > 0) logprobs_join_kernel<T, true><<<(unsigned)a.T, kThreads, 0, st>>>(a);
        else logprobs_join_kernel<T, false><<<(unsigned)a.T, kThreads, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

size_t logprobs_ws(int64_t, int64_t, int top) {
    return kWsHeader + (size_t)kMaxParts * (16 + (size_t)top * sizeof(uint64_t));
}

hipError_t launch_logprobs(int dtype, const void *Z, int64_t T, int64_t V, const int64_t *target, int top, float *logp,
                           float *entropy, float *lse, float *top_logp, int32_t *top_index, uint32_t *flag, void *ws,
                           hipStream_t st) {
    const int splits = plan_splits(T, V);
    const int64_t per = ((V + splits - 1) / splits + 7) / 8 * 8;
    char *base = static_cast<char *>(ws) + kWsHeader;
    // a launch's work-items (512 per row where rows are not split) must stay below 2^32
    constexpr int64_t kRows = (int64_t(1) << 23) - 1;
    for (int64_t r = 0; r < T; r += kRows) {
        LogprobArgs a{static_cast<const char *>(Z) + (size_t)(r * V) * (dtype == kBF16 ? 2 : 4),
                      target ? target + r : nullptr,
                      logp ? logp + r : nullptr,
                      entropy ? entropy + r : nullptr,
                      lse + r,
                      top_logp + r * top,
                      top_index + r * top,
                      flag,
                      reinterpret_cast<Stat *>(base),
                      reinterpret_cast<uint64_t *>(base + kMaxParts * 16),
                      std::min(kRows, T - r),
                      V,
                      per,
                      top,
                      splits};
        const hipError_t e = dtype == kBF16 ? fwd<uint16_t>(a, st) : fwd<float>(a, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_logprobs_bwd(int dtype, const void *Z, int64_t T, int64_t V, const int64_t *target, const float *lse,
                               const float *entropy, const float *d_logp, const float *d_entropy, void *dZ, uint32_t *flag,
                               hipStream_t st) {
    const int64_t chunks = (V + kBwdChunk - 1) / kBwdChunk;
    LogprobBwdArgs a{Z, target, lse, entropy, d_logp, d_entropy, dZ, flag, V, (unsigned)chunks};
    // one launch for as many rows as a grid holds: its work-items (256 per chunk) must stay below 2^32
    const int64_t rows = std::max<int64_t>(1, ((int64_t(1) << 24) - 1) / chunks);
    const size_t esz = dtype == kBF16 ? 2 : 4;
    for (int64_t r = 0; r < T; r += rows) {
        const int64_t n = std::min(rows, T - r);
        LogprobBwdArgs b = a;
        b.Z = static_cast<const char *>(Z) + (size_t)(r * V) * esz;
        b.dZ = static_cast<char *>(dZ) + (size_t)(r * V) * esz;
        b.target = target ? target + r : nullptr;
        b.lse = lse + r;
        b.entropy = entropy ? entropy + r : nullptr;
        b.d_logp = d_logp ? d_logp + r : nullptr;
        b.d_entropy = d_entropy ? d_entropy + r : nullptr;
        const unsigned grid = (unsigned)(n * chunks);
        if (dtype == kBF16) logprobs_bwd_kernel<uint16_t><<<grid, kBwdThreads, 0, st>>>(b);
        else logprobs_bwd_kernel<float><<<grid, kBwdThreads, 0, st>>>(b);
    }
    return hipGetLastError();
}

}  // namespace focus
