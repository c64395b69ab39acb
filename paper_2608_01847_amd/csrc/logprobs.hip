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
// The alternatives: logits are ordered by (value, lower index first), as 64-bit keys. A key `tau` that at least `top` keys of
// the row reach is kept; the few elements that reach it are collected in LDS and ranked at the end (the step that sees
// more of them than there is room first raises tau). Counts do not depend on the order of the LDS additions, nor does
// the ranking, keys being distinct.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kThreads = 512;
constexpr int kWavesL = kThreads / 64;
constexpr int kVecs = 4;                        // vectors of 8 logits per thread and step
constexpr int kStep = kThreads * kVecs * 8;     // logits per step
constexpr int kRoom = 1024;                     // collected keys
constexpr int kFull = 512;                      // keys from which the list is cut to `top` after a step
constexpr int kMaxSplits = 64;
constexpr int kRowsUnsplit = 512;               // rows from which a row is one workgroup's
constexpr int64_t kSplitLogits = 4096;          // logits of a part, at least
constexpr int kMaxParts = 2 * kRowsUnsplit;     // parts of a split launch, at most
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
__device__ __forceinline__ uint64_t shfl_key(uint64_t k, int mask) {
    const uint32_t lo = __shfl_xor((uint32_t)k, mask, 64), hi = __shfl_xor((uint32_t)(k >> 32), mask, 64);
    return ((uint64_t)hi << 32) | lo;
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
    uint64_t group[64];
    uint64_t wave_best[kWavesL];
    int count[3];
    int pos;
};

// The running list of the largest keys of a workgroup's elements. Every member is called by all threads.
struct TopList {
    TopLds &l;
    int top, n = 0, turn = 0;
    uint64_t tau = 0;  // at least `top` of the keys seen so far reach it (0: all do)

    __device__ __forceinline__ TopList(TopLds &lds, int k) : l(lds), top(k) {
        if (threadIdx.x == 0) {
            l.count[0] = l.count[1] = l.count[2] = 0;
            l.pos = 0;
        }
        __syncthreads();
    }

    // sum of c over the workgroup
    __device__ __forceinline__ int total(int c) {
        if (c) atomicAdd(&l.count[turn], c);
        const int next = turn == 2 ? 0 : turn + 1;
        if (threadIdx.x == 0) l.count[next] = 0;  // last read before the previous call's barrier
        __syncthreads();
        const int r = l.count[turn];
        turn = next;
        return r;
    }

    // Keeps the `top` largest of the list, in order.
    __device__ __forceinline__ void cut() {
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t k = l.list[i];
            int rank = 0;
            for (int j = 0; j < n; j++) rank += l.list[j] > k ? 1 : 0;
            if (rank < top) l.cut[rank] = k;
        }
        __syncthreads();
        const int kept = n < top ? n : top;
        for (int i = threadIdx.x; i < kept; i += kThreads) l.list[i] = l.cut[i];
        if (threadIdx.x == 0) l.pos = kept;
        __syncthreads();
        n = kept;
        if (kept == top && l.list[top - 1] > tau) tau = l.list[top - 1];
    }

    // Takes in a thread's E elements; key(e) is an element's key, 0 for none, best(): the largest order_of among them
    template <int E, typename Key>
    __device__ __forceinline__ void add(uint32_t best, Key &&key) {
        auto reach = [&]() {
            int c = 0;
            if (best >= (uint32_t)(tau >> 32)) {
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const uint64_t k = key(e);
                    c += k >= tau && k != 0 ? 1 : 0;
                }
            }
            return c;
        };
        int c = reach(), sum = total(c);
        if (sum == 0) return;
        if (n + sum > kRoom && n > top) {
            cut();
            c = reach();
            sum = total(c);
        }
        if (n + sum > kRoom) {
            // Raise tau: of the largest keys of 64 groups of threads, the top-th is reached by `top` keys at least.
            uint64_t mine = 0;
#pragma unroll
            for (int e = 0; e < E; e++) {
                const uint64_t k = key(e);
                mine = k > mine ? k : mine;
            }
#pragma unroll
            for (int x = 1; x < kThreads / 64; x <<= 1) {
                const uint64_t o = shfl_key(mine, x);
                mine = o > mine ? o : mine;
            }
            if (threadIdx.x % (kThreads / 64) == 0) l.group[threadIdx.x / (kThreads / 64)] = mine;
            __syncthreads();
            uint64_t g = l.group[threadIdx.x & 63];
            int rank = 0;
            for (int j = 0; j < 64; j++) rank += l.group[j] > g || (l.group[j] == g && j < (int)(threadIdx.x & 63)) ? 1 : 0;
            const unsigned long long who = __ballot(rank == top - 1);
            const uint64_t kth = l.group[__builtin_ctzll(who)];
            if (kth > tau) tau = kth;
            c = reach();
            sum = total(c);
        }
        if (n + sum <= kRoom) {
            if (c) {
                int at = atomicAdd(&l.pos, c);
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const uint64_t k = key(e);
                    if (k >= tau && k != 0) l.list[at++] = k;
                }
            }
            n += sum;
        } else {
            // Few threads hold most of the largest keys: take them one by one.
            uint64_t below = ~(uint64_t)0;
            for (int i = 0; i < top; i++) {
                uint64_t mine = 0;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const uint64_t k = key(e);
                    mine = k < below && k > mine ? k : mine;
                }
#pragma unroll
                for (int x = 1; x < 64; x <<= 1) {
                    const uint64_t o = shfl_key(mine, x);
                    mine = o > mine ? o : mine;
                }
                if ((threadIdx.x & 63) == 0) l.wave_best[threadIdx.x >> 6] = mine;
                __syncthreads();
                uint64_t b = 0;
                for (int w = 0; w < kWavesL; w++) b = l.wave_best[w] > b ? l.wave_best[w] : b;
                __syncthreads();
                if (b == 0) break;
                if (threadIdx.x == 0) l.list[n] = b;
                n++;
                below = b;
            }
            if (threadIdx.x == 0) l.pos = n;
        }
        if (n > kFull) cut();
    }
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

// One row's results from its statistics and the ranked list
__device__ __forceinline__ void finish_row(const LogprobArgs &a, int64_t row, const Stat &t, const uint64_t *list, int n,
                                           float target_logit, int64_t target) {
    const bool none = t.m == -__builtin_inff();  // every logit is -inf
    const float lse = none ? -__builtin_inff() : __builtin_fmaf(log2f(t.s), kLn2, t.m);
    if (threadIdx.x == 0) {
        a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = none ? 0.0f : kLn2 * (log2f(t.s) - t.w / t.s);
        if (a.logp) a.logp[row] = target < 0 || target >= a.V ? 0.0f : none ? -__builtin_inff() : target_logit - lse;
        if (t.s != t.s || target >= a.V) *a.flag = 1u;  // a NaN or +inf among the logits, or no such token
    }
    for (int i = threadIdx.x; i < a.top; i += kThreads) {
        const bool in = i < n;
        const uint64_t k = in ? list[i] : 0;
        const float v = value_of((uint32_t)(k >> 32));
        a.top_index[row * a.top + i] = in ? (int32_t)(0xFFFFFFFFu - (uint32_t)k) : -1;
        a.top_logp[row * a.top + i] = !in || none ? -__builtin_inff() : v - lse;
    }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(LogprobArgs a) {
    __shared__ TopLds lds_top;
    __shared__ Stat lds_stat[kWavesL];
    const int64_t row = blockIdx.x / (unsigned)a.splits;
    const int split = (int)(blockIdx.x % (unsigned)a.splits);
    const int64_t v0 = split * a.per, v1 = v0 + a.per < a.V ? v0 + a.per : a.V;
    const T *z = static_cast<const T *>(a.Z) + row * a.V;
    TopList list(lds_top, TOP ? a.top : 1);
    Stat t = {-__builtin_inff(), 0.0f, 0.0f};
    for (int64_t c0 = v0; c0 < v1; c0 += kStep) {
        float v[kVecs][8];
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < kVecs; j++) {
            const int64_t c = c0 + (j * kThreads + (int)threadIdx.x) * 8;
            const int64_t left = v1 - c;
            const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
            if (n > 0) load8_n(z + c, n, v[j]);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                v[j][e] = e < n ? v[j][e] : -__builtin_inff();
                top = fmaxf(top, v[j][e]);
            }
        }
        const float m = fmaxf(t.m, top), base = m == -__builtin_inff() ? 0.0f : m;
        float s = 0.0f, w = 0.0f;
#pragma unroll
        for (int j = 0; j < kVecs; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = (v[j][e] - base) * kLog2e, x = exp2_raw(d);
                s += x;
                w = __builtin_fmaf(x, d, w);
            }
        if (w != w) {  // a -inf among them (0 times -inf), or a NaN, which s keeps
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
        if constexpr (TOP) {
            list.add<kVecs * 8>(order_of(top), [&](int e) {
                const int64_t c = c0 + ((e >> 3) * kThreads + (int)threadIdx.x) * 8 + (e & 7);
                return c < v1 ? key_of(v[e >> 3][e & 7], (uint32_t)c) : (uint64_t)0;
            });
        }
    }
    t = wave_merge(t);
    if ((threadIdx.x & 63) == 0) lds_stat[threadIdx.x >> 6] = t;
    __syncthreads();
    t = lds_stat[0];
#pragma unroll
    for (int i = 1; i < kWavesL; i++) t = merge(t, lds_stat[i]);
    if constexpr (TOP) list.cut();
    if (a.splits == 1) {
        const int64_t target = a.target ? a.target[row] : -1;
        const float zt = target >= 0 && target < a.V ? load_one(z + target) : 0.0f;
        finish_row(a, row, t, lds_top.list, TOP ? list.n : 0, zt, target);
    } else {
        if (threadIdx.x == 0) a.part[blockIdx.x] = t;
        if constexpr (TOP)
            for (int i = threadIdx.x; i < a.top; i += kThreads)
                a.keys[(int64_t)blockIdx.x * a.top + i] = i < list.n ? lds_top.list[i] : 0;
    }
}

// Joins the parts of a row, in order.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_join_kernel(LogprobArgs a) {
    __shared__ TopLds lds_top;
    const int64_t row = blockIdx.x;
    TopList list(lds_top, TOP ? a.top : 1);
    Stat t = {-__builtin_inff(), 0.0f, 0.0f};
    if ((int)(threadIdx.x & 63) < a.splits) t = a.part[row * a.splits + (threadIdx.x & 63)];
    t = wave_merge(t);
    if constexpr (TOP) {
        constexpr int E = kMaxSplits * kMaxTop / kThreads;
        uint64_t k[E];
        uint64_t best = 0;
        const int n = a.splits * a.top;
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int i = e * kThreads + (int)threadIdx.x;
            k[e] = i < n ? a.keys[row * n + i] : 0;
            best = k[e] > best ? k[e] : best;
        }
        list.add<E>((uint32_t)(best >> 32), [&](int e) { return k[e]; });
        list.cut();
    }
    const int64_t target = a.target ? a.target[row] : -1;
    const float zt = target >= 0 && target < a.V ? load_one(static_cast<const T *>(a.Z) + row * a.V + target) : 0.0f;
    finish_row(a, row, t, lds_top.list, TOP ? list.n : 0, zt, target);
}

constexpr int kBwdThreads = 256;
constexpr int kBwdVecs = 4;
constexpr int kBwdChunk = kBwdThreads * kBwdVecs * 8;  // logits per workgroup

struct LogprobBwdArgs {
    const void *Z;
    const int64_t *target;
    const float *lse, *entropy, *d_logp, *d_entropy;
    void *dZ;
    int64_t V;
    unsigned chunks;  // workgroups per row
};

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

int plan_splits(int64_t T, int64_t V) {
    if (T >= kRowsUnsplit) return 1;
    const int64_t want = (kRowsUnsplit + T - 1) / T, parts = (V + kSplitLogits - 1) / kSplitLogits;
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, parts, kMaxSplits}));
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
    LogprobArgs a{Z, target, logp, entropy, lse, top_logp, top_index, flag, reinterpret_cast<Stat *>(base),
                  reinterpret_cast<uint64_t *>(base + kMaxParts * 16), T, V, per, top, splits};
    return dtype == kBF16 ? fwd<uint16_t>(a, st) : fwd<float>(a, st);
}

hipError_t launch_logprobs_bwd(int dtype, const void *Z, int64_t T, int64_t V, const int64_t *target, const float *lse,
                               const float *entropy, const float *d_logp, const float *d_entropy, void *dZ, hipStream_t st) {
    const int64_t chunks = (V + kBwdChunk - 1) / kBwdChunk;
    LogprobBwdArgs a{Z, target, lse, entropy, d_logp, d_entropy, dZ, V, (unsigned)chunks};
    // one launch for as many rows as a grid holds
    const int64_t rows = std::max<int64_t>(1, ((int64_t(1) << 31) - 1) / chunks);
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
