// Pieces shared by the attention kernels: which tile of which sequence a workgroup takes, and the masks.
#pragma once

#include "internal.h"
#include "ops_device.h"

namespace focus {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;

// One sequence's rows of the packed queries and keys.
struct SeqRange {
    int64_t q0, k0;  // first rows
    int lq, lk;
};

// ends that do not rise or that pass the tensors raise the domain flag and leave an empty sequence
__device__ __forceinline__ void set_range(const AttnArgs &a, int qa, int qb, int ka, int kb, SeqRange &r) {
    const bool ok = qa >= 0 && qa <= qb && qb <= a.Tq && ka >= 0 && ka <= kb && kb <= a.Tk;
    if (!ok) *a.flag = 1u;
    r.q0 = ok ? qa : 0;
    r.k0 = ok ? ka : 0;
    r.lq = ok ? qb - qa : 0;
    r.lk = ok ? kb - ka : 0;
}

// Tiles of `rows` rows over packed sequences with ends cu[0..n] (the keys' where KEYS), `each` rows per token: sequence i's
// tiles take the slots from cu[i] each / rows + i on, which leaves room for ceil(length / rows) of them whatever the lengths
// are, so the number of slots, T each / rows + n, needs no look at the lengths on the host. Gives the slot's sequence in r and
// returns its tile, which may lie past the sequence's end or, in slots before the first sequence, be -1: nothing to do (tile_in
// below). Every lane loads one sequence's four ends at once: after the bisection that many sequences need, one trip to memory.
template <bool KEYS>
__device__ __forceinline__ int slot_range(const AttnArgs &a, int rows, int slot, int each, SeqRange &r) {
    if (!a.cu_q) {
        r.q0 = r.k0 = 0;
        r.lq = (int)a.Tq;
        r.lk = (int)a.Tk;
        return slot;
    }
    const int32_t *cu = KEYS ? a.cu_k : a.cu_q;
    // (T each is below 2^31; ends that lie outside give a place of no meaning, and their sequence is empty)
    auto start_of = [&](int end, int i) { return (int)((uint32_t)end * (uint32_t)each / (uint32_t)rows) + i; };
    int lo = 0, len = a.n_seq;  // the answer is in [lo, lo + len)
    while (len > 64) {          // a scalar bisection down to one wave's width
        const int half = len / 2;
        if (start_of(cu[lo + half], lo + half) <= slot) {
            lo += half;
            len -= half;
        } else {
            len = half;
        }
    }
    const int lane = threadIdx.x & 63, i = lo + (lane < len ? lane : len - 1);
    const int qa = a.cu_q[i], qb = a.cu_q[i + 1], ka = a.cu_k[i], kb = a.cu_k[i + 1];
    const int start = start_of(KEYS ? ka : qa, i);
    const unsigned long long below = __ballot(lane < len && start <= slot);
    const int at = __builtin_amdgcn_readfirstlane(below ? 63 - __builtin_clzll(below) : 0);
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
    set_range(a, of(qa), of(qb), of(ka), of(kb), r);
    return below ? slot - of(start) : -1;
}

// Whether a tile of `rows` rows has any of a sequence's n
__device__ __forceinline__ bool tile_in(int tile, int rows, int64_t n) { return tile >= 0 && (int64_t)tile * rows < n; }

// Every pair of ends, by the first workgroup of a launch (the others meet only those of their own tiles)
template <int THREADS>
__device__ __forceinline__ void check_ends(const AttnArgs &a) {
    if (!a.cu_q || blockIdx.x != 0 || blockIdx.y != 0) return;
    SeqRange r;
    for (int s = threadIdx.x; s < a.n_seq; s += THREADS) set_range(a, a.cu_q[s], a.cu_q[s + 1], a.cu_k[s], a.cu_k[s + 1], r);
}

// row of register r in the 32 x 32 accumulator of a lane: 8 (r / 4) + 4 (lane / 32) + r % 4
__device__ __forceinline__ constexpr int acc_row(int r) { return (r & 3) + 8 * (r >> 2); }

// Partial results of a forward whose keys are split: [splits][Hq][Tq] (x D)
struct AttnParts {
    float *m, *l, *o;
};
// Gradients of a backward whose sums are split, fp32: dq [splits][Tq][Hq][D], dk and dv [splits][Tk][Hkv][D]
struct AttnGradParts {
    float *dq, *dk, *dv;
};
struct AttnBwdPlan {
    int q_splits, k_splits;
};
AttnBwdPlan plan_attn_bwd_bf16(int64_t Tq, int64_t Tk, int Hq, int Hkv, int64_t n_seq);
// bytes of m and l, rounded to keep o aligned
inline size_t attn_part_stats(int splits, int64_t rows) { return ((size_t)splits * (size_t)rows * 8 + 255) / 256 * 256; }
int attn_splits_bf16(int64_t Tq, int64_t Tk, int Hq, int Hkv, int64_t n_seq);
hipError_t launch_attn_fwd_bf16(const AttnArgs &a, void *ws, hipStream_t st);
hipError_t launch_attn_bwd_bf16(const AttnArgs &a, float *parts, hipStream_t st);

}  // namespace focus
