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

__device__ __forceinline__ bool ends_ok(const AttnArgs &a, int qa, int qb, int ka, int kb) {
    return qa >= 0 && qa <= qb && qb <= a.Tq && ka >= 0 && ka <= kb && kb <= a.Tk;
}

// ends that do not rise or that pass the tensors raise the domain flag and leave an empty sequence
__device__ __forceinline__ void set_range(const AttnArgs &a, int qa, int qb, int ka, int kb, SeqRange &r) {
    const bool ok = ends_ok(a, qa, qb, ka, kb);
    if (!ok) *a.flag = 1u;
    r.q0 = ok ? qa : 0;
    r.k0 = ok ? ka : 0;
    r.lq = ok ? qb - qa : 0;
    r.lk = ok ? kb - ka : 0;
}

// Tiles of `rows` rows over packed sequences with ends cu[0..n] (the keys' where KEYS), `each` rows per token: sequence i's
// tiles have the slots from cu[i] each / rows + i on, which leaves room for ceil(length / rows) of them whatever the lengths
// are, so the number of slots, T each / rows + n, needs no look at the lengths on the host. Gives the slot's sequence in r and
// returns its tile, which may lie past the sequence's end or be negative: nothing to do (tile_in below).
//
// Under a causal mask a tile's work grows with the rows before it (KEYS: behind it). The slots of kOrdered sequences, one after
// the other, are then given out from the longest tiles to the shortest, over those sequences together: workgroups start in
// the order of the slots, and what starts last should end soonest (backward of 4 x 2,048 tokens, 64/8 heads of 128, 1.11 ms;
// sequence by sequence 1.15; sixteen sequences together, which share less in L2, 2% slower at 32 x 2,048).
//
// Every lane loads one sequence's four ends at once: after the bisection that many sequences need, one trip to memory.
constexpr int kOrdered = 8;

template <bool KEYS>
__device__ __forceinline__ int slot_range(const AttnArgs &a, int rows, int slot, int each, SeqRange &r) {
    // (T each is below 2^31; ends that lie outside give a place of no meaning, and their sequence is empty)
    auto tiles_of = [&](int tokens) { return (int)(((uint32_t)tokens * (uint32_t)each + (uint32_t)rows - 1) / (uint32_t)rows); };
    if (!a.cu_q) {
        r.q0 = r.k0 = 0;
        r.lq = (int)a.Tq;
        r.lk = (int)a.Tk;
        return KEYS || !a.causal ? slot : tiles_of(r.lq) - 1 - slot;
    }
    const int32_t *cu = KEYS ? a.cu_k : a.cu_q;
    auto start_of = [&](int end, int i) { return (int)((uint32_t)end * (uint32_t)each / (uint32_t)rows) + i; };
    int lo = 0, len = a.n_seq;  // the answer is in [lo, lo + len)
    while (len > 64) {          // a scalar bisection down to one wave's width, by whole runs of kOrdered
        const int half = len / 2 / kOrdered * kOrdered;
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
    int at = __builtin_amdgcn_readfirstlane(below ? 63 - __builtin_clzll(below) : 0);
    int tile = below ? slot - __builtin_amdgcn_readlane(start, at) : -1;
    if (a.causal && below) {
        const int first = at / kOrdered * kOrdered, p = slot - __builtin_amdgcn_readlane(start, first);
        const int own = lane < len && ends_ok(a, qa, qb, ka, kb) ? tiles_of(KEYS ? kb - ka : qb - qa) : 0;
        int tiles[kOrdered], most = 0;
#pragma unroll
        for (int j = 0; j < kOrdered; j++) {
            tiles[j] = __builtin_amdgcn_readlane(own, first + j);
            most = tiles[j] > most ? tiles[j] : most;
        }
        auto longer = [&](int v) {  // tiles of more than v units of work
            int n = 0;
#pragma unroll
            for (int j = 0; j < kOrdered; j++) n += tiles[j] > v ? tiles[j] - v : 0;
            return n;
        };
        int v = 0, high = most;  // this slot's work: the least v that no more than p tiles pass
        while (v < high) {
            const int mid = (v + high) / 2;
            if (longer(mid) <= p) high = mid;
            else v = mid + 1;
        }
        int left = p - longer(v);  // tiles of the same work before this one
        tile = -1;
#pragma unroll
        for (int j = 0; j < kOrdered; j++) {
            if (tiles[j] >= v && left-- == 0 && v > 0) {
                at = first + j;
                tile = KEYS ? tiles[j] - v : v - 1;
            }
        }
    }
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
    set_range(a, of(qa), of(qb), of(ka), of(kb), r);
    return tile;
}

// The key-value head, the slot and the part of a split sum that a workgroup takes: heads in turn (consecutive workgroups go to
// different XCDs, so that an XCD's L2 sees few heads), a slot's parts one after the other.
struct Place {
    int hk, slot, part;
};
template <bool SPLIT>
__device__ __forceinline__ Place place(int Hkv) {
    const uint32_t flat = SPLIT ? blockIdx.y * gridDim.x + blockIdx.x : blockIdx.x, rest = flat / (uint32_t)Hkv;
    return {(int)(flat - rest * (uint32_t)Hkv), (int)(SPLIT ? rest / gridDim.y : rest), (int)(SPLIT ? rest % gridDim.y : 0u)};
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
// Gradients of a backward whose sums are split, fp32: dq [splits][Tq][Hq][D], dk and dv [splits][Tk][Hkv][D]; with dq the rows'
// sums of dS [splits][Hq][Tq]
struct AttnGradParts {
    float *rest, *dq, *dk, *dv;
};
inline int64_t attn_rest_floats(int q_splits, int64_t rows) { return q_splits > 1 ? (q_splits * rows + 63) / 64 * 64 : 0; }
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
