// What the kernels of the linear cross entropy share (not part of the public ABI).
#pragma once

#include "internal.h"

namespace focus {

constexpr int kCeTile = 256;  // edge of a tile on the matrix instructions (of a logit tile: or half of it)
constexpr int kCeFew = 16;    // tokens up to which the forward reads the weights straight into registers
constexpr int kCeFewV = 128;  // vocabulary entries of its workgroups
constexpr int64_t kCeMostWidth = int64_t(1) << 20;  // of a piece of the vocabulary

constexpr float kCeMostLogit = 1073741824.0f;       // 2^30: a token whose largest logit reaches that in size raises the domain flag

struct CeArgs {
    const void *X, *W;
    const int64_t *target;
    float *lse, *logp;    // [T]; logp NULL where no targets are given
    const float *g, *h;   // gradients of logp and lse, NULL: 0
    float2 *part;         // [tiles][T] maximum and sum of a tile's exponentials
    float *zt;            // [T] logit of the target
    void *D;              // [T][pitch] of the piece: fp32, or bf16 relative to the token's scale
    const float *scale;   // [T] the power of two at or below the larger of |g| and |h|, what D is relative to
    float *rest;          // [T] what rounding the target's entry of D to bf16 left
    int64_t T, V, K, pitch, v0, t0;  // first vocabulary entry of the piece, first token of the launch
    int tiles_v;
};

// Whether token t has a gradient. One without it takes no part in the sums whatever its row of X and its lse hold, NaN too.
__device__ __forceinline__ bool ce_takes_part(const int64_t *target, const float *g, const float *h, int64_t V, int64_t t) {
    return (g && target[t] >= 0 && target[t] < V && g[t] != 0.0f) || (h && h[t] != 0.0f);
}

// Logit tiles on the matrix instructions (bf16; K a multiple of 16 throughout), of edge x edge: those of `tokens` tokens from a.t0 on
int64_t ce_mfma_tile(int64_t T, int64_t n);
void launch_ce_stats_mfma(const CeArgs &a, int64_t edge, int64_t tokens, hipStream_t st);
void launch_ce_stats_few(const CeArgs &a, hipStream_t st);  // T <= kCeFew
void launch_ce_grad_mfma(const CeArgs &a, int64_t edge, int64_t tokens, uint32_t *flag, hipStream_t st);

// The same on the fp32 matrix instructions, tiles of edge x edge; D's transpose, [entries][pitch_t], goes to Dt;
// with x, the rows of X that have a gradient go there, zeros in place of the others
int64_t ce_f32_tile(int64_t T, int64_t n);
void launch_ce_stats_f32(const CeArgs &a, int64_t edge, int64_t tokens, hipStream_t st);
void launch_ce_grad_f32(const CeArgs &a, int64_t edge, int64_t tokens, float *Dt, int64_t pitch_t, float *x, uint32_t *flag,
                        hipStream_t st);
// out [splits][N][K] = dY^T X over `chunk` rows (a multiple of 32) of dY [M][ldy] (ldy a multiple of 4) and X [M][K] each
hipError_t launch_dw_f32(const float *dY, const float *X, int64_t M, int64_t N, int64_t ldy, int64_t K, int64_t chunk,
                         int64_t splits, float *out, hipStream_t st);

}  // namespace focus
