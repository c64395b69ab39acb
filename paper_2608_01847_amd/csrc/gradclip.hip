// The norm over all gradients of a step and the gradients scaled by it: norm = sqrt(sum g^2) over every element of every tensor,
// out = g min(1, max_norm / norm).
//
// HBM-bound: every gradient is read once for the norm and once more to be scaled. Squares are summed in fp64, so that neither
// the size of a gradient (1e-30 or 1e30) nor their number costs digits. Up to kGroup tensors travel in the arguments of a launch; a
// group's elements are numbered in chunks of one tensor each, which the workgroups take in turn.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kGroup = 112;             // tensors of a launch: 28 bytes each of the 4 KB that a kernel's arguments have
constexpr int kChunk = 8192;            // elements
constexpr int kNormParts = 2048;        // workgroups of a launch at most, each with one partial sum

struct GradGroup {
    const void *g[kGroup];
    void *out[kGroup];
    int64_t n[kGroup];
    uint32_t first[kGroup];             // first chunk of each tensor
    uint32_t bf16[(kGroup + 31) / 32];  // a bit per tensor
    uint32_t chunks;
    int count;
};
static_assert(sizeof(GradGroup) <= 4032, "the group and a kernel's other arguments fit 4 KB");

// The tensor of a chunk: the last one whose first chunk is not behind it
__device__ __forceinline__ int tensor_of(const GradGroup &a, uint32_t chunk) {
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// f(piece start, elements of it) for the 8-element pieces of a chunk that this thread takes
template <typename F>
__device__ __forceinline__ void pieces(int64_t start, int64_t n, F &&f) {
#pragma unroll
    for (int j = 0; j < kChunk / 2048; j++) {
        const int64_t c = start + (j * 256 + (int)threadIdx.x) * 8;
        f(c, (int)(n - c < 8 ? n - c : 8));
    }
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T *g, int64_t start, int64_t n) {
    Raw8<T> v[kChunk / 2048];
    int j = 0;
    pieces(start, n, [&](int64_t c, int m) { v[j++].load(g + c, m); });
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kChunk / 2048; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const double x = (double)v[i][e];
            s = __builtin_fma(x, x, s);
        }
    return s;
}

__global__ void __launch_bounds__(256) grad_norm_kernel(GradGroup a, double *__restrict__ part) {
    __shared__ double lds[4];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(a, c);
        const int64_t start = (int64_t)(c - a.first[i]) * kChunk;
        if (a.bf16[i / 32] >> (i % 32) & 1u) s += chunk_squares(static_cast<const uint16_t *>(a.g[i]), start, a.n[i]);
        else s += chunk_squares(static_cast<const float *>(a.g[i]), start, a.n[i]);
    }
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = lds[0] + lds[1] + lds[2] + lds[3];
}

// The norm from the partial sums, in a fixed order, in every thread of a workgroup of 256
__device__ __forceinline__ double norm_of(const double *__restrict__ part, int64_t parts) {
    __shared__ double lds[4];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < parts; i += 256 * 8) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; u++) v[u] = i + 256 * u < parts ? part[i + 256 * u] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; u++) s += v[u];
    }
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    return sqrt(lds[0] + lds[1] + lds[2] + lds[3]);
}

// The factor as a product x y of two: y = 2^-100 where it is so small that fp32 would lose its digits
__device__ __forceinline__ float2 factor_of(double norm, double max_norm) {
    if (!(norm < (double)__builtin_inff() && norm > max_norm)) return make_float2(1.0f, 1.0f);
    const double f = max_norm / norm;
    return f < 0x1p-100 ? make_float2((float)(f * 0x1p100), 0x1p-100f) : make_float2((float)f, 1.0f);
}

// Writes the norm (one workgroup), and the factor for scaling launches that do not form it themselves
__device__ __forceinline__ void put_norm(double norm, double *out, uint32_t *flag) {
    *out = norm;
    if (!(norm < (double)__builtin_inff())) raise_domain_flag(flag);
}

__global__ void __launch_bounds__(256) grad_finish_kernel(const double *__restrict__ part, int64_t parts, double max_norm,
                                                          double *__restrict__ norm, float2 *__restrict__ factor, uint32_t *flag) {
    const double x = norm_of(part, parts);
    if (threadIdx.x) return;
    put_norm(x, norm, flag);
    *factor = factor_of(x, max_norm);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T *g, T *out, int64_t start, int64_t n, float2 f) {
    Raw8<T> v[kChunk / 2048];
    int j = 0;
    pieces(start, n, [&](int64_t c, int m) { v[j++].load(g + c, m); });
    j = 0;
    pieces(start, n, [&](int64_t c, int m) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = v[j][e] * f.x * f.y;
        j++;
        store8_n(out + c, m, x);
    });
}

// `parts`: the partial sums, of which every workgroup forms the factor itself and the first one writes the norm (a launch less);
// 0: the factor is there
__global__ void __launch_bounds__(256) grad_scale_kernel(GradGroup a, const double *__restrict__ part, int64_t parts, double max_norm,
                                                         double *__restrict__ norm, const float2 *__restrict__ factor, uint32_t *flag) {
    float2 f;
    if (parts) {
        const double x = norm_of(part, parts);
        if (blockIdx.x == 0 && threadIdx.x == 0) put_norm(x, norm, flag);
        f = factor_of(x, max_norm);
    } else {
        f = *factor;
    }
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(a, c);
        if (!a.out[i] || (f.x == 1.0f && a.out[i] == a.g[i])) continue;  // nothing to write
        const int64_t start = (int64_t)(c - a.first[i]) * kChunk;
        if (a.bf16[i / 32] >> (i % 32) & 1u)
            chunk_scale(static_cast<const uint16_t *>(a.g[i]), static_cast<uint16_t *>(a.out[i]), start, a.n[i], f);
        else
            chunk_scale(static_cast<const float *>(a.g[i]), static_cast<float *>(a.out[i]), start, a.n[i], f);
    }
}

// The group of the tensors from `first` on (empty ones are left out); the index behind its last
int64_t next_group(const GradTensor *t, int64_t first, int64_t count, GradGroup &a) {
    a.count = 0, a.chunks = 0;
    for (uint32_t &b : a.bf16) b = 0;
    int64_t i = first;
    for (; i < count && a.count < kGroup; i++) {
        if (t[i].n == 0) continue;
        const int k = a.count++;
        a.g[k] = t[i].grad, a.out[k] = t[i].out, a.n[k] = t[i].n, a.first[k] = a.chunks;
        if (t[i].dtype == kBF16) a.bf16[k / 32] |= 1u << (k % 32);
        a.chunks += (uint32_t)((t[i].n + kChunk - 1) / kChunk);
    }
    return i;
}

}  // namespace

static_assert(kMaxGradElems / kChunk * kGroup < (int64_t(1) << 32), "chunk numbers of a group are 32-bit");

size_t clip_grad_norm_ws(int64_t tensors) {
    return 2 * kWsHeader + (size_t)((tensors + kGroup - 1) / kGroup) * kNormParts * sizeof(double);
}

hipError_t launch_clip_grad_norm(const GradTensor *t, int64_t count, double max_norm, double *norm, uint32_t *flag, void *ws,
                                 hipStream_t st) {
    float2 *const factor = reinterpret_cast<float2 *>(static_cast<char *>(ws) + kWsHeader);
    double *const part = reinterpret_cast<double *>(static_cast<char *>(ws) + 2 * kWsHeader);
    int64_t parts = 0;
    int groups = 0;
    bool scales = false;
    GradGroup a;
    for (int64_t i = 0; i < count;) {
        i = next_group(t, i, count, a);
        if (!a.count) continue;
        for (int k = 0; k < a.count; k++) scales = scales || a.out[k];
        const unsigned grid = std::min<uint32_t>(a.chunks, kNormParts);
        grad_norm_kernel<<<grid, 256, 0, st>>>(a, part + parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        parts += grid;
        groups++;
    }
    const bool alone = scales && groups == 1;  // the one scaling launch finishes the norm as well
    if (!alone) grad_finish_kernel<<<1, 256, 0, st>>>(part, parts, max_norm, norm, factor, flag);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !scales) return e;
    for (int64_t i = 0; i < count;) {
        i = next_group(t, i, count, a);
        if (!a.count) continue;
        grad_scale_kernel<<<std::min<uint32_t>(a.chunks, kNormParts), 256, 0, st>>>(a, part, alone ? parts : 0, max_norm, norm, factor, flag);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace focus
