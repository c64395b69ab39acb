// The norm over all gradients of a step and the gradients scaled by it: norm = sqrt(sum g^2) over every element of every tensor,
// out = g min(1, max_norm / norm).
//
// HBM-bound: every gradient is read once for the norm and once more to be scaled. Squares are summed in fp64, so that neither
// the size of a gradient (1e-30 or 1e30) nor their number costs digits. The tensors travel in the arguments of a launch, as many as
// these hold; a group's elements are numbered in chunks of one tensor each, which the workgroups take in turn.
#include "internal.h"
#include "ops_device.h"

namespace focus {

namespace {

constexpr int kChunk = 8192;            // elements
constexpr int kNormParts = 2048;        // workgroups of a launch at most, each with one partial sum

// Tensors of a launch, as many as fit the 4 KB that a kernel's arguments have: 14 bytes each, or 22 with outputs of their own. 252
// tensors of 169 MB in 3 launches 122 us a pass; with 28 bytes each, in 7, 136.
template <bool OUT>
struct GradGroup {
    static constexpr int kMost = OUT ? 180 : 280;
    const void *g[kMost];
    void *out[OUT ? kMost : 1];
    uint32_t first[kMost + 1];          // first chunk of each tensor, and the number of chunks
    uint16_t tail[kMost];               // elements of its last chunk
    uint32_t bf16[(kMost + 31) / 32];   // a bit per tensor
    int count;
    __host__ __device__ uint32_t chunks() const { return first[count]; }
    __host__ __device__ int64_t n(int i) const { return (int64_t)(first[i + 1] - first[i] - 1) * kChunk + tail[i]; }
};
static_assert(sizeof(GradGroup<false>) <= 4032 && sizeof(GradGroup<true>) <= 4032, "the group and a kernel's other arguments fit 4 KB");

// The tensor of a chunk: the last one whose first chunk is not behind it
template <bool OUT>
__device__ __forceinline__ int tensor_of(const GradGroup<OUT> &a, uint32_t chunk) {
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

// Bound by memory: 14 tensors of 490 MB 113 us, 4.3 TB/s; 169 MB, some of them still in the caches, 28 us, 6 TB/s
__global__ void __launch_bounds__(256) grad_norm_kernel(GradGroup<false> a, double *__restrict__ part) {
    __shared__ double lds[4];
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < a.chunks(); c += gridDim.x) {
        const int i = tensor_of(a, c);
        const int64_t start = (int64_t)(c - a.first[i]) * kChunk;
        if (a.bf16[i / 32] >> (i % 32) & 1u) s += chunk_squares(static_cast<const uint16_t *>(a.g[i]), start, a.n(i));
        else s += chunk_squares(static_cast<const float *>(a.g[i]), start, a.n(i));
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

// `parts`: the partial sums, of which every workgroup forms the factor itself and the first one writes the norm (where `norm` is
// given); 0: the factor is there. Bound by memory: 490 MB read and written 176 us, 5.6 TB/s.
template <bool OUT>
__global__ void __launch_bounds__(256) grad_scale_kernel(GradGroup<OUT> a, const double *__restrict__ part, int64_t parts, double max_norm,
                                                         double *__restrict__ norm, const float2 *__restrict__ factor, uint32_t *flag) {
    float2 f;
    if (parts) {
        const double x = norm_of(part, parts);
        if (norm && blockIdx.x == 0 && threadIdx.x == 0) put_norm(x, norm, flag);
        f = factor_of(x, max_norm);
    } else {
        f = *factor;
    }
    for (uint32_t c = blockIdx.x; c < a.chunks(); c += gridDim.x) {
        const int i = tensor_of(a, c);
        void *const out = OUT ? a.out[OUT ? i : 0] : const_cast<void *>(a.g[i]);
        if (f.x == 1.0f && f.y == 1.0f && out == a.g[i]) continue;  // nothing to write
        const int64_t start = (int64_t)(c - a.first[i]) * kChunk;
        if (a.bf16[i / 32] >> (i % 32) & 1u)
            chunk_scale(static_cast<const uint16_t *>(a.g[i]), static_cast<uint16_t *>(out), start, a.n(i), f);
        else
            chunk_scale(static_cast<const float *>(a.g[i]), static_cast<float *>(out), start, a.n(i), f);
    }
}

// The group of the tensors from `first` on (without empty ones and, where `scaled`, those that are only counted); the index behind
// its last
template <bool OUT>
int64_t next_group(const GradTensor *t, int64_t first, int64_t count, bool scaled, GradGroup<OUT> &a) {
    a.count = 0, a.first[0] = 0;
    for (uint32_t &b : a.bf16) b = 0;
    int64_t i = first;
    for (; i < count && a.count < GradGroup<OUT>::kMost; i++) {
        if (t[i].n == 0 || (scaled && !t[i].out)) continue;
        const int k = a.count++;
        const int64_t chunks = (t[i].n + kChunk - 1) / kChunk;
        a.g[k] = t[i].grad, a.first[k + 1] = a.first[k] + (uint32_t)chunks, a.tail[k] = (uint16_t)(t[i].n - (chunks - 1) * kChunk);
        if constexpr (OUT) a.out[k] = t[i].out;
        if (t[i].dtype == kBF16) a.bf16[k / 32] |= 1u << (k % 32);
    }
    return i;
}

struct Norm {
    const double *part;
    int64_t parts;  // 0: the factor is there
    double max_norm, *out;
    const float2 *factor;
};
template <bool OUT>
hipError_t scale_all(const GradTensor *t, int64_t count, Norm x, uint32_t *flag, hipStream_t st) {
    GradGroup<OUT> a;
    for (int64_t i = 0; i < count;) {
        i = next_group(t, i, count, true, a);
        if (!a.count) continue;
        grad_scale_kernel<OUT><<<std::min<uint32_t>(a.chunks(), kNormParts), 256, 0, st>>>(a, x.part, x.parts, x.max_norm, x.out, x.factor, flag);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        x.out = nullptr;
    }
    return hipSuccess;
}

}  // namespace

static_assert(kMaxGradElems / kChunk * GradGroup<false>::kMost < (int64_t(1) << 32), "chunk numbers of a group are 32-bit");

size_t clip_grad_norm_ws(int64_t tensors) {
    return 2 * kWsHeader + (size_t)((tensors + GradGroup<false>::kMost - 1) / GradGroup<false>::kMost) * kNormParts * sizeof(double);
}

hipError_t launch_clip_grad_norm(const GradTensor *t, int64_t count, double max_norm, double *norm, uint32_t *flag, void *ws,
                                 hipStream_t st) {
    float2 *const factor = reinterpret_cast<float2 *>(static_cast<char *>(ws) + kWsHeader);
    double *const part = reinterpret_cast<double *>(static_cast<char *>(ws) + 2 * kWsHeader);
    int64_t parts = 0, scaled = 0;
    bool in_place = true;
    for (int64_t i = 0; i < count; i++) {
        if (t[i].n == 0 || !t[i].out) continue;
        scaled++;
        in_place = in_place && t[i].out == t[i].grad;
    }
    GradGroup<false> a;
    for (int64_t i = 0; i < count;) {
        i = next_group(t, i, count, false, a);
        if (!a.count) continue;
        const unsigned grid = std::min<uint32_t>(a.chunks(), kNormParts);
        grad_norm_kernel<<<grid, 256, 0, st>>>(a, part + parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        parts += grid;
    }
    // one or two scaling launches form the norm themselves: 1 us each, where a launch for it takes 4.6 and the way to the next
    const bool alone = scaled > 0 && scaled <= 2 * (in_place ? GradGroup<false>::kMost : GradGroup<true>::kMost);
    if (!alone) {
        grad_finish_kernel<<<1, 256, 0, st>>>(part, parts, max_norm, norm, factor, flag);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (scaled == 0) return hipSuccess;
    const Norm x{part, alone ? parts : 0, max_norm, norm, factor};
    return in_place ? scale_all<false>(t, count, x, flag, st) : scale_all<true>(t, count, x, flag, st);
}

}  // namespace focus
