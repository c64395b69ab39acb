// extern "C" entry points of libfocus: host-side argument checks, workspace layout and dispatch.
// Every check runs before anything is launched; a failed check launches nothing.
#include "../../include/focus.h"
#include "focus_device.h"
#include "gemm_common.h"
#include "internal.h"

#include <cmath>
#include <initializer_list>
#include <mutex>
#include <new>

using namespace focus;

namespace {

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxElems = int64_t(1) << 46;

focus_status check_q(const focus_qconfig *q) {
    if (!q) return FOCUS_ERR_NULL;
    if (q->format != FOCUS_MXFP4 && q->format != FOCUS_NVFP4) return FOCUS_ERR_CONFIG;
    const int B = block_of(q->format), sb = q->sub_block;
    if (!(sb == 2 || sb == 4 || sb == 8 || sb == 16 || sb == 32) || B % sb != 0) return FOCUS_ERR_CONFIG;
    if (q->ste_clip != 0 && q->ste_clip != 1) return FOCUS_ERR_CONFIG;
    if (q->scale_layout != FOCUS_SCALES_ROW_MAJOR && q->scale_layout != FOCUS_SCALES_BLOCK_MAJOR) return FOCUS_ERR_CONFIG;
    if (q->e8m0_rounding != FOCUS_E8M0_CEIL && q->e8m0_rounding != FOCUS_E8M0_FLOOR) return FOCUS_ERR_CONFIG;
    if (q->e8m0_rounding == FOCUS_E8M0_FLOOR && q->format != FOCUS_MXFP4) return FOCUS_ERR_CONFIG;
    if (q->code_layout != FOCUS_CODES_ROW_MAJOR && q->code_layout != FOCUS_CODES_K_SLAB) return FOCUS_ERR_CONFIG;
    return FOCUS_OK;
}

int slab_of(const focus_qconfig *q) { return q->code_layout == FOCUS_CODES_K_SLAB ? 1 : 0; }

// codes in K-slabs of 128 elements need whole slabs
focus_status check_code_layout(const focus_qconfig *q, const void *codes, int64_t K) {
    return codes && slab_of(q) && K % 128 != 0 ? FOCUS_ERR_SHAPE : FOCUS_OK;
}

int floor_of(const focus_qconfig *q) { return q->e8m0_rounding == FOCUS_E8M0_FLOOR ? 1 : 0; }

bool dtype_ok(int d) { return d == FOCUS_F32 || d == FOCUS_BF16; }

focus_status check_rows_k(int64_t rows, int64_t K, int B) {
    if (rows < 0 || K < 0 || rows > kMaxDim || K > kMaxDim) return FOCUS_ERR_SHAPE;
    if (K % B != 0) return FOCUS_ERR_SHAPE;
    if (rows > 0 && K > 0 && rows > kMaxElems / K) return FOCUS_ERR_SHAPE;
    return FOCUS_OK;
}

focus_status check_ws(const void *ws, size_t bytes, size_t need) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) % 256) != 0 || bytes < need) return FOCUS_ERR_WORKSPACE;
    return FOCUS_OK;
}

// tensors are read and written with 16-byte vector accesses
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool all_aligned(std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if (p && !aligned16(p)) return false;
    return true;
}

uint32_t *flag_of(void *ws) { return reinterpret_cast<uint32_t *>(ws); }
float *partials_of(void *ws) { return reinterpret_cast<float *>(reinterpret_cast<char *>(ws) + kWsHeader); }

focus_status hip_status(hipError_t e) { return e == hipSuccess ? FOCUS_OK : FOCUS_ERR_HIP; }

size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// The sizes of the forward and of the input gradient do not fall as M grows (a workspace for the largest batch serves
// every smaller one), though their plans take smaller tiles and more splits for fewer tokens.

// Column sums of every tile row and of the whole: rows of 64 at most, or of 32 where fp32 outputs have fewer than 256
// tiles of 64 x 64, whose sums are fewer than 2 x 256 x 64.
size_t fwd_ws(int64_t M, int64_t N) {
    const int64_t rows64 = (M + 63) / 64 * N, rows32 = std::min<int64_t>((M + 31) / 32 * N, 2 * kMfmaConcurrentWgs * kF32Tile);
    return kWsHeader + (size_t)(std::max(rows64, rows32) + N) * sizeof(double);
}

// fp32: the transposed W_hat and the forward's sums; bf16: the splits' sums, as many as any M up to this one takes
size_t dx_ws(int64_t M, int64_t N, int64_t K) {
    const size_t transposed = kWsHeader + round256((size_t)N * (size_t)K * sizeof(float)) + fwd_ws(M, K);
    const int64_t splits = dx_max_splits(N), mk = M * K;
    const int64_t sums = splits > 1 ? (mk > kDxSums / splits ? kDxSums : splits * mk) : 0;
    return std::max(transposed, kWsHeader + (size_t)sums * sizeof(float));
}

size_t bwd_ws(int fmt, int sb, int64_t M, int64_t N, int64_t K) {
    // with G_out there is one split, the least there is
    return std::max(plan_bwd(kF32, fmt, sb, M, N, K, false).ws_bytes, plan_bwd(kBF16, fmt, sb, M, N, K, false).ws_bytes);
}

#define FOCUS_TRY(x)                  \
    do {                              \
        focus_status s_ = (x);        \
        if (s_ != FOCUS_OK) return s_; \
    } while (0)

// argument checks shared by the two entry points of the forward from packed MXFP4 operands
focus_status check_fwd_mx_args(const uint8_t *X_codes, const uint8_t *X_scales, const uint8_t *W_codes,
                               const uint8_t *W_scales, int64_t M, int64_t N, int64_t K, const void *Y_ref,
                               const void *dY, const double *loss_out) {
    if (!X_codes || !X_scales || !W_codes || !W_scales || !dY) return FOCUS_ERR_NULL;
    if (Y_ref && !loss_out) return FOCUS_ERR_NULL;
    if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return FOCUS_ERR_SHAPE;
    if (K % 128 != 0 || N % 8 != 0 || M % 4 != 0) return FOCUS_ERR_SHAPE;
    if ((M > 0 && K > kMaxElems / M) || (N > 0 && K > kMaxElems / N) || (M > 0 && N > kMaxElems / M))
        return FOCUS_ERR_SHAPE;
    if (!all_aligned({X_codes, W_codes, Y_ref, dY})) return FOCUS_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(X_scales) | reinterpret_cast<uintptr_t>(W_scales)) & 3u) return FOCUS_ERR_SHAPE;
    return FOCUS_OK;
}

// ---- fixed device scratch of the allocation-free forward ---------------------------------------
// 32 MiB per GPU: the kWsHeader bytes the workspace layout skips, ceil(M / 256) x N partial sums of
// D^2 (fp64) and, when the caller passes no col_sq, N column sums. Every hidden-2560 layer at 65,536
// tokens fits (at most 20 MB). (Where the forward takes 128 x 128 tiles there are at most 512 of them,
// 0.5 MB of sums.)
constexpr size_t kNoAllocScratchBytes = size_t(32) << 20;

size_t noalloc_fwd_scratch_bytes(int64_t M, int64_t N, bool have_col_sq) {
    const size_t mtiles = (size_t)((M + kMfmaTileM - 1) / kMfmaTileM);
    return kWsHeader + (mtiles * (size_t)N + (have_col_sq ? 0 : (size_t)N)) * sizeof(double);
}

// ---- operators around the linears ---------------------------------------------------------------
focus_status check_norm_shape(int64_t T, int64_t C) {
    return T < 0 || C < 0 || T > kMaxDim || C > (int64_t(1) << 24) ? FOCUS_ERR_SHAPE : FOCUS_OK;
}

focus_status check_logits(int64_t T, int64_t V) {
    return T < 0 || V < 1 || T > kMaxDim || V > kMaxDim || (T > 0 && V > kMaxElems / T) ? FOCUS_ERR_SHAPE : FOCUS_OK;
}

bool aligned_to(std::initializer_list<const void *> ps, uintptr_t bytes) {
    for (const void *p : ps)
        if (reinterpret_cast<uintptr_t>(p) % bytes) return false;
    return true;
}

bool logits_aligned(const void *Z, int dtype) { return aligned_to({Z}, dtype == FOCUS_BF16 ? 2 : 4); }

// checks the shapes of an attention call and fills them in (the pointers stay unset)
focus_status attention_args(const focus_attention_config *cfg, int64_t Tq, int64_t Tk, int64_t n_seq, AttnArgs &a) {
    if (!cfg) return FOCUS_ERR_NULL;
    if (cfg->causal != 0 && cfg->causal != 1) return FOCUS_ERR_CONFIG;
    if (!std::isfinite(cfg->scale) || cfg->reserved != 0) return FOCUS_ERR_CONFIG;
    const int64_t hq = cfg->heads_q, hkv = cfg->heads_kv, d = cfg->head_dim;
    if (hq < 1 || hkv < 1 || hq > 65535 || hq % hkv != 0 || d < 8 || d > 128 || d % 8 != 0) return FOCUS_ERR_SHAPE;
    constexpr int64_t kMaxTokens = int64_t(1) << 30;
    if (Tq < 0 || Tk < 0 || n_seq < 0 || Tq > kMaxTokens || Tk > kMaxTokens || n_seq > (int64_t(1) << 24)) return FOCUS_ERR_SHAPE;
    a = AttnArgs{};
    const int64_t rq = hq * d, rk = hkv * d;
    const int64_t given[6] = {cfg->q_stride, cfg->k_stride, cfg->v_stride, cfg->dq_stride, cfg->dk_stride, cfg->dv_stride};
    int64_t *const out[6] = {&a.q_stride, &a.k_stride, &a.v_stride, &a.dq_stride, &a.dk_stride, &a.dv_stride};
    for (int i = 0; i < 6; i++) {
        const int64_t row = i % 3 == 0 ? rq : rk;
        if (given[i] != 0 && (given[i] < row || given[i] > (int64_t(1) << 24))) return FOCUS_ERR_SHAPE;
        *out[i] = given[i] ? given[i] : row;
    }
    // a launch's work-items in x (256 per workgroup: 32 tokens in fp32, 128 rows of a key-value head in bf16) stay below 2^32
    constexpr int64_t kMaxWgs = (int64_t(1) << 24) - 1;
    const int64_t most = std::max(Tq, Tk);
    if (most / 32 + n_seq > kMaxWgs || (Tq * (hq / hkv) / 128 + n_seq) * hkv > kMaxWgs || (Tk / 128 + n_seq) * hkv > kMaxWgs)
        return FOCUS_ERR_SHAPE;
    a.Tq = Tq, a.Tk = Tk, a.n_seq = (int)n_seq;
    a.Hq = (int)hq, a.Hkv = (int)hkv, a.D = (int)d, a.causal = cfg->causal, a.scale = cfg->scale;
    return FOCUS_OK;
}

// 16-byte rows
bool strides_ok(const AttnArgs &a, int dtype) {
    const int64_t e = dtype == FOCUS_BF16 ? 8 : 4;
    return (a.q_stride | a.k_stride | a.v_stride | a.dq_stride | a.dk_stride | a.dv_stride) % e == 0;
}

// The tokens of an attention tensor in memory: `n` rows of `width` bytes, `stride` apart
struct Rows {
    const void *base;
    int64_t n, stride, width;
};

// Whether two of them share memory. Slices of one fused tensor, whose rows interleave at one stride, need not; rows that
// interleave at different strides are taken to.
bool overlap(Rows a, Rows b) {
    if (a.n == 0 || b.n == 0) return false;
    const int64_t off = (int64_t)((intptr_t)a.base - (intptr_t)b.base);  // of a's row 0 from b's
    if (off >= (b.n - 1) * b.stride + b.width || -off >= (a.n - 1) * a.stride + a.width) return false;
    if (a.n == 1) a.stride = b.stride;
    if (b.n == 1) b.stride = a.stride;
    if (a.stride != b.stride) return true;
    // rows i of a and j of b share memory where -a.width < off + (i - j) stride < b.width: the largest i - j below that bound
    const int64_t most = b.width - 1 - off, up = most >= 0 ? most / a.stride : -((-most + a.stride - 1) / a.stride);
    const int64_t diff = std::min(up, a.n - 1);
    return diff >= -(b.n - 1) && off + diff * a.stride > -a.width;
}

struct AttnRows {
    Rows q, k, v, O, dO, dq, dk, dv;
    AttnRows(const AttnArgs &a, int dtype) {
        const int64_t e = dtype == FOCUS_BF16 ? 2 : 4, wq = (int64_t)a.Hq * a.D * e, wk = (int64_t)a.Hkv * a.D * e;
        q = {a.q, a.Tq, a.q_stride * e, wq}, O = {a.O, a.Tq, wq, wq}, dO = {a.dO, a.Tq, wq, wq}, dq = {a.dq, a.Tq, a.dq_stride * e, wq};
        k = {a.k, a.Tk, a.k_stride * e, wk}, v = {a.v, a.Tk, a.v_stride * e, wk};
        dk = {a.dk, a.Tk, a.dk_stride * e, wk}, dv = {a.dv, a.Tk, a.dv_stride * e, wk};
    }
};

// ---- the rest of a training step ----------------------------------------------------------------
struct Span {
    const void *p;
    int64_t bytes;
};

bool meet(Span a, Span b) {
    if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

// Whether an output shares memory with another output or an input; `in_place`: an output may stand in an input's place
bool clash(std::initializer_list<Span> outs, std::initializer_list<Span> ins, bool in_place) {
    for (const Span *o = outs.begin(); o != outs.end(); o++) {
        for (const Span *q = o + 1; q != outs.end(); q++)
            if (meet(*o, *q)) return true;
        for (const Span &i : ins)
            if (meet(*o, i) && !(in_place && o->p == i.p && o->bytes == i.bytes)) return true;
    }
    return false;
}

focus_status check_sandwich(const focus_sandwich_config *cfg, int dtype, int w_dtype, int64_t T, int64_t C, const void *gate) {
    if (!cfg) return FOCUS_ERR_NULL;
    if (cfg->kind != FOCUS_NORM_LAYER && cfg->kind != FOCUS_NORM_RMS) return FOCUS_ERR_CONFIG;
    if (cfg->gate != FOCUS_GATE_NONE && cfg->gate != FOCUS_GATE_FEATURE && cfg->gate != FOCUS_GATE_TOKEN) return FOCUS_ERR_CONFIG;
    if (!std::isfinite(cfg->eps) || cfg->eps < 0.f || !std::isfinite(cfg->residual_scale)) return FOCUS_ERR_CONFIG;
    if (cfg->gate == FOCUS_GATE_NONE && gate) return FOCUS_ERR_CONFIG;
    if (!dtype_ok(dtype) || !dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_norm_shape(T, C));
    if (T > 0 && C > kMaxElems / T) return FOCUS_ERR_SHAPE;
    return FOCUS_OK;
}

constexpr int64_t kCeMaxRows = int64_t(1) << 24, kCeMaxK = int64_t(1) << 20;
focus_status check_linear_ce(int64_t T, int64_t V, int64_t K, int dtype = FOCUS_BF16) {
    const int64_t most = dtype == FOCUS_BF16 ? kCeMaxRows : kCeMaxRows / 2;  // 32 rows of the fp32 D's transpose stay below 2 GB
    return T < 0 || V < 1 || K < 1 || T > most || V > kCeMaxRows || K > kCeMaxK ? FOCUS_ERR_SHAPE : FOCUS_OK;
}

constexpr int64_t kMaxGradTensors = int64_t(1) << 20;
static_assert(sizeof(focus_grad_tensor) == sizeof(GradTensor), "the ABI's struct is the launcher's");

Span grad_span(const focus_grad_tensor &t, const void *p) { return Span{p, t.n * (t.dtype == FOCUS_BF16 ? 2 : 4)}; }

// An output in a place of its own or its gradient's. Tensors that lie in rising order, as a rule, need one pass; for others
// their outputs are sorted by address (`order`: scratch of n indices).
focus_status check_grad_places(const focus_grad_tensor *t, int64_t n, int32_t *order) {
    int64_t k = 0;
    for (int64_t i = 0; i < n; i++) {
        if (t[i].n == 0 || !t[i].out) continue;
        const Span o = grad_span(t[i], t[i].out), g = grad_span(t[i], t[i].grad);
        if (o.p != g.p && meet(o, g)) return FOCUS_ERR_SHAPE;
        order[k++] = (int32_t)i;
    }
    auto less = [&](int32_t a, int32_t b) { return (uintptr_t)t[a].out < (uintptr_t)t[b].out; };
    if (!std::is_sorted(order, order + k, less)) std::sort(order, order + k, less);
    for (int64_t i = 1; i < k; i++)
        if (meet(grad_span(t[order[i - 1]], t[order[i - 1]].out), grad_span(t[order[i]], t[order[i]].out))) return FOCUS_ERR_SHAPE;
    for (int64_t i = 0; i < n; i++) {
        if (t[i].n == 0) continue;
        const Span g = grad_span(t[i], t[i].grad);
        // the outputs are disjoint: the first one that ends behind the gradient's start is the only one to look at, as far as
        // it is not its own
        const int32_t *at = std::partition_point(order, order + k, [&](int32_t j) {
            return (uintptr_t)t[j].out + (uintptr_t)grad_span(t[j], t[j].out).bytes <= (uintptr_t)g.p;
        });
        for (; at != order + k && meet(grad_span(t[*at], t[*at].out), g); at++)
            if (*at != i) return FOCUS_ERR_SHAPE;
    }
    return FOCUS_OK;
}

focus_status check_ends(const int32_t *cu_q, const int32_t *cu_k, int64_t n_seq) {
    if (!cu_q != !cu_k || (!cu_q && n_seq != 1)) return FOCUS_ERR_NULL;
    return aligned_to({cu_q, cu_k}, 4) ? FOCUS_OK : FOCUS_ERR_SHAPE;
}

}  // namespace

// One copy per GPU, held until the process ends, shared by every call on that GPU (calls that
// overlap on one GPU race). In host code this name stands for a host-side shadow, not a device
// address: only the address scratch_address() looks up may reach a kernel or a copy.
static __device__ __align__(256) double scratch[kNoAllocScratchBytes / sizeof(double)];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void *g_scratch_ptr[kMaxDevices];

// Device address of `scratch` on the current device, looked up once per device with that device
// current (each GPU holds its own copy at its own address).
hipError_t scratch_address(void **out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void *p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return hipSuccess;
}

}  // namespace

extern "C" {

size_t focus_workspace_size(int call, const focus_qconfig *q, int64_t M, int64_t N, int64_t K) {
    if (call == FOCUS_CALL_ADAMW) return kWsHeader;  // the domain flag only; q may be NULL
    if (call == FOCUS_CALL_RECON_GEMM_DX) {            // q may be NULL
        if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return 0;
        return dx_ws(M, N, K);
    }
    if (call == FOCUS_CALL_KL_TOP) {  // M = tokens; q may be NULL
        if (M < 0 || M > kMaxDim) return 0;
        return kWsHeader + round256((size_t)M * sizeof(double)) + sizeof(double);
    }
    if (call == FOCUS_CALL_NORM_FWD || call == FOCUS_CALL_NORM_BWD) {  // the operators around the linears: q may be NULL
        if (check_norm_shape(M, K) != FOCUS_OK) return 0;
        return call == FOCUS_CALL_NORM_FWD ? kWsHeader : norm_bwd_ws(M, K);
    }
    if (call == FOCUS_CALL_TOKEN_LOGPROBS) {
        if (check_logits(M, N) != FOCUS_OK || K < 0 || K > FOCUS_MAX_TOP) return 0;
        return logprobs_ws(M, N, (int)K);
    }
    if (call == FOCUS_CALL_TOKEN_LOGPROBS_BWD) return check_logits(M, N) == FOCUS_OK ? kWsHeader : 0;
    if (call == FOCUS_CALL_SANDWICH_NORM_FWD || call == FOCUS_CALL_SANDWICH_NORM_BWD) {
        if (check_norm_shape(M, K) != FOCUS_OK || (M > 0 && K > kMaxElems / M)) return 0;
        return call == FOCUS_CALL_SANDWICH_NORM_FWD ? kWsHeader : sandwich_bwd_ws(M, K);
    }
    if (call == FOCUS_CALL_LINEAR_CE_FWD || call == FOCUS_CALL_LINEAR_CE_BWD) {
        if (check_linear_ce(M, N, K) != FOCUS_OK) return 0;
        return call == FOCUS_CALL_LINEAR_CE_FWD ? linear_ce_fwd_ws(M, N, K) : linear_ce_bwd_ws(M, N, K);
    }
    if (call == FOCUS_CALL_CLIP_GRAD_NORM) return M < 0 || M > kMaxGradTensors ? 0 : clip_grad_norm_ws(M);
    if (check_q(q) != FOCUS_OK) return 0;
    const int B = block_of(q->format);
    switch (call) {
        case FOCUS_CALL_SCALES_INIT:
        case FOCUS_CALL_FAKEQUANT_FWD:
        case FOCUS_CALL_FAKEQUANT_ACT_BWD:
            return kWsHeader + (kAbsmaxParts + 64) * sizeof(float);  // partial maxima + tensor scale slot
        case FOCUS_CALL_FAKEQUANT_BWD:
        case FOCUS_CALL_EXPORT_PACKED:
        case FOCUS_CALL_FAKEQUANT_WEIGHTS:
            return kWsHeader;
        case FOCUS_CALL_RECON_GEMM_FWD:
            if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return 0;
            return fwd_ws(M, N);
        case FOCUS_CALL_RECON_GEMM_BWD:
            if (check_rows_k(N, K, B) != FOCUS_OK || M < 0 || M > kMaxDim) return 0;
            return bwd_ws(q->format, q->sub_block, M, N, K);
        default:
            return 0;
    }
}

focus_status focus_scales_init(const focus_qconfig *q, const void *W, int w_dtype, int64_t N, int64_t K,
                               float *s_fp, float *c, float *alpha_out, void *ws, size_t ws_bytes,
                               focus_stream stream) {
    FOCUS_TRY(check_q(q));
    if (!W || !s_fp || !c) return FOCUS_ERR_NULL;
    if (q->format == FOCUS_NVFP4 && !alpha_out) return FOCUS_ERR_NULL;
    if (!dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(N, K, block_of(q->format)));
    if (!all_aligned({W})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_SCALES_INIT, q, 0, N, K)));
    if (N == 0 || K == 0) return FOCUS_OK;
    return hip_status(launch_scales_init(q->format, w_dtype, W, N, K, s_fp, c, q->sub_block, floor_of(q), alpha_out,
                                         partials_of(ws), (hipStream_t)stream));
}

focus_status focus_fakequant_fwd(const focus_qconfig *q, const void *X, int x_dtype, int64_t rows, int64_t K,
                                 const float *s_fp, const float *c, const float *alpha, void *X_hat,
                                 int xhat_dtype, uint8_t *codes_opt, uint8_t *scale_bytes_opt,
                                 float *alpha_out_opt, void *ws, size_t ws_bytes, focus_stream stream) {
    FOCUS_TRY(check_q(q));
    // X_hat may be left out when codes are asked for; an empty tensor (rows == 0) may come as NULL
    if (rows != 0 && (!X || (!X_hat && !codes_opt))) return FOCUS_ERR_NULL;
    const bool weight_mode = s_fp != nullptr;
    if (weight_mode && q->format == FOCUS_NVFP4 && !alpha) return FOCUS_ERR_NULL;
    if (!weight_mode && (c || alpha)) return FOCUS_ERR_CONFIG;
    if (!dtype_ok(x_dtype) || !dtype_ok(xhat_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(rows, K, block_of(q->format)));
    FOCUS_TRY(check_code_layout(q, codes_opt, K));
    if (!all_aligned({X, X_hat, codes_opt})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_FAKEQUANT_FWD, q, 0, rows, K)));
    if (rows == 0 || K == 0) return FOCUS_OK;
    hipStream_t st = (hipStream_t)stream;
    if (weight_mode)
        return hip_status(launch_fq_weight(q->format, x_dtype, xhat_dtype, X, rows, K, s_fp, c, q->sub_block,
                                           alpha, floor_of(q), X_hat, codes_opt, scale_bytes_opt, q->scale_layout,
                                           slab_of(q), flag_of(ws), st));
    return hip_status(launch_fq_act(q->format, x_dtype, xhat_dtype, X, rows, K, X_hat, codes_opt,
                                    scale_bytes_opt, q->scale_layout, slab_of(q), floor_of(q), alpha_out_opt, partials_of(ws),
                                    flag_of(ws), st));
}

focus_status focus_fakequant_bwd(const focus_qconfig *q, const float *G, int64_t N, int64_t K, const void *W,
                                 int w_dtype, const float *s_fp, const float *c, const float *alpha,
                                 float *grad_s, float *grad_c, void *ws, size_t ws_bytes, focus_stream stream) {
    FOCUS_TRY(check_q(q));
    if (!G || !W || !s_fp || !grad_s || !grad_c) return FOCUS_ERR_NULL;
    if (q->format == FOCUS_NVFP4 && !alpha) return FOCUS_ERR_NULL;
    if (!dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(N, K, block_of(q->format)));
    if (!all_aligned({G, W})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_FAKEQUANT_BWD, q, 0, N, K)));
    if (N == 0 || K == 0) return FOCUS_OK;
    return hip_status(launch_fq_bwd(q->format, w_dtype, G, N, K, W, s_fp, c, q->sub_block, alpha, q->ste_clip,
                                    floor_of(q), grad_s, grad_c, flag_of(ws), (hipStream_t)stream));
}

focus_status focus_recon_gemm_fwd(const void *X_hat, const void *W_hat, int op_dtype, int64_t M, int64_t N,
                                  int64_t K, const void *Y_ref, void *dY, double *loss_out, double *col_sq_opt,
                                  void *ws, size_t ws_bytes, focus_stream stream) {
    if (!X_hat || !W_hat || !dY) return FOCUS_ERR_NULL;
    if (Y_ref && !loss_out) return FOCUS_ERR_NULL;
    if (!dtype_ok(op_dtype)) return FOCUS_ERR_DTYPE;
    if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return FOCUS_ERR_SHAPE;
    if (K % 16 != 0) return FOCUS_ERR_SHAPE;
    if ((M > 0 && K > kMaxElems / M) || (N > 0 && K > kMaxElems / N) || (M > 0 && N > kMaxElems / M))
        return FOCUS_ERR_SHAPE;
    if (!all_aligned({X_hat, W_hat, Y_ref, dY})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, fwd_ws(M, N)));
    if (M == 0 || N == 0) return FOCUS_OK;
    const FwdPlan p = plan_fwd(op_dtype, M, N, K);
    return hip_status(launch_recon_fwd(p, op_dtype, X_hat, W_hat, M, N, K, Y_ref, dY, loss_out, col_sq_opt, ws,
                                       (hipStream_t)stream));
}

focus_status focus_recon_gemm_fwd_mxfp4(const uint8_t *X_codes, const uint8_t *X_scales, const uint8_t *W_codes,
                                        const uint8_t *W_scales, int64_t M, int64_t N, int64_t K,
                                        const void *Y_ref, void *dY, double *loss_out, double *col_sq_opt,
                                        void *ws, size_t ws_bytes, focus_stream stream) {
    FOCUS_TRY(check_fwd_mx_args(X_codes, X_scales, W_codes, W_scales, M, N, K, Y_ref, dY, loss_out));
    FOCUS_TRY(check_ws(ws, ws_bytes, fwd_ws(M, N)));
    if (M == 0 || N == 0) return FOCUS_OK;
    if (!mfma_fwd_mx_supported(M, N, K)) return FOCUS_ERR_SHAPE;
    return hip_status(launch_recon_fwd_mx(X_codes, X_scales, W_codes, W_scales, M, N, K, Y_ref, dY, loss_out,
                                          col_sq_opt, ws, (hipStream_t)stream));
}

focus_status focus_recon_gemm_fwd_mxfp4_noalloc(const uint8_t *X_codes, const uint8_t *X_scales,
                                                const uint8_t *W_codes, const uint8_t *W_scales, int64_t M, int64_t N,
                                                int64_t K, const void *Y_ref, void *dY, double *loss_out,
                                                double *col_sq_opt, focus_stream stream) {
    FOCUS_TRY(check_fwd_mx_args(X_codes, X_scales, W_codes, W_scales, M, N, K, Y_ref, dY, loss_out));
    if (noalloc_fwd_scratch_bytes(M, N, col_sq_opt != nullptr) > kNoAllocScratchBytes) return FOCUS_ERR_SCRATCH;
    if (M == 0 || N == 0) return FOCUS_OK;
    if (!mfma_fwd_mx_supported(M, N, K)) return FOCUS_ERR_SHAPE;
    void *ptr = nullptr;
    if (scratch_address(&ptr) != hipSuccess) return FOCUS_ERR_HIP;
    // the scratch takes the place of the workspace: its first kWsHeader bytes are left unused, then
    // the per-(m-tile, column) partial sums and, without col_sq_opt, the column sums; the kernels
    // write all of it before it is read, so nothing is cleared
    return hip_status(launch_recon_fwd_mx(X_codes, X_scales, W_codes, W_scales, M, N, K, Y_ref, dY, loss_out,
                                          col_sq_opt, ptr, (hipStream_t)stream));
}

focus_status focus_recon_gemm_bwd(const focus_qconfig *q, const void *dY, const void *X_hat, int op_dtype,
                                  int64_t M, int64_t N, int64_t K, const void *W, int w_dtype,
                                  const float *s_fp, const float *c, const float *alpha, float *grad_s,
                                  float *grad_c, float *G_out_opt, void *ws, size_t ws_bytes,
                                  focus_stream stream) {
    FOCUS_TRY(check_q(q));
    // with no tokens (M == 0) the token operands are never read and may be NULL; the gradients are zero
    if ((M != 0 && (!dY || !X_hat)) || !W || !s_fp || !grad_s || !grad_c) return FOCUS_ERR_NULL;
    if (q->format == FOCUS_NVFP4 && !alpha) return FOCUS_ERR_NULL;
    if (!dtype_ok(op_dtype) || !dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(N, K, block_of(q->format)));
    if (M < 0 || M > kMaxDim || (M > 0 && K > kMaxElems / M) || (M > 0 && N > kMaxElems / M))
        return FOCUS_ERR_SHAPE;
    if (!all_aligned({dY, X_hat, W, G_out_opt})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, bwd_ws(q->format, q->sub_block, M, N, K)));
    if (N == 0 || K == 0) return FOCUS_OK;
    const BwdPlan p = plan_bwd(op_dtype, q->format, q->sub_block, M, N, K, G_out_opt != nullptr);
    return hip_status(launch_recon_bwd(p, op_dtype, q->format, q->sub_block, q->ste_clip, floor_of(q), dY, X_hat, M, N, K, W,
                                       w_dtype, s_fp, c, alpha, grad_s, grad_c, G_out_opt, ws, flag_of(ws),
                                       (hipStream_t)stream));
}

focus_status focus_recon_gemm_bwd_mxfp4(const focus_qconfig *q, const void *dY, const uint8_t *X_codes,
                                        const uint8_t *X_scales, int64_t M, int64_t N, int64_t K, const void *W,
                                        int w_dtype, const float *s_fp, const float *c, float *grad_s,
                                        float *grad_c, void *ws, size_t ws_bytes, focus_stream stream) {
    FOCUS_TRY(check_q(q));
    if (q->format != FOCUS_MXFP4) return FOCUS_ERR_CONFIG;
    // with no tokens (M == 0) the token operands are never read and may be NULL; the gradients are zero
    if ((M != 0 && (!dY || !X_codes || !X_scales)) || !W || !s_fp || !grad_s || !grad_c) return FOCUS_ERR_NULL;
    if (!dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(N, K, 32));
    if (M < 0 || M > kMaxDim || (M > 0 && K > kMaxElems / M) || (M > 0 && N > kMaxElems / M))
        return FOCUS_ERR_SHAPE;
    if (M % 4 != 0 || N % 8 != 0) return FOCUS_ERR_SHAPE;
    if (!all_aligned({dY, X_codes, W})) return FOCUS_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(X_scales) & 3u) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, bwd_ws(q->format, q->sub_block, M, N, K)));
    if (N == 0 || K == 0) return FOCUS_OK;
    if (!mfma_bwd_mx_supported(M, N, K)) return FOCUS_ERR_SHAPE;
    const BwdPlan p = plan_bwd(FOCUS_BF16, q->format, q->sub_block, M, N, K, false);
    return hip_status(launch_recon_bwd_mx(p, q->sub_block, q->ste_clip, floor_of(q), dY, X_codes, X_scales, M, N, K,
                                          W, w_dtype, s_fp, c, grad_s, grad_c, ws, flag_of(ws), (hipStream_t)stream));
}

focus_status focus_export_packed(const focus_qconfig *q, const void *W, int w_dtype, int64_t N, int64_t K,
                                 const float *s_fp, const float *c, const float *alpha, uint8_t *packed,
                                 uint8_t *scale_bytes, void *ws, size_t ws_bytes, focus_stream stream) {
    FOCUS_TRY(check_q(q));
    if (!W || !s_fp || !packed || !scale_bytes) return FOCUS_ERR_NULL;
    if (q->format == FOCUS_NVFP4 && !alpha) return FOCUS_ERR_NULL;
    if (!dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(N, K, block_of(q->format)));
    FOCUS_TRY(check_code_layout(q, packed, K));
    if (!all_aligned({W, packed})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_EXPORT_PACKED, q, 0, N, K)));
    if (N == 0 || K == 0) return FOCUS_OK;
    return hip_status(launch_fq_weight(q->format, w_dtype, w_dtype, W, N, K, s_fp, c, q->sub_block, alpha,
                                       floor_of(q), nullptr, packed, scale_bytes, q->scale_layout, slab_of(q), flag_of(ws),
                                       (hipStream_t)stream));
}

focus_status focus_fakequant_weights(const focus_qconfig *q, int w_dtype, int what_dtype,
                                     const focus_weight_layer *layers, int n_layers, void *ws, size_t ws_bytes,
                                     focus_stream stream) {
    FOCUS_TRY(check_q(q));
    if (n_layers < 0 || n_layers > FOCUS_MAX_WEIGHT_LAYERS) return FOCUS_ERR_SHAPE;
    if (n_layers > 0 && !layers) return FOCUS_ERR_NULL;
    if (!dtype_ok(w_dtype) || !dtype_ok(what_dtype)) return FOCUS_ERR_DTYPE;
    WeightLayer L[FOCUS_MAX_WEIGHT_LAYERS];
    for (int i = 0; i < n_layers; i++) {
        const focus_weight_layer &l = layers[i];
        if (l.rows != 0 && (!l.W || !l.s_fp || (!l.W_hat && !l.codes))) return FOCUS_ERR_NULL;
        if (l.rows != 0 && q->format == FOCUS_NVFP4 && !l.alpha) return FOCUS_ERR_NULL;
        FOCUS_TRY(check_rows_k(l.rows, l.K, block_of(q->format)));
        FOCUS_TRY(check_code_layout(q, l.codes, l.K));
        if (!all_aligned({l.W, l.W_hat, l.codes})) return FOCUS_ERR_SHAPE;
        L[i] = WeightLayer{l.W, l.rows, l.K, l.s_fp, l.c, q->format == FOCUS_NVFP4 ? l.alpha : nullptr,
                           l.W_hat, l.codes, l.scale_bytes};
    }
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_FAKEQUANT_WEIGHTS, q, 0, 0, 0)));
    if (n_layers == 0) return FOCUS_OK;
    return hip_status(launch_fq_weight_group(q->format, w_dtype, what_dtype, L, n_layers, q->sub_block, floor_of(q),
                                             q->scale_layout, slab_of(q), flag_of(ws), (hipStream_t)stream));
}

focus_status focus_recon_gemm_dx(const void *dY, const void *W_hat, int op_dtype, int64_t M, int64_t N, int64_t K,
                                 void *dX_hat, void *ws, size_t ws_bytes, focus_stream stream) {
    if (!dX_hat || (N > 0 && (!dY || !W_hat))) return FOCUS_ERR_NULL;  // empty operands may be NULL
    if (!dtype_ok(op_dtype)) return FOCUS_ERR_DTYPE;
    if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return FOCUS_ERR_SHAPE;
    if (N % 16 != 0) return FOCUS_ERR_SHAPE;  // the contraction runs over N
    if ((M > 0 && K > kMaxElems / M) || (N > 0 && K > kMaxElems / N) || (M > 0 && N > kMaxElems / M))
        return FOCUS_ERR_SHAPE;
    if (!all_aligned({dY, W_hat, dX_hat})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, dx_ws(M, N, K)));
    if (M == 0 || K == 0) return FOCUS_OK;
    const hipStream_t st = (hipStream_t)stream;
    if (N == 0) {  // an empty sum: dX_hat = 0
        const size_t esz = op_dtype == FOCUS_BF16 ? 2 : 4;
        return hip_status(launch_zero_fill(dX_hat, (size_t)M * (size_t)K * esz, st));
    }
    return hip_status(launch_recon_dx(plan_dx(op_dtype, M, N, K), op_dtype, dY, W_hat, M, N, K, dX_hat, ws, st));
}

focus_status focus_fakequant_act_bwd(const focus_qconfig *q, const void *X, int x_dtype, int64_t rows, int64_t K,
                                     const void *dX_hat, int g_dtype, void *dX, void *ws, size_t ws_bytes,
                                     focus_stream stream) {
    FOCUS_TRY(check_q(q));
    if (!X || !dX_hat || !dX) return FOCUS_ERR_NULL;
    if (!dtype_ok(x_dtype) || !dtype_ok(g_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_rows_k(rows, K, block_of(q->format)));
    if (!all_aligned({X, dX_hat, dX})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_FAKEQUANT_ACT_BWD, q, 0, rows, K)));
    if (rows == 0 || K == 0) return FOCUS_OK;
    return hip_status(launch_fq_act_bwd(q->format, x_dtype, g_dtype, X, rows, K, floor_of(q), q->ste_clip, dX_hat, dX,
                                        partials_of(ws), (hipStream_t)stream));
}

focus_status focus_kl_top(const void *Z_student, const void *Z_teacher, int dtype, int64_t T, int64_t V, int32_t k,
                          void *dZ_student, double *loss_out, void *ws, size_t ws_bytes, focus_stream stream) {
    if (!Z_student || !Z_teacher || !dZ_student || !loss_out) return FOCUS_ERR_NULL;
    if (!dtype_ok(dtype)) return FOCUS_ERR_DTYPE;
    if (k < 1) return FOCUS_ERR_CONFIG;
    if (T < 1 || V < 1 || T > kMaxDim || V > (int64_t(1) << 31) || V > kMaxElems / T) return FOCUS_ERR_SHAPE;
    const size_t esz = dtype == FOCUS_BF16 ? 2 : 4;
    if ((reinterpret_cast<uintptr_t>(Z_student) | reinterpret_cast<uintptr_t>(Z_teacher) |
         reinterpret_cast<uintptr_t>(dZ_student)) % esz)
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, focus_workspace_size(FOCUS_CALL_KL_TOP, nullptr, T, V, 0)));
    double *row_loss = reinterpret_cast<double *>(static_cast<char *>(ws) + kWsHeader);
    return hip_status(launch_kl_top(dtype, Z_student, Z_teacher, T, V, k, dZ_student, row_loss, loss_out, flag_of(ws),
                                    (hipStream_t)stream));
}

focus_status focus_adamw_step(const focus_adamw_config *cfg, int64_t t, int64_t n, float *param, const float *grad,
                              float *exp_avg, float *exp_avg_sq, void *ws, size_t ws_bytes, focus_stream stream) {
    if (!cfg) return FOCUS_ERR_NULL;
    const bool finite = std::isfinite(cfg->lr) && std::isfinite(cfg->eps) && std::isfinite(cfg->weight_decay);
    if (!finite || !(cfg->lr >= 0.f) || !(cfg->beta1 >= 0.f && cfg->beta1 < 1.f) ||
        !(cfg->beta2 >= 0.f && cfg->beta2 < 1.f) || !(cfg->eps > 0.f) || !(cfg->weight_decay >= 0.f) ||
        (cfg->log2_domain != 0 && cfg->log2_domain != 1) || t < 1)
        return FOCUS_ERR_CONFIG;
    if (n < 0 || n > (int64_t(1) << 40)) return FOCUS_ERR_SHAPE;  // keeps the grid below 2^31 workgroups
    if (!param || !grad || !exp_avg || !exp_avg_sq) return FOCUS_ERR_NULL;
    if (!all_aligned({param, grad, exp_avg, exp_avg_sq})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, kWsHeader));
    if (n == 0) return FOCUS_OK;
    return hip_status(launch_adamw(cfg->lr, cfg->beta1, cfg->beta2, cfg->eps, cfg->weight_decay, cfg->log2_domain,
                                   t, n, param, grad, exp_avg, exp_avg_sq, flag_of(ws), (hipStream_t)stream));
}

focus_status focus_norm_fwd(int kind, float eps, const void *X, const void *residual_opt, int dtype, int64_t T, int64_t C,
                            const void *weight, const void *bias_opt, int w_dtype, void *H_out, void *Y, float *mean_opt,
                            float *rstd_opt, void *ws, size_t ws_bytes, focus_stream stream) {
    if (kind != FOCUS_NORM_LAYER && kind != FOCUS_NORM_RMS) return FOCUS_ERR_CONFIG;
    if (!std::isfinite(eps) || eps < 0.f || (kind == FOCUS_NORM_RMS && mean_opt)) return FOCUS_ERR_CONFIG;
    if (!dtype_ok(dtype) || !dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_norm_shape(T, C));
    if (T > 0 && C > 0 && (!X || !weight || !Y || (residual_opt && !H_out))) return FOCUS_ERR_NULL;
    if (!residual_opt && H_out) return FOCUS_ERR_CONFIG;
    if (!all_aligned({X, residual_opt, weight, bias_opt, H_out, Y, mean_opt, rstd_opt})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, kWsHeader));
    if (T == 0 || C == 0) return FOCUS_OK;
    return hip_status(launch_norm_fwd(kind == FOCUS_NORM_LAYER, eps, dtype, X, residual_opt, T, C, weight, bias_opt, w_dtype,
                                      H_out, Y, mean_opt, rstd_opt, (hipStream_t)stream));
}

focus_status focus_norm_bwd(int kind, const void *dY, const void *H, int dtype, int64_t T, int64_t C, const void *weight,
                            int w_dtype, const float *mean, const float *rstd, const void *dH_opt, void *dX, float *dweight,
                            float *dbias_opt, void *ws, size_t ws_bytes, focus_stream stream) {
    if (kind != FOCUS_NORM_LAYER && kind != FOCUS_NORM_RMS) return FOCUS_ERR_CONFIG;
    if (kind == FOCUS_NORM_RMS && mean) return FOCUS_ERR_CONFIG;
    if (!dtype_ok(dtype) || !dtype_ok(w_dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_norm_shape(T, C));
    if (C > 0 && !dweight) return FOCUS_ERR_NULL;
    if (T > 0 && C > 0 && (!dY || !H || !weight || !rstd || !dX || (kind == FOCUS_NORM_LAYER && !mean))) return FOCUS_ERR_NULL;
    if (!all_aligned({dY, H, weight, mean, rstd, dH_opt, dX, dweight, dbias_opt})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, norm_bwd_ws(T, C)));
    if (C == 0) return FOCUS_OK;
    const hipStream_t st = (hipStream_t)stream;
    if (T == 0) {  // empty sums
        const hipError_t e = launch_zero_fill(dweight, (size_t)C * sizeof(float), st);
        if (e != hipSuccess || !dbias_opt) return hip_status(e);
        return hip_status(launch_zero_fill(dbias_opt, (size_t)C * sizeof(float), st));
    }
    return hip_status(launch_norm_bwd(kind == FOCUS_NORM_LAYER, dtype, dY, H, T, C, weight, w_dtype, mean, rstd, dH_opt, dX,
                                      dweight, dbias_opt, ws, st));
}

size_t focus_attention_workspace_size(int call, const focus_attention_config *cfg, int64_t Tq, int64_t Tk, int64_t n_seq) {
    AttnArgs a;
    if (attention_args(cfg, Tq, Tk, n_seq, a) != FOCUS_OK) return 0;
    switch (call) {
        case FOCUS_CALL_ATTENTION_FWD: return attn_fwd_ws(FOCUS_BF16, Tq, Tk, a.Hq, a.Hkv, a.D, n_seq);
        case FOCUS_CALL_ATTENTION_BWD: return attn_bwd_ws(FOCUS_BF16, Tq, Tk, a.Hq, a.Hkv, a.D, n_seq);
        case FOCUS_CALL_ATTENTION_FWD_F32: return attn_fwd_ws(FOCUS_F32, Tq, Tk, a.Hq, a.Hkv, a.D, n_seq);
        case FOCUS_CALL_ATTENTION_BWD_F32: return attn_bwd_ws(FOCUS_F32, Tq, Tk, a.Hq, a.Hkv, a.D, n_seq);
    }
    return 0;
}

focus_status focus_attention_fwd(const focus_attention_config *cfg, const void *q, const void *k, const void *v, int dtype,
                                 int64_t Tq, int64_t Tk, const int32_t *cu_q, const int32_t *cu_k, int64_t n_seq, void *O,
                                 float *lse_opt, void *ws, size_t ws_bytes, focus_stream stream) {
    AttnArgs a;
    FOCUS_TRY(attention_args(cfg, Tq, Tk, n_seq, a));
    if (!dtype_ok(dtype)) return FOCUS_ERR_DTYPE;
    if ((Tq > 0 && (!q || !O)) || (Tk > 0 && (!k || !v))) return FOCUS_ERR_NULL;
    FOCUS_TRY(check_ends(cu_q, cu_k, n_seq));
    if (!all_aligned({q, k, v, O}) || !strides_ok(a, dtype) || (reinterpret_cast<uintptr_t>(lse_opt) & 3u))
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, attn_fwd_ws(dtype, Tq, Tk, a.Hq, a.Hkv, a.D, n_seq)));
    if (Tq == 0 || n_seq == 0) return FOCUS_OK;
    a.q = q, a.k = k, a.v = v, a.O = O, a.lse = lse_opt, a.cu_q = cu_q, a.cu_k = cu_k, a.flag = flag_of(ws);
    const AttnRows r(a, dtype);
    const bool in_place = O == q && r.q.stride == r.O.stride;  // a row's queries are read before its output is written
    if (overlap(r.O, r.k) || overlap(r.O, r.v) || (!in_place && overlap(r.O, r.q))) return FOCUS_ERR_SHAPE;
    return hip_status(launch_attn_fwd(dtype, a, ws, (hipStream_t)stream));
}

focus_status focus_attention_bwd(const focus_attention_config *cfg, const void *dO, const void *q, const void *k,
                                 const void *v, const void *O, const float *lse, int dtype, int64_t Tq, int64_t Tk,
                                 const int32_t *cu_q, const int32_t *cu_k, int64_t n_seq, void *dq, void *dk, void *dv,
                                 void *ws, size_t ws_bytes, focus_stream stream) {
    AttnArgs a;
    FOCUS_TRY(attention_args(cfg, Tq, Tk, n_seq, a));
    if (!dtype_ok(dtype)) return FOCUS_ERR_DTYPE;
    if ((Tq > 0 && (!q || !O || !dO || !lse || !dq)) || (Tk > 0 && (!k || !v || !dk || !dv))) return FOCUS_ERR_NULL;
    FOCUS_TRY(check_ends(cu_q, cu_k, n_seq));
    if (!all_aligned({q, k, v, O, dO, dq, dk, dv}) || !strides_ok(a, dtype) || (reinterpret_cast<uintptr_t>(lse) & 3u))
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, attn_bwd_ws(dtype, Tq, Tk, a.Hq, a.Hkv, a.D, n_seq)));
    if ((Tq == 0 && Tk == 0) || n_seq == 0) return FOCUS_OK;
    a.q = q, a.k = k, a.v = v, a.O = const_cast<void *>(O), a.dO = dO, a.lse = const_cast<float *>(lse);
    a.dq = dq, a.dk = dk, a.dv = dv, a.cu_q = cu_q, a.cu_k = cu_k, a.flag = flag_of(ws);
    // the keys' pass reads what the queries' pass, before it, and its own other workgroups would have written over
    const AttnRows r(a, dtype);
    for (const Rows &out : {r.dq, r.dk, r.dv})
        for (const Rows &in : {r.q, r.k, r.v, r.O, r.dO})
            if (overlap(out, in)) return FOCUS_ERR_SHAPE;
    if (overlap(r.dq, r.dk) || overlap(r.dq, r.dv) || overlap(r.dk, r.dv)) return FOCUS_ERR_SHAPE;
    return hip_status(launch_attn_bwd(dtype, a, ws, (hipStream_t)stream));
}

focus_status focus_token_logprobs(const void *Z, int dtype, int64_t T, int64_t V, const int64_t *target_opt, int32_t top,
                                  float *logp_opt, float *entropy_opt, float *lse, float *top_logp, int32_t *top_index,
                                  void *ws, size_t ws_bytes, focus_stream stream) {
    if (!dtype_ok(dtype)) return FOCUS_ERR_DTYPE;
    if (top < 0 || top > FOCUS_MAX_TOP) return FOCUS_ERR_CONFIG;
    FOCUS_TRY(check_logits(T, V));
    if (T > 0 && (!Z || !lse || (top > 0 && (!top_logp || !top_index)) || (logp_opt && !target_opt))) return FOCUS_ERR_NULL;
    if (!logits_aligned(Z, dtype) || !aligned_to({logp_opt, entropy_opt, lse, top_logp, top_index}, 4) ||
        !aligned_to({target_opt}, 8))
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, logprobs_ws(T, V, top)));
    if (T == 0) return FOCUS_OK;
    return hip_status(launch_logprobs(dtype, Z, T, V, target_opt, top, logp_opt, entropy_opt, lse, top_logp, top_index,
                                      flag_of(ws), ws, (hipStream_t)stream));
}

focus_status focus_token_logprobs_bwd(const void *Z, int dtype, int64_t T, int64_t V, const int64_t *target_opt,
                                      const float *lse, const float *entropy_opt, const float *d_logp_opt,
                                      const float *d_entropy_opt, void *dZ, void *ws, size_t ws_bytes, focus_stream stream) {
    if (!dtype_ok(dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_logits(T, V));
    if (T > 0 && (!Z || !lse || !dZ || (!d_logp_opt && !d_entropy_opt) || (d_logp_opt && !target_opt) ||
                  (d_entropy_opt && !entropy_opt)))
        return FOCUS_ERR_NULL;
    if (!logits_aligned(Z, dtype) || !logits_aligned(dZ, dtype) ||
        !aligned_to({lse, entropy_opt, d_logp_opt, d_entropy_opt}, 4) || !aligned_to({target_opt}, 8))
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, kWsHeader));
    if (T == 0) return FOCUS_OK;
    return hip_status(launch_logprobs_bwd(dtype, Z, T, V, target_opt, lse, entropy_opt, d_logp_opt, d_entropy_opt, dZ,
                                          flag_of(ws), (hipStream_t)stream));
}

focus_status focus_sandwich_norm_fwd(const focus_sandwich_config *cfg, const void *X, const void *B, int dtype, int64_t T,
                                     int64_t C, const void *w_post, const void *b_post_opt, const void *gate,
                                     const void *w_pre, const void *b_pre_opt, int w_dtype, void *Y, void *N,
                                     float *stats_opt, void *ws, size_t ws_bytes, focus_stream stream) {
    FOCUS_TRY(check_sandwich(cfg, dtype, w_dtype, T, C, gate));
    if (T > 0 && C > 0 && (!X || !B || !w_post || !w_pre || !Y || !N || (cfg->gate != FOCUS_GATE_NONE && !gate)))
        return FOCUS_ERR_NULL;
    if (!all_aligned({X, B, w_post, b_post_opt, gate, w_pre, b_pre_opt, Y, N, stats_opt})) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, kWsHeader));
    if (T == 0 || C == 0) return FOCUS_OK;
    const bool token = cfg->gate == FOCUS_GATE_TOKEN;
    const int64_t rows = T * C * (dtype == FOCUS_BF16 ? 2 : 4), row = C * (w_dtype == FOCUS_BF16 ? 2 : 4);
    const Span stats{stats_opt, T * (cfg->kind == FOCUS_NORM_LAYER ? 4 : 2) * (int64_t)sizeof(float)};
    if (clash({{Y, rows}, {N, rows}, stats}, {{X, rows}, {B, rows}, {token ? gate : nullptr, rows}}, true) ||
        clash({{Y, rows}, {N, rows}, stats},
              {{w_post, row}, {b_post_opt, row}, {token ? nullptr : gate, row}, {w_pre, row}, {b_pre_opt, row}}, false) ||
        clash({stats}, {{X, rows}, {B, rows}, {gate, token ? rows : row}}, false))
        return FOCUS_ERR_SHAPE;
    SandwichArgs a{};
    a.X = X, a.B = B, a.gate = gate, a.w1 = w_post, a.b1 = b_post_opt, a.w2 = w_pre, a.b2 = b_pre_opt, a.Y = Y, a.N = N;
    a.stats = stats_opt, a.T = T, a.C = (int)C, a.w_dtype = w_dtype, a.layer = cfg->kind == FOCUS_NORM_LAYER;
    a.gate_kind = cfg->gate, a.eps = cfg->eps, a.scale = cfg->residual_scale;
    return hip_status(launch_sandwich_fwd(dtype, a, (hipStream_t)stream));
}

focus_status focus_sandwich_norm_bwd(const focus_sandwich_config *cfg, const void *dN, const void *dY_opt, const void *X,
                                     const void *B, int dtype, int64_t T, int64_t C, const void *w_post,
                                     const void *b_post_opt, const void *gate, const void *w_pre, int w_dtype,
                                     const float *stats, void *dX, void *dB, void *dgate_opt, float *dw_post,
                                     float *db_post_opt, float *dw_pre, float *db_pre_opt, void *ws, size_t ws_bytes,
                                     focus_stream stream) {
    FOCUS_TRY(check_sandwich(cfg, dtype, w_dtype, T, C, gate));
    if (cfg->gate == FOCUS_GATE_NONE && dgate_opt) return FOCUS_ERR_CONFIG;
    if (C > 0 && (!dw_post || !dw_pre)) return FOCUS_ERR_NULL;
    if (T > 0 && C > 0 &&
        (!dN || !X || !B || !w_post || !w_pre || !stats || !dX || !dB || (cfg->gate != FOCUS_GATE_NONE && !gate)))
        return FOCUS_ERR_NULL;
    if (!all_aligned({dN, dY_opt, X, B, w_post, b_post_opt, gate, w_pre, stats, dX, dB, dgate_opt, dw_post, db_post_opt, dw_pre,
                      db_pre_opt}))
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, sandwich_bwd_ws(T, C)));
    if (C == 0) return FOCUS_OK;
    const hipStream_t st = (hipStream_t)stream;
    const bool token = cfg->gate == FOCUS_GATE_TOKEN;
    const int64_t rows = T * C * (dtype == FOCUS_BF16 ? 2 : 4), row = C * (w_dtype == FOCUS_BF16 ? 2 : 4), sums = C * 4;
    const Span dgate_t{token ? dgate_opt : nullptr, rows}, dgate_f{token ? nullptr : dgate_opt, sums};
    const Span given{stats, T * (cfg->kind == FOCUS_NORM_LAYER ? 4 : 2) * (int64_t)sizeof(float)};
    if (clash({{dX, rows}, {dB, rows}, dgate_t, dgate_f, {dw_post, sums}, {db_post_opt, sums}, {dw_pre, sums}, {db_pre_opt, sums}},
              {{w_post, row}, {b_post_opt, row}, {token ? nullptr : gate, row}, {w_pre, row}, given}, false) ||
        clash({{dX, rows}, {dB, rows}, dgate_t},
              {{dN, rows}, {dY_opt, rows}, {X, rows}, {B, rows}, {token ? gate : nullptr, rows}}, true) ||
        clash({dgate_f, {dw_post, sums}, {db_post_opt, sums}, {dw_pre, sums}, {db_pre_opt, sums}},
              {{dN, rows}, {dY_opt, rows}, {X, rows}, {B, rows}, {token ? gate : nullptr, rows}}, false))
        return FOCUS_ERR_SHAPE;
    if (T == 0) {  // empty sums
        for (void *p : {(void *)dw_post, (void *)db_post_opt, (void *)dw_pre, (void *)db_pre_opt, token ? nullptr : dgate_opt}) {
            if (!p) continue;
            const hipError_t e = launch_zero_fill(p, (size_t)sums, st);
            if (e != hipSuccess) return hip_status(e);
        }
        return FOCUS_OK;
    }
    SandwichArgs a{};
    a.X = X, a.B = B, a.gate = gate, a.w1 = w_post, a.b1 = b_post_opt, a.w2 = w_pre, a.stats = const_cast<float *>(stats);
    a.dN = dN, a.dY = dY_opt, a.dX = dX, a.dB = dB, a.dgate = dgate_opt;
    a.dw1 = dw_post, a.db1 = db_post_opt, a.dw2 = dw_pre, a.db2 = db_pre_opt;
    a.T = T, a.C = (int)C, a.w_dtype = w_dtype, a.layer = cfg->kind == FOCUS_NORM_LAYER;
    a.gate_kind = cfg->gate, a.eps = cfg->eps, a.scale = cfg->residual_scale;
    return hip_status(launch_sandwich_bwd(dtype, a, ws, st));
}

focus_status focus_linear_ce_fwd(const void *X, const void *W, int dtype, int64_t T, int64_t V, int64_t K,
                                 const int64_t *target_opt, float *logp_opt, float *lse, void *ws, size_t ws_bytes,
                                 focus_stream stream) {
    if (!dtype_ok(dtype)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_linear_ce(T, V, K, dtype));
    if (T > 0 && (!X || !W || !lse || (logp_opt && !target_opt))) return FOCUS_ERR_NULL;
    if (!all_aligned({X, W}) || !aligned_to({logp_opt, lse}, 4) || !aligned_to({target_opt}, 8)) return FOCUS_ERR_SHAPE;
    const int64_t e = dtype == FOCUS_BF16 ? 2 : 4;
    if (clash({{logp_opt, T * 4}, {lse, T * 4}}, {{X, T * K * e}, {W, V * K * e}, {target_opt, T * 8}}, false)) return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, linear_ce_fwd_ws(T, V, K)));
    if (T == 0) return FOCUS_OK;
    return hip_status(launch_linear_ce_fwd(dtype, X, W, T, V, K, target_opt, logp_opt, lse, flag_of(ws), ws, (hipStream_t)stream));
}

focus_status focus_linear_ce_bwd(const void *X, const void *W, int dtype, int64_t T, int64_t V, int64_t K,
                                 const int64_t *target_opt, const float *lse, const float *d_logp_opt,
                                 const float *d_lse_opt, void *dX_opt, void *dW_opt, int dw_dtype, void *ws,
                                 size_t ws_bytes, focus_stream stream) {
    if (!dtype_ok(dtype) || !dtype_ok(dw_dtype) || (dtype == FOCUS_F32 && dw_dtype != FOCUS_F32)) return FOCUS_ERR_DTYPE;
    FOCUS_TRY(check_linear_ce(T, V, K, dtype));
    if (T > 0 && (!X || !W || !lse || (!dX_opt && !dW_opt) || (!d_logp_opt && !d_lse_opt) || (d_logp_opt && !target_opt)))
        return FOCUS_ERR_NULL;
    if (!all_aligned({X, W, dX_opt, dW_opt}) || !aligned_to({lse, d_logp_opt, d_lse_opt}, 4) || !aligned_to({target_opt}, 8))
        return FOCUS_ERR_SHAPE;
    const int64_t e = dtype == FOCUS_BF16 ? 2 : 4, de = dw_dtype == FOCUS_BF16 ? 2 : 4;
    if (clash({{dX_opt, T * K * e}, {dW_opt, V * K * de}},
              {{X, T * K * e}, {W, V * K * e}, {target_opt, T * 8}, {lse, T * 4}, {d_logp_opt, T * 4}, {d_lse_opt, T * 4}}, false))
        return FOCUS_ERR_SHAPE;
    FOCUS_TRY(check_ws(ws, ws_bytes, linear_ce_bwd_ws(T, V, K)));
    const hipStream_t st = (hipStream_t)stream;
    if (T == 0) return dW_opt ? hip_status(launch_zero_fill(dW_opt, (size_t)(V * K * de), st)) : FOCUS_OK;  // an empty sum
    return hip_status(launch_linear_ce_bwd(dtype, X, W, T, V, K, target_opt, lse, d_logp_opt, d_lse_opt, dX_opt, dW_opt, dw_dtype,
                                           flag_of(ws), ws, st));
}

focus_status focus_clip_grad_norm(const focus_grad_tensor *tensors, int64_t n_tensors, double max_norm, double *norm_out,
                                  void *ws, size_t ws_bytes, focus_stream stream) {
    if (!(max_norm > 0.0)) return FOCUS_ERR_CONFIG;
    if (n_tensors < 0 || n_tensors > kMaxGradTensors) return FOCUS_ERR_SHAPE;
    if (!norm_out || (n_tensors > 0 && !tensors)) return FOCUS_ERR_NULL;
    if (!aligned_to({norm_out}, 8)) return FOCUS_ERR_SHAPE;
    for (int64_t i = 0; i < n_tensors; i++) {
        const focus_grad_tensor &t = tensors[i];
        if (!dtype_ok(t.dtype)) return FOCUS_ERR_DTYPE;
        if (t.reserved != 0) return FOCUS_ERR_CONFIG;
        if (t.n < 0 || t.n > kMaxGradElems || !all_aligned({t.grad, t.out})) return FOCUS_ERR_SHAPE;
        if (t.n > 0 && !t.grad) return FOCUS_ERR_NULL;
        if (meet({norm_out, sizeof(double)}, grad_span(t, t.grad)) || meet({norm_out, sizeof(double)}, grad_span(t, t.out))) return FOCUS_ERR_SHAPE;
    }
    constexpr int kOnStack = 1024;
    int32_t few[kOnStack];
    int32_t *const order = n_tensors <= kOnStack ? few : new (std::nothrow) int32_t[n_tensors];
    if (!order) return FOCUS_ERR_HIP;
    const focus_status places = check_grad_places(tensors, n_tensors, order);
    if (order != few) delete[] order;
    FOCUS_TRY(places);
    FOCUS_TRY(check_ws(ws, ws_bytes, clip_grad_norm_ws(n_tensors)));
    return hip_status(launch_clip_grad_norm(reinterpret_cast<const GradTensor *>(tensors), n_tensors, max_norm, norm_out,
                                            flag_of(ws), ws, (hipStream_t)stream));
}

focus_status focus_check_flags(void *ws, focus_stream stream) {
    if (!ws) return FOCUS_ERR_WORKSPACE;
    if (hipStreamSynchronize((hipStream_t)stream) != hipSuccess) return FOCUS_ERR_HIP;
    uint32_t flag = 0;
    if (hipMemcpy(&flag, ws, sizeof(flag), hipMemcpyDeviceToHost) != hipSuccess) return FOCUS_ERR_HIP;
    if (flag) {
        const uint32_t zero = 0;
        if (hipMemcpy(ws, &zero, sizeof(zero), hipMemcpyHostToDevice) != hipSuccess) return FOCUS_ERR_HIP;
        return FOCUS_ERR_DOMAIN;
    }
    return FOCUS_OK;
}

const char *focus_status_string(int status) {
    switch (status) {
        case FOCUS_OK: return "ok";
        case FOCUS_ERR_NULL: return "a required pointer is NULL";
        case FOCUS_ERR_SHAPE: return "invalid sizes (negative, too large, or K not a multiple of the block size)";
        case FOCUS_ERR_DTYPE: return "unknown or unsupported dtype";
        case FOCUS_ERR_CONFIG: return "invalid quantisation configuration or argument combination";
        case FOCUS_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case FOCUS_ERR_DOMAIN: return "a kernel met a NaN scale or a coefficient c <= 0 or not finite";
        case FOCUS_ERR_HIP: return "HIP runtime error";
        case FOCUS_ERR_SCRATCH: return "the sizes need more scratch than the allocation-free call's fixed 32 MiB";
        default: return "unknown status";
    }
}

}  // extern "C"
