// C ABI of the operators on rows of logits (see include/ears.h): argument checks, the number of CTAs
// per row and the kernel launch.  These calls need no workspace: everything a row's CTAs exchange goes
// through their cluster's shared memory.
#include "../../include/ears.h"

#include <atomic>
#include <climits>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <map>
#include <mutex>
#include <type_traits>
#include <utility>

#include "ears_host.h"
#include "ears_distill.cuh"
#include "ears_rows.cuh"
#include "ears_short.cuh"
#include "ears_token.cuh"
#include "ears_top.cuh"

namespace {

using namespace ears;

std::atomic<int> g_row_cluster{0};   // ears_set_row_cluster

int esize_of(int dtype) { return dtype == EARS_DTYPE_F32 ? 4 : 2; }
bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }

struct RowCall {   // what every entry point is given about its rows
    int dtype; const void* x; int B, R, V; int64_t sb, sr; double T; const float* seq_T;
};

int check_rows(const RowCall& c) {
    if (!c.x) return EARS_ERR_NULL;
    if (c.dtype != EARS_DTYPE_F32 && c.dtype != EARS_DTYPE_BF16 && c.dtype != EARS_DTYPE_F16) return EARS_ERR_PARAM;
    if (c.B < 1 || c.R < 1 || c.V < 1 || c.V > (1 << 30)) return EARS_ERR_SHAPE;
    if ((long long)c.B * c.R > (1ll << 31) / kLMaxCluster - 1) return EARS_ERR_SHAPE;   // CTAs of a launch
    if (c.sb < 0 || c.sr < 0) return EARS_ERR_SHAPE;
    const long double span = (long double)(c.B - 1) * c.sb + (long double)(c.R - 1) * c.sr + c.V;
    if (span * 4 > 4.0e18L) return EARS_ERR_SHAPE;
    if (!c.seq_T) {
        if (!(c.T > 0.0) || !std::isfinite(c.T) || !std::isfinite((float)(kLog2e / c.T))) return EARS_ERR_PARAM;
    }
    if (misaligned(c.x, esize_of(c.dtype)) || misaligned(c.seq_T, 4)) return EARS_ERR_ALIGN;
    return EARS_OK;
}

// The gradient's rows must not share memory with each other, nor with the logits' unless they are the same
// rows (a gradient may be written over its logits).
int check_grad(const RowCall& c, const void* grad, int64_t gsb, int64_t gsr) {
    if (!grad) return EARS_ERR_NULL;
    if (misaligned(grad, esize_of(c.dtype))) return EARS_ERR_ALIGN;
    if (gsb < 0 || gsr < 0) return EARS_ERR_SHAPE;
    const long double last_b = (long double)(c.B - 1) * gsb, last_r = (long double)(c.R - 1) * gsr;
    if ((last_b + last_r + c.V) * 4 > 4.0e18L) return EARS_ERR_SHAPE;
    const bool rows_inside = (c.R == 1 || gsr >= c.V) && (c.B == 1 || gsb >= last_r + c.V);
    const bool batch_inside = (c.B == 1 || gsb >= c.V) && (c.R == 1 || gsr >= last_b + c.V);
    if (!rows_inside && !batch_inside) return EARS_ERR_SHAPE;
    const bool same = grad == c.x && (c.B == 1 || gsb == c.sb) && (c.R == 1 || gsr == c.sr);
    if (!same) {
        const size_t es = (size_t)esize_of(c.dtype);
        const uintptr_t x0 = (uintptr_t)c.x, g0 = (uintptr_t)grad;
        const uintptr_t x1 = x0 + ((size_t)(c.B - 1) * c.sb + (size_t)(c.R - 1) * c.sr + c.V) * es;
        const uintptr_t g1 = g0 + ((size_t)(c.B - 1) * gsb + (size_t)(c.R - 1) * gsr + c.V) * es;
        if (x0 < g1 && g0 < x1) return EARS_ERR_PARAM;
    }
    return EARS_OK;
}

// CTAs per row.  Few rows are split until their CTAs cover half the SMs (slices of min_slice and more), or one and a half per
// SM where the slices stay above 64 KB; a call that fetches a slice twice splits rows so long that the ones in flight (two
// CTAs per SM) would not stay in L2.  More CTAs per row than that cost: the CTAs of a cluster start and end together
// (scoring 256 rows of 256 KB takes 18 us with one, 20 with two, 31 with eight; 64 rows 10, 7.2, 6.4 with four, 9.5).
int choose_cluster(long long rows, size_t row_bytes, bool twice, size_t min_slice, int sms) {
    const int forced = g_row_cluster.load(std::memory_order_relaxed);
    if (forced) return forced;
    int C = 1;
    while (C < 8 && ((rows * C * 2 <= sms && row_bytes / C > min_slice) || (rows * C <= sms && row_bytes / C > (64u << 10)))) C *= 2;
    if (twice)
        while (C < 8 && (size_t)(2 * sms / C) * row_bytes > (100u << 20)) C *= 2;
    return C;
}

int make_span(const RowCall& c, bool twice, RowSpan* out, size_t min_slice = 16u << 10, int max_vectors = INT_MAX) {
    int sms = 0;
    const int rc = host_device_sms(&sms);
    if (rc) return rc;
    RowSpan s;
    s.sms = sms;
    s.x = c.x; s.stride_b = c.sb; s.stride_r = c.sr;
    s.rows = (long long)c.B * c.R;
    s.R = c.R; s.V = c.V; s.T = c.T; s.seq_T = c.seq_T;
    s.C = choose_cluster(s.rows, (size_t)c.V * esize_of(c.dtype), twice, min_slice, sms);
    const int n = 16 / esize_of(c.dtype);
    s.vectors = (int)(((long long)c.V + 2 * n - 2) / n);
    while (s.C < kLMaxCluster && s.vectors / s.C > max_vectors) s.C *= 2;
    const int per = (s.vectors + s.C - 1) / s.C;
    s.slice = (per + kSliceAlign - 1) / kSliceAlign * kSliceAlign;
    *out = s;
    return EARS_OK;
}

// Dynamic shared memory that fits the 48 KB every kernel may have beside what it declares itself.
constexpr size_t kPlainSmem = 32 * 1024;

// Opts a kernel in to more shared memory than that and to clusters of 16, once per kernel and device.
cudaError_t allow_launch(const void* kernel, size_t smem, int C) {
    static std::mutex mutex;
    static std::map<std::pair<const void*, int>, std::pair<size_t, bool>> allowed;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mutex);
    auto& have = allowed[{kernel, dev}];
    if (smem > kPlainSmem && smem > have.first) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        have.first = smem;
    }
    if (C > 8 && !have.second) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        have.second = true;
    }
    return cudaSuccess;
}

template <typename P, typename... Extra>
int launch_rows(void (*kernel)(P, Extra...), const P& p, int threads, size_t smem, cudaStream_t stream, const char* what, Extra... extra) {
    const RowSpan& r = p.rows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(r.rows * r.C), 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // wait_for_stream
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (r.C > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)r.C; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    if (smem > kPlainSmem || r.C > 8) {
        const cudaError_t e = allow_launch((const void*)kernel, smem, r.C);
        if (e != cudaSuccess) return host_cuda_fail(e, what);
    }
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p, extra...);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return host_cuda_fail(e, what);
    }
    return EARS_OK;
}

template <typename F>
int with_type(int dtype, F&& f) {
    if (dtype == EARS_DTYPE_F32) return f((float*)nullptr);
    if (dtype == EARS_DTYPE_F16) return f((f16_t*)nullptr);
    return f((uint16_t*)nullptr);
}

// Threads that have a row to themselves (ears_short.cuh), 0 where it is too long for that or a number of CTAs per row is asked
// for.  Up to 4 KB a warp; up to 16 KB 128 threads, or a warp where there are more than eight rows per SM (steps on 1200
// rows of 12 KB: 12.2 us with 128 threads, 13.3 with a warp; on 8192: 65 and 57, distillation 103 and 77); up to 32 KB a warp
// for forward calls on many rows (4096 of 32 KB: 33 us with a CTA per row, 30 with a warp; steps 74 and 86).  A step on no
// more rows than SMs is done sooner by a CTA each, from a list on twice as many (148 rows of 1991 bf16: policy 6.0 us with a
// warp and 5.5, distillation from 64 entries 10.9 and 8.5; on 592 rows policy 6.2 and 11.1, distillation 11.1 and 16.6).
int short_threads(const RowSpan& r, bool step, bool list) {
    if (g_row_cluster.load(std::memory_order_relaxed)) return 0;
    if (step && r.rows <= (list ? 2ll : 1ll) * r.sms) return 0;
    if (r.vectors <= 32 * kShortSlots) return 32;
    if (r.vectors <= 128 * kShortSlots) return r.rows > 8ll * r.sms ? 32 : 128;
    if (!step && r.vectors <= 32 * kShortSlots * ShortShape<32>::kRounds && r.rows > 16ll * r.sms) return 32;
    return 0;
}

// Calls f with the number of threads as a constant.
template <typename F>
int with_short(int g, F&& f) {
    if (g == 32) return f(std::integral_constant<int, 32>());
    return f(std::integral_constant<int, 128>());
}

template <typename P>
int launch_short(void (*kernel)(P), P p, int threads_per_row, cudaStream_t stream, const char* what) {
    const int rows = threads_per_row == 32 ? kShortWarpRows : 1;   // per CTA
    p.rows.slice = p.rows.vectors;
    p.rows.C = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.rows.rows + rows - 1) / rows), 1, 1);
    cfg.blockDim = dim3((unsigned)(threads_per_row * rows), 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // wait_for_stream
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e == cudaSuccess) return EARS_OK;
    (void)cudaGetLastError();
    return host_cuda_fail(e, what);
}

// Rows that a warp streams (ears_top_warp_kernel): up to 4 KB, and up to 32 KB when there are more of them than CTAs fit on the
// device at once, four per SM; fewer are done sooner by a CTA each.  So are long lists from few rows of any length (128 of 1026
// bf16: 27.9 us with a warp, 10.0 with a CTA on 148 rows, 28.4 and 17.2 on 592, 36.9 and 35.9 on 1200; 64 of 300: 15.9 and 9.0
// on 148, 16.3 and 14.3 on 592, but 64 of 1026 8.1 and 11.7; 8 of 1026: 6.2 and 7.1 on 148).
bool top_by_warps(const RowSpan& r, int k) {
    if (g_row_cluster.load(std::memory_order_relaxed)) return false;
    if ((k > 32 && r.rows <= 2ll * r.sms) || (k > 64 && r.rows <= 4ll * r.sms)) return false;
    return r.vectors <= 32 * kShortSlots || (r.vectors <= 32 * kShortSlots * kWarpTopRounds && r.rows > 4ll * r.sms);
}

template <int MODE>
int launch_token_short(int dtype, const TokenParams& p, bool ent, int g, void* stream) {
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        return with_short(g, [&](auto threads) {
            constexpr int G = decltype(threads)::value;
            return launch_short(ent ? ears_token_short_kernel<E, G, true, MODE> : ears_token_short_kernel<E, G, false, MODE>, p, G,
                                (cudaStream_t)stream, "ears_token_short_kernel launch");
        });
    });
}

template <int MODE>
int launch_distill_short(int dtype, const DistillParams& p, int g, void* stream) {
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        return with_short(g, [&](auto threads) {
            constexpr int G = decltype(threads)::value;
            return launch_short(ears_distill_short_kernel<E, G, MODE>, p, G, (cudaStream_t)stream, "ears_distill_short_kernel launch");
        });
    });
}

template <int MODE>
int launch_token(int dtype, const TokenParams& p, bool ent, void* stream) {
    if (const int g = short_threads(p.rows, false, false)) return launch_token_short<MODE>(dtype, p, ent, g, stream);
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        return launch_rows(ent ? ears_token_kernel<E, true, MODE> : ears_token_kernel<E, false, MODE>, p, kLThreads, 0,
                           (cudaStream_t)stream, "ears_token_kernel launch");
    });
}

int ring_stages(int slice) {
    const int chunks = (slice + kRingVecs - 1) / kRingVecs;
    return chunks < kRingStages ? chunks : kRingStages;
}

int launch_token_step(int dtype, const TokenParams& p, bool ent, void* stream) {
    if (const int g = short_threads(p.rows, true, false)) return launch_token_short<kStep>(dtype, p, ent, g, stream);
    const int stages = ring_stages(p.rows.slice);
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        return launch_rows(ent ? ears_token_step_kernel<E, true> : ears_token_step_kernel<E, false>, p, kRingThreads,
                           (size_t)stages * kRingChunk, (cudaStream_t)stream, "ears_token_step_kernel launch", stages);
    });
}

int launch_distill_step(int dtype, const DistillParams& p, void* stream) {
    if (const int g = short_threads(p.rows, true, true)) return launch_distill_short<kStep>(dtype, p, g, stream);
    int stages = ring_stages(p.rows.slice);
    const size_t flags = (size_t)((p.rows.slice + kRingVecs - 1) / kRingVecs) * kRingVecs;   // a byte per vector
    while (stages > 2 && (size_t)stages * kRingChunk + flags > (100u << 10)) --stages;   // two CTAs per SM
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        return launch_rows(ears_distill_step_kernel<E>, p, kDistillThreads, (size_t)stages * kRingChunk + flags, (cudaStream_t)stream,
                           "ears_distill_step_kernel launch", stages);
    });
}

template <int MODE>
int launch_distill(int dtype, const DistillParams& p, void* stream) {
    if (const int g = short_threads(p.rows, false, true)) return launch_distill_short<MODE>(dtype, p, g, stream);
    const size_t smem = MODE == kBackward ? 0 : (size_t)((p.rows.slice + kLRound - 1) / kLRound) * kLRound;   // a byte per vector
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        return launch_rows(ears_distill_kernel<E, MODE>, p, kLThreads, smem, (cudaStream_t)stream, "ears_distill_kernel launch");
    });
}

int check_words(std::initializer_list<const void*> needed, std::initializer_list<const void*> optional) {
    for (const void* q : needed)
        if (!q) return EARS_ERR_NULL;
    for (auto* list : {&needed, &optional})
        for (const void* q : *list)
            if (misaligned(q, 4)) return EARS_ERR_ALIGN;
    return EARS_OK;
}

int check_policy(double clip_low, double clip_high, double kl_coef, double entropy_coef, const float* ref) {
    if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !std::isfinite(clip_high)) return EARS_ERR_PARAM;
    if (!(kl_coef >= 0.0) || !std::isfinite(kl_coef) || !std::isfinite(entropy_coef)) return EARS_ERR_PARAM;
    if (kl_coef > 0.0 && !ref) return EARS_ERR_PARAM;
    return EARS_OK;
}

int check_distill(int V, int k, int kind, double mix, const float* lse) {
    if (k < 1 || k > EARS_MAX_TOP || V > EARS_MAX_DISTILL_V) return EARS_ERR_SHAPE;
    if (kind != EARS_DISTILL_FORWARD_KL && kind != EARS_DISTILL_REVERSE_KL && kind != EARS_DISTILL_JSD) return EARS_ERR_PARAM;
    if (kind == EARS_DISTILL_JSD && !(mix > 0.0 && mix < 1.0)) return EARS_ERR_PARAM;
    if (kind == EARS_DISTILL_REVERSE_KL && !lse) return EARS_ERR_PARAM;   // infinite: the teacher has nothing outside the list
    return EARS_OK;
}

constexpr int kDistillSlice = 1 << 16;   // vectors per CTA, each with a byte of shared memory
static_assert(kMaxTop == EARS_MAX_TOP, "list length");

}  // namespace

#define EARS_TRY(call)         \
    do {                       \
        const int rc_ = (call); \
        if (rc_) return rc_;   \
    } while (0)

extern "C" {

int ears_set_row_cluster(int cluster) {
    if (cluster != 0 && cluster != 1 && cluster != 2 && cluster != 4 && cluster != 8 && cluster != 16) return EARS_ERR_PARAM;
    g_row_cluster.store(cluster, std::memory_order_relaxed);
    return EARS_OK;
}

int ears_top_logits(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                    double temperature, const float* seq_temperature, const int32_t* accept_len, int k,
                    float* out_values, int32_t* out_ids, float* out_lse, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({out_values, out_ids, out_lse}, {accept_len, status}));
    EARS_TRY(check_rows(c));
    if (k < 1 || k > EARS_MAX_TOP) return EARS_ERR_SHAPE;
    TopParams p{};
    EARS_TRY(make_span(c, false, &p.rows, 64u << 10));   // every CTA has a list of its own to sort
    p.k = k; p.accept_len = accept_len;
    p.out_values = out_values; p.out_ids = out_ids; p.out_lse = out_lse; p.status = status;
    if (top_by_warps(p.rows, p.k))
        return with_type(dtype, [&](auto* e) {
            return launch_short(ears_top_warp_kernel<std::remove_pointer_t<decltype(e)>>, p, 32, (cudaStream_t)stream,
                                "ears_top_warp_kernel launch");
        });
    return with_type(dtype, [&](auto* e) {
        typedef std::remove_pointer_t<decltype(e)> E;
        const bool ahead = p.rows.rows * p.rows.C <= 2ll * p.rows.sms;   // all CTAs run at once, two per SM
        return launch_rows(ahead ? ears_top_kernel<E, true> : ears_top_kernel<E, false>, p, kLThreads, 0, (cudaStream_t)stream,
                           "ears_top_kernel launch");
    });
}

int ears_token_logprobs(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                        double temperature, const float* seq_temperature, const int32_t* tokens,
                        float* out_logp, float* out_entropy, float* out_saved, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({tokens, out_logp}, {out_entropy, status}));
    EARS_TRY(check_rows(c));
    if (misaligned(out_saved, 16)) return EARS_ERR_ALIGN;
    TokenParams p{};
    EARS_TRY(make_span(c, false, &p.rows));
    p.tokens = tokens; p.out_logp = out_logp; p.out_entropy = out_entropy; p.stats = (float4*)out_saved; p.status = status;
    return launch_token<kForward>(dtype, p, out_entropy != nullptr, stream);
}

int ears_token_logprobs_backward(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                                 double temperature, const float* seq_temperature, const int32_t* tokens, const float* saved,
                                 const float* d_logp, const float* d_entropy, void* out_grad, int64_t grad_stride_b,
                                 int64_t grad_stride_r, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({tokens, saved, d_logp}, {d_entropy, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_grad(c, out_grad, grad_stride_b, grad_stride_r));
    if (misaligned(saved, 16)) return EARS_ERR_ALIGN;
    TokenParams p{};
    EARS_TRY(make_span(c, false, &p.rows));
    p.tokens = tokens; p.stats = (float4*)const_cast<float*>(saved); p.d_logp = d_logp; p.d_entropy = d_entropy; p.status = status;
    p.grad = out_grad; p.gsb = grad_stride_b; p.gsr = grad_stride_r;
    return launch_token<kBackward>(dtype, p, d_entropy != nullptr, stream);
}

int ears_token_logprobs_step(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                             double temperature, const float* seq_temperature, const int32_t* tokens, const float* d_logp,
                             const float* d_entropy, float* out_logp, float* out_entropy, void* out_grad,
                             int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({tokens, d_logp, out_logp}, {d_entropy, out_entropy, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_grad(c, out_grad, grad_stride_b, grad_stride_r));
    TokenParams p{};
    EARS_TRY(make_span(c, true, &p.rows));
    p.tokens = tokens; p.d_logp = d_logp; p.d_entropy = d_entropy; p.out_logp = out_logp; p.out_entropy = out_entropy;
    p.grad = out_grad; p.gsb = grad_stride_b; p.gsr = grad_stride_r; p.status = status;
    return launch_token_step(dtype, p, d_entropy != nullptr || out_entropy != nullptr, stream);
}

int ears_policy_loss(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                     double temperature, const float* seq_temperature, const int32_t* tokens, const float* old_logp,
                     const float* ref_logp, const float* advantage, double clip_low, double clip_high, double kl_coef,
                     double entropy_coef, float* out_loss, float* out_logp, float* out_kl, float* out_entropy,
                     float* out_saved, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({tokens, old_logp, advantage, out_loss}, {ref_logp, out_logp, out_kl, out_entropy, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_policy(clip_low, clip_high, kl_coef, entropy_coef, ref_logp));
    if (misaligned(out_saved, 16)) return EARS_ERR_ALIGN;
    TokenParams p{};
    EARS_TRY(make_span(c, false, &p.rows));
    p.policy = 1;
    p.tokens = tokens; p.old_logp = old_logp; p.ref_logp = ref_logp; p.advantage = advantage;
    p.clip_low = clip_low; p.clip_high = clip_high; p.kl_coef = kl_coef; p.entropy_coef = entropy_coef;
    p.out_loss = out_loss; p.out_logp = out_logp; p.out_kl = out_kl; p.out_entropy = out_entropy;
    p.stats = (float4*)out_saved; p.status = status;
    return launch_token<kForward>(dtype, p, entropy_coef != 0.0 || out_entropy != nullptr, stream);
}

int ears_policy_backward(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                         double temperature, const float* seq_temperature, const int32_t* tokens, const float* old_logp,
                         const float* ref_logp, const float* advantage, double clip_low, double clip_high, double kl_coef,
                         double entropy_coef, const float* saved, const float* d_loss, void* out_grad,
                         int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({tokens, old_logp, advantage, saved, d_loss}, {ref_logp, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_policy(clip_low, clip_high, kl_coef, entropy_coef, ref_logp));
    EARS_TRY(check_grad(c, out_grad, grad_stride_b, grad_stride_r));
    if (misaligned(saved, 16)) return EARS_ERR_ALIGN;
    TokenParams p{};
    EARS_TRY(make_span(c, false, &p.rows));
    p.policy = 1;
    p.tokens = tokens; p.old_logp = old_logp; p.ref_logp = ref_logp; p.advantage = advantage; p.weight = d_loss;
    p.clip_low = clip_low; p.clip_high = clip_high; p.kl_coef = kl_coef; p.entropy_coef = entropy_coef;
    p.stats = (float4*)const_cast<float*>(saved); p.status = status;
    p.grad = out_grad; p.gsb = grad_stride_b; p.gsr = grad_stride_r;
    return launch_token<kBackward>(dtype, p, entropy_coef != 0.0, stream);
}

int ears_policy_step(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                     double temperature, const float* seq_temperature, const int32_t* tokens, const float* old_logp,
                     const float* ref_logp, const float* advantage, double clip_low, double clip_high, double kl_coef,
                     double entropy_coef, const float* row_weight, float* out_loss, float* out_logp, float* out_kl,
                     float* out_entropy, void* out_grad, int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status,
                     void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({tokens, old_logp, advantage, out_loss}, {ref_logp, row_weight, out_logp, out_kl, out_entropy, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_policy(clip_low, clip_high, kl_coef, entropy_coef, ref_logp));
    EARS_TRY(check_grad(c, out_grad, grad_stride_b, grad_stride_r));
    TokenParams p{};
    EARS_TRY(make_span(c, true, &p.rows));
    p.policy = 1;
    p.tokens = tokens; p.old_logp = old_logp; p.ref_logp = ref_logp; p.advantage = advantage; p.weight = row_weight;
    p.clip_low = clip_low; p.clip_high = clip_high; p.kl_coef = kl_coef; p.entropy_coef = entropy_coef;
    p.out_loss = out_loss; p.out_logp = out_logp; p.out_kl = out_kl; p.out_entropy = out_entropy; p.status = status;
    p.grad = out_grad; p.gsb = grad_stride_b; p.gsr = grad_stride_r;
    return launch_token_step(dtype, p, entropy_coef != 0.0 || out_entropy != nullptr, stream);
}

int ears_distill_loss(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                      double temperature, const float* seq_temperature, int k, const float* values, const int32_t* ids,
                      const float* lse, int kind, double mix, float* out_loss, float* out_saved, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({values, ids, out_loss}, {lse, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_distill(V, k, kind, mix, lse));
    if (misaligned(out_saved, 16)) return EARS_ERR_ALIGN;
    DistillParams p{};
    EARS_TRY(make_span(c, false, &p.rows, 16u << 10, kDistillSlice));
    p.k = k; p.kind = kind; p.mix = mix; p.values = values; p.ids = ids; p.lse = lse;
    p.out_loss = out_loss; p.stats = (float4*)out_saved; p.status = status;
    return launch_distill<kForward>(dtype, p, stream);
}

int ears_distill_backward(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                          double temperature, const float* seq_temperature, int k, const float* values, const int32_t* ids,
                          const float* lse, int kind, double mix, const float* saved, const float* d_loss, void* out_grad,
                          int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({values, ids, saved, d_loss}, {lse, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_distill(V, k, kind, mix, lse));
    EARS_TRY(check_grad(c, out_grad, grad_stride_b, grad_stride_r));
    if (misaligned(saved, 16)) return EARS_ERR_ALIGN;
    DistillParams p{};
    EARS_TRY(make_span(c, false, &p.rows, 16u << 10, kDistillSlice));
    p.k = k; p.kind = kind; p.mix = mix; p.values = values; p.ids = ids; p.lse = lse; p.weight = d_loss;
    p.stats = (float4*)const_cast<float*>(saved); p.status = status;
    p.grad = out_grad; p.gsb = grad_stride_b; p.gsr = grad_stride_r;
    return launch_distill<kBackward>(dtype, p, stream);
}

int ears_distill_step(int dtype, const void* logits, int B, int R, int V, int64_t stride_b, int64_t stride_r,
                      double temperature, const float* seq_temperature, int k, const float* values, const int32_t* ids,
                      const float* lse, int kind, double mix, const float* row_weight, float* out_loss, void* out_grad,
                      int64_t grad_stride_b, int64_t grad_stride_r, int32_t* status, void* stream) {
    const RowCall c{dtype, logits, B, R, V, stride_b, stride_r, temperature, seq_temperature};
    EARS_TRY(check_words({values, ids, out_loss}, {lse, row_weight, status}));
    EARS_TRY(check_rows(c));
    EARS_TRY(check_distill(V, k, kind, mix, lse));
    EARS_TRY(check_grad(c, out_grad, grad_stride_b, grad_stride_r));
    DistillParams p{};
    EARS_TRY(make_span(c, true, &p.rows, 16u << 10, kDistillSlice));
    p.k = k; p.kind = kind; p.mix = mix; p.values = values; p.ids = ids; p.lse = lse; p.weight = row_weight;
    p.out_loss = out_loss; p.status = status;
    p.grad = out_grad; p.gsb = grad_stride_b; p.gsr = grad_stride_r;
    return launch_distill_step(dtype, p, stream);
}

}  // extern "C"
