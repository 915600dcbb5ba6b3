// C ABI of the key/value cache held in 4 bits (see include/ears.h): argument checks, launch shapes, kernel launches.
#include "../../include/ears.h"

#include <climits>
#include <cmath>
#include <cstdint>
#include <map>
#include <mutex>
#include <type_traits>
#include <utility>

#include "ears_host.h"
#include "ears_kv.cuh"
#include "ears_kv_attention.cuh"

namespace {

using namespace ears;

static_assert(kKvGroup == EARS_KV_GROUP && kDevInvalid == EARS_DEV_INVALID_INPUT, "mirrors of the C header");

bool misaligned(const void* p, size_t a) { return ((uintptr_t)p % a) != 0; }
bool type_ok(int dtype) { return dtype == EARS_DTYPE_F32 || dtype == EARS_DTYPE_BF16 || dtype == EARS_DTYPE_F16; }
int esize_of(int dtype) { return dtype == EARS_DTYPE_F32 ? 4 : 2; }

int check_cache(const ears_kv_cache* c) {
    if (!c || !c->codes || !c->params) return EARS_ERR_NULL;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return EARS_ERR_SHAPE;
    if (c->pages < 1 || c->heads < 1 || c->heads > (1 << 16) || c->page_size < 16 || c->page_size % 16 || c->page_size > (1 << 20)) return EARS_ERR_SHAPE;
    if ((long long)c->heads * c->page_size * c->head_dim > INT_MAX) return EARS_ERR_SHAPE;       // bytes of a page
    if ((long double)c->pages * 2 * c->heads * c->page_size > 3.0e10L) return EARS_ERR_SHAPE;    // sixteenths of rows in 31 bits
    if (misaligned(c->codes, 16) || misaligned(c->params, 16)) return EARS_ERR_ALIGN;
    return EARS_OK;
}

constexpr long long kMaxTokens = INT_MAX - 1024;      // of a table: positions and what is added to them stay in 31 bits

int check_seqs(const ears_kv_cache* c, const KvSeqs& s) {
    if (!s.table || !s.start) return EARS_ERR_NULL;
    if (s.B < 1 || s.Q < 1 || s.width < 1 || s.stride < 0) return EARS_ERR_SHAPE;
    if ((long long)s.width * c->page_size > kMaxTokens) return EARS_ERR_SHAPE;
    if ((long double)(s.B - 1) * s.stride + s.width > 1.0e18L) return EARS_ERR_SHAPE;
    // eights of a call's elements, counted in 31 bits
    if ((long double)s.B * s.Q * 2 * c->heads * (c->head_dim / 8) > (long double)INT_MAX) return EARS_ERR_SHAPE;
    if (misaligned(s.table, 4) || misaligned(s.start, 4) || misaligned(s.counts, 4)) return EARS_ERR_ALIGN;
    return EARS_OK;
}

int check_strides(int B, int Q, int heads, int D, int64_t sb, int64_t sq, int64_t sh) {
    if (sb < 0 || sq < 0 || sh < 0) return EARS_ERR_SHAPE;
    if ((long double)(B - 1) * sb + (long double)(Q - 1) * sq + (long double)(heads - 1) * sh + D > 1.0e18L) return EARS_ERR_SHAPE;
    return EARS_OK;
}
bool vectors(const void* x, int es, int B, int Q, int heads, int64_t sb, int64_t sq, int64_t sh) {
    const int64_t n = 16 / es;
    return !misaligned(x, 16) && (B == 1 || sb % n == 0) && (Q == 1 || sq % n == 0) && (heads == 1 || sh % n == 0);
}

KvCache cache_of(const ears_kv_cache* c) { return KvCache{(uint8_t*)c->codes, (uint32_t*)c->params, c->pages, c->heads, c->page_size}; }

template <typename F>
int with_dim(int D, F&& f) {
    if (D == 64) return f(std::integral_constant<int, 64>());
    if (D == 128) return f(std::integral_constant<int, 128>());
    return f(std::integral_constant<int, 256>());
}
template <typename F>
int with_type(int dtype, F&& f) {
    if (dtype == EARS_DTYPE_F32) return f((float*)nullptr);
    if (dtype == EARS_DTYPE_F16) return f((f16_t*)nullptr);
    return f((uint16_t*)nullptr);
}

template <typename P, typename... Extra>
int launch(void (*kernel)(P, Extra...), const std::decay_t<P>& p, dim3 grid, int threads, size_t smem, void* stream, const char* what, Extra... extra) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // wait_for_stream
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p, extra...);
    if (e == cudaSuccess) return EARS_OK;
    (void)cudaGetLastError();
    return host_cuda_fail(e, what);
}

// Warps per position of a write or a read, and the grid: fewer positions than a few per SM are shared by up to a warp per step.
int share_positions(const KvSeqs& s, const ears_kv_cache* c, int values, int* parts, unsigned* grid) {
    int sms = 0;
    const int rc = host_device_sms(&sms);
    if (rc) return rc;
    const long long positions = (long long)s.B * s.Q;
    const int lanes = c->head_dim / values, steps = 2 * (lanes > 32 ? c->heads * (lanes / 32) : (c->heads + 32 / lanes - 1) / (32 / lanes));
    int n = 1;
    while (n * 2 <= steps && positions * n < 16ll * sms) n *= 2;
    *parts = n;
    *grid = (unsigned)((positions * n + kKvThreads / 32 - 1) / (kKvThreads / 32));
    return EARS_OK;
}

// ---- attention: variant and grid
// Eights of rows per block.  A unit's blocks each read its part of the cache (from L2 all but the first time), which blocks of few rows
// do faster: the time of a block of 1, 2, .. eights, in us for 576000 tokens x 8 heads of 64 or 128, 240000 x 4 of 256.
template <int D> constexpr int kMaxTiles = D == 64 ? 4 : D == 128 ? 4 : 2;
constexpr int kBlockTime[3][4] = {{83, 114, 144, 177}, {127, 169, 228, 322}, {65, 98, 0, 0}};
template <int D>
int choose_rows(int tiles) {
    int best = 1;
    long long least = -1;
    for (int nt = 1; nt <= kMaxTiles<D>; ++nt) {
        const long long time = (long long)((tiles + nt - 1) / nt) * kBlockTime[D == 64 ? 0 : D == 128 ? 1 : 2][nt - 1];
        if (least < 0 || time <= least) { least = time; best = nt; }
    }
    return best;
}

typedef void (*AttentionKernel)(const KaParams);
struct Variant { AttentionKernel attention, join; size_t smem; int nt; };

template <typename E, int D, int NT>
Variant variant_of() { return Variant{ears_kv_attention_kernel<E, D, NT>, ears_kv_join_kernel<E, D, NT>, KaShape<D, NT>::kSmem, NT}; }

template <typename E, int D>
Variant choose_tiles(int nt) {
    if constexpr (kMaxTiles<D> >= 4) { if (nt == 4) return variant_of<E, D, 4>(); }
    if constexpr (kMaxTiles<D> >= 3) { if (nt == 3) return variant_of<E, D, 3>(); }
    if constexpr (kMaxTiles<D> >= 2) { if (nt == 2) return variant_of<E, D, 2>(); }
    return variant_of<E, D, 1>();
}

struct KaPlan { Variant v; int blocks, grid; };

// CTAs of the kernel that are resident at once on the current device; opts in to its shared memory.
int resident(const Variant& v, int* ctas) {
    static std::mutex mutex;
    static std::map<std::pair<const void*, int>, int> known;
    int dev = 0, sms = 0, per_sm = 0;
    const char* what = "cudaGetDevice";
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) {
        const int rc = host_device_sms(&sms);
        if (rc) return rc;
        try {
            std::lock_guard<std::mutex> lock(mutex);
            int& n = known[{(const void*)v.attention, dev}];
            if (!n) {
                what = "cudaFuncSetAttribute";
                e = cudaFuncSetAttribute((const void*)v.attention, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.smem);
                if (e == cudaSuccess) {
                    what = "cudaOccupancyMaxActiveBlocksPerMultiprocessor";
                    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, v.attention, kKaThreads, v.smem);
                }
                if (e == cudaSuccess) n = sms * (per_sm < 1 ? 1 : per_sm);
            }
            *ctas = n;
        } catch (...) {                   // the host is out of memory, or its lock failed: no exception passes the C entry
            what = "the table of resident CTAs";
            e = cudaErrorMemoryAllocation;
        }
    }
    if (e == cudaSuccess) return EARS_OK;
    (void)cudaGetLastError();
    return host_cuda_fail(e, what);
}

int make_plan(int dtype, const ears_kv_cache* c, int B, int Q, int heads_q, int width, int window, int sinks, KaPlan* plan) {
    const int M = Q * (heads_q / c->heads), tiles = (M + 7) / 8;
    int sms = 0;
    const int rc_sms = host_device_sms(&sms);
    if (rc_sms) return rc_sms;
    // chunks of a sequence at the most, whatever its length
    long long tokens = (long long)width * c->page_size;
    if (window && (long long)window + sinks + Q + 3 * kKaTile < tokens) tokens = (long long)window + sinks + Q + 3 * kKaTile;
    const long long chunks = (tokens + kKaChunk - 1) / kKaChunk;
    // Few chunks are bound by latency, and blocks of one eight are done soonest, although each reads the cache: up to 16 chunks per SM, 64
    // counting every block's.  Blocks of one eight and those of choose_rows, us, 8 heads of 128: 3 eights of rows, 1000 tokens (2.6 counting
    // every block's) 12.3 and 13.8, 4000 (10) 14.9 and 20.6; 9 eights, 8000 tokens (61) 25.9 and 28.2; 33 eights, 2000 tokens (57) 26.7 and 25.7,
    // 4000 (112) 39.5 and 34.5, 16000 (446) 112 and 82; 2 eights, 4 sequences of 8000 (54, but 27 chunks) 25.1 and 23.1.
    const long double work = (long double)B * c->heads * chunks;
    const bool few = work <= 16.0L * sms && work * tiles <= 64.0L * sms;
    with_dim(c->head_dim, [&](auto d) {
        constexpr int D = decltype(d)::value;
        const int nt = few ? 1 : choose_rows<D>(tiles);
        plan->v = dtype == EARS_DTYPE_F16 ? choose_tiles<f16_t, D>(nt) : choose_tiles<uint16_t, D>(nt);
        return 0;
    });
    plan->blocks = (tiles + plan->v.nt - 1) / plan->v.nt;
    const int rc = resident(plan->v, &plan->grid);
    if (rc) return rc;
    const long double units = (long double)B * c->heads * plan->blocks;
    if (units * (chunks + kKaAhead) > (long double)INT_MAX) return EARS_ERR_SHAPE;    // the device counts in 31 bits
    if (units * chunks < plan->grid) plan->grid = (int)(units * chunks);
    return EARS_OK;
}

constexpr size_t kWsAlign = 256;
size_t aligned(size_t n) { return (n + kWsAlign - 1) / kWsAlign * kWsAlign; }
size_t carve(const KaPlan& plan, int D, unsigned char* at, KaParams* p) {
    const size_t rows = (size_t)plan.grid * 2 * plan.v.nt * 8;
    const size_t cut = aligned((size_t)plan.grid * sizeof(int4)), ml = aligned(rows * sizeof(float2)), o = aligned(rows * D * sizeof(float));
    if (p) {
        p->cut = (int4*)at;
        p->part_ml = (float2*)(at + cut);
        p->part_o = (float*)(at + cut + ml);
    }
    return cut + ml + o;
}

int check_attention(int dtype, const ears_kv_cache* c, int B, int Q, int heads_q, int width, int window, int sinks) {
    if (dtype != EARS_DTYPE_BF16 && dtype != EARS_DTYPE_F16) return EARS_ERR_PARAM;
    if (heads_q < 1 || heads_q % c->heads) return EARS_ERR_SHAPE;
    if ((long double)B * Q * heads_q > (long double)INT_MAX) return EARS_ERR_SHAPE;
    if (window < 0 || sinks < 0) return EARS_ERR_PARAM;
    return EARS_OK;
}

}  // namespace

#define EARS_TRY(call)         \
    do {                       \
        const int rc_ = (call); \
        if (rc_) return rc_;   \
    } while (0)

extern "C" {

int ears_kv_write(int dtype, const ears_kv_cache* cache, const void* k, const void* v, int B, int Q, int64_t k_stride_b, int64_t k_stride_q,
                  int64_t k_stride_h, int64_t v_stride_b, int64_t v_stride_q, int64_t v_stride_h, const int32_t* page_table,
                  int table_width, int64_t table_stride, const int32_t* start, const int32_t* counts, int32_t* status, void* stream) {
    EARS_TRY(check_cache(cache));
    if (!k || !v) return EARS_ERR_NULL;
    if (!type_ok(dtype)) return EARS_ERR_PARAM;
    KvWriteParams p{};
    p.cache = cache_of(cache);
    p.seqs = KvSeqs{page_table, table_stride, table_width, start, counts, B, Q};
    EARS_TRY(check_seqs(cache, p.seqs));
    EARS_TRY(check_strides(B, Q, cache->heads, cache->head_dim, k_stride_b, k_stride_q, k_stride_h));
    EARS_TRY(check_strides(B, Q, cache->heads, cache->head_dim, v_stride_b, v_stride_q, v_stride_h));
    const int es = esize_of(dtype);
    if (misaligned(k, es) || misaligned(v, es) || misaligned(status, 4)) return EARS_ERR_ALIGN;
    p.x[0] = k; p.sb[0] = k_stride_b; p.sq[0] = k_stride_q; p.sh[0] = k_stride_h;
    p.x[1] = v; p.sb[1] = v_stride_b; p.sq[1] = v_stride_q; p.sh[1] = v_stride_h;
    p.vec[0] = vectors(k, es, B, Q, cache->heads, k_stride_b, k_stride_q, k_stride_h);
    p.vec[1] = vectors(v, es, B, Q, cache->heads, v_stride_b, v_stride_q, v_stride_h);
    p.status = status;
    int parts = 1;
    unsigned grid = 1;
    EARS_TRY(share_positions(p.seqs, cache, 8, &parts, &grid));
    return with_dim(cache->head_dim, [&](auto d) {
        return with_type(dtype, [&](auto* e) {
            return launch(ears_kv_write_kernel<std::remove_pointer_t<decltype(e)>, decltype(d)::value>, p, dim3(grid), kKvThreads, 0, stream,
                          "ears_kv_write_kernel launch", parts);
        });
    });
}

int ears_kv_read(int dtype, const ears_kv_cache* cache, int B, int Q, const int32_t* page_table, int table_width, int64_t table_stride,
                 const int32_t* start, const int32_t* counts, void* out_k, void* out_v, int32_t* status, void* stream) {
    EARS_TRY(check_cache(cache));
    if (!out_k || !out_v) return EARS_ERR_NULL;
    if (!type_ok(dtype)) return EARS_ERR_PARAM;
    KvReadParams p{};
    p.cache = cache_of(cache);
    p.seqs = KvSeqs{page_table, table_stride, table_width, start, counts, B, Q};
    EARS_TRY(check_seqs(cache, p.seqs));
    if (misaligned(out_k, 16) || misaligned(out_v, 16) || misaligned(status, 4)) return EARS_ERR_ALIGN;
    p.out[0] = out_k; p.out[1] = out_v;
    p.status = status;
    int parts = 1;
    unsigned grid = 1;
    EARS_TRY(share_positions(p.seqs, cache, dtype == EARS_DTYPE_F32 ? 4 : 8, &parts, &grid));
    return with_dim(cache->head_dim, [&](auto d) {
        return with_type(dtype, [&](auto* e) {
            return launch(ears_kv_read_kernel<std::remove_pointer_t<decltype(e)>, decltype(d)::value>, p, dim3(grid), kKvThreads, 0, stream,
                          "ears_kv_read_kernel launch", parts);
        });
    });
}

size_t ears_kv_attention_workspace_bytes(int dtype, const ears_kv_cache* cache, int B, int Q, int heads_q, int table_width, int window, int sinks) {
    if (check_cache(cache) || B < 1 || Q < 1 || table_width < 1 || (long long)table_width * cache->page_size > kMaxTokens) return 0;
    if (check_attention(dtype, cache, B, Q, heads_q, table_width, window, sinks)) return 0;
    KaPlan plan;
    if (make_plan(dtype, cache, B, Q, heads_q, table_width, window, sinks, &plan)) return 0;
    return carve(plan, cache->head_dim, nullptr, nullptr);
}

int ears_kv_attention(int dtype, const ears_kv_cache* cache, const void* q, int B, int Q, int heads_q, int64_t q_stride_b, int64_t q_stride_q,
                      int64_t q_stride_h, const int32_t* page_table, int table_width, int64_t table_stride, const int32_t* start,
                      const int32_t* counts, double scale, int window, int sinks, void* out, float* out_lse, void* workspace,
                      size_t workspace_bytes, int32_t* status, void* stream) {
    EARS_TRY(check_cache(cache));
    if (!q || !out || !workspace) return EARS_ERR_NULL;
    KaParams p{};
    p.cache = cache_of(cache);
    p.seqs = KvSeqs{page_table, table_stride, table_width, start, counts, B, Q};
    EARS_TRY(check_seqs(cache, p.seqs));
    EARS_TRY(check_attention(dtype, cache, B, Q, heads_q, table_width, window, sinks));
    EARS_TRY(check_strides(B, Q, heads_q, cache->head_dim, q_stride_b, q_stride_q, q_stride_h));
    if (!std::isfinite(scale) || !std::isfinite((float)(scale * 1.44269504088896340736))) return EARS_ERR_PARAM;
    if (misaligned(q, 2) || misaligned(out, 16) || misaligned(out_lse, 4) || misaligned(workspace, kWsAlign) || misaligned(status, 4))
        return EARS_ERR_ALIGN;
    KaPlan plan;
    EARS_TRY(make_plan(dtype, cache, B, Q, heads_q, table_width, window, sinks, &plan));
    if (carve(plan, cache->head_dim, (unsigned char*)workspace, &p) > workspace_bytes) return EARS_ERR_WORKSPACE;
    p.q = q; p.sb = q_stride_b; p.sq = q_stride_q; p.sh = q_stride_h;
    p.vec = vectors(q, 2, B, Q, heads_q, q_stride_b, q_stride_q, q_stride_h);
    p.group = heads_q / cache->heads;
    p.M = Q * p.group;
    p.blocks = plan.blocks;
    p.scale2 = (float)(scale * 1.44269504088896340736);
    p.window = window; p.sinks = sinks;
    p.out = out; p.lse = out_lse; p.status = status;
    EARS_TRY(launch(plan.v.attention, p, dim3((unsigned)plan.grid), kKaThreads, plan.v.smem, stream, "ears_kv_attention_kernel launch"));
    // few units have many parts each: as many warps per row as leave a warp a dozen of them
    const long long units = (long long)B * cache->heads * plan.blocks;
    const int warps = plan.grid > 24 * units ? 4 : plan.grid > 12 * units ? 2 : 1;
    return launch(plan.v.join, p, dim3((unsigned)plan.grid, (unsigned)(plan.v.nt * 8 / kKaJoinRows)), kKaJoinRows * 32 * warps, 0, stream,
                  "ears_kv_join_kernel launch");
}

}  // extern "C"
