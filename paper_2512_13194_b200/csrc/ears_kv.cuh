// A key/value cache held in 4 bits: its layout, the quantising write and the read as values.
//
// A pool of pages, each with the keys and values of `page` tokens for every head:
//     codes  [P, 2, H, page, D / 2]      two codes a byte, the even dimension's in the low half
//     params [P, 2, H, page, D / 64]     a word per group of 64: the scale s (low half) and the minimum m, bfloat16
// and a code c stands for m + s c.  A token's codes in one head are contiguous, and so are a page's tokens, so that a tile
// of tokens is one run of bytes for whatever reads it.  For a group x_0 .. x_63
//     m = min x, rounded down to bfloat16            s = (max x - m) fl(1 / 15) in 32 bits, rounded up to bfloat16, at least 2^-126
//     c = (x - m) / s to the nearest, ties to even
// with the directed roundings keeping every x inside [m, m + 15 s]: a value comes back within s / 2 of what was written.
// bfloat16 and not half precision, since neither large keys overflow its range nor small values lose their scale.
// A group that holds a NaN or an infinity, or whose range overflows, gets NaN for both parameters and reads back as NaN.
#pragma once
#include <cfloat>

#include "ears_math.cuh"
#include "ears_pipeline.cuh"

namespace ears {

constexpr int kKvGroup = 64;
constexpr int kDevInvalid = 1;            // EARS_DEV_INVALID_INPUT

struct KvCache {
    uint8_t* codes;
    uint32_t* params;
    int pages, heads, page;               // pages in the pool, heads, tokens per page
};

// Where the sequences of a call stand: position i of sequence b is its token start[b] + i, for i < counts[b].
struct KvSeqs {
    const int32_t* table;                 // [B, width] page of each run of `page` tokens
    long long stride;
    int width;
    const int32_t* start;
    const int32_t* counts;                // or NULL: Q for all
    int B, Q;
};

__device__ __forceinline__ int kv_count(const KvSeqs& s, int b) {
    return s.counts ? max(0, min(__ldg(s.counts + b), s.Q)) : s.Q;
}
// Row of token `t` of sequence b for keys in head 0 (rows: [P, 2, H, page]); -1 where the table has no page of the pool for it.
__device__ __forceinline__ long long kv_row(const KvCache& c, const KvSeqs& s, int b, long long t) {
    if (t < 0 || t >= (long long)s.width * c.page) return -1;
    const int slot = (int)t / c.page;     // width * page < 2^31 (the host's check)
    const int id = __ldg(s.table + b * s.stride + slot);
    if (id < 0 || id >= c.pages) return -1;
    return (long long)id * 2 * c.heads * c.page + ((int)t - slot * c.page);
}

__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// eight consecutive elements; `vec`: 16-byte aligned
template <typename E> struct KvEight;
template <> struct KvEight<float> {
    __device__ static __forceinline__ void load(const float* p, bool vec, float (&x)[8]) {
        if (vec) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __ldg(p + i);
        }
    }
    __device__ static __forceinline__ void store(float* p, const float (&x)[8]) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
};
template <typename E> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_pair<uint16_t>(float lo, float hi) {
    uint32_t r; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r;
}
template <> __device__ __forceinline__ uint32_t pack_pair<f16_t>(float lo, float hi) {
    uint32_t r; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r;
}
template <typename E> __device__ __forceinline__ float2 unpack_pair(uint32_t w);
template <> __device__ __forceinline__ float2 unpack_pair<uint16_t>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack_pair<f16_t>(uint32_t w) { return f16x2_to_float2(w); }
template <typename E> struct KvEight {
    __device__ static __forceinline__ void load(const E* p, bool vec, float (&x)[8]) {
        if (vec) {
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
            const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack_pair<E>(v[i]);
                x[2 * i] = f.x; x[2 * i + 1] = f.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = load_logit(p + i);
        }
    }
    __device__ static __forceinline__ void store(E* p, const float (&x)[8]) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_pair<E>(x[0], x[1]), pack_pair<E>(x[2], x[3]), pack_pair<E>(x[4], x[5]), pack_pair<E>(x[6], x[7]));
    }
};

// ---- write ------------------------------------------------------------------------------------------
struct KvWriteParams {
    KvCache cache;
    KvSeqs seqs;
    const void* x[2];                     // keys, values [B, Q, H, D]
    long long sb[2], sq[2], sh[2];        // strides in elements
    bool vec[2];                          // every group starts on 16 bytes
    int32_t* status;
};

constexpr int kKvThreads = 256;
constexpr int kKvTeams = kKvThreads / 8;  // eight threads have a group of 64, eight values each

template <typename E, int D>
__global__ void __launch_bounds__(kKvThreads) ears_kv_write_kernel(const KvWriteParams p) {
    constexpr int NG = D / kKvGroup;
    wait_for_stream();
    const int lane = threadIdx.x & 7;
    const unsigned per_kind = (unsigned)p.cache.heads * NG, per_row = 2 * per_kind;
    const unsigned items = (unsigned)p.seqs.B * p.seqs.Q * per_row;
    const unsigned item = blockIdx.x * kKvTeams + threadIdx.x / 8;
    const unsigned row = min(item, items - 1) / per_row, in_row = min(item, items - 1) - row * per_row;
    const int b = (int)(row / (unsigned)p.seqs.Q), i = (int)(row - (unsigned)b * p.seqs.Q);
    const int kind = in_row >= per_kind;
    const unsigned hg = in_row - kind * per_kind;
    const int h = (int)(hg / NG), g = (int)(hg % NG);
    const bool mine = item < items && i < kv_count(p.seqs, b);

    float x[8];
    long long at = -1;
    if (mine) {
        KvEight<E>::load(reinterpret_cast<const E*>(kind ? p.x[1] : p.x[0]) + b * (kind ? p.sb[1] : p.sb[0]) + i * (kind ? p.sq[1] : p.sq[0]) +
                             h * (kind ? p.sh[1] : p.sh[0]) + g * kKvGroup + lane * 8,
                         kind ? p.vec[1] : p.vec[0], x);
        at = kv_row(p.cache, p.seqs, b, (long long)__ldg(p.seqs.start + b) + i);
        if (at < 0 && lane == 0 && p.status) atomicOr(p.status, kDevInvalid);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
    }
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) { lo = min_nan(lo, x[j]); hi = max_nan(hi, x[j]); }
#pragma unroll
    for (int d = 4; d; d >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    uint32_t mb = __float_as_uint(lo), cut = mb & 0xffff0000u;
    if ((int)mb < 0 && mb != cut) cut += 0x10000u;
    const float m = __uint_as_float(cut);
    const float range = __fmul_rn(__fsub_rn(hi, m), 1.f / 15.f);
    const bool fine = range <= FLT_MAX;               // false for NaN too
    uint32_t sbits = __float_as_uint(range);
    if (sbits & 0xffffu) sbits = (sbits & 0xffff0000u) + 0x10000u;
    float s = __uint_as_float(sbits);
    s = fmaxf(s, 0x1p-126f);
    uint32_t word = 0, par = 0x7fc07fc0u;
    if (fine) {
        par = (__float_as_uint(s) >> 16) | (__float_as_uint(m) & 0xffff0000u);
        const float r = 1.f / s;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // floor of an approximate quotient; the border s (k + 1/2) has 13 bits and is exact, so that the comparison
            // decides as the exact quotient would, also where the floor is one off beside a whole number
            const float t = __fsub_rn(x[j], m);
            const float k = floorf(t * r), border = s * (k + 0.5f);
            int c = (int)k;
            c += t > border || (t == border && (c & 1));
            word |= (uint32_t)min(max(c, 0), 15) << (4 * j);
        }
    }
    if (at < 0) return;
    const long long to = at + ((long long)kind * p.cache.heads + h) * p.cache.page;
    *reinterpret_cast<uint32_t*>(p.cache.codes + to * (D / 2) + g * (kKvGroup / 2) + lane * 4) = word;
    if (lane == 0) p.cache.params[to * NG + g] = par;
}

// ---- read -------------------------------------------------------------------------------------------
struct KvReadParams {
    KvCache cache;
    KvSeqs seqs;
    void* out[2];                         // [B, Q, H, D] each, contiguous
    int32_t* status;
};

template <typename E, int D>
__global__ void __launch_bounds__(kKvThreads) ears_kv_read_kernel(const KvReadParams p) {
    constexpr int NG = D / kKvGroup;
    wait_for_stream();
    const int lane = threadIdx.x & 7;
    const unsigned per_kind = (unsigned)p.cache.heads * NG, per_row = 2 * per_kind;
    const unsigned items = (unsigned)p.seqs.B * p.seqs.Q * per_row;
    const unsigned item = blockIdx.x * kKvTeams + threadIdx.x / 8;
    if (item >= items) return;
    const unsigned row = item / per_row, in_row = item - row * per_row;
    const int b = (int)(row / (unsigned)p.seqs.Q), i = (int)(row - (unsigned)b * p.seqs.Q);
    const int kind = in_row >= per_kind;
    const unsigned hg = in_row - kind * per_kind;
    const int h = (int)(hg / NG), g = (int)(hg % NG);
    float x[8];
    if (i < kv_count(p.seqs, b)) {
        const long long at = kv_row(p.cache, p.seqs, b, (long long)__ldg(p.seqs.start + b) + i);
        uint32_t word = 0, par = 0x7fc07fc0u;
        if (at >= 0) {
            const long long from = at + ((long long)kind * p.cache.heads + h) * p.cache.page;
            word = *reinterpret_cast<const uint32_t*>(p.cache.codes + from * (D / 2) + g * (kKvGroup / 2) + lane * 4);
            par = p.cache.params[from * NG + g];
        } else if (lane == 0 && p.status) {
            atomicOr(p.status, kDevInvalid);
        }
        const float s = __uint_as_float(par << 16), m = __uint_as_float(par & 0xffff0000u);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __fmaf_rn(s, (float)((word >> (4 * j)) & 15u), m);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
    }
    KvEight<E>::store(reinterpret_cast<E*>(kind ? p.out[1] : p.out[0]) + ((long long)row * per_kind + hg) * kKvGroup + lane * 8, x);
}

}  // namespace ears
