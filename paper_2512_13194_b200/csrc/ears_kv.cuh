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
    int pages, heads, page;               // pages in the pool, heads, tokens per page; a page has less than 2^31 bytes (the host's check)
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
template <typename E> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t min2<uint16_t>(uint32_t a, uint32_t b) {
    uint32_t r; asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r;
}
template <> __device__ __forceinline__ uint32_t min2<f16_t>(uint32_t a, uint32_t b) {
    uint32_t r; asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r;
}
__device__ __forceinline__ uint32_t half_bits(const uint16_t* p) { return __ldg(p); }
__device__ __forceinline__ uint32_t half_bits(const f16_t* p) { return __ldg(&p->bits); }
// Eight consecutive elements as they lie (`vec`: 16-byte aligned), their values, and their smallest and largest, NaN if there is one.
template <typename E> struct KvEight {
    uint32_t w[4];
    __device__ __forceinline__ void load(const E* p, bool vec) {
        if (vec) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = half_bits(p + 2 * i) | half_bits(p + 2 * i + 1) << 16;
        }
    }
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ float2 pair(int i) const { return unpack_pair<E>(w[i]); }
    // over the eight lanes of a group: (smallest, minus the largest) travel together, exact in the elements' type
    __device__ __forceinline__ float2 range() const {
        const uint32_t lo = min2<E>(min2<E>(w[0], w[1]), min2<E>(w[2], w[3]));
        const uint32_t hi = min2<E>(min2<E>(w[0] ^ 0x80008000u, w[1] ^ 0x80008000u), min2<E>(w[2] ^ 0x80008000u, w[3] ^ 0x80008000u));
        uint32_t r = min2<E>(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
#pragma unroll
        for (int e = 4; e; e >>= 1) r = min2<E>(r, __shfl_xor_sync(0xffffffffu, r, e));
        const float2 f = unpack_pair<E>(r);
        return make_float2(f.x, -f.y);
    }
};
template <> struct KvEight<float> {
    float x[8];
    __device__ __forceinline__ void load(const float* p, bool vec) {
        if (vec) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __ldg(p + i);
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
    }
    __device__ __forceinline__ float2 pair(int i) const { return make_float2(x[2 * i], x[2 * i + 1]); }
    __device__ __forceinline__ float2 range() const {
        float lo = x[0], hi = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) { lo = min_nan(lo, x[j]); hi = max_nan(hi, x[j]); }
#pragma unroll
        for (int e = 4; e; e >>= 1) {
            lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, e));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, e));
        }
        return make_float2(lo, hi);
    }
};
// 16 bytes; the results are not read again here
__device__ __forceinline__ void kv_store(float* p, const float (&x)[4]) { __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3])); }
template <typename E>
__device__ __forceinline__ void kv_store(E* p, const float (&x)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_pair<E>(x[0], x[1]), pack_pair<E>(x[2], x[3]), pack_pair<E>(x[4], x[5]), pack_pair<E>(x[6], x[7])));
}

__device__ __forceinline__ float rcp_approx(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ uint2 halves_of(f32x2 v) { uint2 r; asm("mov.b64 {%0, %1}, %2;" : "=r"(r.x), "=r"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ f32x2 add2_down(f32x2 a, f32x2 b) { f32x2 r; asm("add.rm.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }

// ---- write ------------------------------------------------------------------------------------------
struct KvWriteParams {
    KvCache cache;
    KvSeqs seqs;
    const void* x[2];                     // keys, values [B, Q, H, D]
    long long sb[2], sq[2], sh[2];        // strides in elements
    bool vec[2];                          // every group starts on 16 bytes
    int32_t* status;
};

// Warps have a position's keys and values of all heads, eight consecutive values per lane and step: a group is eight lanes, a
// position's place is looked up once, and what a warp loads or stores at once is contiguous.  `parts` warps share a position
// where there are few of them.  Measured, 8 heads of 128: 13100 positions of bf16 written in 24 us (11 at the copy rate; issue 75 %:
// some 190 instructions per step of a warp), 65003 read as bf16 in 60 us (52), as fp32 in 98 (93).  A thread team per group, which looks the
// place up for each, took 55, 129 and more.
constexpr int kKvThreads = 128;
constexpr int kKvUnroll = 4;              // steps whose loads are on their way together

struct KvPlace {
    long long row;                        // of the position's keys in head 0; -1: no place
    int b, i, part;
    bool mine;                            // the position is asked for
};
__device__ __forceinline__ KvPlace kv_place(const KvCache& c, const KvSeqs& s, int parts, int32_t* status) {
    const unsigned warp = (blockIdx.x * kKvThreads + threadIdx.x) / 32, at = warp / (unsigned)parts;
    KvPlace p;
    p.part = (int)(warp - at * parts);
    p.b = (int)(at / (unsigned)s.Q);
    p.i = (int)(at - (unsigned)p.b * s.Q);
    p.row = -1;
    p.mine = p.b < s.B && p.i < kv_count(s, p.b);
    if (p.mine) {
        p.row = kv_row(c, s, p.b, (long long)__ldg(s.start + p.b) + p.i);
        if (p.row < 0 && p.part == 0 && threadIdx.x % 32 == 0 && status) atomicOr(status, kDevInvalid);
    }
    return p;
}

template <typename E, int D>
__global__ void __launch_bounds__(kKvThreads) ears_kv_write_kernel(const KvWriteParams p, int parts) {
    constexpr int NG = D / kKvGroup, PER = D / 8, HEADS = 32 / PER;      // lanes per head, heads per step
    wait_for_stream();
    const int lane = threadIdx.x & 31, d = lane % PER;
    const KvPlace at = kv_place(p.cache, p.seqs, parts, p.status);
    if (!at.mine) return;                                  // the whole warp; the place is waited for behind the first loads
    const int per_kind = (p.cache.heads + HEADS - 1) / HEADS, steps = 2 * per_kind;
    const E* const keys = reinterpret_cast<const E*>(p.x[0]) + at.b * p.sb[0] + at.i * p.sq[0] + d * 8;
    const E* const values = reinterpret_cast<const E*>(p.x[1]) + at.b * p.sb[1] + at.i * p.sq[1] + d * 8;
    uint8_t* const codes = p.cache.codes + at.row * (D / 2) + d * 4;
    uint32_t* const params = p.cache.params + at.row * NG + d / 8;
#pragma unroll 1
    for (int s0 = at.part; s0 < steps; s0 += parts * kKvUnroll) {
        KvEight<E> x[kKvUnroll];
        int rows[kKvUnroll];                               // first token of (kind, head) in a page, -1: none
#pragma unroll
        for (int u = 0; u < kKvUnroll; ++u) {
            const int st = s0 + u * parts, kind = st >= per_kind, h = (st - kind * per_kind) * HEADS + lane / PER;
            rows[u] = st < steps && h < p.cache.heads ? (kind * p.cache.heads + h) * p.cache.page : -1;
            if (rows[u] >= 0) x[u].load(kind ? values + h * p.sh[1] : keys + h * p.sh[0], kind ? p.vec[1] : p.vec[0]);
            else x[u].clear();
        }
#pragma unroll
        for (int u = 0; u < kKvUnroll; ++u) {
            if (s0 + u * parts >= steps) break;            // the whole warp
            const float2 ends = x[u].range();
            const float lo = ends.x, hi = ends.y;
            const uint32_t mb = __float_as_uint(lo);
            uint32_t cut = mb & 0xffff0000u;
            if ((int)mb < 0 && mb != cut) cut += 0x10000u;
            const float m = __uint_as_float(cut);
            const float range = __fmul_rn(__fsub_rn(hi, m), 1.f / 15.f);
            const bool fine = range <= FLT_MAX;            // false for NaN too
            uint32_t sbits = __float_as_uint(range);
            if (sbits & 0xffffu) sbits = (sbits & 0xffff0000u) + 0x10000u;
            const float s = fmaxf(__uint_as_float(sbits), 0x1p-126f);
            // k: floor of an approximate quotient, in the low bits of 2^23 + q rounded down.  The border s (k + 1/2) has 13 bits and
            // is exact, so that the comparison decides as the exact quotient would, also where the floor is one off beside a whole
            // number; a tie goes to the even code.  t >= 0 and the border are compared as integers.  The 2^23s add up to kOffset.
            constexpr uint32_t kOffset = 0x4b000000u * 0x11111111u;
            const float r = rcp_approx(s), half = 0.5f * s;      // s in [2^-126, 2^126): so is 1 / s
            const f32x2 m2 = pack2(-m, -m), r2 = pack2(r, r), s2 = pack2(s, s), h2 = pack2(half, half), big = pack2(8388608.f, 8388608.f),
                        less = pack2(-8388608.f, -8388608.f);
            uint32_t word = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 v = x[u].pair(j);
                const f32x2 t = add2(pack2(v.x, v.y), m2), q = add2_down(mul2(t, r2), big), border = fma2(s2, add2(q, less), h2);
                const uint2 tb = halves_of(t), qb = halves_of(q), bb = halves_of(border);
                word += (qb.x + ((bb.x - tb.x - (qb.x & 1u)) >> 31)) << (8 * j);
                word += (qb.y + ((bb.y - tb.y - (qb.y & 1u)) >> 31)) << (8 * j + 4);
            }
            word -= kOffset;
            if (rows[u] >= 0 && at.row >= 0) {
                *reinterpret_cast<uint32_t*>(codes + (unsigned)rows[u] * (D / 2)) = fine ? word : 0u;
                if (lane % 8 == 0) params[(unsigned)rows[u] * NG] = fine ? (__float_as_uint(s) >> 16) | (__float_as_uint(m) & 0xffff0000u) : 0x7fc07fc0u;
            }
        }
    }
}

// ---- read -------------------------------------------------------------------------------------------
struct KvReadParams {
    KvCache cache;
    KvSeqs seqs;
    void* out[2];                         // [B, Q, H, D] each, contiguous
    int32_t* status;
};

template <typename E, int D>
__global__ void __launch_bounds__(kKvThreads) ears_kv_read_kernel(const KvReadParams p, int parts) {
    constexpr int N = sizeof(E) == 4 ? 4 : 8;              // values per lane and step: 16 bytes of the result
    constexpr int NG = D / kKvGroup, PER = D / N, WARPS = PER > 32 ? PER / 32 : 1, HEADS = PER > 32 ? 1 : 32 / PER;   // steps per head, or heads per step
    wait_for_stream();
    const int lane = threadIdx.x & 31;
    const KvPlace at = kv_place(p.cache, p.seqs, parts, p.status);
    if (at.b >= p.seqs.B) return;
    const int per_kind = (p.cache.heads + HEADS - 1) / HEADS * WARPS, steps = 2 * per_kind;
    const long long out = ((long long)at.b * p.seqs.Q + at.i) * p.cache.heads * D;
    const uint8_t* const codes = p.cache.codes + at.row * (D / 2);
    const uint32_t* const params = p.cache.params + at.row * NG;
    const uint32_t none = at.mine ? 0x7fc07fc0u : 0u;      // without a place: NaN where asked for, zeros where not
#pragma unroll 1
    for (int s0 = at.part; s0 < steps; s0 += parts * kKvUnroll) {
        uint32_t word[kKvUnroll], par[kKvUnroll];
        int place[kKvUnroll];                              // of the first value in the position's result, -1: none
#pragma unroll
        for (int u = 0; u < kKvUnroll; ++u) {
            const int st = s0 + u * parts, kind = st >= per_kind, in = st - kind * per_kind;
            const int h = in / WARPS * HEADS + (HEADS > 1 ? lane / PER : 0), d = (in % WARPS * 32 + lane) % PER * N;
            place[u] = st < steps && h < p.cache.heads ? h * D + d : -1;
            word[u] = 0;
            par[u] = none;
            if (place[u] >= 0 && at.row >= 0) {
                const unsigned from = (unsigned)((kind * p.cache.heads + h) * p.cache.page);
                const uint8_t* at_code = codes + from * (D / 2) + d / 2;
                word[u] = N == 8 ? *reinterpret_cast<const uint32_t*>(at_code) : *reinterpret_cast<const uint16_t*>(at_code);
                par[u] = params[from * NG + d / kKvGroup];
            }
        }
#pragma unroll
        for (int u = 0; u < kKvUnroll; ++u) {
            if (place[u] < 0) continue;
            const int kind = s0 + u * parts >= per_kind;
            const float s = __uint_as_float(par[u] << 16), m = __uint_as_float(par[u] & 0xffff0000u);
            const f32x2 s2 = pack2(s, s), m2 = pack2(m, m), less = pack2(-8388608.f, -8388608.f);
            const uint32_t even = word[u] & 0x0f0f0f0fu, odd = (word[u] >> 4) & 0x0f0f0f0fu;
            float x[N];
            // a code in the low byte of 2^23's bits is 2^23 + c
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const f32x2 c2 = add2(pack2(__uint_as_float(__byte_perm(even, 0x4b000000u, 0x7440 + j)), __uint_as_float(__byte_perm(odd, 0x4b000000u, 0x7440 + j))), less);
                unpack2(fma2(s2, c2, m2), x[2 * j], x[2 * j + 1]);
            }
            kv_store(reinterpret_cast<E*>(kind ? p.out[1] : p.out[0]) + out + place[u], x);
        }
    }
}

}  // namespace ears
