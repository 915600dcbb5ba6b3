// Attention of each sequence's newest positions (K drafts and the token before them, or a single token) over the cache of
// ears_kv.cuh, full or with a sliding window and first tokens that stay visible.
//
// For a row q at position p and the tokens t it sees, out = sum_t softmax(scale q . k_t) v_t.  With k_t = m + s c in groups of 64
//     q . k_t = sum_g s_tg (q_g . c_tg) + m_tg sum(q_g),      out_g = sum_t (P_t s_tg) c_tg + sum_t P_t m_tg
// so that the products run on the codes themselves, and scales and minima touch a value per token and row only.
//
// What bounds it: 4.5 bits per value have to be read, and each code turned into a 16-bit operand.  A code c placed in the lowest
// bits of a half-precision number IS the subnormal c 2^-24, and one in bits 4..7 is c 2^-20, which tensor cores take at full
// speed: two masks and one shift make eight operands of a 32-bit word, with nothing to subtract; the powers of two go into q
// (odd dimensions of keys / 16) and into the result (odd dimensions of values).  A product of a subnormal is added to 2^-24 of the largest
// product's exponent as a normal number's would be, that is to 2^-14 of the largest weight in a tile times one code: where one token of a
// tile outweighs the others by 2^15, 5 % of theirs and 2^-15 of its own was seen to go.  (8-bit floating-point operands would take fewer
// operations still, c 2^-9 being one as it stands, but m16n8k32 with them is made of conversions and 16-bit products here:
// 68 conversions per tile of 16 tokens counted, and 437 instructions against 386.)
// Measured: 64 single tokens, 64 / 8 heads of 128, 6000 to 8192 tokens (527 MB): 115 us, 70 % of the copy rate, 266 instructions per tile of
// 16 tokens; 128 x 5 positions, 32 / 8 heads, 680 MB: 246 to 260 us by the lengths drawn, 403 instructions, of them 48 matrix products.
// No unit is full (issue 53 and 44 %, ALU 55 and 35 %, matrix products 27 and 41 %): each scheduler has two or three warps, whose
// matrix products and logic overlap in part only.
//
// The products have 16 tokens (or, for the values, dimensions) as rows and eight of the head group's
// queries as columns: M = Q x heads per key head is seldom more than a few eights, and no work goes into padding a tile of
// 64 or 128.  Scores come out with a token per pair of rows of a thread, where a token's scale and minimum are two registers, and
// become the second product's operand through an 8x8 transpose.  The order of dimensions within a product is free as long as
// both operands agree: a thread takes consecutive codes, 8 (keys) or 4 (values) bytes of a token and group at a time.
//
// Work: a unit is (sequence, key head, block of NT x 8 rows); its tokens are cut into chunks of 64, of which each warp takes a tile of 16.
// Every CTA of the grid, as many as are resident at once, takes an equal run of the chunks of all units, whatever the
// sequences' lengths, which it reads on the device.  Units that are cut are joined by a second small kernel in a fixed order.
// A warp's tiles come through a ring of its own, copied asynchronously two at a time: no barrier among warps until a unit ends.
#pragma once
#include <climits>
#include <type_traits>

#include "ears_kv.cuh"

namespace ears {

constexpr int kKaWarps = 4, kKaThreads = kKaWarps * 32;
constexpr int kKaTile = 16;                         // tokens of a warp's tile
constexpr int kKaChunk = kKaWarps * kKaTile;
constexpr int kKaAhead = 8;                         // what starting and ending a unit costs, in chunks: with 4, 8, 12, 16 of them 277, 247, 246, 251 us
                                                    // for 128 x 5 positions as above, 25.2, 22.9, 23.7, 23.3 for 8 x 6, 49.6, 48.6, 47.1, 47.3 for a window
// A row's weights are P = 2^(score - reference).  The reference, a whole number, is raised when a P passes 2^-18, to where the largest is
// between 2^-31 and 2^-30: their sums with minima up to the type's largest number stay finite, and minima down to 2^-100 keep their bits.
// The second product's half-precision operands are P s cs, with a power of two cs for each group that goes by the largest P s of a warp's tiles: it
// brings that to 2^4 (2^6 to 2^10 for 8192 to 131072 tokens of a warp) when one may pass 2^15.  Not by the largest s, which may be that of a token of no
// weight (131072 tokens, one of them with values 4096 times the others' and a weight of e^-60: an error of 0.08 of the result that way, 0.0015 this
// way, its own rounding).  What falls below half precision's normal numbers is off by 2^-25 at most, so that a warp's n tokens are right to 2^-12 of a
// row's sum of P s cs as long as the largest of its sums of P s cs c is 15 n 2^-13 or more.  That is looked at when the unit's tiles are through; where a
// row has less, as one that does not see a token whose large values another row's result is made of, the warp takes its tiles once more with a cs of
// each row's own (a batch where every last draft is such a token, 128 x 5 positions: 615 us beside 248).  A lower goal than 2^4 leaves no room
// for rows that differ, a higher one has the powers set again more often: 2^6 250 us, 2^8 254, where 2^4 takes 246.
constexpr int kKaLow = 30;
constexpr float kKaTop = -18.f, kKaMost = 0x1p15f;
constexpr int kKaMinGoal = 4, kKaMaxGoal = 10, kKaFar = 1000;

template <int D, int NT> struct KaShape {
    static constexpr int NG = D / kKvGroup;
    static constexpr int RB = D / 2;                // bytes of a token's codes
    static constexpr int kCodes = kKaTile * RB, kPars = kKaTile * NG * 4;
    static constexpr int kTileBytes = 2 * (kCodes + kPars);        // keys' codes, values' codes, keys' parameters, values' parameters
    static constexpr int kStage = 2 * kTileBytes;   // two tiles
    // CTAs per SM that registers allow, and as many stages as their shared memory does
    static constexpr int kCtas = NT == 1 && D <= 128 ? 3 : 2;
    static constexpr int kStages = D == 64 ? (kCtas == 3 ? 8 : 10) : D == 128 ? (kCtas == 3 ? 4 : 5) : NT == 1 ? 3 : 2;
    static constexpr int kSmem = kKaWarps * kStages * kStage;
    // 16-byte pieces of row i are kept in another order, so that what a warp loads at once lies in different banks
    __device__ static __forceinline__ int swizzle(int i) { return RB == 128 ? ((i & 1) << 2) | (i & 2) : RB == 64 ? (i & 2) : 0; }
};
// product row i of each eight holds token (i >> 1) | (i & 1) << 2, so that the values' token pairs lie in different banks
__device__ __forceinline__ int ka_row_of(int t) { return (t & 8) | ((t & 3) << 1) | ((t >> 2) & 1); }

struct KaParams {
    KvCache cache;
    KvSeqs seqs;
    const void* q;
    long long sb, sq, sh;                 // q's strides in elements
    bool vec;
    int group;                            // query heads per key head
    int M, blocks;                        // rows of a unit's sequence and head, Q x group; blocks of NT x 8 of them
    float scale2;                         // scale x log2(e)
    int window, sinks;
    void* out;                            // [B, Q, H x group, D]
    float* lse;                           // [B, Q, H x group] or NULL
    int4* cut;                            // [CTAs] the unit that this CTA begins and leaves to others: (b, unit of it, last CTA), or b = -1
    float* part_o;                        // [CTAs][2][NT x 8][D]
    float2* part_ml;                      // [CTAs][2][NT x 8]
    int32_t* status;
};

// ---- lengths --------------------------------------------------------------------------------------------
struct KaSpan {
    int start, count;
    int sinks, first, tiles;              // tiles 0 .. sinks-1, then first .. first + (tiles - sinks) - 1
    bool bad;
    __device__ __forceinline__ int tile(int i) const { return i < sinks ? i : first + (i - sinks); }
    __device__ __forceinline__ int chunks() const { return max(1, (tiles + kKaWarps - 1) / kKaWarps); }
};
__device__ __forceinline__ KaSpan ka_span(const KaParams& p, int b) {
    KaSpan s;
    s.start = __ldg(p.seqs.start + b);
    s.count = kv_count(p.seqs, b);
    s.bad = s.count > 0 && (s.start < 0 || (long long)s.start + s.count > (long long)p.seqs.width * p.cache.page);
    s.sinks = s.first = s.tiles = 0;
    if (s.bad || s.count == 0) s.start = 0;      // no tile is looked at, and no position that passes 31 bits formed
    if (s.count > 0 && !s.bad) {
        const int last = (s.start + s.count - 1) / kKaTile;
        if (p.window) {
            s.first = max(0, s.start - p.window + 1) / kKaTile;
            s.sinks = min(p.sinks / kKaTile + (p.sinks % kKaTile != 0), s.first);
        }
        s.tiles = s.sinks + last - s.first + 1;
    }
    return s;
}

// ---- instructions -----------------------------------------------------------------------------------------
// c = a b + c (ZERO: a b)
template <bool ZERO = false>
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (ZERO) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    } else {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t r; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(a) : "memory"); return r; }
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory");
    return r;
}
template <int N> __device__ __forceinline__ void lds_words(uint32_t a, uint32_t (&r)[N]) {
    if constexpr (N == 1) {
        r[0] = lds32(a);
    } else if constexpr (N == 2) {
        const uint2 w = lds64(a);
        r[0] = w.x; r[1] = w.y;
    } else {
        static_assert(N == 4, "groups");
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
    }
}
__device__ __forceinline__ float2 apart(f32x2 p) { float2 r; unpack2(p, r.x, r.y); return r; }
__device__ __forceinline__ float scale_of(uint32_t par) { return __uint_as_float(par << 16); }
__device__ __forceinline__ float minimum_of(uint32_t par) { return __uint_as_float(par & 0xffff0000u); }
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) { return pack_pair<f16_t>(lo, hi); }
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}
__device__ __forceinline__ float across_max(float x) {      // over the eight lanes with the same column
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
__device__ __forceinline__ float across_sum(float x) {
    x += __shfl_xor_sync(0xffffffffu, x, 4);
    x += __shfl_xor_sync(0xffffffffu, x, 8);
    return x + __shfl_xor_sync(0xffffffffu, x, 16);
}

template <typename E>
__device__ __noinline__ uint4 ka_unaligned(const E* p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = half_bits(p + 2 * i) | half_bits(p + 2 * i + 1) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- a row's result ------------------------------------------------------------------------------------------
template <typename E, int N>
__device__ __forceinline__ void ka_store(E* out, const float (&x)[N]) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pack_pair<E>(x[2 * i], x[2 * i + 1]);
    if constexpr (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) reinterpret_cast<uint4*>(out)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else if constexpr (N == 4) {
        *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
    } else {
        *reinterpret_cast<uint32_t*>(out) = w[0];
    }
}
// where row `row` of (b, h) goes: [B, Q, H x group]
__device__ __forceinline__ long long ka_out_row(const KaParams& p, int b, int h, int row) {
    const int i = row / p.group, g = row - i * p.group;
    return ((long long)b * p.seqs.Q + i) * ((long long)p.cache.heads * p.group) + (long long)h * p.group + g;
}
__device__ __forceinline__ float ka_lse(float ref, float l) { return l == 0.f ? -INFINITY : ((ref - kKaLow) + __log2f(l * 0x1p30f)) * 0.69314718055994531f; }
// the inverse of a sum of weights; 0 where there are none, NaN where one is
__device__ __forceinline__ float ka_inverse(float sum) { return sum != 0.f ? rcp_approx(sum) : 0.f; }
__device__ __forceinline__ float pow2_of(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }      // -126 <= e <= 127
__device__ __forceinline__ float inverse_pow2(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }       // x >= 0
__device__ __forceinline__ uint32_t upper_halves(float x, float y) { return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632); }
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) { uint32_t r; asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }

// ---- the kernel ------------------------------------------------------------------------------------------------
// E: the queries' type.  FINE: a half-precision weight is off by up to 2^-11 (2^-12.3 in the mean), times codes that lie between 0 and 15:
// nothing beside a bfloat16 result's own 2^-9, but twice a half-precision result's rounding.  For those what a weight lost is
// added back times the middle code, 7.5, with the minima, so that its error meets codes less their middle.  (Weights in two halves
// would be exact and double the second product: 72000 tokens x 8 x 8 heads of 128, 20 rows: 305 us against 253.)
template <typename E, int D, int NT>
__global__ void __launch_bounds__(kKaThreads, KaShape<D, NT>::kCtas) ears_kv_attention_kernel(const KaParams p) {
    using S = KaShape<D, NT>;
    constexpr int NG = S::NG, RB = S::RB, ROWS = NT * 8;
    constexpr bool FINE = std::is_same<E, f16_t>::value;
    // tiles taken together, as registers allow: 128 x 5 positions take 269 us by one, 246 by two
    constexpr int SUB = NT * NG <= 6 ? 2 : 1;
    constexpr bool QREG = NT * NG <= 4;                   // queries' operands stay in registers
    constexpr uint32_t M0 = 0x000f000fu, M1 = 0x00f000f0u;

    extern __shared__ __align__(128) unsigned char ring_mem[];
    // queries' operands; with NT = 1 in the stage of warp 1's ring that is filled last, until they are in registers
    constexpr bool QRING = NT == 1;
    static_assert(!QRING || (QREG && NG * 1024 <= S::kStage), "queries in a stage");
    static_assert(kKaWarps * ROWS * D * 4 <= S::kSmem, "the warps' results meet in the ring's memory");
    __shared__ uint4 s_q_own[QRING ? 1 : NT * NG * 64];
    uint4* const s_q = QRING ? reinterpret_cast<uint4*>(ring_mem + (2 * S::kStages - 1) * S::kStage) : s_q_own;
    __shared__ __align__(8) float s_fr[ROWS], s_qs[NG][ROWS];
    __shared__ float s_m[kKaWarps][ROWS], s_l[kKaWarps][ROWS];
    __shared__ __align__(8) float s_cs[kKaWarps][NG][ROWS];
    __shared__ float2 s_ml[ROWS];
    __shared__ __align__(8) int s_ask[ROWS];
    __shared__ int s_pos[ROWS], s_out[ROWS], s_sum[kKaWarps], s_b, s_off;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, j = lane & 3;
    wait_for_stream();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- this CTA's share of all chunks (their number fits 31 bits: the host's check)
    const int per_seq = p.cache.heads * p.blocks;
    const int each = (p.seqs.B + kKaThreads - 1) / kKaThreads;
    const int b0 = min(p.seqs.B, tid * each), b1 = min(p.seqs.B, b0 + each);
    int own = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) own += ka_span(p, b).chunks() * per_seq;
    int before = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += up;
    }
    if (lane == 31) s_sum[warp] = before;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kKaWarps; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    before -= own;
    // no more chunks than CTAs go one each; else what a unit costs beside its chunks counts as `ahead` more, in front of them
    const int ahead = total > (int)gridDim.x ? kKaAhead : 0;
    before += b0 * per_seq * ahead;
    own += (b1 - b0) * per_seq * ahead;
    total += p.seqs.B * per_seq * ahead;
    const int ctas = min((int)gridDim.x, total), share = total / ctas, longer = total - share * ctas;   // the first `longer` have one more
    if (tid == 0) p.cut[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if (blockIdx.x >= ctas) return;
    const int begin = (int)blockIdx.x * share + min((int)blockIdx.x, longer);
    if (own && before <= begin && begin < before + own) {
        int base = before, b = b0;
#pragma unroll 1
        for (;; ++b) {
            const int n = (ka_span(p, b).chunks() + ahead) * per_seq;
            if (begin < base + n) break;
            base += n;
        }
        s_b = b;
        s_off = begin - base;
    }
    __syncthreads();
    int left = share + (blockIdx.x < longer), b = s_b, off = s_off;        // cost still to do; the sequence it starts in, and where there

    // ---- addresses that do not change
    const uint32_t ring = smem_u32(ring_mem) + warp * (S::kStages * S::kStage);
    const int my_token = (r >> 1) | ((r & 1) << 2);
    const uint32_t get_k = r * RB + ((S::swizzle(r) + (j >> 1)) << 4) + (j & 1) * 8;
    const uint32_t get_v = S::kCodes + j * RB + ((S::swizzle(j) + (r >> 2)) << 4) + (r & 3) * 4;
    const uint32_t get_p = 2 * S::kCodes + my_token * NG * 4;
    // copies: half a warp per tile; a lane has every 16th piece of 16 bytes, its tokens t0, t0 + 256 / RB, ...
    const int l16 = lane & 15, t0 = l16 / (RB / 16), c16 = l16 % (RB / 16);
    const uint32_t put_tile = ring + (lane >> 4) * S::kTileBytes;
    const uint32_t put_k = (uint32_t)(c16 ^ S::swizzle(ka_row_of(t0))) << 4, put_v = (uint32_t)(c16 ^ S::swizzle(t0)) << 4;
    const long long v_bytes = (long long)p.cache.heads * p.cache.page * RB;              // from a page's keys to its values

    KaSpan span = ka_span(p, b);
    while (left > 0) {
        const int chunks = span.chunks(), cost = chunks + ahead, unit = off / cost, at0 = off - unit * cost;
        if (unit >= per_seq) {
            span = ka_span(p, ++b);
            off = 0;
            continue;
        }
        const int taken = min(cost - at0, left), c0 = max(0, at0 - ahead), c1 = max(0, at0 + taken - ahead);
        off += taken;
        left -= taken;
        if (c0 == c1) continue;
        const int h = unit / p.blocks, row0 = (unit - h * p.blocks) * ROWS;
        const int last_pos = span.start + max(span.count - 1, 0);

        // ---- this warp's tiles, first + 4 k; a stage of its ring holds two
        const int first = c0 * kKaWarps + warp;
        const int n_tiles = max(0, (min(c1 * kKaWarps, span.tiles) - first + kKaWarps - 1) / kKaWarps);
        const int n_pairs = (n_tiles + 1) / 2;
        int at = 0;                                         // a sixteenth of the row of tile `lane` of the current 32, -1: no page
        const unsigned char* from_k = p.cache.codes + (long long)h * p.cache.page * RB + l16 * 16;
        const unsigned char* from_p = reinterpret_cast<const unsigned char*>(p.cache.params) + (long long)h * p.cache.page * (NG * 4) +
                                      (NG == 4 ? l16 * 16 : (l16 & (4 * NG - 1)) * 16 + (l16 & (4 * NG) ? v_bytes / 8 : 0));
        auto issue = [&](int i, int slot) {
            if ((i & 15) == 0) {
                at = -1;
                if (2 * i + lane < n_tiles) at = (int)(kv_row(p.cache, p.seqs, b, (long long)span.tile(first + (2 * i + lane) * kKaWarps) * kKaTile) >> 4);
            }
            const int row = __shfl_sync(0xffffffffu, at, ((2 * i) & 31) + (lane >> 4));
            const uint32_t to = put_tile + slot * S::kStage;
            if (row >= 0) {
                const unsigned char *k = from_k + (unsigned long long)(unsigned)row * (16 * RB), *v = k + v_bytes;
                const unsigned char* q = from_p + (unsigned long long)(unsigned)row * (64 * NG);
#pragma unroll
                for (int n = 0; n < RB / 16; ++n) {
                    // token t0 + tn: which bits of the row's number and of its swizzle tn adds is known
                    const int tn = n * (256 / RB), in = ka_row_of(tn);
                    copy16(to + ka_row_of(t0) * RB + (put_k ^ (S::swizzle(in) << 4)) + in * RB, k + n * 256);
                    copy16(to + S::kCodes + t0 * RB + (put_v ^ (S::swizzle(tn) << 4)) + tn * RB, v + n * 256);
                }
                if constexpr (NG == 1) {
                    if (l16 < 8) copy16(to + 2 * S::kCodes + l16 * 16, q);
                } else if constexpr (NG == 2) {
                    copy16(to + 2 * S::kCodes + l16 * 16, q);
                } else {
                    copy16(to + 2 * S::kCodes + l16 * 16, q);
                    copy16(to + 2 * S::kCodes + S::kPars + l16 * 16, q + v_bytes / 8);     // 4 NG bytes a token beside RB = 32 NG
                }
            } else if (2 * i + (lane >> 4) < n_tiles) {
                // no page: its tokens' scales and minima are NaN, and so are the rows that see them
#pragma unroll
                for (int n = 0; n < 2 * NG; ++n) sts32(to + 2 * S::kCodes + (l16 + 16 * n) * 4, 0x7fc07fc0u);
                if (l16 == 0 && p.status) atomicOr(p.status, kDevInvalid);
            }
        };
        // ---- queries, eight elements of a row per thread: on their way while the page table is looked up
        constexpr int TPR = D / 8, RPP = kKaThreads / TPR, PASSES = (ROWS + RPP - 1) / RPP;
        const int q_c = tid % TPR;
        uint4 raw[PASSES];
        int q_at[PASSES], q_pos[PASSES];                   // where the row's result goes, -1: no row; its position in the call
#pragma unroll
        for (int n = 0; n < PASSES; ++n) {
            const int in_block = tid / TPR + n * RPP, row = row0 + in_block, i = row / p.group, head = h * p.group + (row - i * p.group);
            const bool real = in_block < ROWS && row < p.M;
            q_at[n] = real ? i * (p.cache.heads * p.group) + head : -1;
            q_pos[n] = real ? i : (p.M - 1) / p.group;
            raw[n] = make_uint4(0, 0, 0, 0);
            if (real) {
                const E* src = reinterpret_cast<const E*>(p.q) + b * p.sb + i * p.sq + head * p.sh + q_c * 8;
                if (p.vec) raw[n] = __ldg(reinterpret_cast<const uint4*>(src));
                else raw[n] = ka_unaligned(src);
            }
        }
#pragma unroll 1
        for (int i = 0; i < S::kStages - 1; ++i) {
            if (i < n_pairs) issue(i, i);
            copies_commit();
        }

        // normalised to below 2^15 per row, in half precision, odd dimensions / 16
#pragma unroll
        for (int n = 0; n < PASSES; ++n) {
            const int row = tid / TPR + n * RPP;
            const uint32_t w[4] = {raw[n].x, raw[n].y, raw[n].z, raw[n].w};
            float v[8], big = 0.f, sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = unpack_pair<E>(w[e]);
                v[2 * e] = f.x; v[2 * e + 1] = f.y;
                sum += f.x + f.y;
                big = max_nan(big, max_nan(fabsf(f.x), fabsf(f.y)));
            }
#pragma unroll
            for (int d = 1; d < TPR; d <<= 1) {
                big = max_nan(big, __shfl_xor_sync(0xffffffffu, big, d));
                if (d < 8) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            }
            const int ex = max((int)(__float_as_uint(big) >> 23) - 127, -100);
            const float up = __uint_as_float((uint32_t)(127 + 14 - ex) << 23), odd = up * 0.0625f;
            if (row < ROWS) {
                if (q_c % 8 == 0) s_qs[q_c / 8][row] = sum * p.scale2;
                if (q_c == 0) {
                    // a code stands for c 2^-24, the row for q 2^(14 - ex)
                    s_fr[row] = big <= FLT_MAX ? p.scale2 * 1024.f * __uint_as_float((uint32_t)(127 + ex) << 23) : NAN;
                    s_pos[row] = min(last_pos, span.start + q_pos[n]);
                    s_out[row] = q_at[n];
                    s_ask[row] = q_at[n] >= 0 && q_pos[n] < span.count;
                }
                // the order in which codes come out of a word
                s_q[(((row >> 3) * NG + q_c / 8) * 2 + (q_c & 1)) * 32 + (row & 7) * 4 + (q_c % 8) / 2] =
                    make_uint4(f16_pair(v[0] * up, v[4] * up), f16_pair(v[1] * odd, v[5] * odd), f16_pair(v[2] * up, v[6] * up), f16_pair(v[3] * odd, v[7] * odd));
            }
        }
        __syncthreads();
        uint4 qf[QREG ? NT : 1][QREG ? NG : 1][2];
        float fr[QREG ? NT : 1][2], qs[QREG ? NT : 1][2][NG];
        if constexpr (QREG) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int col = 0; col < 2; ++col) {
                    fr[nt][col] = s_fr[nt * 8 + 2 * j + col];
#pragma unroll
                    for (int g = 0; g < NG; ++g) qs[nt][col][g] = s_qs[g][nt * 8 + 2 * j + col];
                }
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int w = 0; w < 2; ++w) qf[nt][g][w] = s_q[((nt * NG + g) * 2 + w) * 32 + lane];
            }
        }
        const int pmin = s_pos[0], pmax = s_pos[ROWS - 1];
        if constexpr (QRING) __syncthreads();
        float mb[NT][2], l[NT][2], om[NT][2][NG], o[NT][NG * 4][4];        // mb: minus the reference
        uint32_t unset;                                     // rows that have seen no token yet, a bit per (nt, column)
        float cs[NG];                                       // powers of two; with a row's own s_cs instead
        auto cs_of = [&](int nt, int g) { return *reinterpret_cast<const f32x2*>(&s_cs[warp][g][nt * 8 + 2 * j]); };

        // tiles [lo, hi) of the unit's list are seen whole by all rows; two of this warp's at once if the first is in [lo, hi - 4)
        const int lo = p.window ? span.sinks + max(0, pmax - p.window + kKaTile) / kKaTile - span.first : 0;
        const int hi = min(span.sinks + (pmin + 1) / kKaTile - span.first, c1 * kKaWarps);
        // Scores of the SUB tiles at `stage` relative to the running maximum, base 2, [nt][2 e + col] for token e of this thread's,
        // and the tokens' parameters for the values.
        auto scores = [&](uint32_t stage, float (&sc)[NT][4 * SUB], uint32_t (&vp)[2 * SUB][NG]) {
            uint32_t kp[2 * SUB][NG];
            f32x2 dot[NT][2 * SUB], part[NT][2 * SUB];
#pragma unroll
            for (int e = 0; e < 2 * SUB; ++e) {
                lds_words<NG>(stage + (e >> 1) * S::kTileBytes + get_p + (e & 1) * 8 * NG * 4, kp[e]);
                lds_words<NG>(stage + (e >> 1) * S::kTileBytes + get_p + S::kPars + (e & 1) * 8 * NG * 4, vp[e]);
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                uint2 kw[SUB][2];
                float acc[SUB][NT][4];
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    const uint32_t from = stage + u * S::kTileBytes + (get_k ^ (g << 5));
                    kw[u][0] = lds64(from);
                    kw[u][1] = lds64(from + 8 * RB);
                }
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint4 q[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (QREG) q[nt] = qf[nt][g][w];
                        else q[nt] = s_q[((nt * NG + g) * 2 + w) * 32 + lane];
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int u = 0; u < SUB; ++u) {
                            const uint32_t x0 = (w ? kw[u][0].y : kw[u][0].x) >> (8 * half), x1 = (w ? kw[u][1].y : kw[u][1].x) >> (8 * half);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const uint32_t b0 = half ? q[nt].z : q[nt].x, b1 = half ? q[nt].w : q[nt].y;
                                if (w == 0 && half == 0) mma_f16<true>(acc[u][nt], x0 & M0, x1 & M0, x0 & M1, x1 & M1, b0, b1);
                                else mma_f16(acc[u][nt], x0 & M0, x1 & M0, x0 & M1, x1 & M1, b0, b1);
                            }
                        }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    f32x2 sums;
                    if constexpr (QREG) sums = pack2(qs[nt][0][g], qs[nt][1][g]);
                    else sums = *reinterpret_cast<const f32x2*>(&s_qs[g][nt * 8 + 2 * j]);
#pragma unroll
                    for (int e = 0; e < 2 * SUB; ++e) {
                        const float sk = scale_of(kp[e][g]), mk = minimum_of(kp[e][g]);
                        const f32x2 x = pack2(acc[e >> 1][nt][2 * (e & 1)], acc[e >> 1][nt][2 * (e & 1) + 1]);
                        dot[nt][e] = g ? fma2(x, pack2(sk, sk), dot[nt][e]) : mul2(x, pack2(sk, sk));
                        part[nt][e] = fma2(pack2(mk, mk), sums, g ? part[nt][e] : pack2(mb[nt][0], mb[nt][1]));
                    }
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                f32x2 f;
                if constexpr (QREG) f = pack2(fr[nt][0], fr[nt][1]);
                else f = *reinterpret_cast<const f32x2*>(&s_fr[nt * 8 + 2 * j]);
#pragma unroll
                for (int e = 0; e < 2 * SUB; ++e) {
                    const float2 x = apart(fma2(dot[nt][e], f, part[nt][e]));
                    sc[nt][2 * e] = x.x;
                    sc[nt][2 * e + 1] = x.y;
                }
            }
        };
        // 2^6 above where a row's products are too small for the warp's tokens
        const int aim = min(kKaMaxGoal, max(kKaMinGoal, 24 - __clz(max(n_tiles, 1) * kKaTile)));
        // ---- all tiles; ROWWISE: with a cs of each row's own
        auto sweep = [&](auto rowwise) {
            constexpr bool ROWWISE = decltype(rowwise)::value;
            unset = (1u << (2 * NT)) - 1;
#pragma unroll
            for (int g = 0; g < NG; ++g) cs[g] = 1.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int col = 0; col < 2; ++col) {
                    mb[nt][col] = 0.f;
                    l[nt][col] = 0.f;
#pragma unroll
                    for (int g = 0; g < NG; ++g) om[nt][col][g] = 0.f;
                }
#pragma unroll
                for (int n = 0; n < NG * 4; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[nt][n][k] = 0.f;
            }
            float sc[NT][4 * SUB];
            uint32_t vp[2 * SUB][NG], stage = ring;
            int slot = 0;
#pragma unroll 1
            for (int k = 0; k < n_tiles; k += SUB) {
                const int place = first + kKaWarps * k;
                {
                    if (SUB == 2 || !(k & 1)) {
                        copies_wait<S::kStages - 1>();
                        __syncwarp();
                    }
                    scores(stage, sc, vp);
                    // masks, where a tile needs them
                    if (place < lo || place + (SUB - 1) * kKaWarps >= hi) {
#pragma unroll
                        for (int u = 0; u < SUB; ++u) {
                            const int tt = k + u < n_tiles ? span.tile(place + u * kKaWarps) * kKaTile : INT_MAX - kKaTile;
#pragma unroll
                            for (int e = 2 * u; e < 2 * u + 2; ++e) {
                                const int t = tt + (e & 1) * 8 + my_token;
                                bool lost = false;                     // values of no use: rows that see the token become NaN by their score
#pragma unroll
                                for (int g = 0; g < NG; ++g)
                                    lost = lost || !(scale_of(vp[e][g]) <= FLT_MAX) || !(fabsf(minimum_of(vp[e][g])) <= FLT_MAX);
                                if (lost || t > pmax || (p.window && t >= p.sinks && t <= pmin - p.window)) {
#pragma unroll
                                    for (int g = 0; g < NG; ++g) vp[e][g] = 0;
                                }
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int col = 0; col < 2; ++col) {
                                        const int pos = s_pos[nt * 8 + 2 * j + col];
                                        float& v = sc[nt][2 * e + col];
                                        if (lost) v = NAN;
                                        if (t > pos || (p.window && t >= p.sinks && t <= pos - p.window)) v = -INFINITY;
                                    }
                            }
                        }
                    }

                    float most = sc[0][0], bound = 0.f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4 * SUB; ++c) most = fmaxf(most, sc[nt][c]);
                    const float heaviest = fmaxf(ex2_approx(most), kKaMost * 0x1p-126f);       // so that s cs alone stays below 2^126, too
                    float sv[NG];
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        sv[g] = 0.f;
#pragma unroll
                        for (int e = 0; e < 2 * SUB; ++e) sv[g] = fmaxf(sv[g], scale_of(vp[e][g]));
                        bound = fmaxf(bound, sv[g] * cs[g] * heaviest);
                    }
                    if (ROWWISE || __any_sync(0xffffffffu, unset != 0 || most > kKaTop || bound > kKaMost)) {
                        const uint32_t fresh = unset;                  // rows without weights so far
                        float top[NT][2];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int col = 0; col < 2; ++col) {
                                top[nt][col] = sc[nt][col];
#pragma unroll
                                for (int e = 1; e < 2 * SUB; ++e) top[nt][col] = fmaxf(top[nt][col], sc[nt][2 * e + col]);
                            }
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1)               // all rows' at once: their latencies overlap
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int col = 0; col < 2; ++col) top[nt][col] = fmaxf(top[nt][col], __shfl_xor_sync(0xffffffffu, top[nt][col], d));
                        int raised[NT][2], lift = kKaFar;              // log2 of what weights shrink by; the least of it among rows that have weights
                        float2 big[ROWWISE ? NT : 1][NG];              // the largest P s 2^18 here, of each row or of all
#pragma unroll
                        for (int nt = 0; nt < (ROWWISE ? NT : 1); ++nt)
#pragma unroll
                            for (int g = 0; g < NG; ++g) big[nt][g] = make_float2(0.f, 0.f);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int col = 0; col < 2; ++col) {
                                const uint32_t bit = 1u << (2 * nt + col);
                                const bool raise = top[nt][col] > -kKaLow || ((fresh & bit) && top[nt][col] > -INFINITY);
                                const float d = raise ? ceilf(top[nt][col] + kKaLow) : 0.f;
                                if (raise) unset &= ~bit;
                                mb[nt][col] -= d;
#pragma unroll
                                for (int e = 0; e < 2 * SUB; ++e) sc[nt][2 * e + col] -= d;
                                raised[nt][col] = (int)fminf(fmaxf(d, 0.f), (float)kKaFar);
                                if (!(fresh & bit)) lift = min(lift, raised[nt][col]);
                                const float alpha = (fresh & bit) || raised[nt][col] > 126 ? 0.f : pow2_of(-raised[nt][col]);
                                l[nt][col] *= alpha;
#pragma unroll
                                for (int g = 0; g < NG; ++g) om[nt][col][g] *= alpha;
                            }
#pragma unroll
                            for (int e = 0; e < 2 * SUB; ++e) {
                                const float wx = ex2_approx(sc[nt][2 * e] + 18.f), wy = ex2_approx(sc[nt][2 * e + 1] + 18.f);
#pragma unroll
                                for (int g = 0; g < NG; ++g) {
                                    float2& b = big[ROWWISE ? nt : 0][g];
                                    b.x = fmaxf(b.x, wx * scale_of(vp[e][g]));
                                    b.y = fmaxf(b.y, wy * scale_of(vp[e][g]));
                                }
                            }
                        }
                        auto scale_o = [&](int nt, int g, int col, int by) {        // times 2^by
                            const float ratio = (fresh >> (2 * nt + col)) & 1 || by < -126 ? 0.f : pow2_of(min(by, 127));
#pragma unroll
                            for (int n = 0; n < 4; ++n) { o[nt][g * 4 + n][col] *= ratio; o[nt][g * 4 + n][2 + col] *= ratio; }
                        };
                        if constexpr (!ROWWISE) {
                            float all[NG];
#pragma unroll
                            for (int g = 0; g < NG; ++g) all[g] = fmaxf(big[0][g].x, big[0][g].y);
                            lift = __reduce_min_sync(0xffffffffu, lift);
#pragma unroll
                            for (int g = 0; g < NG; ++g)           // not negative: ordered as whole numbers are
                                all[g] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(all[g])));
#pragma unroll
                            for (int g = 0; g < NG; ++g) {
                                const int before = exponent_of(cs[g]), size = exponent_of(all[g]) - 18;
                                const int limit = 124 - exponent_of(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(sv[g]))));
                                const int goal = min(aim - size, min(limit, 126));
                                int power = before;
                                // all weights so far have shrunk by 2^lift, from 2^15 at the most
                                if (size + before >= 15 || before > limit) power = goal;
                                else if (lift > 15 - aim) power = max(before, min(before + lift - (15 - aim), goal));
                                cs[g] = pow2_of(power);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int col = 0; col < 2; ++col) scale_o(nt, g, col, power - before - raised[nt][col]);
                            }
                        } else {
                            uint32_t both[NT][NG];                     // the upper 16 bits of two rows' values
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int g = 0; g < NG; ++g) both[nt][g] = upper_halves(big[nt][g].x, big[nt][g].y);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int g = 0; g < NG; ++g) both[nt][g] = max_halves(both[nt][g], __shfl_xor_sync(0xffffffffu, both[nt][g], d));
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int g = 0; g < NG; ++g) {
                                    float2* const own = reinterpret_cast<float2*>(&s_cs[warp][g][nt * 8 + 2 * j]);
                                    const float2 was = *own;
                                    float is[2];
#pragma unroll
                                    for (int col = 0; col < 2; ++col) {
                                        const bool first = (fresh >> (2 * nt + col)) & 1;
                                        const int before = exponent_of(col ? was.y : was.x), size = (int)((both[nt][g] >> (16 * col + 7)) & 255) - 127 - 18;
                                        int power = first ? 126 : min(before + raised[nt][col], 126);
                                        if (first || size + power >= 15) power = min(kKaMaxGoal - size, 126);
                                        scale_o(nt, g, col, power - before - raised[nt][col]);
                                        is[col] = pow2_of(power);
                                    }
                                    __syncwarp();
                                    if (r == 0) *own = make_float2(is[0], is[1]);
                                }
                            __syncwarp();
                        }
                    }

                    // weights
                    f32x2 wt[NT][2 * SUB];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2 * SUB; ++e) {
                            const f32x2 w = pack2(ex2_approx(sc[nt][2 * e]), ex2_approx(sc[nt][2 * e + 1]));
                            wt[nt][e] = w;
                            const float2 sum = apart(add2(pack2(l[nt][0], l[nt][1]), w));
                            l[nt][0] = sum.x; l[nt][1] = sum.y;
#pragma unroll
                            for (int g = 0; g < NG; ++g) {
                                const float m = minimum_of(vp[e][g]);
                                const float2 x = apart(fma2(w, pack2(m, m), pack2(om[nt][0][g], om[nt][1][g])));
                                om[nt][0][g] = x.x; om[nt][1][g] = x.y;
                            }
                        }
                    // values
#pragma unroll
                    for (int u = 0; u < SUB; ++u)
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            const float up = ROWWISE ? 1.f : cs[g], s0 = scale_of(vp[2 * u][g]) * up, s1 = scale_of(vp[2 * u + 1][g]) * up;
                            uint32_t wf[NT][2];
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                f32x2 w0 = wt[nt][2 * u], w1 = wt[nt][2 * u + 1];
                                if constexpr (ROWWISE) { w0 = mul2(w0, cs_of(nt, g)); w1 = mul2(w1, cs_of(nt, g)); }
                                const float2 a = apart(mul2(w0, pack2(s0, s0))), c = apart(mul2(w1, pack2(s1, s1)));
                                const uint32_t x = f16_pair(a.x, a.y), y = f16_pair(c.x, c.y);
                                if constexpr (FINE) {
                                    const float2 fx = f16x2_to_float2(x), fy = f16x2_to_float2(y);
                                    const float2 cu = ROWWISE ? apart(cs_of(nt, g)) : make_float2(cs[g], cs[g]);
                                    const f32x2 less = pack2(-1.f, -1.f), middle = pack2(7.5f * inverse_pow2(cu.x), 7.5f * inverse_pow2(cu.y));
                                    const f32x2 lost = add2(fma2(pack2(fx.x, fx.y), less, pack2(a.x, a.y)), fma2(pack2(fy.x, fy.y), less, pack2(c.x, c.y)));
                                    unpack2(fma2(lost, middle, pack2(om[nt][0][g], om[nt][1][g])), om[nt][0][g], om[nt][1][g]);
                                }
                                wf[nt][0] = transpose_8x8(x);
                                wf[nt][1] = transpose_8x8(y);
                            }
                            const uint32_t from = stage + u * S::kTileBytes + (get_v ^ (g << 5));
                            const uint32_t wa = lds32(from), wb = lds32(from + 4 * RB), wc = lds32(from + 8 * RB), wd = lds32(from + 12 * RB);
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const uint32_t ab = __byte_perm(wa, wb, half ? 0x7632 : 0x5410), cd = __byte_perm(wc, wd, half ? 0x7632 : 0x5410);
#pragma unroll
                                for (int n = 0; n < 2; ++n) {
                                    const uint32_t xa = n ? ab >> 8 : ab, xc = n ? cd >> 8 : cd;
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt) {
                                        mma_f16(o[nt][g * 4 + half * 2 + n], xa & M0, xa & M1, xc & M0, xc & M1, wf[nt][0], wf[nt][1]);
                                    }
                                }
                            }
                        }
                    if (SUB == 2 || (k & 1)) {               // the stage is done with
                        __syncwarp();
                        const int i = k / 2 + S::kStages;
                        if (i < n_pairs) issue(i, slot);
                        copies_commit();
                        slot = slot == S::kStages - 1 ? 0 : slot + 1;
                    }
                    stage = stage + SUB * S::kTileBytes == ring + S::kStages * S::kStage ? ring : stage + SUB * S::kTileBytes;
                }
            }
            copies_wait<0>();
        };
        if (S::kStages - 1 < n_pairs) issue(S::kStages - 1, S::kStages - 1);
        copies_commit();
        sweep(std::false_type());

        // ---- rows whose products were too small for the others' cs
        constexpr int BITS = 2 * NT * NG, WORDS = BITS > 8 ? 2 : 1;        // a bit per row of this lane's and group; four lanes' side by side
        const float least = (float)n_tiles * (kKaTile * 15 * 0x1p-33f);
        uint32_t poor = 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float limit = cs[g] < 0x1p126f ? least : 0.f;
#pragma unroll
                for (int col = 0; col < 2; ++col) {
                    float even = o[nt][g * 4][col], odd = o[nt][g * 4][2 + col];          // c 2^-24, c 2^-20
#pragma unroll
                    for (int n = 1; n < 4; ++n) {
                        even = fmaxf(even, o[nt][g * 4 + n][col]);
                        odd = fmaxf(odd, o[nt][g * 4 + n][2 + col]);
                    }
                    poor |= (uint32_t)(fmaxf(even * 16.f, odd) < limit) << ((nt * NG + g) * 2 + col);
                }
            }
        const int shift = BITS * (WORDS == 2 ? j & 1 : j);
        uint32_t all = 0;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {                   // in none of the eight lanes' dimensions
            const uint32_t seen = __reduce_and_sync(0xffffffffu, WORDS == 2 && (j >> 1) != w ? ~0u : ~(((1u << BITS) - 1) << shift) | poor << shift);
            if (WORDS == 1 || (j >> 1) == w) all = seen >> shift;
        }
        uint32_t asked = 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int2 ask = *reinterpret_cast<const int2*>(&s_ask[nt * 8 + 2 * j]);
            const uint32_t rows = (uint32_t)(ask.x | ask.y << 1) & ~(unset >> (2 * nt)) & 3u;
#pragma unroll
            for (int g = 0; g < NG; ++g) asked |= rows << ((nt * NG + g) * 2);
        }
        const bool rowwise = __any_sync(0xffffffffu, (all & asked) != 0);
        if (rowwise) {
            __syncwarp();
#pragma unroll 1
            for (int i = 0; i < S::kStages; ++i) {
                if (i < n_pairs) issue(i, i);
                copies_commit();
            }
            sweep(std::true_type());
        }

        // ---- the warps' results together: means by their own sums of weights, so that nothing is larger than a value
        // [warp][row][D], pairs of a row in an order that goes by the row: what a warp stores at once lies in different banks
        float2* const red = reinterpret_cast<float2*>(ring_mem);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int col = 0; col < 2; ++col) {
                l[nt][col] = across_sum(l[nt][col]);
#pragma unroll
                for (int g = 0; g < NG; ++g) om[nt][col][g] = across_sum(om[nt][col][g]);
                // a token seen that is not finite in one group makes the row NaN in all, as where masks are looked at
#pragma unroll
                for (int g = 0; g < NG; ++g)
                    if (!(fabsf(om[nt][col][g]) <= FLT_MAX) || !(fabsf(o[nt][g * 4][col]) <= FLT_MAX)) l[nt][col] = NAN;
                if (r == 0) {
                    s_m[warp][nt * 8 + 2 * j + col] = (unset >> (2 * nt + col)) & 1 ? -INFINITY : -mb[nt][col];
                    s_l[warp][nt * 8 + 2 * j + col] = l[nt][col];
                }
            }
        __syncthreads();
        if (tid < ROWS) {
            float top = -INFINITY, sum = 0.f, f[kKaWarps];
#pragma unroll
            for (int w = 0; w < kKaWarps; ++w) top = fmaxf(top, s_m[w][tid]);
#pragma unroll
            for (int w = 0; w < kKaWarps; ++w) {
                f[w] = s_l[w][tid] * (s_m[w][tid] == -INFINITY ? 0.f : ex2_approx(s_m[w][tid] - top));
                sum += f[w];
            }
            const float inv = ka_inverse(sum);
#pragma unroll
            for (int w = 0; w < kKaWarps; ++w) s_l[w][tid] = f[w] * inv;       // a warp's share of the row
            s_ml[tid] = make_float2(top, sum);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float inv[2] = {ka_inverse(l[nt][0]), ka_inverse(l[nt][1])};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float2 up = rowwise ? apart(cs_of(nt, g)) : make_float2(cs[g], cs[g]);
#pragma unroll
                for (int col = 0; col < 2; ++col) {
                    const int row = nt * 8 + 2 * j + col;
                    const float down = inverse_pow2(col ? up.y : up.x), shift = om[nt][col][g] * inv[col];
                    float2* to = red + (warp * ROWS + row) * (D / 2) + r * 4 + g * (kKvGroup / 2);
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        to[n ^ j] = make_float2(fmaf(o[nt][g * 4 + n][col] * (inv[col] * 0x1p24f), down, shift),
                                                fmaf(o[nt][g * 4 + n][2 + col] * (inv[col] * 0x1p20f), down, shift));
                }
            }
        }
        __syncthreads();
        const bool whole = c1 - c0 == chunks;
        const long long part = (long long)blockIdx.x * 2 + (c0 == 0);
#pragma unroll 1
        for (int nt = 0; nt < NT; ++nt) {
            constexpr int PER = D / 16;
            const int in_block = nt * 8 + (tid >> 4), d0 = (tid & 15) * PER, place = s_out[in_block];
            if (place < 0) continue;
            const float2 ml = s_ml[in_block];
            float v[PER];
#pragma unroll
            for (int n = 0; n < PER; ++n) v[n] = 0.f;
#pragma unroll
            for (int w = 0; w < kKaWarps; ++w) {
                const float2* from = red + (w * ROWS + in_block) * (D / 2) + d0 / 2;
                const float f = s_l[w][in_block];
#pragma unroll
                for (int n = 0; n < PER / 2; ++n) {
                    // d0 / 2 + n with the two low bits turned by the row's
                    const float2 x = PER >= 8 ? from[n ^ ((in_block >> 1) & 3)] : red[(w * ROWS + in_block) * (D / 2) + ((d0 / 2 + n) ^ ((in_block >> 1) & 3))];
                    v[2 * n] = fmaf(x.x, f, v[2 * n]);
                    v[2 * n + 1] = fmaf(x.y, f, v[2 * n + 1]);
                }
            }
            if (whole) {
                const bool asked = s_ask[in_block];
                const long long orow = (long long)b * p.seqs.Q * (p.cache.heads * p.group) + place;
                if (!asked || span.bad) {
#pragma unroll
                    for (int n = 0; n < PER; ++n) v[n] = asked ? NAN : 0.f;
                }
                ka_store<E, PER>(reinterpret_cast<E*>(p.out) + orow * D + d0, v);
                if (p.lse && (tid & 15) == 0) p.lse[orow] = !asked ? -INFINITY : span.bad ? NAN : ka_lse(ml.x, ml.y);
            } else {
                float* to = p.part_o + (part * ROWS + in_block) * D + d0;
#pragma unroll
                for (int n = 0; n < PER; n += 4) *reinterpret_cast<float4*>(to + n) = make_float4(v[n], v[n + 1], v[n + 2], v[n + 3]);
                if ((tid & 15) == 0) p.part_ml[part * ROWS + in_block] = ml;
            }
        }
        if (tid == 0) {
            if (span.bad && p.status) atomicOr(p.status, kDevInvalid);
            if (!whole && c0 == 0) {
                // who has the unit's last chunk
                const int end = begin + (share + (blockIdx.x < longer) - left) - taken - at0 + cost - 1, few = longer * (share + 1);
                const bool early = end < few;
                p.cut[blockIdx.x] = make_int4(b, unit, (early ? 0 : longer) + (early ? end : end - few) / (early ? share + 1 : share), 0);
            }
        }
        __syncthreads();
    }
}

// ---- units that several CTAs had parts of: the first CTA's second slot, the others' first, in a fixed order
constexpr int kKaJoinRows = 4;             // per block; each has blockDim / 128 warps, which take every so-manieth part
constexpr int kKaJoinWarps = 4;            // of a row at most
template <typename E, int D, int NT>
__global__ void __launch_bounds__(kKaJoinRows * kKaJoinWarps * 32) ears_kv_join_kernel(const KaParams p) {
    constexpr int ROWS = NT * 8, PER = D / 32;
    __shared__ float2 s_ml[kKaJoinWarps][kKaJoinRows];
    __shared__ float s_v[kKaJoinWarps - 1][kKaJoinRows][D];
    wait_for_stream();
    const int4 cut = p.cut[blockIdx.x];
    if (cut.x < 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp / kKaJoinRows, warps = blockDim.x / (32 * kKaJoinRows);
    const int in_block = blockIdx.y * kKaJoinRows + warp % kKaJoinRows;
    const int b = cut.x, h = cut.y / p.blocks, row = (cut.y - h * p.blocks) * ROWS + in_block;
    const int c0 = blockIdx.x, parts = cut.z - c0 + 1;
    const int own = row < p.M ? (parts - mine + warps - 1) / warps : 0;        // parts mine, mine + warps, ...
    auto place = [&](int k) { const int n = mine + k * warps; return ((long long)(c0 + n) * 2 + (n == 0)) * ROWS + in_block; };
    // one look at the maxima and sums, a lane per part; results of eight parts on their way at once
    float top = -INFINITY, sum = 0.f, v[PER];
    float2 w[8][PER / 2];
    auto fetch = [&](int first, int count) {
#pragma unroll
        for (int m = 0; m < 8; ++m)
#pragma unroll
            for (int i = 0; i < PER / 2; ++i)
                w[m][i] = m < count ? __ldcg(reinterpret_cast<const float2*>(p.part_o + place(first + m) * D + lane * PER) + i) : make_float2(0.f, 0.f);
    };
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = 0.f;
    for (int n0 = 0; n0 < own; n0 += 32) {
        const int count = min(32, own - n0);
        const float2 ml = lane < count ? __ldcg(p.part_ml + place(n0 + lane)) : make_float2(-INFINITY, 0.f);
        fetch(n0, count);                                  // beside the maxima: neither waits for the other
        float most = fmaxf(top, ml.x);
#pragma unroll
        for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        const float had = sum * (top == -INFINITY ? 0.f : ex2_approx(top - most));
        float f = ml.y * (ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - most)), part = f;
        top = most;
#pragma unroll
        for (int d = 16; d; d >>= 1) part += __shfl_xor_sync(0xffffffffu, part, d);
        sum = had + part;
        const float inv = ka_inverse(sum);                 // v stays a mean
        f *= inv;
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] *= had * inv;
        for (int m0 = 0; m0 < count; m0 += 8) {
            if (m0) fetch(n0 + m0, count - m0);
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float g = __shfl_sync(0xffffffffu, f, (m0 + m) & 31);
#pragma unroll
                for (int i = 0; i < PER / 2; ++i) {
                    v[2 * i] = fmaf(w[m][i].x, g, v[2 * i]);
                    v[2 * i + 1] = fmaf(w[m][i].y, g, v[2 * i + 1]);
                }
            }
        }
    }
    if (warps > 1) {
        if (lane == 0) s_ml[mine][warp % kKaJoinRows] = make_float2(top, sum);
        if (mine) {
#pragma unroll
            for (int i = 0; i < PER; ++i) s_v[mine - 1][warp % kKaJoinRows][i * 32 + lane] = v[i];
        }
        __syncthreads();
        if (mine) return;
        float most = top;
        for (int w = 1; w < warps; ++w) most = fmaxf(most, s_ml[w][warp].x);
        auto share = [&](float2 ml) { return ml.y * (ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - most)); };
        const float f0 = share(make_float2(top, sum));
        sum = f0;
        for (int w = 1; w < warps; ++w) sum += share(s_ml[w][warp]);
        const float inv = ka_inverse(sum);
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] *= f0 * inv;
        for (int w = 1; w < warps; ++w) {
            const float f = share(s_ml[w][warp]) * inv;
#pragma unroll
            for (int i = 0; i < PER; ++i) v[i] = fmaf(s_v[w - 1][warp][i * 32 + lane], f, v[i]);
        }
        top = most;
    }
    if (row >= p.M) return;
    const bool asked = row / p.group < kv_count(p.seqs, b);
    if (!asked) {
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = 0.f;
    }
    const long long orow = ka_out_row(p, b, h, row);
    ka_store<E, PER>(reinterpret_cast<E*>(p.out) + orow * D + lane * PER, v);
    if (p.lse && lane == 0) p.lse[orow] = asked ? ka_lse(top, sum) : -INFINITY;
}

}  // namespace ears
