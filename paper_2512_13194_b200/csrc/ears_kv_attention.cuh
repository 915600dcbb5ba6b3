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
// (odd dimensions of keys / 16) and into the result (odd dimensions of values).
//
// The products are m16n8k16 with tokens (or, for the values, dimensions) as the 16 rows and eight of the head group's
// queries as columns: M = Q x heads per key head is seldom more than a few eights, and no work goes into padding a tile of
// 64 or 128.  Scores come out with a token per thread pair of rows, where a token's scale and minimum are two registers, and
// become the second product's operand through an 8x8 transpose.  The order of dimensions within a product is free as long as
// both operands agree: a thread takes consecutive codes, 8 (keys) or 4 (values) bytes of a token and group at a time.
//
// Work: a unit is (sequence, key head, block of NT x 8 rows); its tokens are cut into chunks of 64, of which each warp takes a tile of 16.
// Every CTA of the grid, as many as are resident at once, takes an equal run of the chunks of all units, whatever the
// sequences' lengths, which it reads on the device.  Units that are cut are joined by a second small kernel in a fixed order.
#pragma once
#include <type_traits>

#include "ears_kv.cuh"

namespace ears {

constexpr int kKaWarps = 4, kKaThreads = kKaWarps * 32;
constexpr int kKaTile = 16;                         // tokens of a warp's tile
constexpr int kKaChunk = kKaWarps * kKaTile;
constexpr float kKaSlack = 8.f;                     // the running maximum is raised when a score passes it by this much (base 2)

template <int D> struct KaShape {
    static constexpr int NG = D / kKvGroup;
    static constexpr int RB = D / 2;                // bytes of a token's codes
    static constexpr int kCodes = kKaTile * RB, kParams = kKaTile * NG * 4;
    static constexpr int kStage = 2 * (kCodes + kParams);
    static constexpr int kStages = D == 64 ? 8 : D == 128 ? 5 : 4;
    static constexpr int kSmem = kKaWarps * kStages * kStage;
    static_assert(kSmem >= kKaWarps * 8 * D * 4, "the warps' results meet in the ring's memory");
    // 16-byte pieces of row i are kept in another order, so that what a warp loads at once lies in different banks
    __device__ static __forceinline__ int swizzle(int i) { return RB == 128 ? ((i & 1) << 2) | (i & 2) : RB == 64 ? (i & 2) : 0; }
};

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
    if (s.count > 0 && !s.bad) {
        const int last = (s.start + s.count - 1) / kKaTile;
        if (p.window) {
            s.first = max(0, s.start - p.window + 1) / kKaTile;
            s.sinks = min((p.sinks + kKaTile - 1) / kKaTile, s.first);
        }
        s.tiles = s.sinks + last - s.first + 1;
    }
    return s;
}

// ---- instructions -----------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
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
__device__ __forceinline__ float scale_of(uint32_t par) { return __uint_as_float(par << 16); }
__device__ __forceinline__ float minimum_of(uint32_t par) { return __uint_as_float(par & 0xffff0000u); }
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) { return pack_pair<f16_t>(lo, hi); }
__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
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

// ---- a row's result ------------------------------------------------------------------------------------------
template <typename E, int N>
__device__ __forceinline__ void ka_store(E* out, const float (&x)[N], float factor) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pack_pair<E>(x[2 * i] * factor, x[2 * i + 1] * factor);
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
__device__ __forceinline__ float ka_lse(float m, float l) { return l == 0.f ? -INFINITY : fmaf(m, 0.69314718055994531f, logf(l)); }

// ---- the kernel ------------------------------------------------------------------------------------------------
// E: the queries' type.  SPLIT: weights enter the second product in two halves (22 bits): one half-precision weight is off by
// 2^-12 on average, which is nothing beside a bfloat16 result's 2^-9 but would be as much as a half-precision result's own rounding.
template <typename E, int D, int NT>
__global__ void __launch_bounds__(kKaThreads) ears_kv_attention_kernel(const KaParams p) {
    using S = KaShape<D>;
    constexpr int NG = S::NG, RB = S::RB, ROWS = NT * 8;
    constexpr bool SPLIT = std::is_same<E, f16_t>::value;
    constexpr uint32_t M0 = 0x000f000fu, M1 = 0x00f000f0u;
    constexpr int PIECES = RB / 32;               // 16-byte pieces of a tile's codes per lane

    extern __shared__ __align__(128) unsigned char ring_mem[];
    __shared__ float s_m[kKaWarps][ROWS], s_l[kKaWarps][ROWS];
    __shared__ long long s_sum[kKaWarps], s_base;
    __shared__ int s_b;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, j = lane & 3;
    wait_for_stream();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- this CTA's share of all chunks
    const int per_seq = p.cache.heads * p.blocks;
    const int each = (p.seqs.B + kKaThreads - 1) / kKaThreads;
    const int b0 = min(p.seqs.B, tid * each), b1 = min(p.seqs.B, b0 + each);
    long long own = 0;
    for (int b = b0; b < b1; ++b) own += (long long)ka_span(p, b).chunks() * per_seq;
    long long before = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += up;
    }
    if (lane == 31) s_sum[warp] = before;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < kKaWarps; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    before -= own;
    const long long ctas = min((long long)gridDim.x, total);
    if (tid == 0) p.cut[blockIdx.x] = make_int4(-1, 0, 0, 0);
    if (blockIdx.x >= ctas) return;
    const long long x0 = total * blockIdx.x / ctas, x1 = total * (blockIdx.x + 1) / ctas;
    if (own && before <= x0 && x0 < before + own) {
        long long base = before;
        int b = b0;
        for (;; ++b) {
            const long long n = (long long)ka_span(p, b).chunks() * per_seq;
            if (x0 < base + n) break;
            base += n;
        }
        s_b = b;
        s_base = base;
    }
    __syncthreads();

    // ---- addresses that do not change
    const uint32_t ring = smem_u32(ring_mem) + warp * (S::kStages * S::kStage);
    uint32_t put_k[PIECES], put_v[PIECES];
#pragma unroll
    for (int n = 0; n < PIECES; ++n) {
        const int piece = lane + 32 * n, t = piece / (RB / 16), c = piece % (RB / 16);
        // keys: product row i holds token (i >> 1) | (i & 1) << 2 of each eight, so that the values' token pairs lie in different banks
        const int i = (t & 8) | ((t & 3) << 1) | ((t >> 2) & 1);
        put_k[n] = i * RB + ((c ^ S::swizzle(i)) << 4);
        put_v[n] = S::kCodes + t * RB + ((c ^ S::swizzle(t)) << 4);
    }
    const int my_token = (r >> 1) | ((r & 1) << 2);
    const uint32_t get_k = r * RB + ((S::swizzle(r) + (j >> 1)) << 4) + (j & 1) * 8;
    const uint32_t get_v = S::kCodes + j * RB + ((S::swizzle(j) + (r >> 2)) << 4) + (r & 3) * 4;
    const uint32_t get_p = 2 * S::kCodes + my_token * NG * 4;

    long long x = x0, base = s_base;
    int b = s_b;
    KaSpan span = ka_span(p, b);
    while (x < x1) {
        const int chunks = span.chunks();
        const long long seq_total = (long long)chunks * per_seq;
        if (x >= base + seq_total) {
            base += seq_total;
            span = ka_span(p, ++b);
            continue;
        }
        const int unit = (int)((x - base) / chunks), c0 = (int)((x - base) - (long long)unit * chunks);
        const int take = (int)min((long long)(chunks - c0), x1 - x);
        const int h = unit / p.blocks, row0 = (unit - h * p.blocks) * ROWS;

        // ---- queries: normalised to 2^14 at most per row, halves; odd dimensions / 16
        uint32_t qf[NT][NG][4][2];
        float fr[NT][2], qs[NT][2][NG], mb[NT][2], l[NT][2], om[NT][2][NG], o[NT][NG * 4][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + nt * 8 + r, i = row / p.group, qh = h * p.group + (row - i * p.group);
            float v[NG][16], big = 0.f;
            const bool real = row < p.M;
            const E* src = reinterpret_cast<const E*>(p.q) + (real ? b * p.sb + i * p.sq + qh * p.sh : 0) + j * 16;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float e[8];
                    if (real) KvEight<E>::load(src + g * kKvGroup + half * 8, p.vec, e);
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        v[g][half * 8 + n] = real ? e[n] : 0.f;
                        big = max_nan(big, fabsf(v[g][half * 8 + n]));
                    }
                }
            }
            big = max_nan(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = max_nan(big, __shfl_xor_sync(0xffffffffu, big, 2));
            const int ex = max((int)(__float_as_uint(big) >> 23) - 127, -100);
            const float up = __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
            // scores: codes stand for c 2^-24, the row for q 2^(14 - ex)
            float f = p.scale2 * 1024.f * __uint_as_float((uint32_t)(127 + ex) << 23);
            if (!(big <= FLT_MAX)) f = NAN;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < 16; ++n) sum += v[g][n];
                sum = quad_sum(sum) * p.scale2;
#pragma unroll
                for (int col = 0; col < 2; ++col) qs[nt][col][g] = __shfl_sync(0xffffffffu, sum, (2 * j + col) * 4);
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const float u = (n & 1) ? up * 0.0625f : up;
                        qf[nt][g][2 * w + (n >> 1)][n & 1] = f16_pair(v[g][8 * w + n] * u, v[g][8 * w + n + 4] * u);
                    }
            }
#pragma unroll
            for (int col = 0; col < 2; ++col) {
                fr[nt][col] = __shfl_sync(0xffffffffu, f, (2 * j + col) * 4);
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
        uint32_t unset = (1u << (2 * NT)) - 1;              // rows that have seen no token yet, a bit per (nt, column)
        float cs = 0x1p120f;                                // the values' scales enter times this power of two
        const int last_pos = span.start + max(span.count - 1, 0);
        const int pmin = min(last_pos, span.start + row0 / p.group), pmax = min(last_pos, span.start + (min(row0 + ROWS, p.M) - 1) / p.group);

        // ---- this warp's tiles: first + 4 k
        const int first = c0 * kKaWarps + warp;
        const int n_tiles = max(0, (min((c0 + take) * kKaWarps, span.tiles) - first + kKaWarps - 1) / kKaWarps);
        long long at = 0;                                   // row of the tile of `lane` in the current 32, -1: no page
        uint32_t unusable = 0;
        auto issue = [&](int k) {
            if ((k & 31) == 0) {
                at = -1;
                if (k + lane < n_tiles) at = kv_row(p.cache, p.seqs, b, (long long)span.tile(first + (k + lane) * kKaWarps) * kKaTile);
            }
            const long long row = __shfl_sync(0xffffffffu, at, k & 31);
            unusable = (unusable & ~(1u << (k & 31))) | ((uint32_t)(row < 0) << (k & 31));
            if (row >= 0) {
                const uint32_t to = ring + (k % S::kStages) * S::kStage;
                const long long kr = row + (long long)h * p.cache.page, vr = kr + (long long)p.cache.heads * p.cache.page;
#pragma unroll
                for (int n = 0; n < PIECES; ++n) {
                    copy16(to + put_k[n], p.cache.codes + kr * RB + (lane + 32 * n) * 16);
                    copy16(to + put_v[n], p.cache.codes + vr * RB + (lane + 32 * n) * 16);
                }
                if (lane < 8 * NG) {
                    const long long pr = lane < 4 * NG ? kr : vr;
                    copy16(to + 2 * S::kCodes + lane * 16, reinterpret_cast<const unsigned char*>(p.cache.params + pr * NG) + (lane & (4 * NG - 1)) * 16);
                }
            } else if (lane == 0 && p.status) {
                atomicOr(p.status, kDevInvalid);
            }
        };
#pragma unroll 1
        for (int k = 0; k < S::kStages - 1; ++k) {
            if (k < n_tiles) issue(k);
            copies_commit();
        }
#pragma unroll 1
        for (int k = 0; k < n_tiles; ++k) {
            const bool broken = (unusable >> (k & 31)) & 1;
            copies_wait<S::kStages - 2>();
            __syncwarp();
            if (k + S::kStages - 1 < n_tiles) issue(k + S::kStages - 1);
            copies_commit();
            const uint32_t stage = ring + (k % S::kStages) * S::kStage;

            uint32_t kp[2][NG], vp[2][NG];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                lds_words<NG>(stage + get_p + e * 8 * NG * 4, kp[e]);
                lds_words<NG>(stage + get_p + S::kParams + e * 8 * NG * 4, vp[e]);
            }

            // scores relative to the running maximum, base 2: [nt][2 e + col], token e of this thread's two
            float sc[NT][4], dot[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) { sc[nt][c] = -mb[nt][c & 1]; dot[nt][c] = 0.f; }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                uint2 w0 = lds64(stage + (get_k ^ (g << 5))), w1 = lds64(stage + (get_k ^ (g << 5)) + 8 * RB);
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[nt][c] = 0.f;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t x0w = w ? w0.y : w0.x, x1w = w ? w1.y : w1.x, y0 = x0w >> 8, y1 = x1w >> 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_f16(acc[nt], x0w & M0, x1w & M0, x0w & M1, x1w & M1, qf[nt][g][2 * w][0], qf[nt][g][2 * w][1]);
                        mma_f16(acc[nt], y0 & M0, y1 & M0, y0 & M1, y1 & M1, qf[nt][g][2 * w + 1][0], qf[nt][g][2 * w + 1][1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        dot[nt][c] = fmaf(acc[nt][c], scale_of(kp[c >> 1][g]), dot[nt][c]);
                        sc[nt][c] = fmaf(minimum_of(kp[c >> 1][g]), qs[nt][c & 1][g], sc[nt][c]);
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) sc[nt][c] = fmaf(dot[nt][c], fr[nt][c & 1], sc[nt][c]);

            // masks, where the tile needs them
            const int t0 = span.tile(first + k * kKaWarps) * kKaTile;
            if (broken || t0 + kKaTile - 1 > pmin || (p.window && t0 + kKaTile - 1 >= p.sinks && t0 <= pmax - p.window)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int t = t0 + e * 8 + my_token;
                    bool lost = broken;                        // values of no use: rows that see the token become NaN by their score
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        lost = lost || !(scale_of(vp[e][g]) <= FLT_MAX) || !(fabsf(minimum_of(vp[e][g])) <= FLT_MAX);
                    }
                    if (lost || t > pmax || (p.window && t >= p.sinks && t <= pmin - p.window)) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) vp[e][g] = 0;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int col = 0; col < 2; ++col) {
                            const int row = min(row0 + nt * 8 + 2 * j + col, p.M - 1);
                            const int pos = min(last_pos, span.start + row / p.group);
                            float& v = sc[nt][2 * e + col];
                            if (lost) v = NAN;
                            if (t > pos || (p.window && t >= p.sinks && t <= pos - p.window)) v = -INFINITY;
                        }
                }
            }

            bool raise = unset != 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) raise = raise || sc[nt][c] > kKaSlack;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int g = 0; g < NG; ++g) raise = raise || scale_of(vp[e][g]) * cs > 128.f;
            if (__any_sync(0xffffffffu, raise)) {
                float sv = 0.f;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int g = 0; g < NG; ++g) sv = fmaxf(sv, scale_of(vp[e][g]));
                sv = across_max(sv);
                float ratio = 1.f;
                if (sv * cs > 128.f) {
                    const int ex = (int)(__float_as_uint(sv) >> 23) - 127;           // sv >= 2^-120: a finite normal number
                    const float now = __uint_as_float((uint32_t)(127 + 6 - ex) << 23);
                    ratio = now / cs;
                    cs = now;
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int col = 0; col < 2; ++col) {
                        const float top = across_max(fmaxf(sc[nt][col], sc[nt][2 + col]));
                        const uint32_t bit = 1u << (2 * nt + col);
                        float alpha = 1.f;
                        if (top > kKaSlack || ((unset & bit) && top > -INFINITY)) {
                            alpha = (unset & bit) ? 0.f : ex2_approx(-top);
                            mb[nt][col] += top;
                            sc[nt][col] -= top;
                            sc[nt][2 + col] -= top;
                            unset &= ~bit;
                        }
                        l[nt][col] *= alpha;
#pragma unroll
                        for (int g = 0; g < NG; ++g) om[nt][col][g] *= alpha;
                        alpha *= ratio;
#pragma unroll
                        for (int n = 0; n < NG * 4; ++n) { o[nt][n][col] *= alpha; o[nt][n][2 + col] *= alpha; }
                    }
            }

            // weights
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float w = ex2_approx(sc[nt][c]);
                    sc[nt][c] = w;
                    l[nt][c & 1] += w;
#pragma unroll
                    for (int g = 0; g < NG; ++g) om[nt][c & 1][g] = fmaf(w, minimum_of(vp[c >> 1][g]), om[nt][c & 1][g]);
                }
            // values
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float s0 = scale_of(vp[0][g]) * cs, s1 = scale_of(vp[1][g]) * cs;
                uint32_t wf[NT][2], wl[SPLIT ? NT : 1][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float a = sc[nt][0] * s0, bq = sc[nt][1] * s0, c = sc[nt][2] * s1, d = sc[nt][3] * s1;
                    const uint32_t u = f16_pair(a, bq), v = f16_pair(c, d);
                    if constexpr (SPLIT) {
                        const float2 fu = f16x2_to_float2(u), fv = f16x2_to_float2(v);
                        wl[nt][0] = transpose_8x8(f16_pair(a - fu.x, bq - fu.y));
                        wl[nt][1] = transpose_8x8(f16_pair(c - fv.x, d - fv.y));
                    }
                    wf[nt][0] = transpose_8x8(u);
                    wf[nt][1] = transpose_8x8(v);
                }
                const uint32_t from = stage + (get_v ^ (g << 5));
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
                            if constexpr (SPLIT) mma_f16(o[nt][g * 4 + half * 2 + n], xa & M0, xa & M1, xc & M0, xc & M1, wl[nt][0], wl[nt][1]);
                        }
                    }
                }
            }
        }

        // ---- the warps' results together
        copies_wait<0>();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int col = 0; col < 2; ++col) {
                l[nt][col] = across_sum(l[nt][col]);
#pragma unroll
                for (int g = 0; g < NG; ++g) om[nt][col][g] = across_sum(om[nt][col][g]);
                if (r == 0) {
                    s_m[warp][nt * 8 + 2 * j + col] = (unset >> (2 * nt + col)) & 1 ? -INFINITY : mb[nt][col];
                    s_l[warp][nt * 8 + 2 * j + col] = l[nt][col];
                }
            }
        __syncthreads();
        const bool whole = take == chunks;
        const long long slot = (long long)blockIdx.x * 2 + (c0 == 0);
        float* red = reinterpret_cast<float*>(ring_mem);      // [warp][8][D]
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int col = 0; col < 2; ++col) {
                const int row = nt * 8 + 2 * j + col;
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < kKaWarps; ++w) top = fmaxf(top, s_m[w][row]);
                const float mine = s_m[warp][row], f = mine == -INFINITY ? 0.f : ex2_approx(mine - top);
                const float even = f / cs;                     // cs a power of two
                float* to = red + ((warp * 8 + 2 * j + col) * D) + r * 8;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const float a = o[nt][g * 4 + n][col] * 0x1p24f, c = o[nt][g * 4 + n][2 + col] * 0x1p20f;
                        const float shift = f * om[nt][col][g];
                        *reinterpret_cast<float2*>(to + g * kKvGroup + 2 * n) = make_float2(fmaf(a, even, shift), fmaf(c, even, shift));
                    }
            }
            __syncthreads();
            {
                constexpr int PER = D / 16;
                const int row = tid >> 4, d0 = (tid & 15) * PER, in_block = nt * 8 + row, rr = row0 + in_block;
                float top = -INFINITY, sum = 0.f, v[PER];
#pragma unroll
                for (int w = 0; w < kKaWarps; ++w) top = fmaxf(top, s_m[w][in_block]);
#pragma unroll
                for (int w = 0; w < kKaWarps; ++w) {
                    const float m = s_m[w][in_block];
                    sum = fmaf(s_l[w][in_block], m == -INFINITY ? 0.f : ex2_approx(m - top), sum);
                }
#pragma unroll
                for (int n = 0; n < PER; ++n) v[n] = 0.f;
#pragma unroll
                for (int w = 0; w < kKaWarps; ++w)
#pragma unroll
                    for (int n = 0; n < PER; ++n) v[n] += red[(w * 8 + row) * D + d0 + n];
                if (rr < p.M) {
                    if (whole) {
                        const bool asked = rr / p.group < span.count;
                        const long long orow = ka_out_row(p, b, h, rr);
                        float f = asked && sum != 0.f ? 1.f / sum : 0.f;
                        if (asked && span.bad) f = NAN;
                        if (!asked) {
#pragma unroll
                            for (int n = 0; n < PER; ++n) v[n] = 0.f;
                        }
                        ka_store<E, PER>(reinterpret_cast<E*>(p.out) + orow * D + d0, v, f);
                        if (p.lse && (tid & 15) == 0) p.lse[orow] = !asked ? -INFINITY : span.bad ? NAN : ka_lse(top, sum);
                    } else {
                        float* to = p.part_o + (slot * ROWS + in_block) * D + d0;
#pragma unroll
                        for (int n = 0; n < PER; n += 4) *reinterpret_cast<float4*>(to + n) = make_float4(v[n], v[n + 1], v[n + 2], v[n + 3]);
                        if ((tid & 15) == 0) p.part_ml[slot * ROWS + in_block] = make_float2(top, sum);
                    }
                }
            }
            __syncthreads();
        }
        if (tid == 0) {
            if (span.bad && p.status) atomicOr(p.status, kDevInvalid);
            if (!whole && c0 == 0) {
                const long long end = base + (long long)(unit + 1) * chunks - 1;       // the unit's last chunk, and whose it is
                p.cut[blockIdx.x] = make_int4(b, unit, (int)(((end + 1) * ctas - 1) / total), 0);
            }
        }
        x += take;
    }
}

// ---- units that several CTAs had parts of: the first CTA's second slot, the others' first, in that order
constexpr int kKaJoinRows = 4;             // a warp each
template <typename E, int D, int NT>
__global__ void __launch_bounds__(kKaJoinRows * 32) ears_kv_join_kernel(const KaParams p) {
    constexpr int ROWS = NT * 8, PER = D / 32;
    wait_for_stream();
    const int4 cut = p.cut[blockIdx.x];
    if (cut.x < 0) return;
    const int lane = threadIdx.x & 31, in_block = blockIdx.y * kKaJoinRows + (threadIdx.x >> 5);
    const int b = cut.x, h = cut.y / p.blocks, row = (cut.y - h * p.blocks) * ROWS + in_block;
    if (row >= p.M) return;
    const int c0 = blockIdx.x, parts = cut.z - c0 + 1;
    auto place = [&](int n) { return ((long long)(c0 + n) * 2 + (n == 0)) * ROWS + in_block; };
    float top = -INFINITY;
    for (int n = lane; n < parts; n += 32) top = fmaxf(top, p.part_ml[place(n)].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    float v[PER], sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = 0.f;
#pragma unroll 4
    for (int n = 0; n < parts; ++n) {
        const float2 ml = p.part_ml[place(n)];
        const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
        const float* from = p.part_o + place(n) * D + lane * PER;
        sum = fmaf(ml.y, f, sum);
#pragma unroll
        for (int i = 0; i < PER; i += 2) {
            const float2 w = *reinterpret_cast<const float2*>(from + i);
            v[i] = fmaf(w.x, f, v[i]);
            v[i + 1] = fmaf(w.y, f, v[i + 1]);
        }
    }
    const bool asked = row / p.group < kv_count(p.seqs, b);
    if (!asked) {
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = 0.f;
    }
    const long long orow = ka_out_row(p, b, h, row);
    ka_store<E, PER>(reinterpret_cast<E*>(p.out) + orow * D + lane * PER, v, asked && sum != 0.f ? 1.f / sum : 0.f);
    if (p.lse && lane == 0) p.lse[orow] = asked ? ka_lse(top, sum) : -INFINITY;
}

}  // namespace ears
