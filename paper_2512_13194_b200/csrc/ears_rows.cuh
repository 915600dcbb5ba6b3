// Rows of logits for the operators that train and score with them: where a row lies, the sweep of
// one CTA over its slice of a row, the softmax statistics of the slices of a cluster put together,
// and the dense part of a gradient row.
//
// A row is handled by a thread-block cluster of C CTAs, each with one contiguous slice.  A row of V
// entries need not start on a 16-byte boundary: it is seen as the run of 16-byte vectors that
// cover it, the first and the last possibly in part (the entries beside the row count as -inf and are
// never loaded or stored), so that odd vocabularies and padded rows run at the same speed.
//
// Statistics are (m, s, w): the maximum, s = sum 2^t and, where the entropy is wanted, w = sum 2^t t
// with t = (l - m) c, c = log2(e) / temperature.  The difference is taken before the product: every t
// is <= 0 and neither masks of the type's lowest value nor rows made of nothing else overflow it.  c enters in
// two parts: rounded to 32 bits it would be off by up to 6e-8, the same in every term, and a row's log normaliser
// by that times its mean |t| (13 and more), against 1e-7 from everything else.
#pragma once
#include "ears_cluster.cuh"
#include "ears_common.cuh"
#include "ears_math.cuh"
#include "ears_pipeline.cuh"

namespace ears {

constexpr int kLThreads = 256;
constexpr int kLWarps = kLThreads / 32;
constexpr int kLUnroll = 8;                 // 16-byte vectors in flight per thread
constexpr int kLRound = kLThreads * kLUnroll;
constexpr int kLMaxCluster = 16;
constexpr float kMaskedT = -2000.f;         // t of masked entries in sums of 2^t t (2^-2000 = 0 in fp32)
constexpr double kLn2 = 0.69314718055994530942;
constexpr double kLog2e = 1.44269504088896340736;

struct RowSpan {           // rows r = b R + k of [B, R, V] with strides in entries
    const void* x;
    long long stride_b, stride_r;
    long long rows;
    int R, V;
    double T;
    const float* seq_T;    // [B] temperature per sequence, or NULL
    int vectors;           // 16-byte vectors that a row, starting anywhere, covers at most
    int C;                 // CTAs per row
    int sms;               // of the device
    int slice;             // vectors per CTA (a multiple of kSliceAlign)
};
constexpr int kSliceAlign = 8;   // 128-byte lines are not shared between slices

// c = log2(e) / temperature: hi < c and lo = c - hi > 0, and the nearest 32-bit value.  None of them is 0, since a masked
// entry's -inf times each must stay -inf: from T = 1e29 on lo may round to 0, from 1e45 on the others do, and 2^-149 takes
// its place (2^-149 times the largest difference of two logits is 1e-6, in entries whose exponent is 0).
struct Scale { float hi, lo, near; };

__device__ __forceinline__ Scale make_scale(double T) {
    const double c = kLog2e / T;
    Scale s;
    s.hi = __double2float_rd(c);
    if ((double)s.hi == c) s.hi = __uint_as_float(__float_as_uint(s.hi) - 1u);
    const float least = __uint_as_float(1u);
    s.hi = fmaxf(s.hi, least);
    s.lo = fmaxf((float)(c - (double)s.hi), least);
    s.near = fmaxf((float)c, least);
    return s;
}
__device__ __forceinline__ float scaled(float d, const Scale& c) { return __fmaf_rn(d, c.hi, d * c.lo); }

// The special-function unit's exp2 falls short by this much on average (measured over the fractions; single results by
// up to 2^-22 either way): added to sums of it, all but the maximum's own term, which is exactly 1.
constexpr double kEx2Short = 1.25e-7;
__device__ __forceinline__ double row_mass(float s) { return (double)s + kEx2Short * ((double)s - 1.0); }

// The vectors of one row that one CTA handles.
template <typename E>
struct Slice {
    const E* base;         // 16-byte boundary at or below the row's first entry
    int lead;              // entries between base and the row's first entry
    int end;               // lead + V: entries of the vector run that belong to the row end here
    int v0, n;             // first vector and number of vectors of this slice
    __device__ __forceinline__ bool whole(int v) const { return v * Words<E>::N >= lead && (v + 1) * Words<E>::N <= end; }
};

template <typename E>
__device__ __forceinline__ Slice<E> make_slice(const E* row, int V, int slice, int rank) {
    constexpr int N = Words<E>::N;
    Slice<E> s;
    s.lead = (int)(((uintptr_t)row & 15) / sizeof(E));
    s.base = row - s.lead;
    s.end = s.lead + V;
    const int nv = (s.end + N - 1) / N;
    s.v0 = min(nv, rank * slice);
    s.n = min(nv - s.v0, slice);
    return s;
}

// Loads go past L1 and stay in L2: the statistics pass reads a slice that the gradient pass reads
// again.  Not the read-only path: a gradient may be written over its logits.
__device__ __forceinline__ uint4 ld_row16(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ uint4 ld_row16_hint(const void* p, uint64_t pol) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p), "l"(pol) : "memory");
    return r;
}
__device__ __forceinline__ void st_row16_hint(void* p, uint4 r, uint64_t pol) {
    asm volatile("st.global.L1::no_allocate.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;"
                 :: "l"(p), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "l"(pol) : "memory");
}
__device__ __forceinline__ uint32_t raw_bits(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t raw_bits(const uint16_t* p) { return *p; }
__device__ __forceinline__ uint32_t raw_bits(const f16_t* p) { return p->bits; }

// one entry of a packed vector replaced
__device__ __forceinline__ void put_entry(uint4& w, int i, uint32_t bits, float) {
    if (i == 0) w.x = bits; else if (i == 1) w.y = bits; else if (i == 2) w.z = bits; else w.w = bits;
}
__device__ __forceinline__ void put_half(uint32_t& h, int odd, uint32_t bits) {
    h = odd ? ((h & 0xffffu) | (bits << 16)) : ((h & 0xffff0000u) | bits);
}
__device__ __forceinline__ void put_entry(uint4& w, int i, uint32_t bits, uint16_t) {
    if (i < 2) put_half(w.x, i & 1, bits); else if (i < 4) put_half(w.y, i & 1, bits);
    else if (i < 6) put_half(w.z, i & 1, bits); else put_half(w.w, i & 1, bits);
}
__device__ __forceinline__ void put_entry(uint4& w, int i, uint32_t bits, f16_t) { put_entry(w, i, bits, (uint16_t)0); }
template <typename E> __device__ __forceinline__ uint32_t minus_inf_bits() { return Words<E>::minus_inf().x & (sizeof(E) == 4 ? 0xffffffffu : 0xffffu); }

// Vector v of the run when it is not wholly inside the row.
template <typename E>
__device__ __noinline__ uint4 load_partial(const E* base, int v, int lead, int end) {
    constexpr int N = Words<E>::N;
    uint4 w = Words<E>::minus_inf();
    for (int i = 0; i < N; ++i) {
        const int e = v * N + i;
        if (e >= lead && e < end) put_entry(w, i, raw_bits(base + e), E{});
    }
    return w;
}

// The vectors of one round of one thread: slice-local indices i0 + j kLThreads.
template <typename E>
__device__ __forceinline__ void load_round(const Slice<E>& s, int i0, uint4 (&w)[kLUnroll], uint64_t pol) {
    const uint4* p = reinterpret_cast<const uint4*>(s.base) + s.v0;
    if (i0 + (kLUnroll - 1) * kLThreads < s.n && s.whole(s.v0 + i0) && s.whole(s.v0 + i0 + (kLUnroll - 1) * kLThreads)) {
#pragma unroll
        for (int j = 0; j < kLUnroll; ++j) w[j] = ld_row16_hint(p + i0 + j * kLThreads, pol);
    } else {
#pragma unroll
        for (int j = 0; j < kLUnroll; ++j) {
            const int i = i0 + j * kLThreads;
            w[j] = Words<E>::minus_inf();
            if (i < s.n) {
                if (s.whole(s.v0 + i)) w[j] = ld_row16(p + i);
                else w[j] = load_partial(s.base, s.v0 + i, s.lead, s.end);
            }
        }
    }
}

// f(w, round) for every round of the thread's vectors.  Four CTAs per SM cover the wait for a round's loads.  AHEAD fetches
// the next round while one is worked on, which leaves room for two CTAs per SM: for launches of the top-logits kernel that have no
// more (64 of 250 rows of 128256 bf16: 25.1 us and 22.7; with more CTAs it loses, scoring 2048 rows of 256000 fp32: 306 us
// and 330, and so do the leaner forward kernels, 200 rows of 33000: 6.2 us and 7.2).
template <typename E, bool AHEAD, class F>
__device__ __forceinline__ void sweep_rounds(const Slice<E>& s, uint64_t pol, F f) {
    const int tid = threadIdx.x, rounds = (s.n + kLRound - 1) / kLRound;
    if (!AHEAD) {
        for (int r = 0; r < rounds; ++r) {
            uint4 w[kLUnroll];
            load_round(s, r * kLRound + tid, w, pol);
            f(w, r);
        }
    } else if (rounds > 0) {
        uint4 w[kLUnroll], x[kLUnroll];
        load_round(s, tid, w, pol);
#pragma unroll 1
        for (int r = 0;; r += 2) {
            if (r + 1 < rounds) load_round(s, (r + 1) * kLRound + tid, x, pol);
            f(w, r);
            if (r + 1 >= rounds) break;
            if (r + 2 < rounds) load_round(s, (r + 2) * kLRound + tid, w, pol);
            f(x, r + 1);
            if (r + 2 >= rounds) break;
        }
    }
}

// ---- statistics -------------------------------------------------------------------------
template <bool ENT> struct Stat { float m; f32x2 s[2]; f32x2 w[ENT ? 2 : 1]; };

template <bool ENT>
__device__ __forceinline__ void stat_open(Stat<ENT>& a) {
    a.m = -INFINITY;
    a.s[0] = a.s[1] = pack2(0.f, 0.f);
    a.w[0] = a.w[ENT ? 1 : 0] = pack2(0.f, 0.f);
}

__device__ __forceinline__ f32x2 clamp_masked(f32x2 t) {
    float lo, hi;
    unpack2(t, lo, hi);
    return pack2(fmaxf(lo, kMaskedT), fmaxf(hi, kMaskedT));
}

// G vectors: the maximum first, one rescale of the sums if it grew, then per entry a subtraction, a
// multiplication, a multiply-add, an exp2 and an addition, all but the exp2 on pairs.
// cm: the vectors' maximum.
template <typename E, int G, bool ENT>
__device__ __forceinline__ void stat_add(const uint4 (&w)[G], float cm, const Scale& c, Stat<ENT>& a) {
    constexpr int PN = Words<E>::N / 2;
    if (cm > a.m) {
        const float dl = a.m == -INFINITY ? 0.f : fmaxf(scaled(a.m - cm, c), kMaskedT);
        const float sc = a.m == -INFINITY ? 0.f : ex2_approx(dl);
        const f32x2 sc2 = pack2(sc, sc), dl2 = pack2(dl, dl);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (ENT) a.w[h] = mul2(fma2(dl2, a.s[h], a.w[h]), sc2);
            a.s[h] = mul2(a.s[h], sc2);
        }
        a.m = cm;
    }
    const float ref = a.m == -INFINITY ? 0.f : a.m;
    const f32x2 c2 = pack2(c.hi, c.hi), l2 = pack2(c.lo, c.lo), nr2 = pack2(-ref, -ref);
    // The call's terms are added up among themselves first, in eight lanes: a row with one large entry (a sum of 1.01, say)
    // would otherwise lose most of its small terms, each below half a step of the running sum.
    f32x2 ns[4], nw[ENT ? 2 : 1];
#pragma unroll
    for (int q = 0; q < 4; ++q) ns[q] = pack2(0.f, 0.f);
    nw[0] = nw[ENT ? 1 : 0] = pack2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < G; ++j) {
        f32x2 p[PN];
        Words<E>::pairs(w[j], p);
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            const f32x2 d = add2(p[i], nr2), t = fma2(d, c2, mul2(d, l2));
            const f32x2 e = ex2_pair(t);
            f32x2& lane = ns[(j * PN + i) & 3];
            lane = add2(lane, e);
            if (ENT) nw[i & 1] = fma2(e, clamp_masked(t), nw[i & 1]);
        }
    }
    a.s[0] = add2(a.s[0], add2(ns[0], ns[2]));
    a.s[1] = add2(a.s[1], add2(ns[1], ns[3]));
    if (ENT) {
        a.w[0] = add2(a.w[0], nw[0]);
        a.w[ENT ? 1 : 0] = add2(a.w[ENT ? 1 : 0], nw[ENT ? 1 : 0]);
    }
}
template <typename E, int G, bool ENT>
__device__ __forceinline__ void stat_fold(const uint4 (&w)[G], const Scale& c, Stat<ENT>& a) {
    stat_add<E, G, ENT>(w, Words<E>::template vmax_all<G>(w), c, a);
}

// The statistics of a part: what one warp hands on, and what the whole row ends with.
struct Part { float m, s, w; };

// Merges the 32 lanes' parts; all lanes get the result.
__device__ __forceinline__ Part merge_lanes(Part a, const Scale& c, bool ent) {
    float M = a.m;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    const float dl = a.m == -INFINITY ? 0.f : fmaxf(scaled(a.m - M, c), kMaskedT);   // nothing seen: s is 0, or NaN
    const float sc = exp2f(dl);   // full precision: the factor scales a whole part
    a.w = ent ? sc * __fmaf_rn(dl, a.s, a.w) : 0.f;
    a.s *= sc;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, off);
        if (ent) a.w += __shfl_xor_sync(0xffffffffu, a.w, off);
    }
    a.m = M;
    return a;
}

// The wait that belongs to the arrival of row_setup: from here on every CTA of the cluster has started.
__device__ __forceinline__ void cluster_wait_peers() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One warp: the n parts that the exchange left in xs -> the row's; the same in every warp and CTA.
template <bool ENT>
__device__ __forceinline__ Part merge_parts(const float4* xs, int n, const Scale& c) {
    const int lane = threadIdx.x & 31;
    Part q{-INFINITY, 0.f, 0.f};
    if (n <= 32) {
        if (lane < n) q = Part{xs[lane].x, xs[lane].y, xs[lane].z};
    } else {
        // lane i takes parts i, i + 32, ..
        for (int i = lane; i < n; i += 32) q.m = fmaxf(q.m, xs[i].x);
        for (int i = lane; i < n; i += 32) {
            const float dl = xs[i].x == -INFINITY ? 0.f : fmaxf(scaled(xs[i].x - q.m, c), kMaskedT);
            const float sc = exp2f(dl);
            if (ENT) q.w += sc * __fmaf_rn(dl, xs[i].y, xs[i].z);
            q.s = __fmaf_rn(sc, xs[i].y, q.s);
        }
    }
    return merge_lanes(q, c, ENT);
}

// Every warp's part goes to every CTA of the cluster through distributed shared memory; after one
// barrier every warp merges the same C x WARPS parts in the same order, so all CTAs hold identical bits.
template <bool ENT, int WARPS = kLWarps>
__device__ __forceinline__ Part exchange_parts(const Stat<ENT>& a, float4* xs /* [kLMaxCluster * WARPS] */, int C, int rank, const Scale& c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float s0, s1, w0 = 0.f, w1 = 0.f;
    unpack2(add2(a.s[0], a.s[1]), s0, s1);
    if (ENT) unpack2(add2(a.w[0], a.w[ENT ? 1 : 0]), w0, w1);
    Part p = merge_lanes(Part{a.m, s0 + s1, w0 + w1}, c, ENT);
    const float4 v = make_float4(p.m, p.s, p.w, 0.f);
    if (C == 1) {
        if (lane == 0) xs[warp] = v;
        __syncthreads();
    } else {
        cluster_wait_peers();
        if (lane < C) peer_store(map_to_peer(smem_u32(xs + rank * WARPS + warp), (uint32_t)lane), v);
        __syncwarp();
        cluster_sync_all();
    }
    return merge_parts<ENT>(xs, C * WARPS, c);
}

// The same barriers for a warp that has no part to hand on.
__device__ __forceinline__ void exchange_join(int C) {
    __syncwarp();
    if (C == 1) {
        __syncthreads();
    } else {
        cluster_wait_peers();
        cluster_sync_all();
    }
}

// ---- dense gradient ------------------------------------------------------------------------
__device__ __forceinline__ uint32_t round_pair(float lo, float hi, uint16_t) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t round_pair(float lo, float hi, f16_t) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename E>
__device__ __forceinline__ uint4 pack_words(const f32x2 (&g)[Words<E>::N / 2]) {
    uint32_t h[4];
    if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float lo, hi;
            unpack2(g[i], lo, hi);
            h[2 * i] = __float_as_uint(lo);
            h[2 * i + 1] = __float_as_uint(hi);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            unpack2(g[i], lo, hi);
            h[i] = round_pair(lo, hi, E{});   // the only rounding of a gradient entry, to the logits' type
        }
    }
    return make_uint4(h[0], h[1], h[2], h[3]);
}

__device__ __forceinline__ void store_entry(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_entry(uint16_t* p, float v) { *p = (uint16_t)round_pair(v, 0.f, (uint16_t)0); }
__device__ __forceinline__ void store_entry(f16_t* p, float v) { p->bits = (uint16_t)round_pair(v, 0.f, f16_t{}); }

__device__ __forceinline__ uint32_t entry_of(uint4 w, int i, float) { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
__device__ __forceinline__ uint32_t entry_of(uint4 w, int i, uint16_t) {
    const uint32_t h = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return (i & 1) ? h >> 16 : h & 0xffffu;
}
__device__ __forceinline__ uint32_t entry_of(uint4 w, int i, f16_t) { return entry_of(w, i, (uint16_t)0); }
__device__ __forceinline__ void store_raw(float* p, uint32_t b) { *p = __uint_as_float(b); }
__device__ __forceinline__ void store_raw(uint16_t* p, uint32_t b) { *p = (uint16_t)b; }
__device__ __forceinline__ void store_raw(f16_t* p, uint32_t b) { p->bits = (uint16_t)b; }

// Vector v of a gradient row whose entry e of the run (v N + i) lives at g[e]; entries outside
// [lead, end) are not touched.
template <typename E>
__device__ __noinline__ void store_partial(E* g, int v, uint4 w, int lead, int end) {
    constexpr int N = Words<E>::N;
    for (int i = 0; i < N; ++i) {
        const int e = v * N + i;
        if (e >= lead && e < end) store_raw(g + e, entry_of(w, i, E{}));
    }
}

// 2^t (A + Bt t) of a vector of logits, rounded to their type.
template <typename E, bool ENT>
__device__ __forceinline__ uint4 dense_words(uint4 w, float ref, float c, float A, float Bt) {
    constexpr int PN = Words<E>::N / 2;
    const f32x2 c2 = pack2(c, c), nr2 = pack2(-ref, -ref), a2 = pack2(A, A), b2 = pack2(Bt, Bt);
    f32x2 p[PN];
    Words<E>::pairs(w, p);
#pragma unroll
    for (int i = 0; i < PN; ++i) {
        const f32x2 t = mul2(add2(p[i], nr2), c2);
        const f32x2 e = ex2_pair(t);
        p[i] = mul2(e, ENT ? fma2(b2, clamp_masked(t), a2) : a2);
    }
    return pack_words<E>(p);
}

// The CTA's slice of a gradient row; `zero` writes zeros and reads nothing.  The gradient row's entry
// e of the run lives at g[e] (g = the row's first entry - lead); when g is not on a 16-byte boundary
// entries are stored one by one.
template <typename E, bool ENT>
__device__ __forceinline__ void dense_pass(const Slice<E>& s, E* g, bool zero, float ref, float c, float A, float Bt) {
    const bool aligned = ((uintptr_t)g & 15) == 0;
    uint4* out = reinterpret_cast<uint4*>(g) + s.v0;
    const uint64_t pol = l2_policy_evict_first();
    for (int i0 = threadIdx.x; i0 < s.n; i0 += kLRound) {
        uint4 w[kLUnroll];
        if (!zero) {
            load_round(s, i0, w, pol);
#pragma unroll
            for (int j = 0; j < kLUnroll; ++j) w[j] = dense_words<E, ENT>(w[j], ref, c, A, Bt);
        } else {
#pragma unroll
            for (int j = 0; j < kLUnroll; ++j) w[j] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < kLUnroll; ++j) {
            const int i = i0 + j * kLThreads;
            if (i < s.n) {
                if (aligned && s.whole(s.v0 + i)) st_row16_hint(out + i, w[j], pol);
                else store_partial(g, s.v0 + i, w[j], s.lead, s.end);
            }
        }
    }
}

// Whether entry `col` of the row lies in this CTA's slice.
template <typename E>
__device__ __forceinline__ bool in_slice(const Slice<E>& s, int col) {
    const int v = (s.lead + col) / Words<E>::N;
    return v >= s.v0 && v < s.v0 + s.n;
}

// ---- what every kernel does first ---------------------------------------------------------------
struct RowSetup { long long row; unsigned b, k; int rank; double T; Scale c; bool T_ok; };

__device__ __forceinline__ RowSetup row_setup_at(const RowSpan& p, unsigned row) {   // rows fit 32 bits
    RowSetup r;
    r.rank = 0;
    r.row = row;
    r.b = row / (unsigned)p.R;
    r.k = row - r.b * (unsigned)p.R;
    r.T = p.seq_T ? (double)__ldg(p.seq_T + r.b) : p.T;
    r.c = make_scale(r.T);
    r.T_ok = r.T > 0.0 && r.T < (double)INFINITY && r.c.near < INFINITY;
    return r;
}

__device__ __forceinline__ RowSetup row_setup(const RowSpan& p) {
    wait_for_stream();
    const unsigned row = blockIdx.x / (unsigned)p.C;
    RowSetup r = row_setup_at(p, row);
    r.rank = (int)(blockIdx.x - row * (unsigned)p.C);
    if (p.C > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    return r;
}
template <typename E>
__device__ __forceinline__ const E* row_ptr(const RowSpan& p, const RowSetup& r) {
    return reinterpret_cast<const E*>(p.x) + r.b * p.stride_b + r.k * p.stride_r;
}
template <typename E>
__device__ __forceinline__ E* grad_ptr(void* g, long long gsb, long long gsr, const RowSetup& r) {
    return reinterpret_cast<E*>(g) + r.b * gsb + r.k * gsr;
}

}  // namespace ears
