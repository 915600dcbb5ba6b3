// Short rows: a warp (up to 4 KB of logits) or a CTA of 128 or 256 threads (up to 16 and 32 KB) holds a whole row
// in registers, eight 16-byte vectors per thread, so that it is read once whatever is computed from it.
//
// Bound by latency: a row passes through about 3 us of dependent steps (its token or list, its logits, the
// reduction, the 64-bit scalars), so what counts is the number of rows an SM has in flight, 24 with a warp per row
// against the 3 or 4 that CTAs of 256 threads and more leave room for.  8192 rows of 4 KB take a step of token log
// probabilities from 85 us (a CTA with a ring of stages per row) to the figure in the table of measurements.
#pragma once
#include "ears_distill.cuh"
#include "ears_rows.cuh"
#include "ears_token.cuh"
#include "ears_top.cuh"

namespace ears {

constexpr int kShortSlots = 8;               // vectors per thread
constexpr int kShortWarpRows = 4;            // rows per CTA where a warp has a row

template <int G> struct ShortShape {
    static constexpr int kRows = G == 32 ? kShortWarpRows : 1;   // rows per CTA
    static constexpr int kThreads = G * kRows;
};

// The thread's vectors of a row: vector tid + j G; -inf beyond the row.
template <typename E, int G>
__device__ __forceinline__ void short_load(const Slice<E>& s, int tid, uint4 (&w)[kShortSlots]) {
    const uint4* p = reinterpret_cast<const uint4*>(s.base);
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) {
        const int v = tid + j * G;
        w[j] = Words<E>::minus_inf();
        if (v < s.n) {
            if (s.whole(v)) w[j] = ld_row16(p + v);
            else w[j] = load_partial(s.base, v, s.lead, s.end);
        }
    }
}

template <typename E, int G>
__device__ __forceinline__ void short_store(const Slice<E>& s, int tid, E* g, int j, uint4 d) {
    const int v = tid + j * G;
    if (v < s.n) {
        if (((uintptr_t)g & 15) == 0 && s.whole(v)) reinterpret_cast<uint4*>(g)[v] = d;
        else store_partial(g, v, d, s.lead, s.end);
    }
}

template <typename E, int G>
__device__ __forceinline__ void short_zero(const Slice<E>& s, int tid, E* g) {
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) short_store<E, G>(s, tid, g, j, make_uint4(0, 0, 0, 0));
}

template <typename E, int G, bool ENT>
__device__ __forceinline__ void short_gradient(const Slice<E>& s, int tid, E* g, const uint4 (&w)[kShortSlots], float ref, float c, float A, float Bt) {
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) {
        if (j * G >= s.n) break;
        short_store<E, G>(s, tid, g, j, dense_words<E, ENT>(w[j], ref, c, A, Bt));
    }
}

// The statistics of the whole row, in every thread.
template <int G, bool ENT>
__device__ __forceinline__ Part short_merge(const Stat<ENT>& a, float4* xs, float c) {
    float s0, s1, w0 = 0.f, w1 = 0.f;
    unpack2(add2(a.s[0], a.s[1]), s0, s1);
    if (ENT) unpack2(add2(a.w[0], a.w[ENT ? 1 : 0]), w0, w1);
    const Part p = merge_lanes(Part{a.m, s0 + s1, w0 + w1}, c, ENT);
    if (G == 32) return p;
    if ((threadIdx.x & 31) == 0) xs[threadIdx.x >> 5] = make_float4(p.m, p.s, p.w, 0.f);
    __syncthreads();
    return merge_parts<ENT>(xs, G / 32, c);
}

// The row of this thread, or false when the grid's last CTA has none left for it.
template <int G>
__device__ __forceinline__ bool short_setup(const RowSpan& p, RowSetup* r) {
    const unsigned row = blockIdx.x * (unsigned)ShortShape<G>::kRows + (G == 32 ? threadIdx.x / 32u : 0u);
    if (row >= p.rows) return false;
    *r = row_setup_at(p, row);
    return true;
}

template <typename E, int G, bool ENT, int MODE>
__global__ void __launch_bounds__(ShortShape<G>::kThreads) ears_token_short_kernel(const TokenParams p) {
    __shared__ float4 xs[G / 32];
    __shared__ TokenScalars scalars[ShortShape<G>::kRows];
    RowSetup r;
    if (!short_setup<G>(p.rows, &r)) return;
    const int tid = threadIdx.x % G;
    TokenScalars& sc = scalars[threadIdx.x / G];
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, 0);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const int tok = __ldg(p.tokens + r.row);
    const bool absent = tok == -1, bad = tok < -1 || tok >= p.rows.V;
    if (absent || bad) {
        if (tid == 0) token_unused<MODE>(p, r.row, bad);
        if (MODE != kForward) short_zero<E, G>(s, tid, grad);
        return;
    }
    TokenInputs in{};
    if (tid == 0) in = token_inputs<E, ENT, MODE>(p, row, r.row, tok);
    uint4 w[kShortSlots];
    short_load<E, G>(s, tid, w);
    Part st;
    if (MODE == kBackward) {
        const float4 q = p.stats[r.row];
        st = token_saved<ENT>(q);
    } else {
        Stat<ENT> a;
        stat_open(a);
        stat_fold<E, kShortSlots, ENT>(w, r.c, a);
        st = short_merge<G, ENT>(a, xs, r.c);
    }
    if (tid == 0) sc = token_scalars<ENT, MODE>(p, r.row, 0, r.T, r.T_ok, in, st);
    if (MODE == kForward) return;
    row_sync<G>();
    const TokenScalars t = sc;
    if (t.zero) {
        short_zero<E, G>(s, tid, grad);
        return;
    }
    short_gradient<E, G, ENT>(s, tid, grad, w, st.m, r.c, t.A, t.Bt);
    row_sync<G>();   // the dense value of the token's entry has been written
    if (tid == 0) store_entry(grad + s.lead + tok, t.entry);
}

template <typename E, int G, int MODE>
__global__ void __launch_bounds__(ShortShape<G>::kThreads) ears_distill_short_kernel(const DistillParams p) {
    __shared__ float4 xs[G / 32];
    __shared__ ListSmem lists[ShortShape<G>::kRows];
    __shared__ uint32_t all_flags[ShortShape<G>::kThreads / 4];
    RowSetup r;
    if (!short_setup<G>(p.rows, &r)) return;
    const int tid = threadIdx.x % G, k = p.k;
    ListSmem& sm = lists[threadIdx.x / G];
    uint32_t* flags = all_flags + threadIdx.x / G * (G / 4);
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, 0);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const int seen = distill_list<E, kShortSlots, G, G>(p, sm, flags, tid, r.row, row, s.lead, 0, s.n);
    if (seen != 1) {
        if (tid == 0) distill_unused<MODE>(p, r.row, (seen & 2) != 0);
        if (MODE != kForward) short_zero<E, G>(s, tid, grad);
        return;
    }
    uint4 w[kShortSlots];
    short_load<E, G>(s, tid, w);
    Part st;
    if (MODE == kBackward) {
        const float4 q = p.stats[r.row];
        st = Part{q.x, q.y, 0.f};
    } else {
        // the gradient of a listed entry is written on its own, so its place may go to -inf for good
        const unsigned f = reinterpret_cast<const unsigned char*>(flags)[tid];
        if (f) {
#pragma unroll
            for (int j = 0; j < kShortSlots; ++j)
                if (f >> j & 1u) mask_listed<E>(sm, s.lead, tid + j * G, w[j]);
        }
        Stat<false> a;
        stat_open(a);
        stat_fold<E, kShortSlots, false>(w, r.c, a);
        st = short_merge<G, false>(a, xs, r.c);
    }
    const bool empty = tail_empty(st);
    if (tid < 32) {
        const double invT = 1.0 / r.T;
        const float weight = MODE != kForward && p.weight ? __ldg(p.weight + r.row) : 1.f;
        distill_scalars<MODE>(p, sm, r.row, 0, invT, r.T_ok && (empty || rowstat_ok(st.m, st.s)), teacher_part(p, sm, r.row, invT),
                              weight, st);
    }
    if (MODE == kForward) return;
    row_sync<G>();
    if (sm.zero) {
        short_zero<E, G>(s, tid, grad);
        return;
    }
    short_gradient<E, G, false>(s, tid, grad, w, empty ? 0.f : st.m, r.c, sm.factor, 0.f);
    row_sync<G>();   // the dense values of the listed entries have been written
    for (int j = tid; j < k; j += G)
        if (sm.col[j] >= 0) store_entry(grad + s.lead + sm.col[j], sm.entry[j]);
}

// ---- top logits of short rows: a warp per row -------------------------------------------------------
constexpr int kShortTopBuf = 256;            // candidates per row; kMaxTop and more

struct ShortTopSmem { alignas(16) top_key buf[kShortTopBuf]; int total; };

// kth_prefix for one warp: the largest 16-bit t (from the bits given) that at least k of the warp's values reach.
template <int PER>
__device__ __forceinline__ uint32_t warp_kth(const uint32_t (&v)[PER], int per, int k) {
    uint32_t t = 0;
#pragma unroll 1
    for (int s = 14; s >= 0; s -= 2) {
        const uint32_t t1 = t | 1u << s, t2 = t | 2u << s, t3 = t | 3u << s;
        uint32_t a = 0, b = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i >= per) break;
            a += (v[i] >= t1 ? 1u : 0u) + (v[i] >= t2 ? 1u << 16 : 0u);
            b += v[i] >= t3 ? 1u : 0u;
        }
        a = __reduce_add_sync(0xffffffffu, a);
        b = __reduce_add_sync(0xffffffffu, b);
        if ((int)b >= k) t = t3;
        else if ((int)(a >> 16) >= k) t = t2;
        else if ((int)(a & 0xffffu) >= k) t = t1;
    }
    return max(t, kLowestPrefix);
}

template <typename E>
__global__ void __launch_bounds__(ShortShape<32>::kThreads) ears_top_short_kernel(const TopParams p) {
    constexpr int N = Words<E>::N;
    __shared__ ShortTopSmem rows[ShortShape<32>::kRows];
    RowSetup r;
    if (!short_setup<32>(p.rows, &r)) return;
    const int lane = threadIdx.x & 31, k = p.k;
    ShortTopSmem& sm = rows[threadIdx.x / 32];
    float* values = p.out_values + r.row * k;
    int32_t* ids = p.out_ids + r.row * k;
    const bool live = !p.accept_len || (int)r.k <= __ldg(p.accept_len + r.b);
    const Slice<E> s = make_slice<E>(row_ptr<E>(p.rows, r), p.rows.V, p.rows.slice, 0);
    Part st{-INFINITY, 0.f, 0.f};
    uint4 w[kShortSlots];
    if (live) {
        short_load<E, 32>(s, lane, w);
        Stat<false> a;
        stat_open(a);
        stat_fold<E, kShortSlots, false>(w, r.c, a);
        st = short_merge<32, false>(a, nullptr, r.c);
    }
    const bool ok = live && r.T_ok && rowstat_ok(st.m, st.s);
    if (lane == 0) {
        p.out_lse[r.row] = !live ? -INFINITY : ok ? (float)((double)st.m / r.T + log((double)st.s)) : __int_as_float(0x7fc00000);
        if (live && !ok && p.status) atomicOr(p.status, kDevInvalidInput);
        sm.total = 0;
    }
    __syncwarp();
    if (!ok) {
        for (int j = lane; j < k; j += 32) { values[j] = -INFINITY; ids[j] = -1; }
        return;
    }
    // threshold from the vectors' maxima
    const int per = (s.n + 31) / 32;
    uint32_t v[kShortSlots];
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) {
        const uint4 one[1] = {w[j]};
        v[j] = order_bits(Words<E>::template vmax_all<1>(one)) >> 16;
    }
    const uint32_t t16 = warp_kth(v, per, k);
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) {
        if (v[j] < t16) continue;
        float x[N];
        Words<E>::unpack(w[j], x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if ((order_bits(x[i]) >> 16) < t16) continue;
            const int at = atomicAdd(&sm.total, 1);
            if (at < kShortTopBuf) sm.buf[at] = make_key(x[i], (lane + 32 * j) * N + i - s.lead);
        }
    }
    __syncwarp();
    int n = sm.total;
    if (n > kShortTopBuf) {
        // too many reach it: the k-th largest value bit by bit, then all entries above it and the first equal ones
        uint32_t u = 0;
#pragma unroll 1
        for (int b = 31; b >= 0; --b) {
            const uint32_t t = u | 1u << b;
            int c = 0;
#pragma unroll
            for (int j = 0; j < kShortSlots; ++j) {
                float x[N];
                Words<E>::unpack(w[j], x);
#pragma unroll
                for (int i = 0; i < N; ++i) c += order_bits(x[i]) >= t ? 1 : 0;
            }
            if (__reduce_add_sync(0xffffffffu, c) >= k) u = t;
        }
        int above = 0;
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) {
            float x[N];
            Words<E>::unpack(w[j], x);
#pragma unroll
            for (int i = 0; i < N; ++i) above += order_bits(x[i]) > u ? 1 : 0;
        }
        above = __reduce_add_sync(0xffffffffu, above);
        __syncwarp();
        if (lane == 0) sm.total = 0;
        __syncwarp();
        int equal = 0;   // equal entries before slot j
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) {
            float x[N];
            Words<E>::unpack(w[j], x);
            int mine = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) mine += order_bits(x[i]) == u ? 1 : 0;
            int before = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, before, off);
                if (lane >= off) before += o;
            }
            const int all = __shfl_sync(0xffffffffu, before, 31);
            before += equal - mine;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t o = order_bits(x[i]);
                if (o > u || (o == u && above + before++ < k)) {
                    const int at = atomicAdd(&sm.total, 1);
                    if (at < kShortTopBuf) sm.buf[at] = make_key(x[i], (lane + 32 * j) * N + i - s.lead);
                }
            }
            equal += all;
        }
        __syncwarp();
        n = min(sm.total, kShortTopBuf);
    }
    if (lane == 0 && (n & 1)) sm.buf[n] = 0ull;   // kShortTopBuf is even
    __syncwarp();
    const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(sm.buf);
    for (int at = lane; at < n; at += 32) {
        const top_key mine = sm.buf[at];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < (n + 1) / 2; ++j) {
            const ulonglong2 q = pairs[j];
            rank += (q.x > mine) + (q.y > mine);
        }
        if (rank < k) {
            values[rank] = unorder_bits((uint32_t)(mine >> 32));
            ids[rank] = (int32_t)~(uint32_t)mine;
        }
    }
    for (int j = n + lane; j < k; j += 32) { values[j] = -INFINITY; ids[j] = -1; }   // fewer than k finite entries
}

}  // namespace ears
