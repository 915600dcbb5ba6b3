// The k largest logits of every row, with the row's log normaliser.
//
// Entries are ordered by (value, lower index first), so that the result does not depend on how the
// row was split: an entry's key is its value as an order-preserving 32-bit integer followed by the
// complement of its index, all keys of a row are distinct, and the k largest keys are unique.
//
// One sweep of the slice, with the statistics of the row's softmax on the way.  A CTA keeps a buffer of
// candidates and a threshold below which nothing can be among the slice's k largest:
//   * first round: the k-th largest of the threads' maxima (k entries are at least that large).  For
//     rows in no particular order a slice then yields about 256 ln(256 / (256 - k)) candidates a round,
//     falling with the rounds behind it;
//   * candidates are appended to the buffer.  When it cannot take them all, its k largest are
//     sorted to its front, the threshold rises to the k-th and what is still pending is offered again:
//     rows in ascending order or with most entries equal run slower, never wrong.
// The rank of a candidate is the number of larger keys: one comparison with every other, read from
// shared memory two to a load, without a barrier.  The C sorted lists of a cluster are handed to every
// CTA, and each CTA finds the final ranks of its own entries by binary search in the others.
//
// Bound by HBM for long rows, by latency for few: a row of 256 KB in one CTA takes 18 us at a CTA's
// share of the bandwidth, its ranks about 1.
#pragma once
#include "ears_distill.cuh"   // kMaxTop
#include "ears_rows.cuh"

namespace ears {

typedef unsigned long long top_key;
constexpr int kTopBuf = 2048;                // candidates a CTA holds: 128 + 64 < 2048, so each offer takes one thread's at least

struct TopParams {
    RowSpan rows;
    int k;
    const int32_t* accept_len;   // [B] or NULL: rows behind a sequence's first rejection are left out
    float* out_values;           // [rows, k]
    int32_t* out_ids;
    float* out_lse;
    int32_t* status;
};

struct TopSmem {
    float4 xs[kLMaxCluster * kLWarps];
    alignas(16) top_key buf[kTopBuf];
    top_key list[kLMaxCluster][kMaxTop];     // sorted lists of the cluster's CTAs
    int count[kLMaxCluster];
    alignas(16) float tmax[kLThreads];
    int total;                               // places of buf given out
    int overflow[2];                         // alternating by offer
    top_key threshold;
};

// larger float -> larger integer; -0 and 0 are one value
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unorder_bits(uint32_t u) {
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ top_key make_key(float x, int col) { return ((top_key)order_bits(x) << 32) | (uint32_t)~col; }

// The k largest of buf[0 .. n) sorted to its front.  All threads; buf is final when it returns.
__device__ __forceinline__ int compact_candidates(TopSmem& sm, int n, int k) {
    constexpr int PER = kTopBuf / kLThreads;
    const int tid = threadIdx.x;
    if (tid == 0 && (n & 1)) sm.buf[n] = 0ull;   // kTopBuf is even
    __syncthreads();
    top_key mine[PER];
    int rank[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = tid + i * kLThreads;
        mine[i] = at < n ? sm.buf[at] : 0ull;
        rank[i] = 0;
    }
    const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(sm.buf);
    const int n2 = (n + 1) / 2;
    // as many of a thread's candidates as there are (n is the same for all threads)
    if (n <= kLThreads) {
#pragma unroll 4
        for (int j = 0; j < n2; ++j) {
            const ulonglong2 q = pairs[j];
            rank[0] += (q.x > mine[0]) + (q.y > mine[0]);
        }
    } else if (n <= 2 * kLThreads) {
#pragma unroll 4
        for (int j = 0; j < n2; ++j) {
            const ulonglong2 q = pairs[j];
#pragma unroll
            for (int i = 0; i < 2; ++i) rank[i] += (q.x > mine[i]) + (q.y > mine[i]);
        }
    } else {
        for (int j = 0; j < n2; ++j) {
            const ulonglong2 q = pairs[j];
#pragma unroll
            for (int i = 0; i < PER; ++i) rank[i] += (q.x > mine[i]) + (q.y > mine[i]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (mine[i] != 0ull && rank[i] < k) sm.buf[rank[i]] = mine[i];
    __syncthreads();
    return min(n, k);
}

// Calls f(value, column) for every entry of the thread's round whose value is at least `floor`.  The vectors
// are fetched again (from L2, and seldom): keeping all eight for this path would cost the sweep its registers.
template <typename E, class F>
__device__ __forceinline__ void each_candidate(const Slice<E>& s, int i0, float floor, F f) {
    constexpr int N = Words<E>::N;
#pragma unroll 1
    for (int i = i0; i < s.n && i < i0 + kLRound; i += kLThreads) {
        const int v = s.v0 + i;
        const uint4 w = s.whole(v) ? ld_row16(reinterpret_cast<const uint4*>(s.base) + v) : load_partial(s.base, v, s.lead, s.end);
        const uint4 one[1] = {w};
        if (Words<E>::template vmax_all<1>(one) >= floor) {
            float x[N];
            Words<E>::unpack(w, x);
            const int col = v * N - s.lead;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (x[j] >= floor && x[j] > -INFINITY) f(x[j], col + j);
        }
    }
}

template <typename E>
__global__ void __launch_bounds__(kLThreads) ears_top_kernel(const TopParams p) {
    __shared__ TopSmem sm;
    const int tid = threadIdx.x, k = p.k;
    const RowSetup r = row_setup(p.rows);
    if (p.accept_len && (int)r.k > __ldg(p.accept_len + r.b)) {   // the same in the whole cluster
        if (r.rank == 0) {
            if (tid < k) {
                p.out_values[r.row * k + tid] = -INFINITY;
                p.out_ids[r.row * k + tid] = -1;
            }
            if (tid == 0) p.out_lse[r.row] = -INFINITY;
        }
        return;
    }
    const Slice<E> s = make_slice<E>(row_ptr<E>(p.rows, r), p.rows.V, p.rows.slice, r.rank);
    if (tid == 0) { sm.total = 0; sm.overflow[0] = sm.overflow[1] = 0; sm.threshold = 0ull; }
    Stat<false> a;
    stat_open(a);
    const uint64_t pol = l2_policy_evict_first();
    float floor = -INFINITY;
    top_key threshold = 0;
    int offers = 0;
    const int rounds = (s.n + kLRound - 1) / kLRound;
    for (int round = 0; round < rounds; ++round) {
        const int i0 = round * kLRound + tid;
        uint4 w[kLUnroll];
        load_round(s, i0, w, pol);   // beyond the slice: -inf
        stat_fold<E, kLUnroll, false>(w, r.c, a);
        float top = Words<E>::template vmax_all<kLUnroll>(w);
        if (!(top > -INFINITY)) top = -INFINITY;   // nothing but NaN
        if (round == 0) {
            // the k-th largest of the threads' maxima
            sm.tmax[tid] = top;
            __syncthreads();
            int larger = 0;
            const float4* q4 = reinterpret_cast<const float4*>(sm.tmax);
#pragma unroll 4
            for (int q = 0; q < kLThreads / 4; ++q) {
                const float4 v = q4[q];
                // equal maxima in thread order: the ranks are a permutation
                larger += (v.x > top || (v.x == top && 4 * q < tid)) + (v.y > top || (v.y == top && 4 * q + 1 < tid))
                        + (v.z > top || (v.z == top && 4 * q + 2 < tid)) + (v.w > top || (v.w == top && 4 * q + 3 < tid));
            }
            if (larger == k - 1) sm.threshold = top > -INFINITY ? ((top_key)order_bits(top) << 32) : 0ull;
            __syncthreads();
            threshold = sm.threshold;
            floor = threshold ? unorder_bits((uint32_t)(threshold >> 32)) : -INFINITY;
        }
        bool pending = top >= floor && top > -INFINITY;
        for (;; ++offers) {
            if (pending) {
                int n = 0;
                each_candidate(s, i0, floor, [&](float x, int col) { n += make_key(x, col) >= threshold; });
                const int at = n ? atomicAdd(&sm.total, n) : 0;
                if (at + n <= kTopBuf) {
                    int o = at;
                    each_candidate(s, i0, floor, [&](float x, int col) {
                        const top_key key = make_key(x, col);
                        if (key >= threshold) sm.buf[o++] = key;
                    });
                    pending = false;
                } else {
                    for (int o = at; o < kTopBuf; ++o) sm.buf[o] = 0ull;   // places given out and not used
                    sm.overflow[offers & 1] = 1;
                }
            }
            __syncthreads();
            if (!sm.overflow[offers & 1]) break;
            const int n = compact_candidates(sm, min(sm.total, kTopBuf), k);
            if (tid == 0) { sm.total = n; sm.overflow[offers & 1] = 0; }
            threshold = sm.buf[n - 1];
            if (n == k) floor = unorder_bits((uint32_t)(threshold >> 32));
            else threshold = 0;
            __syncthreads();
        }
        ++offers;
    }
    // the slice's k largest, sorted
    __syncthreads();
    const int got = compact_candidates(sm, min(sm.total, kTopBuf), k);
    const Part st = exchange_parts<false>(a, sm.xs, p.rows.C, r.rank, r.c);
    const bool ok = r.T_ok && rowstat_ok(st.m, st.s);
    if (r.rank == 0 && tid == 0) {
        p.out_lse[r.row] = ok ? (float)((double)st.m / r.T + log((double)st.s)) : __int_as_float(0x7fc00000);
        if (!ok && p.status) atomicOr(p.status, kDevInvalidInput);
    }
    const int C = p.rows.C;
    if (!ok) {   // the same in every CTA
        if (r.rank == 0 && tid < k) {
            p.out_values[r.row * k + tid] = -INFINITY;
            p.out_ids[r.row * k + tid] = -1;
        }
        return;
    }
    if (C == 1) {
        if (tid < k) {
            const bool have = tid < got;
            const top_key key = have ? sm.buf[tid] : 0ull;
            p.out_values[r.row * k + tid] = have ? unorder_bits((uint32_t)(key >> 32)) : -INFINITY;
            p.out_ids[r.row * k + tid] = have ? (int32_t)~(uint32_t)key : -1;
        }
        return;
    }
    // every CTA gets every list
    for (int i = tid; i < C * kMaxTop; i += kLThreads) {
        const int to = i / kMaxTop, at = i % kMaxTop;
        if (at < got) {
            const uint32_t addr = map_to_peer(smem_u32(&sm.list[r.rank][at]), (uint32_t)to);
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(sm.buf[at]) : "memory");
        }
        if (at == 0) peer_store(map_to_peer(smem_u32(&sm.count[r.rank]), (uint32_t)to), got);
    }
    __syncwarp();
    cluster_sync_all();
    int all = 0;
    for (int c = 0; c < C; ++c) all += sm.count[c];
    if (tid < got) {
        const top_key key = sm.buf[tid];
        int rank = tid;
        for (int c = 0; c < C; ++c) {
            if (c == r.rank) continue;
            int lo = 0, hi = sm.count[c];   // keys larger than `key`
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (sm.list[c][mid] > key) lo = mid + 1; else hi = mid;
            }
            rank += lo;
        }
        if (rank < k) {
            p.out_values[r.row * k + rank] = unorder_bits((uint32_t)(key >> 32));
            p.out_ids[r.row * k + rank] = (int32_t)~(uint32_t)key;
        }
    }
    if (r.rank == 0 && tid < k && tid >= all) {   // fewer than k finite entries
        p.out_values[r.row * k + tid] = -INFINITY;
        p.out_ids[r.row * k + tid] = -1;
    }
}

}  // namespace ears
