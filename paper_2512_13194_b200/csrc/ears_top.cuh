// The k largest logits of every row, with the row's log normaliser.
//
// Entries are ordered by (value, lower index first), so that the result does not depend on how the
// row was split: an entry's key is its value as an order-preserving 32-bit integer followed by the
// complement of its index, all keys of a row are distinct, and the k largest keys are unique.
//
// One sweep of the slice yields the statistics of the row's softmax and, as a by-product, the maximum of
// every group of entries that one thread held in registers together (64 of them; at most kTopRounds groups
// per thread).  Of these maxima, folded to kTopBest per thread, the k-th largest is a threshold: at least k
// entries reach it.  For rows in no particular order few others do (of G folded groups about G ln(G / (G - k))
// entries: 137 for k = 128 and G = 1024, 177 had each thread one), so only the groups that reach it are
// fetched again, and their entries are candidates.
//   * thresholds and group maxima are compared by the upper 16 bits of their ordered pattern, which is
//     exact for bf16 and a threshold a little lower for the others; the k-th largest is found two bits at a time by
//     counting;
//   * the rank of a candidate is the number of larger keys: one comparison with every other, read from
//     shared memory two to a load, without a barrier;
//   * when too many entries reach the threshold (rows with most entries equal), they are offered to the buffer
//     round by round instead, and whenever it is full its k largest stay and the threshold rises to the k-th:
//     slower, never wrong.
// The C sorted lists of a cluster are handed to every CTA, and each CTA finds the final ranks of its own
// entries by binary search in the others.
#pragma once
#include "ears_distill.cuh"   // kMaxTop
#include "ears_rows.cuh"

namespace ears {

typedef unsigned long long top_key;
constexpr int kTopBuf = 2048;                // candidates a CTA holds: 128 + 64 < 2048, so each offer takes one thread's at least
constexpr int kTopRounds = 16;               // groups per thread: round r of the sweep counts to group r % kTopRounds
constexpr int kTopGroups = 1024;             // groups fetched again
constexpr int kTopBest = 4;                  // maxima per thread that the threshold is taken from

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
    union {
        top_key list[kLMaxCluster][kMaxTop];          // sorted lists of the cluster's CTAs
        uint16_t group[kTopRounds][kLThreads];        // before them: 16-bit prefixes of the group maxima
    };
    int count[kLMaxCluster];
    uint16_t reach[kTopGroups];              // groups that reach the threshold
    uint2 tally[2][kLWarps];
    int total;                               // places of buf given out
    int groups;                              // places of reach given out
    int overflow[2];                         // alternating by offer
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

constexpr uint32_t kLowestPrefix = 0x0080u;   // of the lowest finite value; -inf lies below it

// The largest 16-bit t >= kLowestPrefix that at least k of the threads' values v reach (kLowestPrefix if fewer do).
// All threads; values below kLowestPrefix stand for nothing.
template <int PER>
__device__ __forceinline__ uint32_t kth_prefix(const uint32_t (&v)[PER], int per, int k, TopSmem& sm) {
    uint32_t t = 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
        uint2* tally = sm.tally[(s >> 1) & 1];
        if (lane == 0) tally[warp] = make_uint2(a, b);
        __syncthreads();
        a = b = 0;
#pragma unroll
        for (int w = 0; w < kLWarps; ++w) { a += tally[w].x; b += tally[w].y; }
        if ((int)b >= k) t = t3;
        else if ((int)(a >> 16) >= k) t = t2;
        else if ((int)(a & 0xffffu) >= k) t = t1;
    }
    return max(t, kLowestPrefix);
}

// The k largest of buf[0 .. n) sorted to its front.  All threads; buf is final when it returns.
__device__ __forceinline__ int compact_candidates(TopSmem& sm, int n, int k) {
    constexpr int PER = kTopBuf / kLThreads;
    const int tid = threadIdx.x;
    if (n > kLThreads && n > k) {
        // drop what the k-th largest prefix leaves behind, so that the ranking has little more than k to compare
        top_key mine[PER];
        uint32_t v[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = tid + i * kLThreads;
            mine[i] = at < n ? sm.buf[at] : 0ull;
            v[i] = (uint32_t)(mine[i] >> 48);
        }
        if (tid == 0) sm.total = 0;
        const uint32_t t = kth_prefix(v, (n + kLThreads - 1) / kLThreads, k, sm);   // its barriers part the reads from the writes
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (v[i] >= t) sm.buf[atomicAdd(&sm.total, 1)] = mine[i];
        __syncthreads();
        n = sm.total;
    }
    if (tid == 0 && (n & 1)) sm.buf[n] = 0ull;   // kTopBuf is even
    __syncthreads();
    const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(sm.buf);
    const int n2 = (n + 1) / 2;
    top_key mine[PER];
    int rank[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = tid + i * kLThreads;
        mine[i] = 0ull;
        if (at >= n) continue;
        mine[i] = sm.buf[at];
        rank[i] = 0;
#pragma unroll 4
        for (int j = 0; j < n2; ++j) {
            const ulonglong2 q = pairs[j];
            rank[i] += (q.x > mine[i]) + (q.y > mine[i]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (mine[i] != 0ull && rank[i] < k) sm.buf[rank[i]] = mine[i];
    __syncthreads();
    return min(n, k);
}

// Calls f(value, column) for every finite entry of vector i of the slice whose prefix is at least t16.
template <typename E, class F>
__device__ __forceinline__ void each_candidate(const Slice<E>& s, int i, uint32_t t16, F f) {
    constexpr int N = Words<E>::N;
    const int v = s.v0 + i;
    const uint4 w = s.whole(v) ? ld_row16(reinterpret_cast<const uint4*>(s.base) + v) : load_partial(s.base, v, s.lead, s.end);
    float x[N];
    Words<E>::unpack(w, x);
    const int col = v * N - s.lead;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if ((order_bits(x[j]) >> 16) >= t16) f(x[j], col + j);
}

// Too many entries reach the threshold: every thread offers its entries round by round, and when the buffer cannot take
// them all, its k largest stay, the threshold rises to the k-th and what is still pending is offered again.
template <typename E>
__device__ __noinline__ void offer_rounds(const Slice<E>& s, TopSmem& sm, int rounds, uint32_t t16, int k) {
    const int tid = threadIdx.x;
    top_key threshold = (top_key)t16 << 48;
    int offers = 0;
    __syncthreads();
    if (tid == 0) sm.total = 0;
    __syncthreads();
    for (int round = 0; round < rounds; ++round) {
        const int i0 = round * kLRound + tid;
        bool pending = true;
        for (;; ++offers) {
            if (pending) {
                int n = 0;
                for (int i = i0; i < s.n && i < i0 + kLRound; i += kLThreads)
                    each_candidate(s, i, t16, [&](float x, int col) { n += make_key(x, col) >= threshold; });
                const int at = n ? atomicAdd(&sm.total, n) : 0;
                if (at + n <= kTopBuf) {
                    int o = at;
                    for (int i = i0; i < s.n && i < i0 + kLRound; i += kLThreads)
                        each_candidate(s, i, t16, [&](float x, int col) {
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
            const int held = min(sm.total, kTopBuf);
            __syncthreads();
            const int n = compact_candidates(sm, held, k);
            threshold = n == k ? sm.buf[k - 1] : threshold;
            if (tid == 0) { sm.total = n; sm.overflow[offers & 1] = 0; }
            __syncthreads();
        }
        ++offers;
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
    if (tid == 0) { sm.total = sm.groups = 0; sm.overflow[0] = sm.overflow[1] = 0; }
    Stat<false> a;
    stat_open(a);
    const uint64_t pol = l2_policy_evict_first();
    const int rounds = (s.n + kLRound - 1) / kLRound, groups = min(rounds, kTopRounds);
    uint32_t best[kTopBest];   // the thread's group maxima, folded
#pragma unroll
    for (int i = 0; i < kTopBest; ++i) best[i] = 0u;
    sweep_rounds(s, pol, [&](uint4 (&w)[kLUnroll], int round) {
        const float top = stat_fold<E, kLUnroll, false>(w, r.c, a);
        const uint32_t prefix = top > -INFINITY ? order_bits(top) >> 16 : 0u;   // NaN: the row is unusable anyway
        uint16_t* g = &sm.group[round % kTopRounds][tid];
        *g = (uint16_t)(round < kTopRounds ? prefix : max((uint32_t)*g, prefix));
#pragma unroll
        for (int i = 0; i < kTopBest; ++i)
            if (round % kTopBest == i) best[i] = max(best[i], prefix);
    });
    const uint32_t t16 = kth_prefix(best, min(rounds, kTopBest), k, sm);
    for (int i = 0; i < groups; ++i) {
        if (sm.group[i][tid] >= t16) {   // the thread's own
            const int at = atomicAdd(&sm.groups, 1);
            if (at < kTopGroups) sm.reach[at] = (uint16_t)(i * kLThreads + tid);
        }
    }
    __syncthreads();
    const int reached = sm.groups;
    if (reached <= kTopGroups) {
        // eight threads to a group, one vector each
        for (int q = tid / kLUnroll; q < reached; q += kLThreads / kLUnroll) {
            const int g = sm.reach[q];
            for (int round = g / kLThreads; round < rounds; round += kTopRounds) {
                const int i = round * kLRound + (tid % kLUnroll) * kLThreads + g % kLThreads;
                if (i < s.n)
                    each_candidate(s, i, t16, [&](float x, int col) {
                        const int at = atomicAdd(&sm.total, 1);
                        if (at < kTopBuf) sm.buf[at] = make_key(x, col);
                    });
            }
        }
    }
    __syncthreads();
    if (reached > kTopGroups || sm.total > kTopBuf) offer_rounds(s, sm, rounds, t16, k);
    // the slice's k largest, sorted
    const int found = sm.total;
    __syncthreads();
    const int got = compact_candidates(sm, found, k);
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
