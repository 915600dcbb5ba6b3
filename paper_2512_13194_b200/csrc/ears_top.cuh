// The k largest logits of every row, with the row's log normaliser.
//
// Entries are ordered by (value, lower index first), so that the result does not depend on how the
// row was split: an entry's key is its value as an order-preserving 32-bit integer followed by the
// complement of its index, all keys of a row are distinct, and the k largest keys are unique.
//
// One sweep of the slice yields the statistics of the row's softmax and, as a by-product, the maximum of
// every group of entries that one thread held in registers together (two vectors, 16 entries of two bytes; rounds
// beyond kTopRounds share groups with earlier ones).  Of these maxima, folded to two per thread, the k-th largest is
// a threshold: at least k entries reach it.  For rows in no particular order few others do (of G folded groups about G ln(G / (G - k))
// entries: 147 for k = 128 and G = 512, 177 had each thread one, 137 four), so only the groups that reach it are
// fetched again, and their entries are candidates.
//   * the threshold is kept as the upper 16 bits of an ordered pattern, which is exact for bf16 and a little lower
//     for the others; the k-th largest is found two bits at a time by counting, by one warp: what follows the
//     sweep is bound by the number of instructions, since the CTAs of a launch reach it together;
//   * the rank of a candidate is the number of larger keys: one comparison with every other, read from
//     shared memory two to a load, without a barrier;
//   * when too many entries reach the threshold (rows with most entries equal), they are offered to the buffer
//     round by round instead, and whenever it is full its k largest stay and the threshold rises to the k-th:
//     slower, never wrong.
// The C sorted lists of a cluster are handed to every CTA, and each CTA finds the final ranks of its own
// entries by binary search in the others.
//
// Bound by HBM and by what follows the sweep: of 47 us for 128 of 512 rows of 152064 bf16 (0.51 of the copy rate; the
// CTAs of one launch run side by side and finish together) the sweep takes 39 (33 without the group maxima), the candidates 5, their
// ranks 3.  A first build that ranked every candidate of a per-thread threshold by counting took 465 us, fetching all eight
// vectors of a round again 53.
#pragma once
#include "ears_distill.cuh"   // kMaxTop
#include "ears_rows.cuh"

namespace ears {

typedef unsigned long long top_key;
constexpr int kTopBuf = 1024;                // candidates a CTA holds: 128 + 64 < 1024, so each offer takes one thread's at least
constexpr int kTopRounds = 16;               // round r of the sweep counts to the groups of r % kTopRounds
constexpr int kTopParts = 4;                 // groups per thread and round: two vectors each
constexpr int kTopGroups = 1024;             // groups fetched again
constexpr int kTopBatch = 6;                 // groups fetched at a time by eight lanes: 192 by the CTA

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
        uint2 group[kTopRounds][kLThreads];           // before them: the upper halves of the group maxima, four a round
    };
    float best[2 * kLThreads];
    int count[kLMaxCluster];
    uint16_t reach[kTopGroups];              // groups that reach the threshold
    uint2 tally[2][kLWarps];
    int total;                               // places of buf given out
    int groups;                              // places of reach given out
    int overflow[2];                         // alternating by offer
    uint32_t t16;
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

// The largest 16-bit t >= kLowestPrefix that at least k of one warp's values v reach (kLowestPrefix if fewer do); values
// below kLowestPrefix stand for nothing.
template <int PER>
__device__ __forceinline__ uint32_t warp_kth(const uint32_t (&v)[PER], int per, int k) {
    // the leading bits that the largest and the smallest share are the threshold's as well
    uint32_t hi = 0, lo = 0xffffu;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i >= per) break;
        hi = max(hi, v[i]);
        lo = min(lo, v[i]);
    }
    hi = __reduce_max_sync(0xffffffffu, hi);
    lo = __reduce_min_sync(0xffffffffu, lo);
    if (hi == lo || per * 32 < k) return max(lo, kLowestPrefix);
    const int top = (31 - __clz(hi ^ lo)) & ~1;   // of the two bits tried first
    uint32_t t = hi >> (top + 2) << (top + 2);
#pragma unroll 1
    for (int s = top; s >= 0; s -= 2) {
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

// Places for n entries of every lane, one atomic for the warp.  -> the lane's first place.
__device__ __forceinline__ int warp_reserve(int n, int* counter) {
    const int lane = threadIdx.x & 31;
    int sum = n;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, sum, off);
        if (lane >= off) sum += o;
    }
    int base = 0;
    if (lane == 31 && sum > 0) base = atomicAdd(counter, sum);
    return __shfl_sync(0xffffffffu, base, 31) + sum - n;
}

// warp_kth over the values of all threads of the CTA.
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

// One 32-bit word of the row's vector run: entry e and what shares its word, -inf beyond the row.
template <typename E> constexpr int kTopWord = 4 / (int)sizeof(E);   // entries in it
template <typename E>
__device__ __forceinline__ uint32_t load_word(const Slice<E>& s, int e) {
    constexpr int W = kTopWord<E>;
    if (e >= s.lead && e + W <= s.end) return *reinterpret_cast<const uint32_t*>(s.base + e);
    uint32_t w = Words<E>::minus_inf().x;
    if (W == 2) {
        if (e >= s.lead && e < s.end) put_half(w, 0, raw_bits(s.base + e));
        if (e + 1 >= s.lead && e + 1 < s.end) put_half(w, 1, raw_bits(s.base + e + 1));
    }
    return w;
}
__device__ __forceinline__ void unpack_word(uint32_t w, float (&x)[1], float) { x[0] = __uint_as_float(w); }
__device__ __forceinline__ void unpack_word(uint32_t w, float (&x)[2], uint16_t) { x[0] = __uint_as_float(w << 16); x[1] = __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void unpack_word(uint32_t w, float (&x)[2], f16_t) { const float2 v = f16x2_to_float2(w); x[0] = v.x; x[1] = v.y; }

template <typename E>
__device__ __forceinline__ uint4 slice_vector(const Slice<E>& s, int i) {
    const int v = s.v0 + i;
    return s.whole(v) ? ld_row16(reinterpret_cast<const uint4*>(s.base) + v) : load_partial(s.base, v, s.lead, s.end);
}

// Calls f(value, column) for every finite entry of w, vector i of the slice, whose prefix is at least t16.
template <typename E, class F>
__device__ __forceinline__ void each_candidate(const Slice<E>& s, uint4 w, int i, uint32_t t16, F f) {
    constexpr int N = Words<E>::N;
    const uint4 one[1] = {w};
    const float top = Words<E>::template vmax_all<1>(one);
    if ((order_bits(top) >> 16) < t16) return;   // false for NaN: the row is unusable anyway
    float x[N];
    Words<E>::unpack(w, x);
    const int col = (s.v0 + i) * N - s.lead;
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
                    each_candidate(s, slice_vector(s, i), i, t16, [&](float x, int col) { n += make_key(x, col) >= threshold; });
                const int at = n ? atomicAdd(&sm.total, n) : 0;
                if (at + n <= kTopBuf) {
                    int o = at;
                    for (int i = i0; i < s.n && i < i0 + kLRound; i += kLThreads)
                        each_candidate(s, slice_vector(s, i), i, t16, [&](float x, int col) {
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

// Group q of a round: its maximum with the lower half of its bits cut off, which a threshold without those bits (or, below
// zero, with all of them set) does not notice.
__device__ __forceinline__ float group_max(uint2 g, int q) {
    const uint32_t two = q < 2 ? g.x : g.y;
    return __uint_as_float(q & 1 ? two & 0xffff0000u : two << 16);
}

template <typename E, bool AHEAD>
__global__ void __launch_bounds__(kLThreads, AHEAD ? 2 : 4) ears_top_kernel(const TopParams p) {
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
    const uint64_t pol = l2_policy_normal();   // some of it is fetched again
    const int rounds = (s.n + kLRound - 1) / kLRound, groups = min(rounds, kTopRounds);
    float best[2] = {-INFINITY, -INFINITY};   // the thread's group maxima, folded to those of even and of odd rounds
    sweep_rounds<E, AHEAD>(s, pol, [&](uint4 (&w)[kLUnroll], int round) {
        float part[kTopParts];
#pragma unroll
        for (int q = 0; q < kTopParts; ++q) {
            const uint4 two[2] = {w[2 * q], w[2 * q + 1]};
            part[q] = Words<E>::template vmax_all<2>(two);
        }
        const float top = fmaxf(max3(part[0], part[1], part[2]), part[3]);
        uint2* g = &sm.group[round % kTopRounds][tid];
        if (round >= kTopRounds) {
            const uint2 old = *g;
#pragma unroll
            for (int q = 0; q < kTopParts; ++q) part[q] = fmaxf(part[q], group_max(old, q));
        }
        *g = make_uint2(__byte_perm(__float_as_uint(part[0]), __float_as_uint(part[1]), 0x7632),
                        __byte_perm(__float_as_uint(part[2]), __float_as_uint(part[3]), 0x7632));
        best[round & 1] = fmaxf(best[round & 1], top);
        stat_add<E, kLUnroll, false>(w, top, r.c, a);
    });
    sm.best[tid] = best[0];
    sm.best[kLThreads + tid] = best[1];
    __syncthreads();
    if (tid < 32) {
        uint32_t v[2 * kLWarps];
#pragma unroll
        for (int i = 0; i < 2 * kLWarps; ++i) v[i] = order_bits(sm.best[tid + 32 * i]) >> 16;
        const uint32_t t = warp_kth(v, rounds > 1 ? 2 * kLWarps : kLWarps, k);
        if (tid == 0) sm.t16 = t;
    }
    __syncthreads();
    const uint32_t t16 = sm.t16;
    const float reach = unorder_bits(t16 << 16);
    // the thread's own groups; false for NaN: the row is unusable anyway
    int mine = 0;
    for (int i = 0; i < groups; ++i) {
        const uint2 g = sm.group[i][tid];
#pragma unroll
        for (int q = 0; q < kTopParts; ++q) mine += group_max(g, q) >= reach ? 1 : 0;
    }
    int place = warp_reserve(mine, &sm.groups);
    if (mine > 0 && place + mine <= kTopGroups) {
        for (int i = 0; i < groups; ++i) {
            const uint2 g = sm.group[i][tid];
#pragma unroll
            for (int q = 0; q < kTopParts; ++q)
                if (group_max(g, q) >= reach) sm.reach[place++] = (uint16_t)((i * kTopParts + q) * kLThreads + tid);
        }
    }
    __syncthreads();
    const int reached = sm.groups;
    if (reached <= kTopGroups) {
        // eight lanes to a group's two vectors, kTopBatch groups of theirs in flight
        constexpr int TEAMS = kLThreads / 8;
        for (int q0 = tid / 32 * 4; q0 < reached; q0 += kTopBatch * TEAMS) {   // the same for a warp
            const int team = (tid & 31) / 8, sub = tid & 7;
            for (int turn = 0; turn < rounds; turn += kTopRounds) {   // once, unless a slice has more rounds than groups
                uint32_t w[kTopBatch];
                const auto entry = [&](int j) {   // of the run: vector, word sub % 4
                    const int q = q0 + team + j * TEAMS, g = q < reached ? sm.reach[q] : 0;
                    const int round = turn + g / (kTopParts * kLThreads), part = g / kLThreads % kTopParts;
                    return ((s.v0 + round * kLRound + (2 * part + sub / 4) * kLThreads + g % kLThreads) * 4 + sub % 4) * kTopWord<E>;
                };
#pragma unroll
                for (int j = 0; j < kTopBatch; ++j) {
                    w[j] = Words<E>::minus_inf().x;
                    if (q0 + team + j * TEAMS < reached) {
                        const int e = entry(j);
                        if (e < (s.v0 + s.n) * Words<E>::N) w[j] = load_word(s, e);
                    }
                }
                int hits = 0;
#pragma unroll
                for (int j = 0; j < kTopBatch; ++j) {
                    float x[kTopWord<E>];
                    unpack_word(w[j], x, E{});
#pragma unroll
                    for (int i = 0; i < kTopWord<E>; ++i) hits += x[i] >= reach ? 1 : 0;
                }
                int at = warp_reserve(hits, &sm.total);
                if (hits > 0 && at + hits <= kTopBuf) {
#pragma unroll
                    for (int j = 0; j < kTopBatch; ++j) {
                        float x[kTopWord<E>];
                        unpack_word(w[j], x, E{});
#pragma unroll
                        for (int i = 0; i < kTopWord<E>; ++i)
                            if (x[i] >= reach) sm.buf[at++] = make_key(x[i], entry(j) + i - s.lead);
                    }
                }
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
        p.out_lse[r.row] = ok ? (float)((double)st.m / r.T + log(row_mass(st.s))) : __int_as_float(0x7fc00000);
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
