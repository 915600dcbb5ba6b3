// Short rows: a warp, or a CTA of 128 threads, has a row to itself.  It takes the row in rounds of eight 16-byte vectors
// per thread and keeps the last round in registers, so that a row of one round (4 KB for a warp, 16 KB for 128 threads) is
// read once whatever is computed from it; the gradient of a longer one fetches the other rounds again, out of L2.
//
// Bound by latency: a row passes through some 3 us of dependent steps (its token or list, its logits, the
// reduction, the 64-bit scalars), so what counts is the number of rows an SM has in flight: 24 with a warp per row, 6 with
// 128 threads, 2 to 4 with the CTAs of the other kernels.  Token steps on 8192 rows of bf16: 85 us with the ring at 2000
// entries, 22 so; 98 and 56 at 6000 (floor 30).
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
    static constexpr int kRounds = G == 32 ? 8 : 1;              // longest rows: 32 and 16 KB
    // Per SM: leaves 80 registers a thread, at which forward calls spill little or nothing (40 bytes a thread at most), token
    // steps 16 to 168, distillation's backward calls 236 and 332 and its steps 328 to 440.
    static constexpr int kCtas = 6;
};

// A row's whole vectors, in rounds: vector (round kShortSlots + j) G + tid in w[j]; and the one vector at an end that the row
// covers in part which falls to this thread: thread 0 has the first, thread 1 the last (index `edge`, -1: none).  Beyond
// the row: -inf.
template <typename E, int G>
struct ShortRow {
    const Slice<E>& s;
    int tid, v0, vecs, edge, rounds;
    uint4 w[kShortSlots], we;

    __device__ __forceinline__ ShortRow(const Slice<E>& slice, int thread) : s(slice), tid(thread) {
        v0 = s.lead > 0 ? 1 : 0;
        vecs = max(0, s.end / Words<E>::N - v0);
        rounds = (vecs + kShortSlots * G - 1) / (kShortSlots * G);
        edge = -1;
        if (tid == 0 && v0 > 0) edge = 0;
        if (tid == 1 && s.n > v0 + vecs) edge = s.n - 1;
        we = Words<E>::minus_inf();
        if (edge >= 0) we = load_partial(s.base, edge, s.lead, s.end);
    }
    __device__ __forceinline__ void load(int round) {
        const int first = round * kShortSlots * G + tid;
        const uint4* p = reinterpret_cast<const uint4*>(s.base) + v0 + first;
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) {
            w[j] = Words<E>::minus_inf();
            if (first + j * G < vecs) w[j] = ld_row16(p + j * G);
        }
    }
};

// The statistics of the thread's vectors; mask(w, round) may take entries out, of the last round for good.
template <typename E, int G, bool ENT, class F>
__device__ __forceinline__ Stat<ENT> short_stats(ShortRow<E, G>& x, const Scale& c, F mask) {
    Stat<ENT> a;
    stat_open(a);
    for (int round = 0; round < x.rounds; ++round) {
        x.load(round);
        mask(x.w, round);
        stat_fold<E, kShortSlots, ENT>(x.w, c, a);
    }
    if (x.edge >= 0) {
        const uint4 one[1] = {x.we};
        stat_fold<E, 1, ENT>(one, c, a);
    }
    return a;
}

// The gradient row, 2^t (A + Bt t) or zeros: the last round, which w holds, first.
template <typename E, int G, bool ENT>
__device__ __forceinline__ void short_gradient(ShortRow<E, G>& x, E* g, bool zero, float ref, float c, float A, float Bt) {
    const Slice<E>& s = x.s;
    const bool aligned = ((uintptr_t)g & 15) == 0;
    for (int round = x.rounds - 1; round >= 0; --round) {
        if (round < x.rounds - 1 && !zero) x.load(round);
        const int first = round * kShortSlots * G + x.tid;
        uint4* out = reinterpret_cast<uint4*>(g) + x.v0 + first;
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) {
            const uint4 d = zero ? make_uint4(0, 0, 0, 0) : dense_words<E, ENT>(x.w[j], ref, c, A, Bt);
            if (first + j * G < x.vecs) {
                if (aligned) out[j * G] = d;
                else store_partial(g, x.v0 + first + j * G, d, s.lead, s.end);
            }
        }
    }
    if (x.edge >= 0)
        store_partial(g, x.edge, zero ? make_uint4(0, 0, 0, 0) : dense_words<E, ENT>(x.we, ref, c, A, Bt), s.lead, s.end);
}

// A gradient row of zeros of which nothing was read.
template <typename E, int G>
__device__ __forceinline__ void short_zero(const Slice<E>& s, int tid, E* g) {
    const bool aligned = ((uintptr_t)g & 15) == 0;
#pragma unroll 1
    for (int v = tid; v < s.n; v += G) {
        if (aligned && s.whole(v)) reinterpret_cast<uint4*>(g)[v] = make_uint4(0, 0, 0, 0);
        else store_partial(g, v, make_uint4(0, 0, 0, 0), s.lead, s.end);
    }
}

// The statistics of the whole row, in every thread.
template <int G, bool ENT>
__device__ __forceinline__ Part short_merge(const Stat<ENT>& a, float4* xs, const Scale& c) {
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
    wait_for_stream();
    const unsigned row = blockIdx.x * (unsigned)ShortShape<G>::kRows + (G == 32 ? threadIdx.x / 32u : 0u);
    if (row >= p.rows) return false;
    *r = row_setup_at(p, row);
    return true;
}

template <typename E, int G, bool ENT, int MODE>
__global__ void __launch_bounds__(ShortShape<G>::kThreads, ShortShape<G>::kCtas) ears_token_short_kernel(const TokenParams p) {
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
    ShortRow<E, G> x(s, tid);
    Part st;
    if (MODE == kBackward) {
        if (x.rounds > 0) x.load(x.rounds - 1);
        st = token_saved<ENT>(p.stats[r.row]);
    } else {
        st = short_merge<G, ENT>(short_stats<E, G, ENT>(x, r.c, [](uint4 (&)[kShortSlots], int) {}), xs, r.c);
    }
    if (tid == 0) sc = token_scalars<ENT, MODE>(p, r.row, 0, r.T, r.T_ok, in, st);
    if (MODE == kForward) return;
    row_sync<G>();
    const TokenScalars t = sc;
    short_gradient<E, G, ENT>(x, grad, t.zero != 0, st.m, r.c.near, t.A, t.Bt);
    if (t.zero) return;
    row_sync<G>();   // the dense value of the token's entry has been written
    if (tid == 0) store_entry(grad + s.lead + tok, t.entry);
}

template <typename E, int G, int MODE>
__global__ void __launch_bounds__(ShortShape<G>::kThreads, ShortShape<G>::kCtas) ears_distill_short_kernel(const DistillParams p) {
    __shared__ float4 xs[G / 32];
    __shared__ ListSmem lists[ShortShape<G>::kRows];
    __shared__ alignas(16) uint2 all_bits[ShortShape<G>::kThreads * ShortShape<G>::kRounds];
    RowSetup r;
    if (!short_setup<G>(p.rows, &r)) return;
    const int tid = threadIdx.x % G, k = p.k;
    ListSmem& sm = lists[threadIdx.x / G];
    uint2* bits = all_bits + threadIdx.x / G * (G * ShortShape<G>::kRounds);
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, 0);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const int v0 = s.lead > 0 ? 1 : 0;   // the first whole vector
    const int seen = distill_list<E, kShortSlots, G, G>(p, sm, reinterpret_cast<uint32_t*>(bits), tid, r.row, s.lead, v0,
                                                             max(0, s.end / Words<E>::N - v0));
    if (seen != 1) {
        if (tid == 0) distill_unused<MODE>(p, r.row, (seen & 2) != 0);
        if (MODE != kForward) short_zero<E, G>(s, tid, grad);
        return;
    }
    DraftLogits dl{};
    if (tid < 32) dl = draft_logits(p, sm, row);
    ShortRow<E, G> x(s, tid);
    Part st;
    if (MODE == kBackward) {
        if (x.rounds > 0) x.load(x.rounds - 1);
        const float4 q = p.stats[r.row];
        st = Part{q.x, q.y, 0.f};
    } else {
        // the gradient of a listed entry is written on its own, so its place may go to -inf for good
        if (x.edge >= 0) mask_entries<E>(x.we, sm.edge[x.edge < v0 ? 0 : 1]);
        st = short_merge<G, false>(short_stats<E, G, false>(x, r.c, [&](uint4 (&w)[kShortSlots], int round) {
            mask_listed<E>(w, bits[round * G + tid]);
        }), xs, r.c);
    }
    const bool empty = tail_empty(st);
    if (tid < 32) {
        const double invT = 1.0 / r.T;
        const float weight = MODE != kForward && p.weight ? __ldg(p.weight + r.row) : 1.f;
        distill_scalars<MODE>(p, sm, r.row, 0, invT, r.T_ok && (empty || rowstat_ok(st.m, st.s)), teacher_part(p, sm, r.row, invT),
                              draft_part(p, sm, dl, invT), weight, st, [] {});
    }
    if (MODE == kForward) return;
    row_sync<G>();
    const bool zero = sm.zero != 0;
    short_gradient<E, G, false>(x, grad, zero, empty ? 0.f : st.m, r.c.near, sm.factor, 0.f);
    if (zero) return;
    row_sync<G>();   // the dense values of the listed entries have been written
    for (int j = tid; j < k; j += G)
        if (sm.col[j] >= 0) store_entry(grad + s.lead + sm.col[j], sm.entry[j]);
}

// ---- top logits: a warp streams its row ----------------------------------------------------------------
// The CTA-wide kernel spends some 10 us on a row whatever its length, with four rows in flight per SM; here 24 are
// (8192 rows of 6000 bf16: 147 us and 50).  Where the vectors' maxima leave too many candidates, as in a row with few more
// vectors than the list has entries, warp_top_exact narrows them (128 of 20000 x 1026 bf16: 383 us, of 20000 x 2000 183).
constexpr int kShortTopBuf = 256;            // candidates per row; kMaxTop and more
constexpr int kWarpTopRounds = 8;            // of 32 lanes x kShortSlots vectors: rows up to 32 KB
constexpr int kWarpTopReach = 384;           // vectors fetched again

// One warp: the candidates from + lane, from + lane + 32, .. (W of a lane) to their ranks among buf[0 .. n).
template <int W>
__device__ __forceinline__ void rank_some(const top_key* buf, int from, int n, int k, float* values, int32_t* ids) {
    const int at = from + (threadIdx.x & 31);
    const ulonglong2* pairs = reinterpret_cast<const ulonglong2*>(buf);
    top_key mine[W];
    int rank[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const bool have = at + 32 * i < n;
        mine[i] = have ? buf[at + 32 * i] : 0ull;
        rank[i] = have ? 0 : k;
    }
#pragma unroll 4
    for (int j = 0; j < (n + 1) / 2; ++j) {
        const ulonglong2 q = pairs[j];
#pragma unroll
        for (int i = 0; i < W; ++i) rank[i] += (q.x > mine[i]) + (q.y > mine[i]);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (rank[i] < k) {
            values[rank[i]] = unorder_bits((uint32_t)(mine[i] >> 32));
            ids[rank[i]] = (int32_t)~(uint32_t)mine[i];
        }
    }
}

// One warp: the candidates buf[0 .. n) to their ranks below k, absent entries behind them.
__device__ __forceinline__ void write_ranked(top_key* buf, int n, int k, float* values, int32_t* ids) {
    const int lane = threadIdx.x & 31;
    if (lane == 0 && (n & 1)) buf[n] = 0ull;   // kShortTopBuf is even
    __syncwarp();
    int from = 0;
    for (; n - from > 64; from += 128) rank_some<4>(buf, from, n, k, values, ids);
    for (; n - from > 0; from += 32) rank_some<1>(buf, from, n, k, values, ids);
    for (int j = n + lane; j < k; j += 32) { values[j] = -INFINITY; ids[j] = -1; }   // fewer than k finite entries
}

struct WarpTopSmem {
    alignas(16) top_key buf[kShortTopBuf];
    uint4 peak[kWarpTopRounds][32];          // upper halves of the vectors' maxima, eight a round and lane
    uint16_t reach[kWarpTopReach];
    int total, vectors;
};

__device__ __forceinline__ float peak_of(uint4 p, int j) {
    const uint32_t two = j < 2 ? p.x : j < 4 ? p.y : j < 6 ? p.z : p.w;
    return __uint_as_float(j & 1 ? two & 0xffff0000u : two << 16);
}

// Too many entries reach `lo`, the threshold from the vectors' maxima: the k-th largest value is approached two bits at a
// time, from the bits that lo and the row's largest share, the row fetched again for every step, until no more entries reach
// the threshold than buf holds.  If its last bit leaves too many (equal entries), buf gets those above it and the first
// equal ones.  -> entries in buf, k or more.
template <typename E>
__device__ __noinline__ int warp_top_exact(const Slice<E>& s, WarpTopSmem& sm, int k, uint32_t lo, uint32_t hi) {
    constexpr int N = Words<E>::N;
    const int lane = threadIdx.x & 31;
    uint32_t u = hi;
    int reaching = kShortTopBuf + 1;
    if (hi != lo) {
        int b = (31 - __clz(hi ^ lo)) & ~1;   // of the two bits tried first
        u = b == 30 ? 0u : hi >> (b + 2) << (b + 2);
        for (; b >= 0 && reaching > kShortTopBuf; b -= 2) {
            // all of k reach lo, and what lies below it need not be told apart (nor be the order of a number)
            const float t1 = unorder_bits(max(u | 1u << b, lo)), t2 = unorder_bits(max(u | 2u << b, lo)), t3 = unorder_bits(max(u | 3u << b, lo));
            uint32_t c12 = 0, c3 = 0;
            for (int v0 = lane; v0 < s.n; v0 += 32 * kShortSlots) {
                uint4 w[kShortSlots];
#pragma unroll
                for (int j = 0; j < kShortSlots; ++j) w[j] = v0 + 32 * j < s.n ? slice_vector(s, v0 + 32 * j) : Words<E>::minus_inf();
#pragma unroll
                for (int j = 0; j < kShortSlots; ++j) {
                    float x[N];
                    Words<E>::unpack(w[j], x);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        c12 += (x[i] >= t1 ? 1u : 0u) + (x[i] >= t2 ? 1u << 16 : 0u);
                        c3 += x[i] >= t3 ? 1u : 0u;
                    }
                }
            }
            c12 = __reduce_add_sync(0xffffffffu, c12);   // at most 16384 each
            c3 = __reduce_add_sync(0xffffffffu, c3);
            const int n3 = (int)c3, n2 = (int)(c12 >> 16), n1 = (int)(c12 & 0xffffu);
            if (n3 >= k) { u |= 3u << b; reaching = n3; }
            else if (n2 >= k) { u |= 2u << b; reaching = n2; }
            else if (n1 >= k) { u |= 1u << b; reaching = n1; }
        }
        u = max(u, lo);
    }
    const bool ties = reaching > kShortTopBuf;
    const int room = ties ? k : kShortTopBuf;
    const uint32_t over = ties ? u : u - 1;
    int above = 0, equal = 0;   // entries above the value so far, equal ones so far, in the order of the columns
    for (int pass = 0; pass < (ties ? 2 : 1); ++pass) {
        for (int v0 = 0; v0 < s.n; v0 += 32) {
            const int v = v0 + lane;
            const uint4 w = v < s.n ? slice_vector(s, v) : Words<E>::minus_inf();
            float x[N];
            Words<E>::unpack(w, x);
            int mine = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) mine += (pass == 0 ? order_bits(x[i]) > over : order_bits(x[i]) == u) ? 1 : 0;
            int sum = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, sum, off);
                if (lane >= off) sum += o;
            }
            int at = above + (pass == 0 ? 0 : equal) + sum - mine;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (pass == 0 ? order_bits(x[i]) > over : order_bits(x[i]) == u) {
                    if (at < room) sm.buf[at] = make_key(x[i], v * N + i - s.lead);
                    ++at;
                }
            }
            const int all = __shfl_sync(0xffffffffu, sum, 31);
            if (pass == 0) above += all; else equal += all;
        }
    }
    __syncwarp();
    return min(above + equal, room);
}

template <typename E>
__global__ void __launch_bounds__(ShortShape<32>::kThreads, ShortShape<32>::kCtas) ears_top_warp_kernel(const TopParams p) {
    constexpr int N = Words<E>::N;
    __shared__ WarpTopSmem rows[ShortShape<32>::kRows];
    RowSetup r;
    if (!short_setup<32>(p.rows, &r)) return;
    const int lane = threadIdx.x & 31, k = p.k;
    WarpTopSmem& sm = rows[threadIdx.x / 32];
    float* values = p.out_values + r.row * k;
    int32_t* ids = p.out_ids + r.row * k;
    const bool live = !p.accept_len || (int)r.k <= __ldg(p.accept_len + r.b);
    const Slice<E> s = make_slice<E>(row_ptr<E>(p.rows, r), p.rows.V, p.rows.slice, 0);
    const int rounds = live ? (s.n + 32 * kShortSlots - 1) / (32 * kShortSlots) : 0;
    Stat<false> a;
    stat_open(a);
    float best[kShortSlots];   // of the vectors at the same place of every round
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) best[j] = -INFINITY;
    for (int round = 0; round < rounds; ++round) {
        uint4 w[kShortSlots];
        uint32_t half[kShortSlots];
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) {
            const int v = (round * kShortSlots + j) * 32 + lane;
            w[j] = Words<E>::minus_inf();
            if (v < s.n) w[j] = slice_vector(s, v);
        }
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) {
            const uint4 one[1] = {w[j]};
            const float m = Words<E>::template vmax_all<1>(one);
            half[j] = __float_as_uint(m);
            best[j] = fmaxf(best[j], m);
            top = fmaxf(top, m);
        }
        sm.peak[round][lane] = make_uint4(__byte_perm(half[0], half[1], 0x7632), __byte_perm(half[2], half[3], 0x7632),
                                          __byte_perm(half[4], half[5], 0x7632), __byte_perm(half[6], half[7], 0x7632));
        stat_add<E, kShortSlots, false>(w, top, r.c, a);
    }
    const Part st = short_merge<32, false>(a, nullptr, r.c);
    const bool ok = live && r.T_ok && rowstat_ok(st.m, st.s);
    if (lane == 0) {
        p.out_lse[r.row] = !live ? -INFINITY : ok ? (float)((double)st.m / r.T + log(row_mass(st.s))) : __int_as_float(0x7fc00000);
        if (live && !ok && p.status) atomicOr(p.status, kDevInvalidInput);
        sm.total = sm.vectors = 0;
    }
    __syncwarp();
    if (!ok) {
        for (int j = lane; j < k; j += 32) { values[j] = -INFINITY; ids[j] = -1; }
        return;
    }
    uint32_t bv[kShortSlots];
#pragma unroll
    for (int j = 0; j < kShortSlots; ++j) bv[j] = order_bits(best[j]) >> 16;
    const uint32_t reach_bits = warp_kth(bv, kShortSlots, k) << 16;
    const float reach = unorder_bits(reach_bits);
    // the lane's own vectors that reach it
    int mine = 0;
    for (int round = 0; round < rounds; ++round) {
        const uint4 q = sm.peak[round][lane];
#pragma unroll
        for (int j = 0; j < kShortSlots; ++j) mine += peak_of(q, j) >= reach ? 1 : 0;
    }
    int place = warp_reserve(mine, &sm.vectors);
    if (mine > 0 && place + mine <= kWarpTopReach) {
        for (int round = 0; round < rounds; ++round) {
            const uint4 q = sm.peak[round][lane];
#pragma unroll
            for (int j = 0; j < kShortSlots; ++j)
                if (peak_of(q, j) >= reach) sm.reach[place++] = (uint16_t)((round * kShortSlots + j) * 32 + lane);
        }
    }
    __syncwarp();
    const int reached = sm.vectors;
    int n = kShortTopBuf + 1;
    if (reached <= kWarpTopReach) {
        constexpr int BATCH = 4;
        for (int q0 = 0; q0 < reached; q0 += 32 * BATCH) {
            uint4 w[BATCH];
            int v[BATCH], hits = 0;
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int q = q0 + j * 32 + lane;
                v[j] = q < reached ? sm.reach[q] : 0;
                w[j] = q < reached ? slice_vector(s, v[j]) : Words<E>::minus_inf();
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                float x[N];
                Words<E>::unpack(w[j], x);
#pragma unroll
                for (int i = 0; i < N; ++i) hits += x[i] >= reach ? 1 : 0;
            }
            int at = warp_reserve(hits, &sm.total);
            if (hits > 0 && at + hits <= kShortTopBuf) {
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    float x[N];
                    Words<E>::unpack(w[j], x);
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (x[i] >= reach) sm.buf[at++] = make_key(x[i], v[j] * N + i - s.lead);
                }
            }
        }
        __syncwarp();
        n = sm.total;
    }
    if (n > kShortTopBuf) n = warp_top_exact(s, sm, k, reach_bits, order_bits(st.m));
    write_ranked(sm.buf, n, k, values, ids);
}

}  // namespace ears
