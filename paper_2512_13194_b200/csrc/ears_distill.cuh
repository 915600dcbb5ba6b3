// Distillation of a draft row from a teacher's top logits.
//
// The teacher's row is known by k entries (id, logit) and, optionally, by its log normaliser L_t at the
// temperature T.  With p_j = exp(t_j / T - L_t) for the listed entries, r = 1 - sum p_j for everything
// else, and the draft's q_j = softmax(l / T) at the same ids, rho = 1 - sum q_j, the loss is a divergence
// between the two distributions over k + 1 outcomes:
//   forward KL    sum p ln(p / q)                      gradient by q_u:  -p_u / q_u
//   reverse KL    sum q ln(q / p)                                        ln(q_u / p_u)  (+ 1)
//   JSD, mix a    a sum p ln(p / m) + (1 - a) sum q ln(q / m), m = a p + (1 - a) q:   (1 - a) ln(q_u / m_u)
// Without L_t the listed entries are renormalised and r = 0.  With g_u the gradient by outcome u's
// probability and cbar = sum q g, a logit of outcome u has the gradient q_v (g_u - cbar) / T: all entries
// outside the list share one factor, so a gradient row is factor * 2^t plus k entries of their own.
//
// rho is the sum over the entries outside the list, never 1 - sum q (a trained draft leaves a tail of
// 1e-4 and less, of which the difference would keep no digits): the sweep skips the listed entries, found by one bit
// per logit in shared memory, looked at a word per thread and round.
//
// Bound by HBM like ears_token.cuh; what comes on top is the list (two dependent loads before the sweep may begin, hidden by the
// ring's first loads) and the scalars, which a warp of their own prepares during the sweep.  2044 rows of 128256 bf16
// with 64 listed entries: 354 us with a linear search for the listed entries, 203 with a slot table, 194 with the bits and with the
// forward divergence's gradient published before its logarithms (0.78 of the measured copy rate).
#pragma once
#include "ears_ring.cuh"
#include "ears_rows.cuh"
#include "ears_token.cuh"   // LossMode

namespace ears {

constexpr int kMaxTop = 128;                 // EARS_MAX_TOP
enum DistillKind : int { kForwardKl = 0, kReverseKl = 1, kJsd = 2 };
constexpr double kTailFloor = 9.5367431640625e-07;   // 2^-20: a smaller tail is not resolved by a 32-bit L_t

struct DistillParams {
    RowSpan rows;
    int k, kind;
    double mix;
    const float* values;         // [rows, k]
    const int32_t* ids;          // [rows, k]; -1: absent
    const float* lse;            // [rows] or NULL
    const float* weight;         // [rows] gradient of the summed loss by this row's loss; NULL: 1
    float* out_loss;
    float4* stats;               // (m, s of the entries outside the list, 0, 0): forward writes, backward reads
    void* grad;
    long long gsb, gsr;
    int32_t* status;
};

struct ListSmem {
    alignas(16) int col[kMaxTop];   // listed ids, -1: absent
    float t[kMaxTop];            // teacher logit
    float entry[kMaxTop];        // gradient of the listed entry
    float factor;
    int zero;
    int seen;                    // bit 0: an entry is present, bit 1: something is wrong
    uint32_t edge[2];            // listed entries of the vectors just before and just behind those with bits
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, off));
    return v;
}

// One warp of every CTA works out the row's scalars in 64 bits: lane i has the entries i, i + 32, .., sums over
// lanes in one fixed order, identical in every CTA.  The teacher's part first: it needs nothing of the draft.
constexpr int kTopPer = kMaxTop / 32;
struct TeacherPart { double lp[kTopPer], pr[kTopPer], ps, L; };

__device__ __forceinline__ bool listed(const DistillParams& p, const ListSmem& sm, int i) {
    const int j = (threadIdx.x & 31) + 32 * i;
    return j < p.k && sm.col[j] >= 0;
}

__device__ __forceinline__ TeacherPart teacher_part(const DistillParams& p, const ListSmem& sm, long long row, double invT) {
    const int lane = threadIdx.x & 31;
    TeacherPart t;
    if (p.lse) {
        t.L = (double)__ldg(p.lse + row);
    } else {
        double tm = -INFINITY, ts = 0.0;
#pragma unroll
        for (int i = 0; i < kTopPer; ++i)
            if (listed(p, sm, i)) tm = fmax(tm, (double)sm.t[lane + 32 * i]);
        tm = warp_max(tm);
#pragma unroll
        for (int i = 0; i < kTopPer; ++i)
            if (listed(p, sm, i)) ts += exp(((double)sm.t[lane + 32 * i] - tm) * invT);
        t.L = tm * invT + log(warp_sum(ts));
    }
    t.ps = 0.0;
#pragma unroll
    for (int i = 0; i < kTopPer; ++i) {
        t.lp[i] = t.pr[i] = 0.0;
        if (listed(p, sm, i)) {
            t.lp[i] = (double)sm.t[lane + 32 * i] * invT - t.L;
            t.pr[i] = exp(t.lp[i]);
            t.ps += t.pr[i];
        }
    }
    t.ps = warp_sum(t.ps);
    return t;
}

// The draft's logits of the listed entries: asked for when the list stands, used later.
struct DraftLogits { float x[kTopPer]; };

template <typename E>
__device__ __forceinline__ DraftLogits draft_logits(const DistillParams& p, const ListSmem& sm, const E* row) {
    const int lane = threadIdx.x & 31;
    DraftLogits d;
#pragma unroll
    for (int i = 0; i < kTopPer; ++i) {
        d.x[i] = -INFINITY;
        if (listed(p, sm, i)) {
            float x[Words<E>::N];
            Words<E>::unpack(make_uint4(raw_bits(row + sm.col[lane + 32 * i]), 0, 0, 0), x);
            d.x[i] = x[0];
        }
    }
    return d;
}

// The draft's listed entries, relative to their own maximum.
struct DraftPart { double xm, lq[kTopPer], e[kTopPer], sum; };

__device__ __forceinline__ DraftPart draft_part(const DistillParams& p, const ListSmem& sm, const DraftLogits& dl, double invT) {
    DraftPart d;
    d.xm = -INFINITY;
#pragma unroll
    for (int i = 0; i < kTopPer; ++i)
        if (listed(p, sm, i)) d.xm = fmax(d.xm, (double)dl.x[i]);
    d.xm = warp_max(d.xm);
    const double ref = d.xm > -INFINITY ? d.xm : 0.0;   // every listed entry masked: e = 0
    d.sum = 0.0;
#pragma unroll
    for (int i = 0; i < kTopPer; ++i) {
        d.lq[i] = d.e[i] = 0.0;
        if (listed(p, sm, i)) {
            d.lq[i] = ((double)dl.x[i] - ref) * invT;
            d.e[i] = exp(d.lq[i]);
            d.sum += d.e[i];
        }
    }
    d.sum = warp_sum(d.sum);
    return d;
}

// published() is called when the gradient's scalars stand in sm.
template <int MODE, class F>
__device__ __forceinline__ void distill_scalars(const DistillParams& p, ListSmem& sm, long long row, int rank, double invT, bool ok,
                                                const TeacherPart& te, const DraftPart& dr, float weight, Part tail, F published) {
    const int lane = threadIdx.x & 31;
    double lq[kTopPer], qr[kTopPer], gs[kTopPer];
    const bool has_tail = tail.m > -INFINITY;
    const double M = fmax(dr.xm, (double)tail.m);
    // Z relative to M
    const double td = dr.xm > -INFINITY ? (dr.xm - M) * invT : 0.0, fd = exp(td);
    const double tt = has_tail ? ((double)tail.m - M) * invT : 0.0;
    const double mass = row_mass(tail.s), zt = has_tail ? exp(tt) * mass : 0.0;
    const double Z = dr.sum * fd + zt, invZ = 1.0 / Z;
    const double rho = zt * invZ;
#pragma unroll
    for (int i = 0; i < kTopPer; ++i) {
        qr[i] = dr.e[i] * (fd * invZ);
        gs[i] = 0.0;
    }
    double rt = 0.0;
    if (p.lse) {
        rt = 1.0 - te.ps;
        if (rt < kTailFloor) rt = rho > 0.0 ? kTailFloor : 0.0;
    }
    ok = ok && M > -INFINITY && M < INFINITY && isfinite(te.L);
    const double w = (double)weight * invT;
    double gt = 0.0;
    // sm gets q (g - cbar) of the listed entries and the factor of the others
    const auto publish = [&] {
        if (MODE == kForward) return;
        bool finite = true;
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) {
            if (listed(p, sm, i)) {
                sm.entry[lane + 32 * i] = (float)(w * gs[i]);
                finite = finite && isfinite(gs[i]);
            }
        }
        // relative to the tail's own maximum: nothing underflows before the product
        const double f = has_tail ? gt / mass : 0.0;
        finite = __all_sync(0xffffffffu, finite) && isfinite(f);
        ok = ok && finite;
        if (lane == 0) {
            sm.factor = (float)(w * f);
            sm.zero = (!ok || w == 0.0) ? 1 : 0;
        }
        __syncwarp();
        published();
    };
    if (p.kind == kForwardKl) {   // needs no logarithm for the gradient
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) gs[i] = qr[i] * (te.ps + rt) - te.pr[i];
        gt = rho * (te.ps + rt) - rt;
        publish();
        if (MODE == kBackward) {
            if (lane == 0 && rank == 0 && !ok && p.status) atomicOr(p.status, kDevInvalidInput);
            return;
        }
    }
    const double lnZ = log(Z);
    const double ln_rho = has_tail ? tt + log(mass) - lnZ : -INFINITY;
    const double ln_rt = log(rt);
#pragma unroll
    for (int i = 0; i < kTopPer; ++i) lq[i] = dr.lq[i] + td - lnZ;
    // loss; q (g - cbar) of every outcome.  Entries that are not listed have p = q = 0 and stay out of every sum.
    const double a = p.mix;
    double part = 0.0, loss;
    if (p.kind == kForwardKl) {
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) part += te.pr[i] > 0.0 ? te.pr[i] * (te.lp[i] - lq[i]) : 0.0;
        loss = warp_sum(part) + (rt > 0.0 ? rt * (ln_rt - ln_rho) : 0.0);
    } else if (p.kind == kReverseKl) {
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) {
            gs[i] = qr[i] > 0.0 ? lq[i] - te.lp[i] : 0.0;
            part += qr[i] * gs[i];
        }
        gt = rho > 0.0 ? ln_rho - ln_rt : 0.0;
        loss = warp_sum(part) + rho * gt;
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) gs[i] = qr[i] * (gs[i] - loss);
        gt = rho * (gt - loss);
    } else {
        double cq = 0.0;
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) {
            if (listed(p, sm, i)) {
                const double lm = log(a * te.pr[i] + (1.0 - a) * qr[i]);
                gs[i] = qr[i] > 0.0 ? lq[i] - lm : 0.0;
                part += te.pr[i] > 0.0 ? te.pr[i] * (te.lp[i] - lm) : 0.0;
                cq += qr[i] * gs[i];
            }
        }
        const double lmt = log(a * rt + (1.0 - a) * rho);
        const double kt = rho > 0.0 ? ln_rho - lmt : 0.0;
        cq = (1.0 - a) * (warp_sum(cq) + rho * kt);
        loss = a * (warp_sum(part) + (rt > 0.0 ? rt * (ln_rt - lmt) : 0.0)) + cq;
#pragma unroll
        for (int i = 0; i < kTopPer; ++i) gs[i] = qr[i] * ((1.0 - a) * gs[i] - cq);
        gt = rho * ((1.0 - a) * kt - cq);
    }
    ok = ok && loss == loss;
    if (p.kind != kForwardKl) publish();
    if (lane == 0 && rank == 0) {
        const float nan = __int_as_float(0x7fc00000);
        if (MODE != kBackward) p.out_loss[row] = ok ? (float)loss : nan;
        if (MODE == kForward && p.stats) p.stats[row] = make_float4(tail.m, ok ? tail.s : nan, 0.f, 0.f);
        if (!ok && p.status) atomicOr(p.status, kDevInvalidInput);
    }
}

// The threads that share a row: a warp, or all threads of the CTA.
template <int THREADS>
__device__ __forceinline__ void row_sync() {
    if (THREADS == 32) __syncwarp();
    else __syncthreads();
}

// Of every vector the bits of its listed entries, one byte: byte q of word (i / (PER SWEEP)) SWEEP + i % SWEEP, q = i / SWEEP % PER,
// for vector base + i -- what the thread that folds PER vectors a round, one of SWEEP, looks at in one load.
template <int PER> struct ListWord;
template <> struct ListWord<4> { typedef uint32_t type; };
template <> struct ListWord<8> { typedef uint2 type; };

// The row's list, by the THREADS threads that share the row (tid among them): into sm, and the bits of the vectors
// among [base, base + count) into bits.  -> sm.seen.
template <typename E, int PER, int SWEEP, int THREADS>
__device__ __forceinline__ int distill_list(const DistillParams& p, ListSmem& sm, uint32_t* bits, int tid, long long row_index, int lead,
                                            int base, int count) {
    constexpr int N = Words<E>::N;
    constexpr int HAND = THREADS < kMaxTop ? kMaxTop / THREADS : 1;   // entries per thread
    const int k = p.k;
    int id[HAND];
    float tv[HAND];
#pragma unroll
    for (int h = 0; h < HAND; ++h) {
        const int j = tid + h * THREADS;
        id[h] = -1;
        tv[h] = -INFINITY;
        if (j < k) {
            id[h] = __ldg(p.ids + row_index * k + j);
            tv[h] = __ldg(p.values + row_index * k + j);
        }
    }
    if (tid == 0) sm.seen = 0, sm.edge[0] = sm.edge[1] = 0;
    const int words = (count + PER * SWEEP - 1) / (PER * SWEEP) * (SWEEP * PER / 4);
    for (int i = tid; i < words / 4; i += THREADS) reinterpret_cast<uint4*>(bits)[i] = make_uint4(0, 0, 0, 0);
    bool wrong = false, present[HAND];
#pragma unroll
    for (int h = 0; h < HAND; ++h) {
        const int j = tid + h * THREADS;
        const bool off = id[h] < -1 || id[h] >= p.rows.V || (id[h] >= 0 && !(tv[h] < INFINITY));   // NaN and +inf
        wrong = wrong || off;
        present[h] = !off && id[h] >= 0 && tv[h] > -INFINITY;
        if (j < kMaxTop) {
            sm.col[j] = present[h] ? id[h] : -1;
            sm.t[j] = tv[h];
        }
    }
    row_sync<THREADS>();
    if (tid < kMaxTop) {   // whole warps
        bool any = false;
#pragma unroll
        for (int h = 0; h < HAND; ++h) {
            if (!present[h]) continue;
            any = true;
            // an id listed twice
            const int4* c4 = reinterpret_cast<const int4*>(sm.col);
            int same = 0;
#pragma unroll 4
            for (int j = 0; j < (k + 3) / 4; ++j) {
                const int4 c = c4[j];
                same += (c.x == id[h]) + (c.y == id[h]) + (c.z == id[h]) + (c.w == id[h]);
            }
            wrong = wrong || same > 1;
            const int e = lead + id[h], i = e / N - base;
            if (i >= 0 && i < count) {
                const int byte = ((i / (PER * SWEEP)) * SWEEP + i % SWEEP) * PER + i / SWEEP % PER;
                atomicOr(&bits[byte >> 2], 1u << ((byte & 3) * 8 + e % N));
            } else if (i == -1 || i == count) {
                atomicOr(&sm.edge[i < 0 ? 0 : 1], 1u << e % N);
            }
        }
        const unsigned some = __ballot_sync(0xffffffffu, any), bad = __ballot_sync(0xffffffffu, wrong);
        if ((tid & 31) == 0 && (some | bad)) atomicOr(&sm.seen, (some ? 1 : 0) | (bad ? 2 : 0));
    }
    row_sync<THREADS>();
    return sm.seen;
}

// The entries of w whose bits are set go to -inf.
__device__ __forceinline__ void mask_half(uint32_t& h, uint32_t two, uint32_t ninf) {
    if (two & 1u) h = (h & 0xffff0000u) | ninf;
    if (two & 2u) h = (h & 0xffffu) | (ninf << 16);
}
template <typename E>
__device__ __forceinline__ void mask_entries(uint4& w, uint32_t b) {
    const uint32_t ninf = minus_inf_bits<E>();
    if constexpr (sizeof(E) == 4) {
        if (b & 1u) w.x = ninf;
        if (b & 2u) w.y = ninf;
        if (b & 4u) w.z = ninf;
        if (b & 8u) w.w = ninf;
    } else {
        mask_half(w.x, b, ninf);
        mask_half(w.y, b >> 2, ninf);
        mask_half(w.z, b >> 4, ninf);
        mask_half(w.w, b >> 6, ninf);
    }
}
template <typename E>
__device__ __forceinline__ void mask_listed(uint4 (&w)[4], uint32_t b) {
    if (b == 0) return;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (b >> 8 * q & 0xffu) mask_entries<E>(w[q], b >> 8 * q);
}
template <typename E>
__device__ __forceinline__ void mask_listed(uint4 (&w)[8], uint2 b) {
    if ((b.x | b.y) == 0) return;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const uint32_t v = (q < 4 ? b.x : b.y) >> 8 * (q & 3) & 0xffu;
        if (v) mask_entries<E>(w[q], v);
    }
}
// Nothing listed, or a list that cannot be used.
template <int MODE>
__device__ __forceinline__ void distill_unused(const DistillParams& p, long long row, bool bad) {
    if (MODE != kBackward) p.out_loss[row] = bad ? __int_as_float(0x7fc00000) : 0.f;
    if (MODE == kForward && p.stats) p.stats[row] = make_float4(0.f, __int_as_float(0x7fc00000), 0.f, 0.f);
    if (bad && p.status) atomicOr(p.status, kDevInvalidInput);
}

// The tail's statistics are usable, or there is no tail (no entry outside the list is finite).
__device__ __forceinline__ bool tail_empty(Part st) { return st.m == -INFINITY && st.s == 0.f; }

// Forward and backward calls: one sweep, straight from memory.
template <typename E, int MODE>
__global__ void __launch_bounds__(kLThreads, 4) ears_distill_kernel(const DistillParams p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ ListSmem sm;
    __shared__ float4 xs[kLMaxCluster * kLWarps];
    uint32_t* flags = reinterpret_cast<uint32_t*>(smem_raw);
    const int tid = threadIdx.x, k = p.k;
    const RowSetup r = row_setup(p.rows);
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, r.rank);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const int seen = distill_list<E, kLUnroll, kLThreads, kLThreads>(p, sm, flags, tid, r.row, s.lead, s.v0, MODE == kBackward ? 0 : s.n);
    if (seen != 1) {   // the same in every CTA of the cluster
        if (tid == 0 && r.rank == 0) distill_unused<MODE>(p, r.row, (seen & 2) != 0);
        if (MODE != kForward) dense_pass<E, false>(s, grad, true, 0.f, 0.f, 0.f, 0.f);
        return;
    }
    DraftLogits dl{};
    if (tid < 32) dl = draft_logits(p, sm, row);
    Part st;
    if (MODE == kBackward) {
        const float4 q = p.stats[r.row];
        st = Part{q.x, q.y, 0.f};
        if (p.rows.C > 1) {
            // the gradient may overwrite the logits: no slice is written before every CTA has its list's logits
            cluster_wait_peers();
            cluster_sync_all();
        }
    } else {
        Stat<false> a;
        stat_open(a);
        const uint64_t pol = l2_policy_evict_first();
        const uint2* bits = reinterpret_cast<const uint2*>(flags) + tid;
        sweep_rounds<E, false>(s, pol, [&](uint4 (&w)[kLUnroll], int round) {
            mask_listed<E>(w, bits[round * kLThreads]);
            stat_fold<E, kLUnroll, false>(w, r.c, a);
        });
        st = exchange_parts<false>(a, xs, p.rows.C, r.rank, r.c);
    }
    const bool empty = tail_empty(st);
    if (tid < 32) {
        const double invT = 1.0 / r.T;
        const float weight = MODE != kForward && p.weight ? __ldg(p.weight + r.row) : 1.f;
        distill_scalars<MODE>(p, sm, r.row, r.rank, invT, r.T_ok && (empty || rowstat_ok(st.m, st.s)),
                              teacher_part(p, sm, r.row, invT), draft_part(p, sm, dl, invT), weight, st, [] {});
    }
    if (MODE == kForward) return;
    __syncthreads();
    const bool zero = sm.zero != 0;
    dense_pass<E, false>(s, grad, zero, empty ? 0.f : st.m, r.c.near, sm.factor, 0.f);
    if (zero) return;
    __syncthreads();   // the dense values of the listed entries have been written
    if (tid < k && sm.col[tid] >= 0 && in_slice(s, sm.col[tid])) store_entry(grad + s.lead + sm.col[tid], sm.entry[tid]);
}

// Loss and gradient in one call: the slice through the ring of ears_ring.cuh, with one more warp for the
// scalars, which has the teacher's part done while the others sweep.
constexpr int kDistillThreads = kRingThreads + 32;

template <typename E>
__global__ void __launch_bounds__(kDistillThreads, 2) ears_distill_step_kernel(const DistillParams p, int stages) {
    extern __shared__ __align__(128) unsigned char ring_buf[];
    __shared__ ListSmem sm;
    __shared__ float4 xs[kLMaxCluster * kRingWarps];
    __shared__ RingBars bars;
    uint32_t* flags = reinterpret_cast<uint32_t*>(ring_buf + (size_t)stages * kRingChunk);
    const int tid = threadIdx.x, k = p.k, C = p.rows.C;
    const RowSetup r = row_setup(p.rows);
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, r.rank);
    E* grad = grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const Ring<E> ring = make_ring(s, ring_buf, &bars, stages);
    const uint64_t keep = l2_policy_evict_last(), drop = l2_policy_evict_first();
    int issued = 0;
    if (tid >= kRingConsumers && tid < kRingThreads) {
        // loads begin as soon as the list is known not to be empty
        bool any = false;
        for (int j = tid - kRingConsumers; j < k; j += 32)
            any = any || (__ldg(p.ids + r.row * k + j) >= 0 && __ldg(p.values + r.row * k + j) > -INFINITY);
        any = __any_sync(0xffffffffu, any);
        if (tid == kRingConsumers) {
            ring_init(&bars, stages);
            if (any) issued = ring_load(ring, 0, ring.H, keep, drop);
        }
    }
    const int seen = distill_list<E, kRingPer, kRingConsumers, kDistillThreads>(p, sm, flags, tid, r.row, s.lead, ring.v0, ring.vecs);
    if (seen != 1) {   // the same in every CTA of the cluster
        if (tid == 0 && r.rank == 0) distill_unused<kStep>(p, r.row, (seen & 2) != 0);
        if (tid < kLThreads) dense_pass<E, false>(s, grad, true, 0.f, 0.f, 0.f, 0.f);
        if (tid == kRingConsumers) ring_drain(ring, issued);
        return;
    }
    if (tid >= kRingThreads) {   // scalars
        const double invT = 1.0 / r.T;
        const float weight = p.weight ? __ldg(p.weight + r.row) : 1.f;
        const DraftLogits dl = draft_logits(p, sm, row);
        const TeacherPart te = teacher_part(p, sm, r.row, invT);
        const DraftPart dr = draft_part(p, sm, dl, invT);
        exchange_join(C);
        const Part st = merge_parts<false>(xs, C * kRingWarps, r.c);
        distill_scalars<kStep>(p, sm, r.row, r.rank, invT, r.T_ok && (tail_empty(st) || rowstat_ok(st.m, st.s)), te, dr, weight, st,
                               [] { asm volatile("bar.arrive 1, %0;" ::"n"(kRingConsumers + 32) : "memory"); });
        return;
    }
    if (tid >= kRingConsumers) {
        ring_loader_warp(ring, issued, C, keep, drop);
        return;
    }
    Stat<false> a;
    stat_open(a);
    const auto* bits = reinterpret_cast<const typename ListWord<kRingPer>::type*>(flags) + tid;
    const bool swept = ring_stats(ring, [&](uint4 (&w)[kRingPer], int chunk) {
        mask_listed<E>(w, bits[chunk * kRingConsumers]);
        stat_fold<E, kRingPer, false>(w, r.c, a);
    });
    if (!swept) {
        a.s[0] = pack2(__int_as_float(0x7fc00000), 0.f);   // the row counts as unusable in every CTA
        if (p.status) atomicOr(p.status, kDevTimeout);
    }
    const int v = edge_vector(ring, s);
    if (v >= 0) {
        uint4 w[1] = {load_partial(s.base, v, s.lead, s.end)};
        mask_entries<E>(w[0], sm.edge[v < ring.v0 ? 0 : 1]);
        stat_fold<E, 1, false>(w, r.c, a);
    }
    const Part st = exchange_parts<false, kRingWarps>(a, xs, C, r.rank, r.c);
    asm volatile("bar.sync 1, %0;" ::"n"(kRingConsumers + 32) : "memory");   // the scalars
    const bool zero = sm.zero != 0;
    ring_gradient<E, false>(ring, s, grad, zero, tail_empty(st) ? 0.f : st.m, r.c.near, sm.factor, 0.f, drop, p.status);
    if (zero) return;
    asm volatile("bar.sync 2, %0;" ::"n"(kRingConsumers) : "memory");   // the dense values of the listed entries have been written
    if (tid < k && sm.col[tid] >= 0 && in_slice(s, sm.col[tid])) store_entry(grad + s.lead + sm.col[tid], sm.entry[tid]);
}

}  // namespace ears
