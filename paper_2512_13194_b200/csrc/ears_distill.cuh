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
// 1e-4 and less, of which the difference would keep no digits): the sweep skips the listed entries.  One
// byte of shared memory per thread and round says which of its eight vectors hold any.
#pragma once
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

struct DistillSmem {
    float4 xs[kLMaxCluster * kLWarps];
    int vec[kMaxTop];            // vector that holds the listed entry, -1: absent
    int col[kMaxTop];
    float x[kMaxTop];            // draft logit of the listed entry
    float t[kMaxTop];            // teacher logit
    float entry[kMaxTop];        // gradient of the listed entry
    float factor;
    int zero;
    int seen;                    // bit 0: an entry is present, bit 1: something is wrong
};

// Warp 0 of every CTA: loss, the factor of the entries outside the list, the listed entries' gradients.
// Lane i has the entries i, i + 32, ..; sums over lanes in one fixed order, identical in every CTA.
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

template <int MODE>
__device__ void distill_scalars(const DistillParams& p, DistillSmem& sm, long long row, int rank, double T, bool ok, Part tail) {
    constexpr int PER = kMaxTop / 32;
    const int lane = threadIdx.x & 31;
    const double invT = 1.0 / T;
    bool on[PER];
    double lp[PER], lq[PER], pr[PER], qr[PER];
    double xm = -INFINITY, tm = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int j = lane + 32 * i;
        on[i] = j < p.k && sm.vec[j] >= 0;
        lq[i] = on[i] ? (double)sm.x[j] : -INFINITY;
        lp[i] = on[i] ? (double)sm.t[j] : -INFINITY;
        xm = fmax(xm, lq[i]);
        tm = fmax(tm, lp[i]);
    }
    const bool has_tail = tail.m > -INFINITY;
    const double M = fmax(warp_max(xm), (double)tail.m);
    tm = warp_max(tm);
    // draft: Z relative to M
    double zs = 0.0, ps = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        lq[i] = (lq[i] - M) * invT;
        qr[i] = on[i] ? exp(lq[i]) : 0.0;
        zs += qr[i];
    }
    const double zt = has_tail ? exp(((double)tail.m - M) * invT) * (double)tail.s : 0.0;
    const double Z = warp_sum(zs) + zt, lnZ = log(Z);
    const double rho = zt / Z;
    const double ln_rho = has_tail ? ((double)tail.m - M) * invT + log((double)tail.s) - lnZ : -INFINITY;
    // teacher
    double L;
    if (p.lse) {
        L = (double)__ldg(p.lse + row);
    } else {
        double ts = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) ts += on[i] ? exp((lp[i] - tm) * invT) : 0.0;
        L = tm * invT + log(warp_sum(ts));
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        lq[i] -= lnZ;
        qr[i] /= Z;
        lp[i] = lp[i] * invT - L;
        pr[i] = on[i] ? exp(lp[i]) : 0.0;
        ps += pr[i];
    }
    ps = warp_sum(ps);
    double rt = 0.0;
    if (p.lse) {
        rt = 1.0 - ps;
        if (rt < kTailFloor) rt = rho > 0.0 ? kTailFloor : 0.0;
    }
    const double ln_rt = log(rt);
    // loss; q (g - cbar) of every outcome
    const double a = p.mix;
    double part = 0.0, loss, gt, gs[PER];
    if (p.kind == kForwardKl) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            part += pr[i] > 0.0 ? pr[i] * (lp[i] - lq[i]) : 0.0;
            gs[i] = qr[i] * (ps + rt) - pr[i];
        }
        loss = warp_sum(part) + (rt > 0.0 ? rt * (ln_rt - ln_rho) : 0.0);
        gt = rho * (ps + rt) - rt;
    } else if (p.kind == kReverseKl) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            gs[i] = qr[i] > 0.0 ? lq[i] - lp[i] : 0.0;
            part += qr[i] * gs[i];
        }
        gt = rho > 0.0 ? ln_rho - ln_rt : 0.0;
        loss = warp_sum(part) + rho * gt;
#pragma unroll
        for (int i = 0; i < PER; ++i) gs[i] = qr[i] * (gs[i] - loss);
        gt = rho * (gt - loss);
    } else {
        double cq = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const double lm = log(a * pr[i] + (1.0 - a) * qr[i]);
            gs[i] = qr[i] > 0.0 ? lq[i] - lm : 0.0;
            part += pr[i] > 0.0 ? pr[i] * (lp[i] - lm) : 0.0;
            cq += qr[i] * gs[i];
        }
        const double lmt = log(a * rt + (1.0 - a) * rho);
        const double kt = rho > 0.0 ? ln_rho - lmt : 0.0;
        cq = (1.0 - a) * (warp_sum(cq) + rho * kt);
        loss = a * (warp_sum(part) + (rt > 0.0 ? rt * (ln_rt - lmt) : 0.0)) + cq;
#pragma unroll
        for (int i = 0; i < PER; ++i) gs[i] = qr[i] * ((1.0 - a) * gs[i] - cq);
        gt = rho * ((1.0 - a) * kt - cq);
    }
    ok = ok && M > -INFINITY && M < INFINITY && isfinite(L) && loss == loss;
    if (MODE != kForward) {
        const double w = (p.weight ? (double)__ldg(p.weight + row) : 1.0) * invT;
        bool finite = true;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = lane + 32 * i;
            const float e = (float)(w * gs[i]);
            if (on[i]) {
                sm.entry[j] = e;
                finite = finite && isfinite(gs[i]);
            }
        }
        // relative to the tail's own maximum: nothing underflows before the product
        const double f = has_tail ? gt / (double)tail.s : 0.0;
        finite = __all_sync(0xffffffffu, finite) && isfinite(f);
        ok = ok && finite;
        if (lane == 0) {
            sm.factor = (float)(w * f);
            sm.zero = (!ok || w == 0.0) ? 1 : 0;
        }
    }
    if (lane == 0 && rank == 0) {
        const float nan = __int_as_float(0x7fc00000);
        if (MODE != kBackward) p.out_loss[row] = ok ? (float)loss : nan;
        if (MODE == kForward && p.stats) p.stats[row] = make_float4(tail.m, ok ? tail.s : nan, 0.f, 0.f);
        if (!ok && p.status) atomicOr(p.status, kDevInvalidInput);
    }
}

template <typename E, int MODE>
__global__ void __launch_bounds__(kLThreads) ears_distill_kernel(const DistillParams p) {
    constexpr int N = Words<E>::N;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ DistillSmem sm;
    uint32_t* flags = reinterpret_cast<uint32_t*>(smem_raw);   // byte (round * kLThreads + thread): bit j = vector j of the round
    const int tid = threadIdx.x, k = p.k;
    const RowSetup r = row_setup(p.rows);
    const E* row = row_ptr<E>(p.rows, r.row);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, r.rank);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.rows, p.gsb, p.gsr, r.row) - s.lead;
    // the list
    int id = -1;
    float tv = -INFINITY;
    if (tid < k) {
        id = __ldg(p.ids + r.row * k + tid);
        tv = __ldg(p.values + r.row * k + tid);
    }
    bool wrong = id < -1 || id >= p.rows.V || (id >= 0 && !(tv < INFINITY));   // NaN and +inf
    const bool present = !wrong && id >= 0 && tv > -INFINITY;
    if (tid == 0) sm.seen = 0;
    if (MODE != kBackward) {
        const int rounds = (s.n + kLRound - 1) / kLRound;
        for (int i = tid; i < rounds * (kLThreads / 4); i += kLThreads) flags[i] = 0;
    }
    if (tid < kMaxTop) {
        float x = -INFINITY;
        if (present) {
            float xx[N];
            Words<E>::unpack(make_uint4(raw_bits(row + id), 0, 0, 0), xx);
            x = xx[0];
        }
        sm.vec[tid] = present ? (s.lead + id) / N : -1;
        sm.col[tid] = present ? id : -1;
        sm.x[tid] = x;
        sm.t[tid] = tv;
    }
    __syncthreads();
    if (tid < k && present) {
        for (int j = 0; j < tid; ++j) wrong = wrong || sm.col[j] == id;   // an id listed twice
        const int i = sm.vec[tid] - s.v0;
        if (MODE != kBackward && i >= 0 && i < s.n) {
            const int byte = (i / kLRound) * kLThreads + i % kLThreads, bit = (i / kLThreads) % kLUnroll;
            atomicOr(&flags[byte >> 2], 1u << ((byte & 3) * 8 + bit));
        }
    }
    if (tid < kMaxTop) {
        const unsigned any = __ballot_sync(0xffffffffu, present), bad = __ballot_sync(0xffffffffu, wrong);
        if ((tid & 31) == 0 && (any | bad)) atomicOr(&sm.seen, (any ? 1 : 0) | (bad ? 2 : 0));
    }
    __syncthreads();
    if (sm.seen != 1) {   // nothing listed, or a list that cannot be used: the same in every CTA of the cluster
        const bool bad = (sm.seen & 2) != 0;
        if (tid == 0 && r.rank == 0) {
            if (MODE != kBackward) p.out_loss[r.row] = bad ? __int_as_float(0x7fc00000) : 0.f;
            if (MODE == kForward && p.stats) p.stats[r.row] = make_float4(0.f, __int_as_float(0x7fc00000), 0.f, 0.f);
            if (bad && p.status) atomicOr(p.status, kDevInvalidInput);
        }
        if (MODE != kForward) dense_pass<E, false>(s, grad, true, 0.f, 0.f, 0.f, 0.f);
        return;
    }
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
        const unsigned char* flag_bytes = reinterpret_cast<const unsigned char*>(flags);
        for (int i0 = tid, round = 0; i0 < s.n; i0 += kLRound, ++round) {
            uint4 w[kLUnroll];
            load_round(s, i0, w);
            const unsigned f = flag_bytes[round * kLThreads + tid];
            if (f) {
#pragma unroll
                for (int j = 0; j < kLUnroll; ++j) {
                    if (f >> j & 1u) {
                        const int v = s.v0 + i0 + j * kLThreads;
                        for (int q = 0; q < k; ++q)
                            if (sm.vec[q] == v) put_entry(w[j], (s.lead + sm.col[q]) % N, minus_inf_bits<E>(), E{});
                    }
                }
            }
            stat_fold<E, kLUnroll, false>(w, r.c, a);
        }
        st = exchange_parts<false>(a, sm.xs, p.rows.C, r.rank, r.c);
    }
    // no entry outside the list is finite: the tail is empty
    const bool empty = st.m == -INFINITY && st.s == 0.f;
    const bool ok = r.T_ok && (empty || rowstat_ok(st.m, st.s));
    if (tid < 32) distill_scalars<MODE>(p, sm, r.row, r.rank, r.T, ok, st);
    if (MODE == kForward) return;
    __syncthreads();
    const bool zero = sm.zero != 0;
    dense_pass<E, false>(s, grad, zero, empty ? 0.f : st.m, r.c, sm.factor, 0.f);
    if (zero) return;
    __syncthreads();   // the dense values of the listed entries have been written
    if (tid < k && present && in_slice(s, id)) store_entry(grad + s.lead + id, sm.entry[tid]);
}

}  // namespace ears
