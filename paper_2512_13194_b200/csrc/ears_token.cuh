// Log probabilities of one token per row, and the clipped policy loss built on them.
//
// With z = l / T, L = ln sum exp z, q = exp(z - L) and the row's token x:
//   log probability      logp = z_x - L
//   entropy              H = -sum q ln q
//   gradients            d logp / d l_v = (1[v = x] - q_v) / T,   d H / d l_v = -q_v (ln q_v + H) / T
// Policy loss of a token sampled with log probability `old`, advantage A, reference `ref`:
//   rho = exp(logp - old);  pg = -min(rho A, clip(rho, 1 - lo, 1 + hi) A)
//   kl  = exp(ref - logp) - (ref - logp) - 1        (never negative, unbiased under the policy)
//   loss = pg + kl_coef kl - entropy_coef H
// so that every gradient row is q_v (a + b ln q_v) plus one entry at x: the same dense pass serves
// the log probabilities' upstream gradients (g, h) and the policy loss (g = w d loss / d logp,
// h = -w entropy_coef).
//
// Bound by HBM: a forward call reads each logit once, a gradient call reads and writes once, a step (loss and gradient
// together) reads once and writes once through the ring of ears_ring.cuh.  Forward and backward calls stream straight from
// memory, eight 16-byte loads in flight per thread and four CTAs per SM: scoring 2048 rows of 256000 fp32 with the entropy
// takes 305 to 340 us depending on the card (6.2 to 6.9 TB/s), 2048 rows of 128256 bf16 84 us (0.95 of the copy rate).
// The scalars are taken in 64 bits by one thread (a logarithm 271 clocks, an exponential 158, a division 80), the
// row's own inputs having been asked for before the sweep.
#pragma once
#include "ears_ring.cuh"
#include "ears_rows.cuh"

namespace ears {

enum LossMode : int { kForward = 0, kBackward = 1, kStep = 2 };

struct TokenParams {
    RowSpan rows;
    const int32_t* tokens;       // [rows]; -1: the row is left out
    // token log probabilities: upstream gradients (backward and step)
    const float* d_logp;
    const float* d_entropy;      // or NULL
    // policy loss
    int policy;
    const float* old_logp;
    const float* ref_logp;       // or NULL
    const float* advantage;
    const float* weight;         // gradient of the summed loss by this row's loss; NULL: 1
    double clip_low, clip_high, kl_coef, entropy_coef;
    float* out_loss;
    float* out_logp;
    float* out_kl;               // NULL allowed, as all outputs below
    float* out_entropy;
    float4* stats;               // (M, Z, W, 1 if W was summed): written by a forward call, read by a backward call
    void* grad;
    long long gsb, gsr;
    int32_t* status;
};

// The row's own inputs: asked for at the start, used after the sweep.
struct TokenInputs { float lt, old_logp, ref_logp, advantage, weight, d_logp, d_entropy; };

template <typename E, bool ENT, int MODE>
__device__ __forceinline__ TokenInputs token_inputs(const TokenParams& p, const E* row, long long r, int tok) {
    TokenInputs in;
    float x[Words<E>::N];
    Words<E>::unpack(make_uint4(raw_bits(row + tok), 0, 0, 0), x);
    in.lt = x[0];
    in.old_logp = p.policy ? __ldg(p.old_logp + r) : 0.f;
    in.advantage = p.policy ? __ldg(p.advantage + r) : 0.f;
    in.ref_logp = p.policy && p.ref_logp ? __ldg(p.ref_logp + r) : 0.f;
    in.weight = MODE != kForward && p.weight ? __ldg(p.weight + r) : 1.f;
    in.d_logp = MODE != kForward && !p.policy ? __ldg(p.d_logp + r) : 0.f;
    in.d_entropy = MODE != kForward && ENT && !p.policy && p.d_entropy ? __ldg(p.d_entropy + r) : 0.f;
    return in;
}

// What the row's scalars come to, in 64 bits: one lane of one warp per CTA, identical in all of them.
struct TokenScalars { float A, Bt, entry; int zero; };

template <bool ENT, int MODE>
__device__ __forceinline__ TokenScalars token_scalars(const TokenParams& p, long long row, int rank, double T, bool T_ok, const TokenInputs& in, Part st) {
    const float lt = in.lt;
    const bool ok = T_ok && rowstat_ok(st.m, st.s) && (!ENT || st.w == st.w);
    const double Z = row_mass(st.s), lnZ = log(Z), invT = 1.0 / T;
    double logp = ((double)lt - (double)st.m) * invT - lnZ;
    double H = ENT ? lnZ - kLn2 * ((1.0 + kEx2Short) * (double)st.w) / Z : 0.0;
    double loss = 0.0, kl = 0.0, g = 0.0, h = 0.0;
    bool fine = ok;
    if (p.policy) {
        const double old = in.old_logp, A = in.advantage;
        const double rho = exp(logp - old);
        const double plain = rho * A, clipped = fmin(fmax(rho, 1.0 - p.clip_low), 1.0 + p.clip_high) * A;
        loss = -fmin(plain, clipped);
        g = plain <= clipped ? -plain : 0.0;
        if (p.ref_logp) {
            const double d = (double)in.ref_logp - logp, ed = exp(d);
            kl = d < INFINITY ? ed - d - 1.0 : d;
            if (p.kl_coef != 0.0) {   // an infinite term without weight is reported, no more
                loss += p.kl_coef * kl;
                g += p.kl_coef * (1.0 - ed);
            }
        }
        if (ENT) loss -= p.entropy_coef * H;
        fine = fine && isfinite(old) && isfinite(A) && isfinite(loss) && isfinite(g);
        if (MODE != kForward) {
            const double w = in.weight;
            g *= w;
            h = -w * p.entropy_coef;
        }
    } else if (MODE != kForward) {
        g = in.d_logp;
        h = in.d_entropy;
    }
    TokenScalars r{0.f, 0.f, 0.f, 1};
    if (MODE != kForward) {
        // g (1[v = x] - q) - h q (ln q + H), with ln q = t ln 2 - ln Z and q = 2^t / Z
        const double a = (-g - h * (H - lnZ)) * invT / Z, b = -h * kLn2 * invT / Z;
        const double tx = ((double)lt - (double)st.m) * invT;
        double entry = g * invT;
        if (lt > -INFINITY) entry += exp(tx) * (a + b * tx * kLog2e);
        r = TokenScalars{(float)a, (float)b, (float)entry, 0};
        // a row without weight is left out of the gradient whatever it holds
        if ((g == 0.0 && h == 0.0) || !fine) r.zero = 1;
        else if (p.policy && !(isfinite(r.A) && isfinite(r.Bt) && isfinite(r.entry))) { fine = false; r.zero = 1; }
    }
    if (rank == 0) {
        if (MODE != kBackward) {
            const float nan = __int_as_float(0x7fc00000);
            if (p.out_logp) p.out_logp[row] = fine ? (float)logp : nan;
            if (p.out_loss) p.out_loss[row] = fine ? (float)loss : nan;
            if (p.out_kl) p.out_kl[row] = fine ? (float)kl : nan;
            if (p.out_entropy) p.out_entropy[row] = fine ? (float)H : nan;
            if (MODE == kForward && p.stats) p.stats[row] = make_float4(st.m, fine ? st.s : nan, st.w, ENT ? 1.f : 0.f);
        }
        if (!fine && p.status) atomicOr(p.status, kDevInvalidInput);
    }
    return r;
}

// What a forward call left for the backward call; an entropy gradient needs the sum that only a forward call with
// the entropy leaves.
template <bool ENT>
__device__ __forceinline__ Part token_saved(float4 q) { return Part{q.x, !ENT || q.w == 1.f ? q.y : __int_as_float(0x7fc00000), q.z}; }

// A row that is left out, or whose token is no index: outputs of 0 or NaN.
template <int MODE>
__device__ __forceinline__ void token_unused(const TokenParams& p, long long row, bool bad) {
    const float v = bad ? __int_as_float(0x7fc00000) : 0.f;
    if (MODE != kBackward) {
        if (p.out_logp) p.out_logp[row] = v;
        if (p.out_loss) p.out_loss[row] = v;
        if (p.out_kl) p.out_kl[row] = v;
        if (p.out_entropy) p.out_entropy[row] = v;
        if (MODE == kForward && p.stats) p.stats[row] = make_float4(0.f, __int_as_float(0x7fc00000), 0.f, 0.f);
    }
    if (bad && p.status) atomicOr(p.status, kDevInvalidInput);
}

// Forward and backward calls: one sweep, straight from memory.
template <typename E, bool ENT, int MODE>
__global__ void __launch_bounds__(kLThreads, 4) ears_token_kernel(const TokenParams p) {
    __shared__ float4 xs[kLMaxCluster * kLWarps];
    __shared__ TokenScalars sc;
    const RowSetup r = row_setup(p.rows);
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, r.rank);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const int tok = __ldg(p.tokens + r.row);
    const bool absent = tok == -1, bad = tok < -1 || tok >= p.rows.V;
    if (absent || bad) {   // the same in every CTA of the cluster
        if (threadIdx.x == 0 && r.rank == 0) token_unused<MODE>(p, r.row, bad);
        if (MODE != kForward) dense_pass<E, ENT>(s, grad, true, 0.f, 0.f, 0.f, 0.f);
        return;
    }
    TokenInputs in{};
    if (threadIdx.x == 0) in = token_inputs<E, ENT, MODE>(p, row, r.row, tok);
    Part st;
    if (MODE == kBackward) {
        const float4 q = p.stats[r.row];
        st = token_saved<ENT>(q);
    } else {
        Stat<ENT> a;
        stat_open(a);
        const uint64_t pol = l2_policy_evict_first();
        sweep_rounds<E, false>(s, pol, [&](uint4 (&w)[kLUnroll], int) { stat_fold<E, kLUnroll, ENT>(w, r.c, a); });
        st = exchange_parts<ENT>(a, xs, p.rows.C, r.rank, r.c);
    }
    if (threadIdx.x == 0) sc = token_scalars<ENT, MODE>(p, r.row, r.rank, r.T, r.T_ok, in, st);
    if (MODE == kForward) return;
    if (MODE == kBackward && p.rows.C > 1) {
        // the gradient may overwrite the logits: no slice is written before every CTA has its token logit
        cluster_wait_peers();
        cluster_sync_all();
    }
    __syncthreads();
    const TokenScalars t = sc;
    dense_pass<E, ENT>(s, grad, t.zero != 0, st.m, r.c.near, t.A, t.Bt);
    if (!t.zero && in_slice(s, tok)) {
        __syncthreads();   // the dense value of this entry has been written
        if (threadIdx.x == 0) store_entry(grad + s.lead + tok, t.entry);
    }
}

// Loss and gradient in one call: the slice through the ring of ears_ring.cuh.
template <typename E, bool ENT>
__global__ void __launch_bounds__(kRingThreads, 2) ears_token_step_kernel(const TokenParams p, int stages) {
    extern __shared__ __align__(128) unsigned char ring_buf[];
    __shared__ float4 xs[kLMaxCluster * kRingWarps];
    __shared__ TokenScalars sc;
    __shared__ RingBars bars;
    const RowSetup r = row_setup(p.rows);
    const E* row = row_ptr<E>(p.rows, r);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, r.rank);
    E* grad = grad_ptr<E>(p.grad, p.gsb, p.gsr, r) - s.lead;
    const int tid = threadIdx.x;
    const int tok = __ldg(p.tokens + r.row);
    const bool absent = tok == -1, bad = tok < -1 || tok >= p.rows.V;
    if (absent || bad) {   // the same in every CTA of the cluster
        if (tid == 0 && r.rank == 0) token_unused<kStep>(p, r.row, bad);
        if (tid < kLThreads) dense_pass<E, ENT>(s, grad, true, 0.f, 0.f, 0.f, 0.f);
        return;
    }
    const Ring<E> ring = make_ring(s, ring_buf, &bars, stages);
    const uint64_t keep = l2_policy_evict_last(), drop = l2_policy_evict_first();
    if (tid == kRingConsumers) {
        ring_init(&bars, stages);
        ring_load(ring, 0, ring.H, keep, drop);
    }
    TokenInputs in{};
    if (tid == 0) in = token_inputs<E, ENT, kStep>(p, row, r.row, tok);
    __syncthreads();
    if (tid >= kRingConsumers) {
        ring_loader_warp(ring, ring.H, p.rows.C, keep, drop);
        return;
    }
    Stat<ENT> a;
    stat_open(a);
    if (!ring_stats(ring, [&](uint4 (&w)[kRingPer], int) { stat_fold<E, kRingPer, ENT>(w, r.c, a); })) {
        a.s[0] = pack2(__int_as_float(0x7fc00000), 0.f);   // the row counts as unusable in every CTA
        if (p.status) atomicOr(p.status, kDevTimeout);
    }
    const int v = edge_vector(ring, s);
    if (v >= 0) {
        const uint4 w[1] = {load_partial(s.base, v, s.lead, s.end)};
        stat_fold<E, 1, ENT>(w, r.c, a);
    }
    const Part st = exchange_parts<ENT, kRingWarps>(a, xs, p.rows.C, r.rank, r.c);
    if (tid == 0) sc = token_scalars<ENT, kStep>(p, r.row, r.rank, r.T, r.T_ok, in, st);
    ring_sync_consumers();
    const TokenScalars t = sc;
    ring_gradient<E, ENT>(ring, s, grad, t.zero != 0, st.m, r.c.near, t.A, t.Bt, drop, p.status);
    if (!t.zero && in_slice(s, tok)) {
        ring_sync_consumers();   // the dense value of this entry has been written
        if (tid == 0) store_entry(grad + s.lead + tok, t.entry);
    }
}

}  // namespace ears
