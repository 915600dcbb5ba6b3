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
// Bound by HBM: a forward call reads each logit once, a gradient call reads and writes once.  A step
// (loss and gradient together) sweeps the slice twice, the second time out of L2: the rows in
// flight (CTAs on the device / C of them) are far smaller than L2.
#pragma once
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

// What the row's scalars come to, in 64 bits: one lane of one warp per CTA, identical in all of them.
struct TokenScalars { float A, Bt, entry; int zero; };

template <bool ENT, int MODE>
__device__ __forceinline__ TokenScalars token_scalars(const TokenParams& p, long long row, int rank, double T, bool T_ok, float lt, Part st) {
    const bool ok = T_ok && rowstat_ok(st.m, st.s) && (!ENT || st.w == st.w);
    const double Z = st.s, lnZ = log(Z), invT = 1.0 / T;
    double logp = ((double)lt - (double)st.m) * invT - lnZ;
    double H = ENT ? lnZ - kLn2 * (double)st.w / Z : 0.0;
    double loss = 0.0, kl = 0.0, g = 0.0, h = 0.0;
    bool fine = ok;
    if (p.policy) {
        const double old = __ldg(p.old_logp + row), A = __ldg(p.advantage + row);
        const double rho = exp(logp - old);
        const double plain = rho * A, clipped = fmin(fmax(rho, 1.0 - p.clip_low), 1.0 + p.clip_high) * A;
        loss = -fmin(plain, clipped);
        g = plain <= clipped ? -plain : 0.0;
        if (p.ref_logp) {
            const double d = (double)__ldg(p.ref_logp + row) - logp, ed = exp(d);
            kl = ed - d - 1.0;
            loss += p.kl_coef * kl;
            g += p.kl_coef * (1.0 - ed);
        }
        if (ENT) loss -= p.entropy_coef * H;
        fine = fine && isfinite(old) && isfinite(A) && isfinite(loss) && isfinite(g);
        if (MODE != kForward) {
            const double w = p.weight ? (double)__ldg(p.weight + row) : 1.0;
            g *= w;
            h = -w * p.entropy_coef;
        }
    } else if (MODE != kForward) {
        g = __ldg(p.d_logp + row);
        if (ENT && p.d_entropy) h = __ldg(p.d_entropy + row);
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

template <typename E, bool ENT, int MODE>
__global__ void __launch_bounds__(kLThreads) ears_token_kernel(const TokenParams p) {
    __shared__ float4 xs[kLMaxCluster * kLWarps];
    __shared__ TokenScalars sc;
    const RowSetup r = row_setup(p.rows);
    const E* row = row_ptr<E>(p.rows, r.row);
    const Slice<E> s = make_slice<E>(row, p.rows.V, p.rows.slice, r.rank);
    E* grad = MODE == kForward ? nullptr : grad_ptr<E>(p.grad, p.rows, p.gsb, p.gsr, r.row) - s.lead;
    const int tok = __ldg(p.tokens + r.row);
    const bool absent = tok == -1, bad = tok < -1 || tok >= p.rows.V;
    if (absent || bad) {   // the same in every CTA of the cluster
        if (threadIdx.x == 0 && r.rank == 0) {
            const float v = bad ? __int_as_float(0x7fc00000) : 0.f;
            if (MODE != kBackward) {
                if (p.out_logp) p.out_logp[r.row] = v;
                if (p.out_loss) p.out_loss[r.row] = v;
                if (p.out_kl) p.out_kl[r.row] = v;
                if (p.out_entropy) p.out_entropy[r.row] = v;
                if (MODE == kForward && p.stats) p.stats[r.row] = make_float4(0.f, __int_as_float(0x7fc00000), 0.f, 0.f);
            }
            if (bad && p.status) atomicOr(p.status, kDevInvalidInput);
        }
        if (MODE != kForward) dense_pass<E, ENT>(s, grad, true, 0.f, 0.f, 0.f, 0.f);
        return;
    }
    // asked for now, used after the sweep
    float lt = 0.f;
    if (threadIdx.x == 0) {
        float x[Words<E>::N];
        Words<E>::unpack(make_uint4(raw_bits(row + tok), 0, 0, 0), x);
        lt = x[0];
    }
    Part st;
    if (MODE == kBackward) {
        const float4 q = p.stats[r.row];
        // an entropy gradient needs the sum that only a forward call with the entropy leaves
        st = Part{q.x, !ENT || q.w == 1.f ? q.y : __int_as_float(0x7fc00000), q.z};
    } else {
        Stat<ENT> a;
        stat_open(a);
        for (int i0 = threadIdx.x; i0 < s.n; i0 += kLRound) {
            uint4 w[kLUnroll];
            load_round(s, i0, w);
            stat_fold<E, kLUnroll, ENT>(w, r.c, a);
        }
        st = exchange_parts<ENT>(a, xs, p.rows.C, r.rank, r.c);
    }
    if (threadIdx.x == 0) sc = token_scalars<ENT, MODE>(p, r.row, r.rank, r.T, r.T_ok, lt, st);
    if (MODE == kForward) return;
    if (MODE == kBackward && p.rows.C > 1) {
        // the gradient may overwrite the logits: no slice is written before every CTA has its token logit
        cluster_wait_peers();
        cluster_sync_all();
    }
    __syncthreads();
    const TokenScalars t = sc;
    dense_pass<E, ENT>(s, grad, t.zero != 0, st.m, r.c, t.A, t.Bt);
    if (!t.zero && in_slice(s, tok)) {
        __syncthreads();   // the dense value of this entry has been written
        if (threadIdx.x == 0) store_entry(grad + s.lead + tok, t.entry);
    }
}

}  // namespace ears
