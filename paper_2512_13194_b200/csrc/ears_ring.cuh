// The slice of a row that is needed twice -- for the statistics, then for the gradient -- streamed
// through a ring of shared-memory stages by bulk asynchronous copies.
//
// A loader thread runs ahead of the kRingWarps consumer warps through the sequence of loads
//     pass 1: chunks 0 .. n-1;   pass 2: chunks 0 .. n-H-1      (H = min(stages, n))
// The last H chunks of pass 1 stay where they are and pass 2 begins with them, so that a slice of at most
// `stages` chunks is read once, a longer one has the rest fetched again (from L2: those loads carry an
// evict-last hint and are evict-first the second time), and the gradient's first chunks are ready the
// moment the row's scalars are.  Load number i lies in stage i % stages.  A stage is released by its
// consumers only if a later load wants it: in pass 1 if i + stages < n, in pass 2 if i + stages < loads in all.
//
// Chunks cover the slice's whole vectors; a vector that the row covers in part (at its ends, when the row
// does not start or end on a 16-byte boundary) is fetched by one thread with plain loads.
//
// Two CTAs per SM, each with its own row: while one is between its passes (the exchange, the scalars), the other
// streams, and the rows in flight (296 of 304 KB) leave what is fetched again in L2.  A policy step on 4096 rows of 152064
// bf16 took 1024 us with plain loads and clusters of eight CTAs (L2 hit rate of the second sweep: 3 %), 542 with one CTA per
// row, 506 with the eviction hints, 413 through this ring (0.85 of the measured copy rate; its DRAM reads are 1.20 times the
// logits of the rows that count, its special-function pipe 60 % busy).  Longer rows are split over a cluster until those in
// flight fit L2 again (256000 fp32: 689 us with one CTA, 577 with four).
#pragma once
#include "ears_pipeline.cuh"
#include "ears_rows.cuh"

namespace ears {

constexpr int kRingWarps = kLWarps;                      // consumers; 16 of them were slower (223 us against 206)
constexpr int kRingConsumers = kRingWarps * 32;
constexpr int kRingThreads = kRingConsumers + 32;        // and one loader warp
constexpr int kRingChunk = 16384;                        // bytes per stage
constexpr int kRingVecs = kRingChunk / 16;
constexpr int kRingPer = kRingVecs / kRingConsumers;          // vectors per thread and chunk
// Six stages for each of two CTAs per SM: 4 -> 194 us, 5 -> 181, 6 -> 179 (token step on 2048 x 128256 bf16)
constexpr int kRingStages = 6;

struct RingBars {
    uint64_t full[kRingStages], empty[kRingStages];
    int abort_flag;      // a wait gave up
    int never;           // stays 0: the abort flag of the final wait for copies in flight
};

// Place of a load in the ring, stepped along with the load number.
struct RingPos {
    int stage;
    uint32_t phase;
    __device__ __forceinline__ void step(int S) {
        if (++stage == S) { stage = 0; phase ^= 1u; }
    }
};

template <typename E>
struct Ring {
    unsigned char* buf;
    RingBars* bars;
    const uint4* src;    // first whole vector
    int v0;              // its index in the row's vector run
    int vecs, n, S, H, loads;

    __device__ __forceinline__ int chunk_vecs(int c) const { return min(kRingVecs, vecs - c * kRingVecs); }
    __device__ __forceinline__ const uint4* stage(int i) const { return reinterpret_cast<const uint4*>(buf + (size_t)i * kRingChunk); }
    __device__ __forceinline__ RingPos place(int load) const { return RingPos{load % S, (uint32_t)(load / S) & 1u}; }
    // whole warps
    __device__ __forceinline__ bool wait(RingPos at) const {
        return __all_sync(0xffffffffu, mbar_wait(&bars->full[at.stage], at.phase, &bars->abort_flag));
    }
    __device__ __forceinline__ void release(RingPos at) const {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&bars->empty[at.stage]);
    }
};

template <typename E>
__device__ __forceinline__ Ring<E> make_ring(const Slice<E>& s, unsigned char* buf, RingBars* bars, int stages) {
    constexpr int N = Words<E>::N;
    Ring<E> r;
    r.buf = buf;
    r.bars = bars;
    r.v0 = max(s.v0, s.lead > 0 ? 1 : 0);
    r.vecs = max(0, min(s.v0 + s.n, s.end / N) - r.v0);
    r.src = reinterpret_cast<const uint4*>(s.base) + r.v0;
    r.n = (r.vecs + kRingVecs - 1) / kRingVecs;
    r.S = stages;
    r.H = min(stages, r.n);
    r.loads = 2 * r.n - r.H;
    return r;
}

// One thread; the barriers are visible to the others after the next __syncthreads.
__device__ __forceinline__ void ring_init(RingBars* bars, int stages) {
    for (int i = 0; i < stages; ++i) {
        mbar_init(&bars->full[i], 1);
        mbar_init(&bars->empty[i], kRingWarps);
    }
    bars->abort_flag = bars->never = 0;
    mbar_init_fence();
}

// The loader thread: loads [from, to).  -> how many loads are out in all (fewer than `to` after a failed wait).
template <typename E>
__device__ __forceinline__ int ring_load(const Ring<E>& r, int from, int to, uint64_t keep, uint64_t drop) {
    RingPos at = r.place(from);
    for (int i = from; i < to; ++i, at.step(r.S)) {
        if (i >= r.S && !mbar_wait(&r.bars->empty[at.stage], at.phase ^ 1u, &r.bars->abort_flag)) return i;
        const int c = i < r.n ? i : i - r.n;
        const uint32_t bytes = (uint32_t)r.chunk_vecs(c) * 16u;
        uint64_t* bar = &r.bars->full[at.stage];
        mbar_arrive_expect_tx(bar, bytes);
        bulk_load_hint(r.buf + (size_t)at.stage * kRingChunk, r.src + (size_t)c * kRingVecs, bytes, bar, i < r.n - r.H ? keep : drop);
    }
    return to;
}

// The loader thread at its end: no copy may be in flight when the CTA ends, whatever its consumers did.
template <typename E>
__device__ __forceinline__ void ring_drain(const Ring<E>& r, int issued) {
    for (int i = max(0, issued - r.S); i < issued; ++i) {
        const RingPos at = r.place(i);
        mbar_wait(&r.bars->full[at.stage], at.phase, &r.bars->never);
    }
}

// Pass 1, the consumers: fold(w, chunk) takes the thread's kRingPer vectors of a chunk (-inf beyond its end).
template <typename E, class F>
__device__ __forceinline__ bool ring_stats(const Ring<E>& r, F fold) {
    RingPos at{0, 0};
    for (int i = 0; i < r.n; ++i, at.step(r.S)) {
        if (!r.wait(at)) return false;
        const uint4* p = r.stage(at.stage) + threadIdx.x;
        const int left = r.vecs - i * kRingVecs;
        uint4 w[kRingPer];
        if (left >= kRingVecs) {
#pragma unroll
            for (int q = 0; q < kRingPer; ++q) w[q] = p[q * kRingConsumers];
        } else {
#pragma unroll
            for (int q = 0; q < kRingPer; ++q) {
                w[q] = Words<E>::minus_inf();
                if ((int)threadIdx.x + q * kRingConsumers < left) w[q] = p[q * kRingConsumers];
            }
        }
        fold(w, i);
        if (i + r.S < r.n) r.release(at);
    }
    return true;
}

__device__ __forceinline__ void st_row16(void* p, uint4 w, uint64_t policy) {
    asm volatile("st.global.L1::no_allocate.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;"
                 ::"l"(p), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w), "l"(policy) : "memory");
}

// Pass 2, the consumers: the gradient of every chunk, 2^t (A + Bt t) or zeros, to g (see dense_pass).
template <typename E, bool ENT>
__device__ __forceinline__ bool ring_dense(const Ring<E>& r, const Slice<E>& s, E* g, bool zero, float ref, float c, float A, float Bt, uint64_t drop) {
    const bool aligned = ((uintptr_t)g & 15) == 0;
    uint4* out = reinterpret_cast<uint4*>(g) + r.v0 + threadIdx.x;
    RingPos at = r.place(r.n - r.H);
    for (int t = 0; t < r.n; ++t, at.step(r.S)) {
        const int chunk = t < r.H ? r.n - r.H + t : t - r.H;
        if (t >= r.H && !r.wait(at)) return false;
        const uint4* p = r.stage(at.stage) + threadIdx.x;
        const int first = chunk * kRingVecs, left = r.vecs - first;
        if (left >= kRingVecs && aligned && !zero) {
            uint4 w[kRingPer];
#pragma unroll
            for (int q = 0; q < kRingPer; ++q) w[q] = p[q * kRingConsumers];
#pragma unroll
            for (int q = 0; q < kRingPer; ++q)
                st_row16(out + first + q * kRingConsumers, dense_words<E, ENT>(w[q], ref, c, A, Bt), drop);
        } else {
            for (int u = threadIdx.x, q = 0; u < left && q < kRingPer; u += kRingConsumers, ++q) {
                const uint4 d = zero ? make_uint4(0, 0, 0, 0) : dense_words<E, ENT>(p[q * kRingConsumers], ref, c, A, Bt);
                if (aligned) st_row16(out + first + q * kRingConsumers, d, drop);
                else store_partial(g, r.v0 + first + u, d, s.lead, s.end);
            }
        }
        if (r.n - r.H + t + r.S < r.loads) r.release(at);
    }
    return true;
}

// The vectors of the slice that its chunks leave out, at most two: thread 0 has the one before the first
// whole vector, thread 32 the one behind the last.  -> the vector's index or -1.
template <typename E>
__device__ __forceinline__ int edge_vector(const Ring<E>& r, const Slice<E>& s) {
    if (threadIdx.x == 0 && s.n > 0 && r.v0 > s.v0) return s.v0;
    if (threadIdx.x == 32 && s.v0 + s.n > r.v0 + r.vecs && s.n > 0 && s.v0 + s.n - 1 >= r.v0) return s.v0 + s.n - 1;
    return -1;
}

// The consumers' barrier; the loader warp does not take part.
__device__ __forceinline__ void ring_sync_consumers() { asm volatile("bar.sync 1, %0;" ::"n"(kRingConsumers) : "memory"); }

// The loader warp from the first loads on: the rest of pass 1, its part in the barriers of exchange_parts, pass 2.
template <typename E>
__device__ __forceinline__ void ring_loader_warp(const Ring<E>& r, int issued, int C, uint64_t keep, uint64_t drop) {
    const bool lead = (threadIdx.x & 31) == 0;
    if (lead) issued = ring_load(r, issued, r.n, keep, drop);
    exchange_join(C);
    if (lead) {
        if (issued == r.n) issued = ring_load(r, r.n, r.loads, keep, drop);
        ring_drain(r, issued);
    }
}

// The consumers' pass 2 over the whole slice, edges included; a wait that gave up leaves zeros and the status.
template <typename E, bool ENT>
__device__ __forceinline__ void ring_gradient(const Ring<E>& r, const Slice<E>& s, E* g, bool zero, float ref, float c, float A, float Bt,
                                              uint64_t drop, int32_t* status) {
    if (!ring_dense<E, ENT>(r, s, g, zero, ref, c, A, Bt, drop)) {
        if (status) atomicOr(status, kDevTimeout);
        if (threadIdx.x < kLThreads) dense_pass<E, ENT>(s, g, true, 0.f, 0.f, 0.f, 0.f);
        return;
    }
    const int v = edge_vector(r, s);
    if (v >= 0) {
        const uint4 d = zero ? make_uint4(0, 0, 0, 0) : dense_words<E, ENT>(load_partial(s.base, v, s.lead, s.end), ref, c, A, Bt);
        store_partial(g, v, d, s.lead, s.end);
    }
}

}  // namespace ears
