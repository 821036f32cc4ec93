// What the streaming kernels over logit rows that keep a list of the largest ones share: the list's end, where it did not hold what passed,
// and sums of exponentials with whole numbers as references.
#pragma once
#include "gr_scan.cuh"

namespace gr {

// (as many listed vectors, and elements of them that pass the last threshold, as leave room for the CTAs of an SM)
template <int NTHR> using BeamSm = ScanShared<NTHR, 4 * NTHR, 8 * NTHR, 1>;

// v 2^k, k a whole number at or below 0 (what falls below 2^-1000 of v is dropped); a NaN stays one
__device__ __forceinline__ double times_pow2(double v, float k)
{
    if (!(k > -1000.f)) return v != v || k != k ? __longlong_as_double(0x7ff8000000000000ll) : 0.0;
    return v * __hiloint2double((1023 + (int)k) << 20, 0);
}

// Cuts the `listed` keys to those above `least`, in place (at most GR_MAX_SELECT of them: one for each thread).
template <class SS>
__device__ __forceinline__ void keep_keys(SS& sh, int listed, unsigned long long least)
{
    const unsigned long long k = (int)threadIdx.x < listed ? sh.keys[threadIdx.x] : 0ull;
    if (threadIdx.x == 0) sh.kept = 0;
    __syncthreads();
    if (k > least) sh.keys[atomicAdd(&sh.kept, 1)] = k;
    __syncthreads();
}

// push_vector; a list that is full puts the threshold out of reach, as what follows would wait for its counter in vain (128 groups of 8
// rows of 128256 with one token unmasked 272 -> 251 us).  Decides nothing but that: the list is taken for over in any case.
template <class SS>
__device__ __forceinline__ void push_or_stop(SS& sh, const ulonglong2& v, int id) {
    const int slot = atomicAdd(&sh.cnt, 1);
    if (slot < SS::kList) {
        GR_ARRAY_AS(ulonglong2, sh.keys, slot) = v;
        GR_ARRAY_AS(int, sh.keys, 4 * SS::kList + slot) = id;
    } else *((volatile float*)&sh.tau) = INFINITY;
}

// Where the list did not hold what passed: mostly ties, of a value that masks tokens or of few values in all.  The K-th largest
// of the threads' largest logits, to the last bit, is a value t that K elements reach.  What is above it is listed in one more
// pass, and what holds t as long as that is not much; else the places that are left go to the first ids that hold t, looked for from
// the first of them on.  The number of keys in sh.keys, or -1 where the elements above t are too many (then few threads met them all).
// (By radix passes alone those rows 1791 us, rows of whole numbers 1305 for 188, in bf16 1174 for 143.)
template <typename T, class SS>
__device__ __noinline__ int tied_select(SS& sh, const T* x, int V, int head, int nch, int first, int stride, int K, float largest)
{
    using VT = VecTraits<T>;
    constexpr int N = VT::N, S = kChunk / (32 * N), U = S < 4 ? S : 4, kWarps = SS::kThr / 32;
    constexpr int kAbove = SS::kCap / 2, kTies = SS::kCap / 4, kAhead = 4;
    static_assert(S % U == 0 && kTies >= GR_MAX_SELECT, "keys");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int vec_end = head + ((V - head) / N) * N;
    const unsigned mine = fkey(largest);
    unsigned t = 0;
#pragma unroll 1
    for (unsigned bit = 1u << 31; bit; bit >>= 1) if (__syncthreads_count(mine >= (t | bit)) >= K) t |= bit;
    if (tid == 0) { sh.kept = 0; sh.cnt = 0; sh.need = V; }
    __syncthreads();
    int id = V;                                            // the first that holds t
    auto look = [&](float v, int i) {
        const unsigned k = fkey(v);
        if (k > t) {
            const int slot = atomicAdd(&sh.kept, 1);
            if (slot < kAbove) sh.keys[slot] = ckey(v, i);
        } else if (k == t) {
            id = min(id, i);
            if (*((volatile int*)&sh.cnt) <= kTies) {
                const int slot = atomicAdd(&sh.cnt, 1);
                if (slot < kTies) sh.keys[kAbove + slot] = ckey(v, i);
            }
        }
    };
#pragma unroll 1
    for (int c = first + warp; c < nch; c += stride) {
        if (c == 0 && lane < head) look(load_logit<T>(x, lane), lane);
        if (c == nch - 1 && vec_end + lane < V) look(load_logit<T>(x, vec_end + lane), vec_end + lane);
#pragma unroll 1
        for (int u0 = 0; u0 < S; u0 += U) {
            const int base = head + c * kChunk + (u0 * 32 + lane) * N;
            ulonglong2 v[U];
#pragma unroll
            for (int u = 0; u < U; u++) if (base + u * 32 * N + N <= vec_end) v[u] = ldg_stream(x + base + u * 32 * N);
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (base + u * 32 * N + N > vec_end || fkey(VT::largest(v[u])) < t) continue;
#pragma unroll
                for (int i = 0; i < N; i++) look(VT::element(v[u], i), base + u * 32 * N + i);
            }
        }
    }
    id = __reduce_min_sync(0xffffffffu, id);
    if (lane == 0) atomicMin(&sh.need, id);
    __syncthreads();
    int have = sh.kept;
    const int from = sh.need, ties = sh.cnt;
    if (have > kAbove) return -1;
    if (have >= K || t <= fkey(-INFINITY)) return have;    // (masked tokens are no continuations)
    if (ties <= kTies) {
        // (they move to places at or before their own: a round's are read before any of them is written)
#pragma unroll 1
        for (int e0 = 0; e0 < ties; e0 += SS::kThr) {
            const int e = e0 + tid;
            const unsigned long long k = e < ties ? sh.keys[kAbove + e] : 0ull;
            __syncthreads();
            if (e < ties) sh.keys[have + e] = k;
            __syncthreads();
        }
        return have + ties;
    }
#pragma unroll 1
    for (int c = first; c < nch && have < K; c += stride) {
        const int end = chunk_end(min(c + kWarps, nch) - 1, head, nch, V);
#pragma unroll 1
        for (int i0 = max(chunk_begin(c, head), from); i0 < end && have < K; i0 += kAhead * SS::kThr) {
            float v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++) v[u] = i0 + u * SS::kThr + tid < end ? load_logit<T>(x, i0 + u * SS::kThr + tid) : NAN;
#pragma unroll
            for (int u = 0; u < kAhead; u++) {
                if (have >= K) break;
                const bool holds = v[u] == v[u] && fkey(v[u]) == t;
                const unsigned mask = __ballot_sync(0xffffffffu, holds);
                if (lane == 0) sh.hist[warp] = __popc(mask);
                __syncthreads();
                int at = have + __popc(mask & ((1u << lane) - 1u));
                for (int w = 0; w < kWarps; w++) { const int n = sh.hist[w]; if (w < warp) at += n; have += n; }
                if (holds && at < K) sh.keys[at] = ckey(v[u], i0 + u * SS::kThr + tid);
                __syncthreads();
            }
        }
    }
    return min(have, K);                                   // (of the last round's ties those that were listed)
}

// The K largest keys (but for masked tokens') of what the list holds, handed to `take(rank, key)`; their number.  use_tau: the list was made
// by a threshold; g0: this thread's largest logit.
template <typename T, class SS, class F>
__device__ __forceinline__ int best_listed(SS& sh, const T* x, int V, int head, int nch, int first, int stride, int K, bool use_tau, float g0, F take)
{
    using VT = VecTraits<T>;
    constexpr int N = VT::N;
    const int tid = threadIdx.x;
    // ---- candidates: a last threshold from the list itself, then keys of those that pass it
    int M = sh.cnt;
    bool over = M > SS::kList;
    if (!over) {
        constexpr int kPer = (SS::kList + SS::kThr - 1) / SS::kThr;
        // (the keys take the list's place: what a thread lists is in its registers before)
        ulonglong2 vv[kPer];
        int id[kPer];
        float own = -INFINITY;
#pragma unroll
        for (int u = 0; u < kPer; u++) {
            const int e = tid + u * SS::kThr;
            vv[u].x = VT::kNone; vv[u].y = VT::kNone; id[u] = 0;
            if (e < M) { vv[u] = GR_ARRAY_AS(ulonglong2, sh.keys, e); id[u] = GR_ARRAY_AS(int, sh.keys, 4 * SS::kList + e); }
            own = fmaxf(own, VT::largest(vv[u]));
        }
        // (a short list is ranked as it is, in less time than a threshold takes; not one of whole vectors from a short row)
        if (M > SS::kThr / 2 || (!use_tau && M * N > kRankKeys)) refine_tau(sh, own, K);
        const float tau = sh.tau;
        if (tid == 0) sh.kept = 0;
        __syncthreads();
        if (own >= tau) {
#pragma unroll
            for (int u = 0; u < kPer; u++) {
                if (VT::largest(vv[u]) < tau) continue;
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const float w = VT::element(vv[u], i);
                    if (w >= tau && w > -INFINITY) {
                        const int slot = atomicAdd(&sh.kept, 1);
                        if (slot < SS::kCap) sh.keys[slot] = ckey(w, id[u] + i);
                    }
                }
            }
        }
        __syncthreads();
        M = sh.kept;
        over = M > SS::kCap;
    }
    if (over) {
        __syncthreads();
        M = tied_select<T>(sh, x, V, head, nch, first, stride, K, g0);
        over = M < 0;
    }
    if (over) {
        __syncthreads();
        exact_select_slow<T>(sh, x, V, head, nch, first, stride, K);
        // (masked tokens come last in that order; they are not continuations)
        const unsigned long long masked = ((unsigned long long)fkey(-INFINITY) << 32) | 0xffffffffull;
        const int listed = min(sh.cnt, K);
        M = __syncthreads_count(tid < listed && sh.keys[min(tid, K - 1)] > masked);
        if (M < listed) keep_keys(sh, listed, masked);
    }
    const int nsel = min(K, M);
    rank_select(sh, M, nsel, take);
    return nsel;
}

}  // namespace gr
