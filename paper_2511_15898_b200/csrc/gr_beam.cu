// gr_beam_select: the best continuations of groups of hypotheses.
//
// The first kernel streams the logit rows once, every row in one or several parts of a CTA each: a part leaves its
// `select` largest logits in descending order and the sum of its exponentials.  The second, a CTA per group, puts the sums
// together, turns the listed logits into scores and ranks them.  Groups in which two continuations lie too close for the sums are
// left to a third, a cluster of CTAs per group, that takes sums again in 64 bits (few groups: it makes the choice of all).
//
// The sum.  With s = log2(e) / T split into two fp32 numbers (s_hi + s_lo, both positive) an element contributes
// 2^(x s - R), R a whole number near x s of the largest element met: two FMAs and one ex2 an element, no
// systematic error from the rounding of s (which alone costs 4e-7 of a log-sum over 10^5 ids), exact factors between sums of
// different R, fp32 sums over one batch of vectors, fp64 from there on.  R is one for a warp and follows the maximum only where
// that is kRise above it (more would cost accuracy: the products' rounding grows with the distance from R).  An element that is -infinity gives 0; NaN and
// +infinity make the sum NaN, as does a maximum whose product with s overflows: such rows' sums are taken again in fp64, where the
// two are told apart.
//
// The order.  Within a row it is that of the logits.  Between rows scores are compared in fp64, and where two continuations lie
// closer than the bounds of their rows' errors the sums are taken again in fp64, so that the order is that of the 64-bit scores.
// (Neighbours in the order are looked at, and what lies near the last that is taken: were any two in the wrong order, two neighbours
// would be, of different rows.)  The bound of a streamed log-sum, with Z = sum 2^(x s - R) and p the elements' shares of it:
//   ex2          1.46e-7, the largest relative error over all arguments from -126 to 2 (documented: 2^-22)
//   fp32 sums    of 8 or 16 terms by vectors, and of the pair's two: 7 roundings of 2^-24 at most
//   exponents    two roundings, of the distance y from R: half a unit in its last place is 2^-24 max(|y|, 1) at most, so
//                2 ln 2 2^-24 E max(|y|, 1) in all, E the mean under p.  The shares' entropy, E log2(1 / p) = log2 Z + E(-y), is
//                largest where all but the first token are alike: with p1 the first's share and q = 1 - p1 the others',
//                E max(|y|, 1) <= p1 + q (log2(V / q) - log2 Z + 2)   (y <= 1, and R only rises).
//   s            known to 2^-48 of itself: 2^-46 |R|.
// and of a key 2^-51 of itself, as 64-bit roundings may fall on the other side.
// Together 1e-6 to 2e-6 a row (measured on rows of one value, of two, of whole numbers and of normal ones: 5.5e-7 at most).
//
// HBM bounds it in fp32 (128 groups of 8 rows of 128256: 95 us, 86 % of the measured copy rate), issue slots and the exponentials' pipe
// in bf16 (256 groups of 16 rows of 152064: 245 us, 78 %), latency where there are few rows (4 of 32000: 12.1 us).
#include <limits.h>
#include <math.h>
#include <algorithm>
#include "gr_host.h"
#include "gr_list.cuh"

namespace gr {

constexpr int kBeamThreads = 256;
constexpr int kBeamWarps = kBeamThreads / 32;
constexpr int kBeamMaxParts = 16;
constexpr int kBeamMaxLists = 256;             // rows of a group times parts
constexpr int kBeamMaxListed = 4096;           // entries of a group's lists
static_assert(GR_MAX_BEAMS * GR_MAX_SELECT <= kBeamMaxListed && GR_MAX_SELECT <= kMaxSupport, "lists");
constexpr double kErrSum = 1.46e-7 + 7.0 / 16777216, kErrDepth = 0.69314718055994530942 / 8388608, kErrRef = 1.0 / (1ll << 46);
constexpr double kErrKey = 1.0 / (1ll << 51);  // a key's roundings, in which an error of the sum may tell
constexpr float kLargestRef = 1048576.f;       // (products of s_lo stay below 1/8, and R + kRise is a number)
constexpr int kSettle = 8;                     // most CTAs of a cluster that takes sums again
constexpr float kRise = 1.f;

// what a part leaves: this, then its keys (ckey) in descending order
struct __align__(16) BeamPart {
    double sum;              // of 2^(x s - ref)
    float ref;
    int count;               // keys that follow
    int state;               // kPartSkipped, kPartCheck
    int pad;
};
constexpr int kPartSkipped = 1, kPartCheck = 2;
static_assert(sizeof(BeamPart) == 32, "workspace layout");

struct BeamArgs {
    const void* logits; const float* scores; const int* lengths; const unsigned char* done;
    long long ld;
    int V, beams, select, keep, parts, eos;        // keep: keys per part
    float s_hi, s_lo;
    double temp, penalty;
    char* ws; int* flags; int batch, team;         // flags: groups that are left to be settled; team: CTAs of a cluster for each
    int* out_token; int* out_parent; float* out_score; int* out_length; unsigned char* out_done; int* status;
};

__host__ __device__ inline int beam_stride(int keep) { return (int)sizeof(BeamPart) + 8 * ((keep + 1) & ~1); }

// ---------------------------------------------------------------- streaming

template <typename T, int U, int NTHR, int CTAS>
__global__ void __launch_bounds__(NTHR, CTAS)
beam_stream_kernel(const __grid_constant__ BeamArgs A)
{
    using VT = VecTraits<T>;
    using Sm = BeamSm<NTHR>;
    constexpr int kWarps = NTHR / 32;
    constexpr int N = VT::N, S = kChunk / (32 * N), NB = S / U;
    static_assert(S % U == 0, "a chunk is a whole number of batches");
    __shared__ Sm sh;
    __shared__ float s_ref[kWarps];
    __shared__ double s_sum[kWarps];
    pdl_wait();
    GR_CHECK_FLAG_DECL;
    GR_CHECK_FLAG_INIT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long row = blockIdx.x / A.parts;
    const int part = blockIdx.x % A.parts;
    BeamPart* rec = reinterpret_cast<BeamPart*>(A.ws + (size_t)blockIdx.x * beam_stride(A.keep));
    GR_PTR(unsigned long long) rec_keys = GR_MKPTR(unsigned long long, reinterpret_cast<unsigned long long*>(rec + 1), A.keep, GR_CHECK_FLAG);
    if (A.scores[row] == -INFINITY || (A.done && A.done[row])) {
        if (tid == 0) { BeamPart p = {0.0, -INFINITY, 0, kPartSkipped, 0}; *rec = p; }
        return;
    }
    const int V = A.V, K = A.keep;
    const T* x = (const T*)A.logits + row * A.ld;
    const int head = row_head(x, 0, V, (int)sizeof(T));
    const int nch = num_chunks(V, head);
    // this part's chunks: first + warp, + stride, ...
    const int first = part * kWarps, stride = A.parts * kWarps;
    const bool use_tau = V > Sm::kCap;             // (else every element may be listed)
    const int vec_end = head + ((V - head) / N) * N, tail = V - vec_end;
    if (tid == 0) { sh.cnt = 0; sh.tau = -3.402823466e38f; sh.reset_checks(); }
    __syncthreads();

    float g0 = -INFINITY, ref = -INFINITY;             // this thread's largest logit; the warp's whole number near the products with s
    double acc = 0.0;
    const unsigned long long hi2 = f_pack(A.s_hi, A.s_hi), lo2 = f_pack(A.s_lo, A.s_lo);
    const int rounds = first < nch ? (nch - first + stride - 1) / stride : 0;
    // the reference follows the maximum of the warp, where that is kRise above it (a logit above `limit`); what has been added up
    // moves there by an exact factor
    float limit = -INFINITY;
    auto raise = [&](float m) {
        const float to = ceilf(warp_max(m) * A.s_hi);
        if (acc != 0.0) acc = times_pow2(acc, ref - to);
        ref = to;
        limit = (to + kRise) / A.s_hi;
    };
    // the elements before the first and behind the last vector of the row, by the warps that the first and last chunk fall to
    float e0 = -INFINITY, e1 = -INFINITY;
    auto push_edges = [&](float tau) {
        if (e0 >= tau) push_vector(sh, VT::alone(e0), lane);
        if (e1 >= tau) push_vector(sh, VT::alone(e1), vec_end + lane);
    };
    {
        const bool has_first = first + warp == 0 && head > 0, has_last = (nch - 1) % stride == first + warp && tail > 0;
        if (has_first && lane < head) e0 = load_logit<T>(x, lane);
        if (has_last && lane < tail) e1 = load_logit<T>(x, vec_end + lane);
        if (has_first || has_last) {
            g0 = fmaxf(e0, e1);
            raise(g0);
            const float down = ref == -INFINITY ? 0.f : -ref;
            acc = (double)ex2(fmaf(e0, A.s_lo, fmaf(e0, A.s_hi, down))) + (double)ex2(fmaf(e1, A.s_lo, fmaf(e1, A.s_hi, down)));
        }
        if (!use_tau) push_edges(-3.402823466e38f);
    }
    // Rounds up to the next threshold.  About A = K + K^2 / NTHR elements of what a threshold was taken from reach it, so A of
    // each further part of that size are listed, with a deviation of a sqrt(A)-th: twice as many have to find room.
    const int A_K = K + K * K / NTHR;
    int r = 0, upto = !use_tau ? rounds : 2 * 4 * NB * A_K <= Sm::kList ? 4 : 1;
    int expected = upto * NB * A_K;
#pragma unroll 1
    while (true) {
#pragma unroll 1
        for (; r < min(upto, rounds); r++) {
            const int c = first + r * stride + warp;
            const bool cvalid = c < nch;
            const bool whole = cvalid && head + (c + 1) * kChunk <= vec_end;
#pragma unroll 1
            for (int nb = 0; nb < NB; nb++) {
                const int base = head + c * kChunk + (nb * U * 32 + lane) * N;
                const bool sample = use_tau && r == 0 && nb == 0;
                const float tau = sample ? INFINITY : *((volatile float*)&sh.tau);
                ulonglong2 v[U];
                auto batch = [&](auto all) {
                    auto in = [&](int i0) { return decltype(all)::value || i0 + N <= vec_end; };
#pragma unroll
                    for (int u = 0; u < U; u++) {
                        const int i0 = base + u * 32 * N;
                        v[u].x = VT::kNone; v[u].y = VT::kNone;
                        bool ok = in(i0);
#ifdef GR_CHECK
                        if (ok && (i0 < 0 || i0 + N > V || ((size_t)(x + i0) & 15))) { *GR_CHECK_FLAG = 1; ok = false; }
#endif
                        if (ok) v[u] = ldg_stream(x + i0);
                    }
                    float each[U];
                    each[0] = VT::largest(v[0]);
                    float most = each[0];
#pragma unroll
                    for (int u = 1; u < U; u++) { each[u] = VT::largest(v[u]); most = fmaxf(most, each[u]); }
                    g0 = fmaxf(g0, most);
                    if (__any_sync(0xffffffffu, most > limit)) raise(most);
                    // (an element that is -infinity gives 0 whatever the reference, as long as that is finite)
                    const float down = ref == -INFINITY ? 0.f : -ref;
                    const unsigned long long down2 = f_pack(down, down);
                    // (a vector's sum, then those of the vectors, in fp32 by halves: equal terms one after another in one sum would
                    // round the same way each time.  By halves in bf16 too: 262 -> 279 us for 256 groups of 16 rows of 152064, by its registers)
                    unsigned long long sum2[U];
#pragma unroll
                    for (int u = 0; u < U; u++) {
#pragma unroll
                        for (int i = 0; i < VT::kPairs; i++) {
                            const unsigned long long w = VT::pair(v[u], i);
                            const unsigned long long y = fma2(w, lo2, fma2(w, hi2, down2));
                            const unsigned long long e = f_pack(ex2(f_lo(y)), ex2(f_hi(y)));
                            sum2[u] = i == 0 ? e : add2(sum2[u], e);
                        }
                        if (VT::kPairs == 2) {
#pragma unroll
                            for (int k = 1; (u & k) && k < U; k *= 2) sum2[u] = add2(sum2[u - k], sum2[u]);
                        } else if (u > 0) sum2[u] = add2(sum2[u - 1], sum2[u]);
                    }
                    acc += (double)(f_lo(sum2[U - 1]) + f_hi(sum2[U - 1]));
                    if (most >= tau) {
#pragma unroll
                        for (int u = 0; u < U; u++) if (each[u] >= tau) push_or_stop(sh, v[u], base + u * 32 * N);
                    }
                };
                if (whole) batch(std::true_type());
                else if (cvalid) batch(std::false_type());
                if (sample) {
                    // the first batch had no threshold: it gives one, and is tested now
                    refine_tau(sh, g0, K);
                    const float t1 = *((volatile float*)&sh.tau);
                    push_edges(t1);
                    if (cvalid) {
#pragma unroll
                        for (int u = 0; u < U; u++) {
                            if ((whole || base + u * 32 * N + N <= vec_end) && VT::largest(v[u]) >= t1) push_or_stop(sh, v[u], base + u * 32 * N);
                        }
                    }
                }
            }
        }
        if (r >= rounds) break;
        upto *= 4;
        // A better threshold whenever the part read has grown fourfold, unless less is to come than has been read and there is
        // room for it; and a shorter list where it would not hold what is to come.
        // (Decided by expected lengths, the same for every thread: the list itself may still be growing.)
        if (rounds < 2 * r && 2 * (expected * r + A_K * (rounds - r)) < Sm::kList * r) { upto = rounds; continue; }
        const int listed = refine_tau(sh, g0, K);
        expected = min(expected + 3 * A_K, Sm::kList);
        const int more = A_K * min(3 * r, rounds - r);                                    // times r
        if (listed <= Sm::kList && 2 * more > (Sm::kList - listed) * r) keep_listed<T>(sh, listed);
    }
    // ---- the part's sum
    {
        // (a thread that met NaN or +infinity holds NaN; one that met nothing, or -infinity only, 0)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
        if (lane == 0) { s_ref[warp] = ref; s_sum[warp] = acc; }
    }
    __syncthreads();
    const int nsel = best_listed<T>(sh, x, V, head, nch, first, stride, K, use_tau, g0, [&](int rank, unsigned long long key) { rec_keys[rank] = key; });
    if (tid == 0) {
        float top = s_ref[0];
        for (int w = 1; w < kWarps; w++) top = fmaxf(top, s_ref[w]);
        double sum = 0.0;
        for (int w = 0; w < kWarps; w++) {
            if (s_sum[w] != 0.0) sum += s_ref[w] == top ? s_sum[w] : times_pow2(s_sum[w], s_ref[w] - top);
        }
        BeamPart p = {sum, top, nsel, sh.checks() | GR_CHECK_VALUE ? kPartCheck : 0, 0};
        *rec = p;
    }
}

// ---------------------------------------------------------------- the group's choice

struct BeamGroup {
    double lse[GR_MAX_BEAMS], scale[GR_MAX_BEAMS], score[GR_MAX_BEAMS];
    double red[kBeamWarps], table[64];
    double part_sum[kBeamMaxLists];
    float part_ref[kBeamMaxLists];
    int count[kBeamMaxLists];
    int length[GR_MAX_BEAMS];
    unsigned char row[kBeamMaxLists];          // a list's row
    unsigned char kind[GR_MAX_BEAMS];
    unsigned char again[GR_MAX_BEAMS];         // the row's sum is to be taken again (2: it was of no use)
    unsigned char exact[GR_MAX_BEAMS];         // ... and has been
    int bad, check, survivors, redo;
    double err[GR_MAX_BEAMS];                  // bound of the error of the row's keys by that of its log-sum
    unsigned long long least;                  // a bound below the last key that is taken (as an integer that orders like it)
    double slack;                              // the largest distance of keys at which sums are taken again
    int best_at[GR_MAX_SELECT + 1];
    double share[2][kSettle];                  // what the cluster's CTAs tell one another
};
constexpr int kRowNone = 0, kRowDone = 1, kRowLive = 2;

// What every CTA of the cluster has to tell (the same `mine` in all of its threads), in all of them.  (Two sets of places, used in
// turn: a CTA writes to one of them again only after all have read it, as they come to the barrier between.)
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ const double* cluster_share(BeamGroup& g, int& turn, int team, double mine)
{
    double* place = g.share[turn++ & 1];
    if ((int)threadIdx.x < team) {
        unsigned at = (unsigned)__cvta_generic_to_shared(place + blockIdx.x % team);
        asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"((unsigned)threadIdx.x));
        asm volatile("st.shared::cluster.f64 [%0], %1;" :: "r"(at), "d"(mine) : "memory");
    }
    cluster_meet();
    return place;
}

// log sum exp(x / T) of a row in fp64 by the CTAs of a cluster, the same for every thread of all of them; -infinity for a row that is
// masked as a whole; `bad` set for one with a NaN or +infinity.  `known`: its largest logit where that is known (then there is no NaN in
// it), else NaN.  (Every thread takes the elements of its index modulo the cluster's size, so that equal rows give equal sums wherever they lie.)
// exp(-d) = 2^-n 2^(j / 64) exp(-r) by a table and five terms, |r| <= ln 2 / 128: a row of 152064 in 60 us by one CTA, for 100 by exp_neg, and in
// 10 by a cluster of eight.
template <typename T>
__device__ __noinline__ double row_lse(BeamGroup& g, int& turn, int team, const T* x, int V, double temp, float known)
{
    constexpr int kAhead = 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, first = (int)(blockIdx.x % team) * kBeamThreads + tid, step = team * kBeamThreads;
    double* red = g.red;
    double top = (double)known;
    if (known != known) {
        float m = -INFINITY;
        int wrong = 0;
        for (int i = first; i < V; i += step) {
            const float v = load_logit<T>(x, i);
            if (!(v < INFINITY)) wrong = 1;
            m = fmaxf(m, v);
        }
        if (wrong) m = INFINITY;
        m = warp_max(m);
        if (lane == 0) red[warp] = (double)m;
        __syncthreads();
        top = red[0];
        for (int w = 1; w < kBeamWarps; w++) top = fmax(top, red[w]);
        const double* all = cluster_share(g, turn, team, top);
        for (int c = 0; c < team; c++) top = fmax(top, all[c]);
        __syncthreads();
        if (top == INFINITY) { if (tid == 0) g.bad = 1; return 0.0; }
    }
    if (top == -INFINITY) return -INFINITY;
    // (kAhead elements at a time, without a branch between them: an element is a chain of twelve dependent operations.  Whole
    // numbers by the sum with 1.5 2^52, whose low word they are: conversions have a sixteenth of the multiplications' rate.)
    const double scale = 64.0 * 1.4426950408889634074 / temp, magic = 6755399441055744.0, unit = 0.69314718055994530942 / 64.0;
    const double c1 = unit, c2 = unit * c1 / 2.0, c3 = unit * c2 / 3.0, c4 = unit * c3 / 4.0, c5 = unit * c4 / 5.0;
    const float lowest = (float)fmax(top - 690.0 * temp, -3.4028234663852886e38);   // exp(-690): nothing beside the largest
    double sum0 = 0.0, sum1 = 0.0;
    float next[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; u++) next[u] = first + u * step < V ? load_logit<T>(x, first + u * step) : -INFINITY;
#pragma unroll 1
    for (int i0 = first; i0 < V; i0 += kAhead * step) {
        float v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int i = i0 + (kAhead + u) * step;
            v[u] = next[u];
            next[u] = i < V ? load_logit<T>(x, i) : -INFINITY;
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const double y = ((double)fmaxf(v[u], lowest) - top) * scale;   // in units of log 2 / 64
            const double whole = fmax(y, -64000.0) + magic;
            const int k = __double2loint(whole);
            const double z = y - (whole - magic);
            const double p = z * fma(z, fma(z, fma(z, fma(z, c5, c4), c3), c2), c1);
            const double t = g.table[k & 63];
            const double f = __hiloint2double(__double2hiint(t) + ((k >> 6) << 20), __double2loint(t));
            const double e = k > -64000 && v[u] > -INFINITY ? fma(f, p, f) : 0.0;
            if (u & 1) sum1 += e; else sum0 += e;
        }
    }
    double sum = sum0 + sum1;
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) red[warp] = sum;
    __syncthreads();
    double mine = 0.0, sum_all = 0.0;
    for (int w = 0; w < kBeamWarps; w++) mine += red[w];
    const double* all = cluster_share(g, turn, team, mine);
    for (int c = 0; c < team; c++) sum_all += all[c];
    __syncthreads();
    return top / temp + m_log(sum_all);
}

// n^a, a >= 0: products for whole numbers a, with a square root for half ones, so that equal keys come out equal (pow is off by a
// unit in the last place in one of twenty cases, at a = 1 too)
__device__ __noinline__ double length_power(int n, double a)
{
    const double twice = 2.0 * a;
    if (twice != floor(twice) || twice > 64.0) return pow((double)n, a);
    double r = 1.0, base = (double)n;
    const int k = (int)twice;
    for (int e = k >> 1; e; e >>= 1, base *= base) if (e & 1) r *= base;
    return k & 1 ? r * sqrt((double)n) : r;
}

// order-preserving map double -> integer (integers compare faster), and back; the two zeros get one key
__device__ __forceinline__ unsigned long long sortable(double v) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double unsortable(unsigned long long k) {
    return __longlong_as_double((long long)((k >> 63) ? (k & 0x7fffffffffffffffull) : ~k));
}

// Shared memory of the choice: `most` entries of lists (a list takes 1 << shift of them), then as many survivors.
__host__ __device__ inline int list_shift(int keep) { int s = 0; while ((1 << s) < keep) s++; return s; }
__host__ __device__ inline size_t choose_bytes(int lists, int keep) { return ((size_t)lists << list_shift(keep)) * 36; }

// One CTA per group, or (kSettles) a cluster: then all of its CTAs make the same choice, take sums again together where that is needed,
// and the first one writes what comes out.  A CTA alone leaves such a group to be settled.  (What it costs is latency: it runs once,
// mostly with its instructions not yet fetched.  So no integer division in the loops, and the survivors next to one another: with
// indices to follow and lists to divide out, ranking 71 of them took 13 us, now 1.)
template <typename T, bool kSettles>
__device__ __forceinline__ void choose(const BeamArgs& A, BeamGroup& g, unsigned char* s_dyn, long long b, int& turn)
{
    GR_CHECK_FLAG_DECL;
    GR_CHECK_FLAG_INIT;
    const int tid = threadIdx.x;
    const int W = A.beams, P = A.parts, K = A.select, keep = A.keep, lists = W * P, shift = list_shift(keep), most = lists << shift;
    GR_PTR(double) key = GR_MKPTR(double, reinterpret_cast<double*>(s_dyn), most, GR_CHECK_FLAG);
    GR_PTR(unsigned long long) raw = GR_MKPTR(unsigned long long, reinterpret_cast<unsigned long long*>(s_dyn) + most, most, GR_CHECK_FLAG);
    // (survivors: the key as an integer that orders like it, and the logit and token)
    GR_PTR(ulonglong2) sv = GR_MKPTR(ulonglong2, reinterpret_cast<ulonglong2*>(s_dyn) + most, most, GR_CHECK_FLAG);
    GR_PTR(int) sv_row = GR_MKPTR(int, reinterpret_cast<int*>(s_dyn + 32 * (size_t)most), most, GR_CHECK_FLAG);
    const int stride = beam_stride(keep);
    const char* recs = A.ws + (size_t)b * lists * stride;
    if (tid == 0) { g.bad = 0; g.check = 0; g.redo = 0; }
    __syncthreads();
    // ---- what the parts left (entries behind a list's count are whatever the workspace held: they are not looked at)
    for (int l = tid; l < lists; l += kBeamThreads) {
        const BeamPart r = *reinterpret_cast<const BeamPart*>(recs + (size_t)l * stride);
        g.part_sum[l] = r.sum; g.part_ref[l] = r.ref; g.count[l] = r.count;
        g.row[l] = (unsigned char)(l / P);
        if (r.state & kPartCheck) g.check = 1;
    }
    for (int e = tid; e < most; e += kBeamThreads) {
        const int l = e >> shift, i = e & ((1 << shift) - 1);
        if (i < keep) raw[e] = reinterpret_cast<const unsigned long long*>(recs + (size_t)l * stride + sizeof(BeamPart))[i];
    }
    static_assert(GR_MAX_BEAMS <= 32, "a lane of the first warp for each row");
    // (a quotient, as the key is defined: by a product with 1 / L^a the keys -49 / 49 and -1 / 1 would differ)
    auto key_of = [&](int w, double total) {
        if (A.penalty == 0.0) return total;
        return A.penalty > 0.0 ? total / g.scale[w] : fmax(total * g.scale[w], -1.7976931348623157e308);
    };
    float score = -INFINITY;
    bool fin = false;
    if (tid < W) {
        score = A.scores[b * W + tid];
        const int n = A.lengths ? A.lengths[b * W + tid] : 0;
        fin = A.done && A.done[b * W + tid];
        g.length[tid] = max(1, fin ? n : (n < INT_MAX ? n + 1 : n));
        g.scale[tid] = A.penalty != 0.0 ? length_power(g.length[tid], fabs(A.penalty)) : 1.0;
        if (!(score < INFINITY)) g.bad = 1;
    }
    __syncthreads();
    // ---- rows
    if (tid < 32) {
        if (tid < W) {
            const int w = tid;
            g.score[w] = (double)score;
            g.kind[w] = score == -INFINITY ? kRowNone : fin ? kRowDone : kRowLive;
            g.again[w] = 0; g.exact[w] = 0; g.err[w] = 0.0;
            double lse = 0.0;
            if (g.kind[w] == kRowLive) {
                float top = -INFINITY;
                for (int l = w * P; l < (w + 1) * P; l++) top = fmaxf(top, g.part_ref[l]);
                double sum = 0.0;
                int listed = 0;
                for (int l = w * P; l < (w + 1) * P; l++) {
                    const double v = g.part_sum[l];
                    if (v != 0.0) sum += g.part_ref[l] == top ? v : times_pow2(v, g.part_ref[l] - top);
                    listed += g.count[l];
                }
                const double units = log2(sum);
                lse = ((double)top + units) * 0.69314718055994530942;
                // NaN, an infinity, or logits so large that R, an fp32 number, is not the whole number near their product with s
                // to within a few units: in fp64.  (Not where every token is masked: nothing depends on that sum.)
                float first = -INFINITY;
                for (int l = w * P; l < (w + 1) * P; l++) if (g.count[l] > 0) first = fmaxf(first, fkey_inv((unsigned)(raw[l << shift] >> 32)));
                if (!(fabsf(top) <= kLargestRef) || !(sum < INFINITY)) g.again[w] = listed > 0 || sum != 0.0 ? 2 : 0;
                else if (listed > 0) {
                    // (the shares to 1e-5 on the side of the larger bound; two units in ten for the products of s_lo)
                    const float p = fminf(1.f, __expf((float)((double)first / A.temp - lse))), q = fminf(1.f, 1.f - p + 1e-5f);
                    const float depth = 1.2f + q * (log2f((float)A.V / q) - (float)units + 2.f);
                    g.err[w] = key_of(w, kErrSum + kErrDepth * (double)depth + kErrRef * fabs((double)top));
                }
            } else if (g.kind[w] == kRowDone) {
                // a finished hypothesis has one continuation, in its first part's list
                g.count[w * P] = 1;
                raw[w * P << shift] = ckey(0.f, A.eos);
            }
            g.lse[w] = lse;
            if (g.again[w]) g.redo = 1;
        }
        double largest = tid < W ? 2.0 * g.err[tid] : 0.0;
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) largest = fmax(largest, __shfl_xor_sync(0xffffffffu, largest, o));
        if (tid == 0) g.slack = largest;
    }
    __syncthreads();
    // (the quotient as in the sum's reference: with a product by 1 / T the largest logit's would be off it by a rounding, which for
    // quotients of 10^16 and more is as large as any difference)
    auto total_of = [&](int w, unsigned long long k) {
        return g.kind[w] == kRowDone ? g.score[w] : g.score[w] + ((double)fkey_inv((unsigned)(k >> 32)) / A.temp - g.lse[w]);
    };
    int M = 0;
#pragma unroll 1
    while (true) {
        // ---- sums that are to be taken again
        if (!kSettles && g.redo) break;
        if (kSettles && g.redo) {
            cluster_meet();                                // (the others have begun)
            if (tid < 64) g.table[tid] = exp2((double)tid * (1.0 / 64.0));
            __syncthreads();
#pragma unroll 1
            for (int w = 0; w < W; w++) {
                if (!g.again[w]) continue;
                // (the largest logit heads one of the row's lists, unless the streamed sum was of no use)
                float known = -INFINITY;
                for (int l = w * P; l < (w + 1) * P; l++) if (g.count[l] > 0) known = fmaxf(known, fkey_inv((unsigned)(raw[l << shift] >> 32)));
                if (g.again[w] == 2) known = __int_as_float(0x7fc00000);
                const double lse = row_lse<T>(g, turn, A.team, (const T*)A.logits + (b * W + w) * A.ld, A.V, A.temp, known);
                __syncthreads();
                if (tid == 0) { g.lse[w] = lse; g.err[w] = 0.0; g.again[w] = 0; g.exact[w] = 1; }
                __syncthreads();
            }
        }
        if (g.bad) break;
        __syncthreads();
        if (tid == 0) { g.survivors = 0; g.redo = 0; g.least = sortable(-INFINITY); }
        // ---- scores, and a bound below the select-th: of the q-th entries of the lists the ceil(K / q)-th largest, q the
        // smallest power of two that leaves at most half of the lists above it
        for (int e = tid; e < most; e += kBeamThreads) {
            const int l = e >> shift, i = e & ((1 << shift) - 1), w = g.row[l];
            key[e] = i < g.count[l] ? key_of(w, total_of(w, raw[e])) : -INFINITY;
        }
        // (few lists: every power of two, and the largest of the bounds)
        int lg0 = 0;
        while ((1 << lg0) < keep && 2 * ((K + (1 << lg0) - 1) >> lg0) > lists) lg0++;
        const int lg1 = lists <= 64 ? shift : lg0;
        if (lists <= 64) lg0 = 0;
        __syncthreads();
        for (int t = tid; t < lists * (lg1 - lg0 + 1); t += kBeamThreads) {
            const int level = t / lists, l = t - level * lists;
            const int q = min(1 << (lg0 + level), keep), place = (K + q - 1) / q;
            if (place > lists) continue;
            const double mine = key[(l << shift) + q - 1];
            int rank = 0;
#pragma unroll 4
            for (int o = 0; o < lists; o++) {
                const double k = key[(o << shift) + q - 1];
                rank += k > mine || (k == mine && o < l) ? 1 : 0;
            }
            if (rank == place - 1) atomicMax(&g.least, sortable(mine));
        }
        __syncthreads();
        // (those a little below the bound too: they may have to be told from the last ones)
        const double bound = unsortable(g.least), least = bound - (g.slack + 2.0 * kErrKey * fabs(bound));
        for (int e = tid; e < most; e += kBeamThreads) {
            const int l = e >> shift;
            if ((e & ((1 << shift) - 1)) < g.count[l] && !(key[e] < least)) {
                const int at = atomicAdd(&g.survivors, 1);
                sv[at] = make_ulonglong2(sortable(key[e]), raw[e]); sv_row[at] = g.row[l];
            }
        }
        __syncthreads();
        M = g.survivors;
        // ---- ranks: larger key, then the row before, then the place in the row (by logit, then by token).  Several threads to
        // a survivor where there are enough.
        const int team = 16 * M <= kBeamThreads ? 16 : 8 * M <= kBeamThreads ? 8 : 4 * M <= kBeamThreads ? 4 : 2 * M <= kBeamThreads ? 2 : 1;
#pragma unroll 1
        for (int a0 = 0; a0 < M; a0 += kBeamThreads / team) {
            const int a = a0 + tid / team;
            int rank = 0;
            unsigned long long mine = 0ull;
            if (a < M) {
                const int w = sv_row[a];
                const ulonglong2 own = sv[a];
                mine = own.x;
#pragma unroll 4
                for (int o = tid & (team - 1); o < M; o += team) {
                    const int v = sv_row[o];
                    const ulonglong2 k = sv[o];
                    const bool within = k.y > own.y, across = k.x > own.x || (k.x == own.x && v < w);
                    rank += (v == w ? within : across) ? 1 : 0;
                }
            }
            __syncwarp();
            for (int o = 1; o < team; o <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
            if (a < M && (tid & (team - 1)) == 0 && rank <= K) g.best_at[rank] = a;
        }
        __syncthreads();
        // ---- continuations of different rows that lie too close for the streamed sums: neighbours, and those near the last one.  (A
        // token masked by a value like -1e30 has its quotient as total, whatever the sum: less than a quarter of a unit in its last
        // place is added to it.)
        const int pairs = min(M, K + 1) - 1;
#pragma unroll 1
        for (int i = tid; i < (M > K ? pairs + M : pairs); i += kBeamThreads) {
            const int e = i < pairs ? g.best_at[i] : i - pairs, f = g.best_at[i < pairs ? i + 1 : K - 1];
            const int w = sv_row[e], v = sv_row[f];
            if (w == v) continue;
            const double key_e = unsortable(sv[e].x), key_f = unsortable(sv[f].x);
            if (fabs(key_e - key_f) > g.err[w] + g.err[v] + kErrKey * (fabs(key_e) + fabs(key_f))) continue;
#pragma unroll 1
            for (int side = 0; side < 2; side++) {
                const int at = side ? f : e, row = side ? v : w;
                const double x = (double)fkey_inv((unsigned)(sv[at].y >> 32)) / A.temp;
                if (g.kind[row] != kRowLive || g.exact[row] || fabs(x) > 72057594037927936.0 * (1.0 + fabs(g.lse[row]) + fabs(g.score[row]))) continue;  // 2^56
                g.again[row] = 1; g.redo = 1;
            }
        }
        __syncthreads();
        if (!g.redo) break;
    }
    // ---- results
    const bool left = !kSettles && g.redo && !g.bad;
    if (!kSettles && tid == 0) A.flags[b] = left ? 1 : 0;
    if (left || (kSettles && blockIdx.x % A.team != 0)) return;
    const bool bad = g.bad != 0;
    for (int i = tid; i < K; i += kBeamThreads) {
        const size_t at = (size_t)b * K + i;
        int token = -1, parent = -1, length = 0;
        float total = -INFINITY;
        unsigned char ended = 0;
        if (!bad && i < M) {
            const int e = g.best_at[i];
            parent = sv_row[e];
            token = (int)(0xffffffffu - (unsigned)sv[e].y);
            total = (float)total_of(parent, sv[e].y);
            length = g.length[parent];
            ended = g.kind[parent] == kRowDone || token == A.eos;
        }
        A.out_token[at] = token; A.out_parent[at] = parent; A.out_score[at] = total; A.out_done[at] = ended;
        if (A.out_length) A.out_length[at] = length;
    }
    if (tid == 0) {
        A.status[b] = bad ? GR_BAD_LOGITS : g.check ? GR_CHECK_FAILED : GR_OK;
#ifdef GR_CHECK
        if (GR_CHECK_VALUE) A.status[b] = GR_CHECK_FAILED;
#endif
    }
}

template <typename T>
__global__ void __launch_bounds__(kBeamThreads, 3)
beam_choose_kernel(const __grid_constant__ BeamArgs A)
{
    extern __shared__ __align__(16) unsigned char s_dyn[];
    __shared__ BeamGroup g;
    pdl_wait();
    int turn = 0;
    choose<T, false>(A, g, s_dyn, blockIdx.x, turn);
}

// The groups that the choice has left (all, where there are no flags), a cluster for each in turn.
template <typename T>
__global__ void __launch_bounds__(kBeamThreads, 2)
beam_settle_kernel(const __grid_constant__ BeamArgs A)
{
    extern __shared__ __align__(16) unsigned char s_dyn[];
    __shared__ BeamGroup g;
    __shared__ unsigned s_left[kBeamWarps];
    pdl_wait();
    int turn = 0;
    const int tid = threadIdx.x, clusters = gridDim.x / A.team;
#pragma unroll 1
    for (long long b0 = blockIdx.x / A.team; b0 < A.batch; b0 += (long long)clusters * kBeamThreads) {
        const long long b = b0 + (long long)tid * clusters;
        const unsigned left = __ballot_sync(0xffffffffu, b < A.batch && (!A.flags || A.flags[b]));
        if ((tid & 31) == 0) s_left[tid >> 5] = left;
        __syncthreads();
#pragma unroll 1
        for (int w = 0; w < kBeamWarps; w++) {
#pragma unroll 1
            for (unsigned more = s_left[w]; more; more &= more - 1) {
                choose<T, true>(A, g, s_dyn, b0 + (long long)(32 * w + __ffs(more) - 1) * clusters, turn);
                __syncthreads();
            }
        }
        __syncthreads();
    }
}

// parts of a row: as many as there are CTAs of one wave for, each with a chunk per warp at least
static int beam_parts(int V, int rows, int beams, int keep)
{
    const int chunks = (V + kChunk - 1) / kChunk;
    int most = (chunks + kBeamWarps - 1) / kBeamWarps;
    if (most > kBeamMaxParts) most = kBeamMaxParts;
    int parts = (4 * kSms) / (rows > 0 ? rows : 1);
    if (parts > most) parts = most;
    if (parts > kBeamMaxLists / beams) parts = kBeamMaxLists / beams;
    const int per = beams << list_shift(keep);
    if (parts > kBeamMaxListed / per) parts = kBeamMaxListed / per;
    return parts < 1 ? 1 : parts;
}

static bool beam_shape_ok(int V, int beams, int select, int batch)
{
    return V >= 1 && V <= (1 << 21) && beams >= 1 && beams <= GR_MAX_BEAMS && select >= 1 && select <= GR_MAX_SELECT
        && batch >= 0 && (long long)batch * beams <= (1 << 26);
}

template <typename T>
static int launch_beam(const BeamArgs& A, int batch, cudaStream_t st)
{
    const int smem = (int)choose_bytes(A.beams * A.parts, A.keep);
    static bool raised[kMaxDevices] = {false};
    if (smem > 24 * 1024) {
        int dev = -1;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return GR_E_LAUNCH; }
        if (!raised[dev]) {
            if (cudaFuncSetAttribute(beam_choose_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 36 * kBeamMaxListed) != cudaSuccess
                || cudaFuncSetAttribute(beam_settle_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 36 * kBeamMaxListed) != cudaSuccess) {
                cudaGetLastError();
                return GR_E_LAUNCH;
            }
            raised[dev] = true;
        }
    }
    // More than one wave of four CTAs per SM: eight smaller ones (a row's thresholds and its selection at the end leave gaps that
    // seven other rows fill better than three: 1024 rows of 50257 fp32 58 -> 49 us, of 128256 115 -> 108).  In fp32 where they do not
    // leave a larger part of their last wave empty or where there are more than two waves of them (1200 rows of 128256, just over
    // one wave, 131 -> 143); in bf16, which waits for instructions and not for bytes, always, and twelve per SM where that saves a
    // quarter of the waves (1200 rows of 128256 88 us by four, 93 by eight, 81 by twelve; 2000 rows 124, 117, 126; 4096 of 152064 261,
    // 244, 233).  The smaller ones' lists hold 4 A + 5 deviations up to 48 keys.
    const int ctas = batch * A.beams * A.parts;
    auto waves = [&](int per) { return (ctas + per * kSms - 1) / (per * kSms); };
    constexpr bool kNarrow = sizeof(T) == 2;
    const bool small = A.keep <= 48 && ctas > 4 * kSms && (kNarrow || ctas > 16 * kSms || 2 * waves(8) <= waves(4));
    // Few CTAs: a whole chunk per warp in flight, so that a short part needs one trip to memory and one threshold.
    if (ctas <= 2 * kSms) launch_pdl(beam_stream_kernel<T, kChunk / (32 * VecTraits<T>::N), 256, 2>, ctas, 256, 0, st, A);
    else if (small && kNarrow && 4 * waves(12) <= 3 * waves(8)) launch_pdl(beam_stream_kernel<T, 4, 128, kNarrow ? 12 : 8>, ctas, 128, 0, st, A);
    else if (small) launch_pdl(beam_stream_kernel<T, 4, 128, 8>, ctas, 128, 0, st, A);
    else launch_pdl(beam_stream_kernel<T, 4, 256, 4>, ctas, 256, 0, st, A);
    // Few groups: a cluster chooses for each at once, of as many CTAs as leave every group's an SM.  Else a CTA for each, and then
    // clusters for what these leave (74 groups of 4 rows of 32000: 19.7 us by clusters of two, 20.6 by a CTA each and a second
    // launch).  A CTA of theirs to an SM: with two the launch takes 0.7 us longer where no group is left, and where all are 3.5 ms for
    // 3.9 (256 groups of 16 equal rows of 152064).
    BeamArgs B = A;
    B.team = kSettle;
    while (B.team > 2 && batch * B.team > kSms) B.team /= 2;
    if (batch * B.team <= kSms) {
        B.flags = nullptr;
        launch_pdl_cluster(B.team, beam_settle_kernel<T>, batch * B.team, kBeamThreads, smem, st, B);
    } else {
        B.team = kSettle;
        launch_pdl(beam_choose_kernel<T>, batch, kBeamThreads, smem, st, B);
        launch_pdl_cluster(kSettle, beam_settle_kernel<T>, std::min(batch, kSms / kSettle) * kSettle, kBeamThreads, smem, st, B);
    }
    return GR_OK;
}

}  // namespace gr

extern "C" {

size_t gr_beam_workspace_bytes(int V, int beams, int select, int batch)
{
    if (!gr::beam_shape_ok(V, beams, select, batch)) return 0;
    const int keep = select < V ? select : V, rows = (batch > 0 ? batch : 1) * beams;
    return (size_t)rows * gr::beam_parts(V, rows, beams, keep) * gr::beam_stride(keep) + 4 * (((size_t)batch + 3) & ~(size_t)3);
}

int gr_beam_select(const void* logits, int dtype, int V, long long ld, int beams, int batch, float temperature,
                   const float* scores, const int* lengths, const unsigned char* done, int eos,
                   float length_penalty, int select, void* workspace, int* out_token, int* out_parent,
                   float* out_score, int* out_length, unsigned char* out_done, int* status, void* stream)
{
    if (!gr::beam_shape_ok(V, beams, select, batch)) return GR_E_INVALID;
    if (dtype != GR_F32 && dtype != GR_BF16) return GR_E_INVALID;
    if (!(temperature > 0.f) || !isfinite(temperature) || !(fabsf(length_penalty) <= 32.f)) return GR_E_INVALID;
    if (ld < V || ld > (1ll << 32)) return GR_E_INVALID;
    if (eos < -1 || eos >= V || (done && eos < 0) || (!lengths && length_penalty != 0.f)) return GR_E_INVALID;
    if (batch == 0) return GR_OK;
    if (!logits || !scores || !workspace || !out_token || !out_parent || !out_score || !out_done || !status) return GR_E_NULL;
    if (((uintptr_t)logits & (dtype == GR_F32 ? 3 : 1)) || ((uintptr_t)workspace & 15)) return GR_E_ALIGN;
    gr::BeamArgs A;
    A.logits = logits; A.scores = scores; A.lengths = lengths; A.done = done; A.ld = ld; A.V = V; A.beams = beams;
    A.select = select; A.keep = select < V ? select : V; A.eos = eos;
    A.parts = gr::beam_parts(V, batch * beams, beams, A.keep);
    A.temp = (double)temperature; A.penalty = (double)length_penalty;
    // log2(e) / T in two parts, both positive: a logit of -infinity times either is -infinity, never NaN
    const double s = 1.4426950408889634074 / A.temp;
    A.s_hi = nextafterf((float)s, 0.f);
    if ((double)A.s_hi >= s) A.s_hi = nextafterf(A.s_hi, 0.f);
    A.s_lo = (float)(s - (double)A.s_hi);
    A.ws = (char*)workspace; A.batch = batch;
    A.flags = (int*)(A.ws + (size_t)(batch * beams) * A.parts * gr::beam_stride(A.keep));
    A.out_token = out_token; A.out_parent = out_parent; A.out_score = out_score; A.out_length = out_length;
    A.out_done = out_done; A.status = status;
    gr::NvtxRange whole("gr_beam_select");
    const int rc = dtype == GR_F32 ? gr::launch_beam<float>(A, batch, (cudaStream_t)stream)
                                   : gr::launch_beam<__nv_bfloat16>(A, batch, (cudaStream_t)stream);
    if (rc != GR_OK) return rc;
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
