// gr_token_logprobs: log probabilities of given tokens under logit rows, the rows' entropies, and their likeliest tokens.
//
// One pass over a row, by a CTA or by a cluster that shares it.  With s = log2(e) / T rounded to fp32 and y = x s - R, R a whole number that
// follows the warp's largest x s, an element adds e = 2^y to S and e y to U: one FMA, one ex2, an addition and an FMA, two elements at a time
// in fp32, batches in fp64.  Then, with q = s exactly over s rounded,
//   log sum exp(x / T) = ln 2 (R q + log2 S),      entropy = ln 2 (log2 S - q U / S),
// in which nothing cancels (log2 S >= 0 >= U where R is the largest x s), and what the rounding of s leaves is 2^-24 of the mean distance
// from R.  Errors: ex2 2^-22.7, y two roundings of 2^-24 |y|, sums of 8 to 32 terms in fp32: 5e-7 to 2e-6 of a log probability.
// Elements far below R are raised to R - 200 before (their exponentials are 0 either way), so that masked ones, -infinity or the type's lowest
// value, do not make 0 times infinity.  The list of the likeliest is the beam selection's (thresholds from running maxima).
// Rows with a NaN or +infinity leave a sum that is no number; those, and rows whose x s is beyond 2^20, are taken again in fp64.
//
// HBM bounds it in fp32 (1024 rows of 128256, 20 alternatives: 95 us, 84 % of the copy rate); in bf16 (2048 rows of 152064, 8 alternatives: 149 us, 64 %)
// instruction issue and the exponentials' pipe, half of each: 80 instructions for 8 ids of 32 lanes, eight of them exponentials.  A batch ahead in
// registers, with six CTAs per SM for eight, takes 159 (and 124 in fp32), twelve CTAs of 40 registers 183.  Latency bounds few rows (4 of
// 50257: 9.7 us, clusters of eight: a trip to memory, a threshold, the selection, the parts' merge).
#include <math.h>
#include <algorithm>
#include "gr_host.h"
#include "gr_list.cuh"
#include "gr_cache.cuh"

namespace gr {

constexpr int kProbCluster = 8;                // most CTAs that share a row
constexpr float kFarRef = 1048576.f;
constexpr float kFloor = 200.f;                // 2^-200 is 0 in fp32

struct ProbArgs {
    const void* logits; long long ld;
    int V, rows, given, top, keep, team;       // keep: entries of a list; team: CTAs of a row
    float s; double ratio, temp;               // s: log2(e) / T in fp32; ratio: exactly over that
    const int* tokens;
    float* logprob; float* entropy; int* top_token; float* top_logprob; int* status;
};

// what a part of a row tells the first one
struct ProbPart { double sum, mean; float ref; int count, some, pad; };       // some: it has an element that is not masked

template <typename T> struct Floor;
template <> struct Floor<float> {
    // (a NaN stays one)
    __device__ static float of(float x) { return x; }
    __device__ static float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
    __device__ static ulonglong2 raise(const ulonglong2& v, float f) {
        ulonglong2 r;
        r.x = f_pack(max_nan(f_lo(v.x), f), max_nan(f_hi(v.x), f)); r.y = f_pack(max_nan(f_lo(v.y), f), max_nan(f_hi(v.y), f));
        return r;
    }
};
template <> struct Floor<__nv_bfloat16> {
    // (down: what is above the bound stays as it is)
    __device__ static float of(float x) { return __bfloat162float(__float2bfloat16_rd(x)); }
    __device__ static float max_nan(float a, float b) { return Floor<float>::max_nan(a, b); }
    __device__ static unsigned two(unsigned a, unsigned f) { unsigned r; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(f)); return r; }
    __device__ static ulonglong2 raise(const ulonglong2& v, float x) {
        const unsigned f = __float_as_uint(x) & 0xffff0000u | __float_as_uint(x) >> 16;
        ulonglong2 r;
        r.x = (unsigned long long)two((unsigned)(v.x >> 32), f) << 32 | two((unsigned)v.x, f);
        r.y = (unsigned long long)two((unsigned)(v.y >> 32), f) << 32 | two((unsigned)v.y, f);
        return r;
    }
};

// The K largest of the parts' keys, part p in descending order at sh.keys[p GR_MAX_SELECT ...]: a key's rank is its place in its own part and the numbers
// of larger keys in the others, by bisection in all of them at once.  (Only the K places of a part that may be taken: with all 128 of them, as where a
// support is selected, eight parts of five keys took 6 us longer.)
template <class SS, class F>
__device__ __forceinline__ void merge_parts(SS& sh, int parts, int K, F take)
{
    int from = 1;
    while (from < K) from *= 2;
#pragma unroll 1
    for (int e = threadIdx.x; e < parts * K; e += SS::kThr) {
        const int part = e / K, at = e - part * K;
        if (at >= sh.part_cnt[part]) continue;
        const unsigned long long me = sh.keys[part * GR_MAX_SELECT + at];
        int pos[kProbCluster];
#pragma unroll
        for (int p = 0; p < kProbCluster; p++) pos[p] = 0;
#pragma unroll 1
        for (int s = from; s > 0; s >>= 1) {
#pragma unroll
            for (int p = 0; p < kProbCluster; p++)
                if (p < parts && pos[p] + s <= sh.part_cnt[p] && sh.keys[p * GR_MAX_SELECT + pos[p] + s - 1] > me) pos[p] += s;
        }
        int rank = 0;
#pragma unroll
        for (int p = 0; p < kProbCluster; p++) rank += pos[p];
        if (rank < K) take(rank, me);
    }
}

// (sum, mean) of a part moves to the reference `to` at or above its own
__device__ __forceinline__ void move_to(double& sum, double& mean, float ref, float to)
{
    if (sum == 0.0) return;
    const float d = ref - to;
    mean = times_pow2(fma((double)d, sum, mean), d);
    sum = times_pow2(sum, d);
}

// log sum exp((x - shift) / T) and entropy of a row in fp64, by this CTA, shift the row's largest; false: a NaN or +infinity in it.
template <typename T, int NTHR>
__device__ __noinline__ bool row_in_64(const T* x, int V, double temp, double* red, double& shift, double& lse, double& entropy)
{
    const int tid = threadIdx.x;
    auto all = [&](double v, bool largest) {
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) { const double w = __shfl_xor_sync(0xffffffffu, v, o); v = largest ? fmax(v, w) : v + w; }
        __syncthreads();
        if ((tid & 31) == 0) red[tid >> 5] = v;
        __syncthreads();
        double r = red[0];
        for (int w = 1; w < NTHR / 32; w++) r = largest ? fmax(r, red[w]) : r + red[w];
        return r;
    };
    float m = -INFINITY;
    bool wrong = false;
    for (int i = tid; i < V; i += NTHR) {
        const float v = load_logit<T>(x, i);
        if (!(v < INFINITY)) wrong = true;
        m = fmaxf(m, v);
    }
    if (__syncthreads_or(wrong)) return false;
    const double top = all((double)m, true);
    lse = entropy = 0.0;
    if (top == -INFINITY) return true;
    shift = top;
    double sum = 0.0, mean = 0.0;
    for (int i = tid; i < V; i += NTHR) {
        const double d = (top - (double)load_logit<T>(x, i)) / temp, e = d < 700.0 ? exp_neg(d) : 0.0;
        sum += e;
        if (e > 0.0) mean = fma(e, d, mean);
    }
    sum = all(sum, false);
    mean = all(mean, false);
    lse = m_log(sum);
    entropy = lse + mean / sum;
    return true;
}

template <typename T, int U, int NTHR, int CTAS>
__global__ void __launch_bounds__(NTHR, CTAS)
logprobs_kernel(const __grid_constant__ ProbArgs A)
{
    using VT = VecTraits<T>;
    using Sm = BeamSm<NTHR>;
    constexpr int kWarps = NTHR / 32, N = VT::N, S = kChunk / (32 * N), NB = S / U;
    static_assert(S % U == 0, "a chunk is a whole number of batches");
    static_assert(sizeof(((Sm*)0)->keys) >= 8 * kProbCluster * GR_MAX_SELECT || CTAS > 4, "the parts' keys");
    __shared__ Sm sh;
    __shared__ float s_ref[kWarps];
    __shared__ double s_sum[kWarps], s_mean[kWarps];
    __shared__ unsigned long long s_best[GR_MAX_SELECT];
    __shared__ ProbPart s_part[kProbCluster];
    __shared__ double s_lse, s_entropy;
    __shared__ int s_state;
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long row = blockIdx.x / A.team;
    const int part = blockIdx.x % A.team;
    const int V = A.V, K = A.keep;
    const T* x = (const T*)A.logits + row * A.ld;
    const int head = row_head(x, 0, V, (int)sizeof(T));
    const int nch = num_chunks(V, head);
    const int first = part * kWarps, stride = A.team * kWarps;     // this part's chunks: first + warp, + stride, ...
    const bool use_tau = V > Sm::kCap || K == 0;                   // (else every element may be listed)
    const int vec_end = head + ((V - head) / N) * N, tail = V - vec_end;
    if (tid == 0) { sh.cnt = 0; sh.tau = K == 0 ? INFINITY : -3.402823466e38f; sh.reset_checks(); }
    __syncthreads();

    float g0 = -INFINITY, ref = -INFINITY, floor_x = Floor<T>::of(-kFloor / A.s), limit = -INFINITY;
    double acc = 0.0, mean = 0.0;
    const unsigned long long s2 = f_pack(A.s, A.s);
    const int rounds = first < nch ? (nch - first + stride - 1) / stride : 0;
    auto raise = [&](float m) {
        const float to = ceilf(warp_max(m) * A.s);
        move_to(acc, mean, ref, to);
        ref = to;
        limit = (to + 1.f) / A.s;
        if (to > -INFINITY) floor_x = Floor<T>::of((to - kFloor) / A.s);
    };
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
            const float y0 = fmaf(Floor<T>::max_nan(e0, floor_x), A.s, down), y1 = fmaf(Floor<T>::max_nan(e1, floor_x), A.s, down);
            acc = (double)ex2(y0) + (double)ex2(y1);
            mean = (double)(ex2(y0) * y0) + (double)(ex2(y1) * y1);
        }
        if (!use_tau) push_edges(-3.402823466e38f);
    }
    // (thresholds and the list's room as in the beam selection's streaming pass)
    const int A_K = K + K * K / NTHR;
    int r = 0, upto = !use_tau || K == 0 ? rounds : 2 * 4 * NB * A_K <= Sm::kList ? 4 : 1;
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
                const bool sample = use_tau && K > 0 && r == 0 && nb == 0;
                const float tau = sample ? INFINITY : *((volatile float*)&sh.tau);
                ulonglong2 v[U];
                auto batch = [&](auto all) {
#pragma unroll
                    for (int u = 0; u < U; u++) {
                        const int i0 = base + u * 32 * N;
                        v[u].x = VT::kNone; v[u].y = VT::kNone;
                        if (decltype(all)::value || i0 + N <= vec_end) v[u] = ldg_stream(x + i0);
                    }
                    float each[U];
                    each[0] = VT::largest(v[0]);
                    float most = each[0];
#pragma unroll
                    for (int u = 1; u < U; u++) { each[u] = VT::largest(v[u]); most = fmaxf(most, each[u]); }
                    g0 = fmaxf(g0, most);
                    if (__any_sync(0xffffffffu, most > limit)) raise(most);
                    const float down = ref == -INFINITY ? 0.f : -ref;
                    const unsigned long long down2 = f_pack(down, down);
                    unsigned long long sum2 = 0ull, mean2 = 0ull;
#pragma unroll
                    for (int u = 0; u < U; u++) {
                        const ulonglong2 w = Floor<T>::raise(v[u], floor_x);
                        unsigned long long s1 = 0ull, m1 = 0ull;
#pragma unroll
                        for (int i = 0; i < VT::kPairs; i++) {
                            const unsigned long long y = fma2(VT::pair(w, i), s2, down2);
                            const unsigned long long e = f_pack(ex2(f_lo(y)), ex2(f_hi(y)));
                            s1 = i == 0 ? e : add2(s1, e);
                            m1 = i == 0 ? mul2(e, y) : fma2(e, y, m1);
                        }
                        sum2 = u == 0 ? s1 : add2(sum2, s1);
                        mean2 = u == 0 ? m1 : add2(mean2, m1);
                    }
                    acc += (double)(f_lo(sum2) + f_hi(sum2));
                    mean += (double)(f_lo(mean2) + f_hi(mean2));
                    if (most >= tau) {
#pragma unroll
                        for (int u = 0; u < U; u++) if (each[u] >= tau) push_or_stop(sh, v[u], base + u * 32 * N);
                    }
                };
                if (whole) batch(std::true_type());
                else if (cvalid) batch(std::false_type());
                if (sample) {
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
        if (rounds < 2 * r && 2 * (expected * r + A_K * (rounds - r)) < Sm::kList * r) { upto = rounds; continue; }
        const int listed = refine_tau(sh, g0, K);
        expected = min(expected + 3 * A_K, Sm::kList);
        const int more = A_K * min(3 * r, rounds - r);                                    // times r
        if (listed <= Sm::kList && 2 * more > (Sm::kList - listed) * r) keep_listed<T>(sh, listed);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { acc += __shfl_xor_sync(0xffffffffu, acc, o); mean += __shfl_xor_sync(0xffffffffu, mean, o); }
    if (lane == 0) { s_ref[warp] = ref; s_sum[warp] = acc; s_mean[warp] = mean; }
    const int some = __syncthreads_or(g0 > -INFINITY);
    int count = 0;
    if (K > 0) count = best_listed<T>(sh, x, V, head, nch, first, stride, K, use_tau, g0, [&](int rank, unsigned long long key) { s_best[rank] = key; });
    __syncthreads();
    if (tid == 0) {
        float top = s_ref[0];
        for (int w = 1; w < kWarps; w++) top = fmaxf(top, s_ref[w]);
        double sum = 0.0, m = 0.0;
        for (int w = 0; w < kWarps; w++) {
            double a = s_sum[w], b = s_mean[w];
            move_to(a, b, s_ref[w], top);
            sum += a; m += b;
        }
        s_part[0] = ProbPart{sum, m, top, count, some, 0};
    }
    if (A.team > 1) {
        // the parts' sums and keys to the first of them
        cluster_barrier();                     // (its keys are done with, as are all others' own sums)
        if (part > 0) {
            if (tid == 0) {
                const unsigned long long* p = reinterpret_cast<const unsigned long long*>(&s_part[0]);
                const unsigned at = cluster_addr(&s_part[part], 0);
                for (int i = 0; i < (int)(sizeof(ProbPart) / 8); i++) st_cluster(at + 8 * i, p[i]);
            }
            for (int e = tid; e < count; e += NTHR) st_cluster(cluster_addr(&sh.keys, 0) + 8 * (unsigned)(part * GR_MAX_SELECT + e), s_best[e]);
        } else for (int e = tid; e < count; e += NTHR) sh.keys[e] = s_best[e];
        cluster_barrier();
        if (part > 0) return;
        if (K > 0) {
            if (tid < A.team) sh.part_cnt[tid] = s_part[tid].count;
            __syncthreads();
            int listed = 0;
            for (int p = 0; p < A.team; p++) listed += s_part[p].count;
            count = min(K, listed);
            merge_parts(sh, A.team, K, [&](int rank, unsigned long long key) { s_best[rank] = key; });
        }
    }
    __syncthreads();
    if (tid == 0) {
        float top = s_part[0].ref;
        for (int p = 1; p < A.team; p++) top = fmaxf(top, s_part[p].ref);
        double sum = 0.0, m = 0.0;
        bool live = false;
        for (int p = 0; p < A.team; p++) {
            live |= s_part[p].some != 0;
            double a = s_part[p].sum, b = s_part[p].mean;
            move_to(a, b, s_part[p].ref, top);
            sum += a; m += b;
        }
        int state = 0;                         // 1: in fp64, 2: masked as a whole
        // (logits whose products with s overflow leave no reference either: those rows are not masked)
        if (!live && sum == 0.0) state = 2;
        else if (!(fabsf(top) <= kFarRef) || !(sum < INFINITY) || !(A.s > 1e-30f && A.s < 1e30f)) state = 1;
        const double units = log2(sum);
        s_lse = state == 2 ? 0.0 : 0.69314718055994530942 * ((double)top * A.ratio + units);
        s_entropy = state == 2 ? 0.0 : fmax(0.0, 0.69314718055994530942 * (units - A.ratio * (m / sum)));
        s_state = state;
    }
    __syncthreads();
    double shift = 0.0, lse = s_lse, entropy = s_entropy;
    bool good = true;
    if (s_state == 1) good = row_in_64<T, NTHR>(x, V, A.temp, s_sum, shift, lse, entropy);
    // ---- results
    auto logprob_of = [&](float v) { return !good ? NAN : v == -INFINITY ? -INFINITY : (float)(((double)v - shift) / A.temp - lse); };
    for (int i = tid; i < A.given; i += NTHR) {
        const int t = A.tokens[row * A.given + i];
        A.logprob[row * A.given + i] = t >= 0 && t < V ? logprob_of(load_logit<T>(x, t)) : good ? -INFINITY : NAN;
    }
    if (!good) count = 0;
    for (int i = tid; i < A.top; i += NTHR) {
        const bool some = i < count;
        const unsigned long long key = some ? s_best[i] : 0ull;
        A.top_token[row * A.top + i] = some ? (int)(0xffffffffu - (unsigned)key) : -1;
        A.top_logprob[row * A.top + i] = some ? logprob_of(fkey_inv((unsigned)(key >> 32))) : -INFINITY;
    }
    if (tid == 0) {
        if (A.entropy) A.entropy[row] = good ? (float)entropy : NAN;
        A.status[row] = sh.checks() ? GR_CHECK_FAILED : good ? GR_OK : GR_BAD_LOGITS;
    }
}

// CTAs that share a row: as many as there is room for, with a chunk for every other warp at least.
static int prob_team(int V, int rows)
{
    const int chunks = (V + kChunk - 1) / kChunk;
    int team = 1;
    while (team < kProbCluster && 2 * team * 4 <= chunks && rows * team * 2 <= 2 * kSms) team *= 2;
    return team;
}

template <typename T>
static int launch_logprobs(const ProbArgs& A, cudaStream_t st)
{
    // CTAs of 128 threads, eight to an SM, finish a wave of rows sooner than four of 256 (128256 fp32 logits, us: 600 rows 77 for 86, 1184: 102 for 107,
    // 4200: 352 for 369; bf16, 2000: 130 for 139, 4800: 285 for 310), unless they need two waves where those take three (fp32, 1500: 164 for
    // 144), which evens out with more waves (4800: 417 for 416).  In bf16 a wave of twelve to an SM goes before two of eight (1300 rows
    // 97 for 107, 1700: 117 for 119), but not three of them before four (3600: 236 for 224).
    const long long ctas = (long long)A.rows * A.team;
    auto waves = [&](int per) { return (ctas + per * kSms - 1) / (per * kSms); };
    constexpr bool kNarrow = sizeof(T) == 2;
    const bool small = A.keep <= 48 && ctas > 4 * kSms && (kNarrow || ctas > 16 * kSms || 2 * waves(8) <= waves(4));
    cudaError_t rc;
    if (A.team > 1 || ctas <= 2 * kSms) rc = launch_pdl_cluster(A.team, logprobs_kernel<T, kChunk / (32 * VecTraits<T>::N), 256, 2>, (int)ctas, 256, 0, st, A);
    else if (small && kNarrow && waves(12) == 1 && waves(8) == 2) rc = launch_pdl(logprobs_kernel<T, 4, 128, kNarrow ? 12 : 8>, (int)ctas, 128, 0, st, A);
    else if (small) rc = launch_pdl(logprobs_kernel<T, 4, 128, 8>, (int)ctas, 128, 0, st, A);
    else rc = launch_pdl(logprobs_kernel<T, 4, 256, 4>, (int)ctas, 256, 0, st, A);
    return rc == cudaSuccess ? GR_OK : GR_E_LAUNCH;
}

}  // namespace gr

extern "C" {

int gr_token_logprobs(const void* logits, int dtype, int V, long long ld, int rows, float temperature, const int* tokens, int given,
                      int top, float* logprob, float* entropy, int* top_token, float* top_logprob, int* status, void* stream)
{
    if (V < 1 || V > (1 << 21) || rows < 0 || rows > (1 << 26) || (dtype != GR_F32 && dtype != GR_BF16)) return GR_E_INVALID;
    if (!(temperature > 0.f) || !isfinite(temperature) || ld < V || ld > (1ll << 32)) return GR_E_INVALID;
    if (given < 0 || given > GR_MAX_GIVEN || top < 0 || top > GR_MAX_SELECT) return GR_E_INVALID;
    if (rows == 0) return GR_OK;
    if (!logits || (given > 0 && (!tokens || !logprob)) || (top > 0 && (!top_token || !top_logprob))) return GR_E_NULL;
    const int e = gr::type_size(dtype);
    if ((uintptr_t)logits & (uintptr_t)(e - 1)) return GR_E_ALIGN;
    const uintptr_t lists = (given > 0 ? (uintptr_t)tokens | (uintptr_t)logprob : 0) | (top > 0 ? (uintptr_t)top_token | (uintptr_t)top_logprob : 0);
    if ((lists | (uintptr_t)entropy | (uintptr_t)status) & 3) return GR_E_ALIGN;
    // (outputs lie apart from one another and from what is read; the status, looked at last, behind the others)
    const long long step = ld * e, size = rows;
    auto of = [&](const void* p, long long each) { return gr::bytes_at(p, p ? 4 * each * rows : 0); };
    const gr::Places read[2] = {gr::places_of(logits, (long long)V * e, &step, &size, 1), of(tokens, given)};
    const gr::Places written[5] = {of(logprob, given), of(entropy, 1), of(top_token, top), of(top_logprob, top), of(status, 1)};
    for (int i = 0; i < 5; i++) {
        if (i == 4 && !status) return GR_E_NULL;
        for (int j = 0; j < i + 2; j++) if (gr::meet(written[i], j < 2 ? read[j] : written[j - 2])) return GR_E_INVALID;
    }
    gr::ProbArgs A;
    A.logits = logits; A.ld = ld; A.V = V; A.rows = rows; A.given = given; A.top = top; A.keep = std::min(top, V);
    A.team = gr::prob_team(V, rows);
    A.temp = (double)temperature;
    const double s = 1.4426950408889634074 / A.temp;
    A.s = (float)std::min(s, 3e38);
    A.ratio = s / (double)A.s;
    A.tokens = tokens; A.logprob = logprob; A.entropy = entropy; A.top_token = top_token; A.top_logprob = top_logprob; A.status = status;
    gr::NvtxRange whole("gr_token_logprobs");
    const int rc = dtype == GR_F32 ? gr::launch_logprobs<float>(A, (cudaStream_t)stream) : gr::launch_logprobs<__nv_bfloat16>(A, (cudaStream_t)stream);
    if (rc != GR_OK || cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
