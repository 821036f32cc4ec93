// gr_cache_append and gr_cache_read: new tokens' keys and values into a paged cache, rotated by their positions on the way, and out again.
//
// Both move bytes.  A CTA takes the tokens of one window (one token where there are few, for latency; eight or sixteen otherwise) and all
// their heads, so that slots, runs and angles are worked out once: position x frequency in fp64, brought to [-pi / 4, pi / 4] in fp64 (far
// positions lose nothing), sine and cosine by their Taylor series, rounded to fp32 once.  The rotation takes fp32 products and sums
// without contraction, each rounded, so that what is held follows from the formula whatever computes it.
// In a 4-bit cache the unit is the octet: a run of a call's tokens that lie one after another in one octet is taken by one CTA, the
// one whose window its first token is in, so that a prompt's octets are written whole.
//
// Measured (bytes that it cannot do without, against the copy rate): 9000 tokens of 12 ragged prompts, 8 heads and 32 query heads of 128 dims,
// fp16: 38 to 41 us, 82 to 89 %; the same keys and values from bf16 into 4 bits and out of them 49 to 52, where the bytes of both take 14 (9000 tokens without
// ragged ends 29 and 12): instructions bound both, 250 for a row of 128 numbers of two tokens at half of the issue rate.  65536 tokens
// out of 4 bits as bf16: 64 us, 83 %; out of 16 bits 99 and out of 32 171 us, 83 and 96 %.  One token for each of 64 rows: 2.5 us into 16 bits, with
// 32 query heads; 6.4 into 4: latency.
#include <math.h>
#include <algorithm>
#include "gr_host.h"
#include "gr_cache.cuh"

namespace gr {

constexpr int kCacheThreads = 256, kCacheWarps = kCacheThreads / 32;
constexpr int kCacheWindow = 16;               // most tokens of a CTA
constexpr int kCacheSeen = kCacheWindow + 7;   // and those that it looks at
constexpr int kCacheMany = 16 * kSms;          // from so many tokens on

struct CacheArgs {
    char* keys; char* values;
    long long block_stride, token_stride, head_stride;     // elements of the cache (4 bits: bytes, the first only)
    int heads, dim, block, num_blocks, four;
    gr_cache_tokens x;
    int tokens, window, split;                 // split: CTAs that share a window's rows
    const long long* slots; const int* positions; const double* freq;
    int half, interleaved;                     // half: pairs of dims that are rotated
    int team, queries_vec;                     // team: threads of a row
    // whole quotients that loops go on by, and 1 / n for first places (small numbers: exact with a half added)
    int by_half, by_heads, by_queries;
    float of_half, of_heads, of_queries;
    GR_SPAN(in_k); GR_SPAN(in_v); GR_SPAN(in_q); GR_SPAN(out_q); GR_SPAN(held_k); GR_SPAN(held_v);
};

// ---------------------------------------------------------------- angles

// cosine and sine of a, rounded to fp32; NaN from 2^50 on
__device__ __forceinline__ float2 cos_sin(double a)
{
    if ((__double2hiint(a) & 0x7fffffff) >= 0x43100000) a = NAN;
    // (whole numbers by the sum with 1.5 2^52, whose low word they are, up to 2^51: conversions have a fraction of the multiplications' rate)
    const double magic = 6755399441055744.0, whole = fma(a, 0.63661977236758134308, magic), k = whole - magic;     // 2 / pi
    double r = fma(-k, 1.57079632679489655800e+00, a);                      // pi / 2 in two parts
    r = fma(-k, 6.12323399573676603587e-17, r);
    const double z = r * r;
    // Taylor series to r^15 and r^16: below 1e-16 of the value up to pi / 4
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = fma(s, z, 1.0 / 6227020800.0);  c = fma(c, z, -1.0 / 87178291200.0);
    s = fma(s, z, -1.0 / 39916800.0);   c = fma(c, z, 1.0 / 479001600.0);
    s = fma(s, z, 1.0 / 362880.0);      c = fma(c, z, -1.0 / 3628800.0);
    s = fma(s, z, -1.0 / 5040.0);       c = fma(c, z, 1.0 / 40320.0);
    s = fma(s, z, 1.0 / 120.0);         c = fma(c, z, -1.0 / 720.0);
    s = fma(s, z, -1.0 / 6.0);          c = fma(c, z, 1.0 / 24.0);
    s = fma(s * z, r, r);               c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    const int quadrant = __double2loint(whole) & 3;
    const double cq = quadrant & 1 ? s : c, sq = quadrant & 1 ? c : s;
    return make_float2((float)(quadrant == 1 || quadrant == 2 ? -cq : cq), (float)(quadrant >= 2 ? -sq : sq));
}

// A window's tokens, in shared memory: where each goes, and (cos, sin) of its pairs behind that.  Windows of a 4-bit cache look at the
// seven tokens behind them too, which a run that begins in the window may hold.
struct Tokens {
    long long slot[kCacheSeen];
    long long at[kCacheSeen];                  // elements (4 bits: bytes, of the octet) from the cache's beginning to the token's first head; -1: nowhere
    double angle[kCacheSeen];                  // the position, as a factor
    int position[kCacheSeen];
    int runs, first[kCacheWindow], size[kCacheWindow];     // 4 bits: runs that begin in the window, by their first token
};
__device__ __forceinline__ void window_tokens(const CacheArgs& A, Tokens& w, int i0, int n)
{
    const int t = threadIdx.x;
    if (t < n) {
        const long long slot = A.slots[i0 + t];
        const int position = A.positions ? A.positions[i0 + t] : 0;
        w.position[t] = position; w.angle[t] = (double)position;
        w.slot[t] = slot;
        long long at = -1;
        if (slot >= 0 && slot < (long long)A.num_blocks * A.block) {
            // (32 bits divide in a quarter of the time)
            const long long block = slot >> 32 ? slot / A.block : (long long)((unsigned)slot / (unsigned)A.block);
            const int in = (int)(slot - block * A.block);
            at = block * A.block_stride + (A.four ? (long long)(in >> 3) * octet_bytes(A.dim) : in * A.token_stride);
        }
        w.at[t] = at;
    }
    __syncthreads();
}
// Of tokens from..to - 1: cs[token][pairs], with room so that threads eight pairs apart meet different banks.
__host__ __device__ inline int angle_step(int half) { return (half + 1) / 2 * 2 + 2 * ((half + 7) >> 3); }
__device__ __forceinline__ int angle_at(int f) { return f + 2 * (f >> 3); }
__device__ __forceinline__ void window_angles(const CacheArgs& A, const Tokens& w, float2* cs, int from, int to)
{
    if (A.half == 0) return;
    const int step = angle_step(A.half);
    // (a thread's pair and token go on by fixed steps: no divisions in the loop)
    int tok = (int)(((float)threadIdx.x + 0.5f) * A.of_half), f = threadIdx.x - tok * A.half;
    const int by_tok = A.by_half, by_f = kCacheThreads - by_tok * A.half;
    for (tok += from; tok < to;) {
        const float2 turn = cos_sin(w.angle[tok] * A.freq[f]);
        if (GR_WITHIN(shared_span(cs), cs + tok * step + angle_at(f), sizeof(float2))) cs[tok * step + angle_at(f)] = turn;
        tok += by_tok; f += by_f;
        if (f >= A.half) { f -= A.half; tok++; }
    }
    __syncthreads();
}

// a rotated number: x the element itself, y the other of its pair
__device__ __forceinline__ float turned(float x, float y, float2 cs, bool second)
{
    const float p = __fmul_rn(x, cs.x), q = __fmul_rn(y, cs.y);
    return second ? __fadd_rn(p, q) : __fsub_rn(p, q);
}

// N elements as they are held, as numbers and back: 16-bit ones by words of two
template <typename T, int N> struct Raw { T x[N]; };
template <int N> struct Raw<__nv_bfloat16, N> { unsigned w[(N + 1) / 2]; };
template <int N> struct Raw<__half, N> { unsigned w[(N + 1) / 2]; };
template <typename T, int N>
__device__ __forceinline__ Raw<T, N> load_raw(const T* p)
{
    Raw<T, N> r;
    if constexpr (sizeof(T) == 2 && N == 1) r.w[0] = *reinterpret_cast<const unsigned short*>(p);
    else {
        constexpr int kWords = N * (int)sizeof(T) / 4, kEach = kWords < 4 ? kWords : 4;
        unsigned* to = reinterpret_cast<unsigned*>(&r);
#pragma unroll
        for (int i = 0; i < kWords; i += kEach) {
            const Pack<unsigned, kEach> v = *reinterpret_cast<const Pack<unsigned, kEach>*>(reinterpret_cast<const unsigned*>(p) + i);
#pragma unroll
            for (int z = 0; z < kEach; z++) to[i + z] = v.x[z];
        }
    }
    return r;
}
template <int N> __device__ __forceinline__ void unpack(float (&x)[N], const Raw<float, N>& r)
{
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = r.x[i];
}
template <int N> __device__ __forceinline__ void unpack(float (&x)[N], const Raw<__nv_bfloat16, N>& r)
{
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = __uint_as_float(i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
}
template <int N> __device__ __forceinline__ void unpack(float (&x)[N], const Raw<__half, N>& r)
{
#pragma unroll
    for (int i = 0; i < N; i++) {
        const __half2 h = *reinterpret_cast<const __half2*>(&r.w[i / 2]);
        x[i] = i & 1 ? __high2float(h) : __low2float(h);
    }
}
__device__ __forceinline__ unsigned two_of(float a, float b, __nv_bfloat16) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const unsigned*>(&h); }
__device__ __forceinline__ unsigned two_of(float a, float b, __half) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const unsigned*>(&h); }
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&x)[N])
{
    if constexpr (N == 1) *p = from_f32<T>(x[0]);
    else {
        constexpr int kWords = N * (int)sizeof(T) / 4, kEach = kWords < 4 ? kWords : 4;
        unsigned w[kWords];
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
            else w[i] = two_of(x[2 * i], x[2 * i + 1], T());
        }
#pragma unroll
        for (int i = 0; i < kWords; i += kEach) {
            Pack<unsigned, kEach> v;
#pragma unroll
            for (int z = 0; z < kEach; z++) v.x[z] = w[i + z];
            *reinterpret_cast<Pack<unsigned, kEach>*>(reinterpret_cast<unsigned*>(p) + i) = v;
        }
    }
}

// ---------------------------------------------------------------- 16- and 32-bit caches, and queries
//
// A row (token, head) is taken by a team of threads, two pieces of N elements each to a thread: where pairs are halves apart
// a piece and its partners, so that both are read before either is written and queries can be rotated in place; else two pieces anywhere.
// N is 8 where both sides have 16 bits and everything is aligned to 16 bytes, 4 where it is to four elements, else 1.

struct Pieces { int c0, c1, turn; };           // turn: 0 not, 1 one with the other, 2 neighbours within a piece
template <int N>
__device__ __forceinline__ Pieces pieces_of(int e, int D, int half, bool interleaved)
{
    if (interleaved) return N > 1 ? Pieces{e * N, D / 2 + e * N, 2} : Pieces{2 * e, 2 * e + 1, e < half ? 1 : 0};
    const int turned = half / N;
    if (e < turned) return Pieces{e * N, e * N + half, 1};
    return Pieces{2 * half + (e - turned) * N, half + D / 2 + (e - turned) * N, 0};
}

// (cs: of the token)
template <int N>
__device__ __forceinline__ void turn_pieces(float (&a)[N], float (&b)[N], const Pieces& p, const float2* cs, int half, bool interleaved)
{
    if (p.turn == 1) {
        // (N pairs from a multiple of N on: next to one another)
        const float2* at = cs + angle_at(interleaved ? p.c0 / 2 : p.c0);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float4 t = N > 1 ? *reinterpret_cast<const float4*>(at + i) : make_float4(at[i].x, at[i].y, 0.f, 0.f);
            const float x = a[i], y = b[i];
            a[i] = turned(x, y, make_float2(t.x, t.y), false); b[i] = turned(y, x, make_float2(t.x, t.y), true);
            if (N > 1) {
                const float x1 = a[i + (N > 1)], y1 = b[i + (N > 1)];
                a[i + (N > 1)] = turned(x1, y1, make_float2(t.z, t.w), false); b[i + (N > 1)] = turned(y1, x1, make_float2(t.z, t.w), true);
            }
        }
    } else if (p.turn == 2) {
        const float2 *at = cs + angle_at(p.c0 / 2), *bt = cs + angle_at(p.c1 / 2);
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            if (p.c0 + i < 2 * half) {
                const float2 t = at[i / 2];
                const float x = a[i], y = a[i + 1];
                a[i] = turned(x, y, t, false); a[i + 1] = turned(y, x, t, true);
            }
            if (p.c1 + i < 2 * half) {
                const float2 t = bt[i / 2];
                const float x = b[i], y = b[i + 1];
                b[i] = turned(x, y, t, false); b[i + 1] = turned(y, x, t, true);
            }
        }
    }
}

// The rows of a window's tokens: keys and values (but for a 4-bit cache, whose queries alone come here), queries.  A team takes a row (a
// head of keys, values or queries) of two tokens at a time; rows and pairs of tokens go on by fixed steps, without divisions.  With kEarly
// what a team reads first, which depends on neither slots nor angles, is under way while `before` (the window's prologue) runs: for few tokens, where
// that is a trip to memory less; where there are many, those without a place are not read.
template <typename T, typename C, int N, bool kQueries, bool kEarly, class F>
__device__ __forceinline__ void append_rows(const CacheArgs& A, const Tokens& w, const float2* cs, int i0, int n, int part, F before)
{
    constexpr int kTok = kEarly ? 1 : 2;
    const int D = A.dim, chunks = D / (2 * N), team = A.team, in_team = threadIdx.x & (team - 1), teams = kCacheThreads / team;
    const int kv = kQueries ? 0 : 2 * A.heads, per = kv + A.x.q_heads, stride = A.split * teams, step = angle_step(A.half);
    const int by_tok = stride / per, by_row = stride - by_tok * per;
    int row = part * teams + threadIdx.x / team, tok = row / per;
    row -= tok * per;
    tok *= kTok;
    bool early = kEarly;
    do {
        // (a row's kind, and where it begins)
        const bool live = tok < n, values = row >= A.heads && row < kv, queries = row >= kv;
        const int head = queries ? row - kv : values ? row - A.heads : row, half = values ? 0 : A.half;
        const bool interleaved = !values && A.interleaved;
        const long long src_step = queries ? A.x.q_token : values ? A.x.v_token : A.x.k_token;
        const T* src = (const T*)(queries ? A.x.q : values ? A.x.v : A.x.k) + (long long)head * (queries ? A.x.q_head : values ? A.x.v_head : A.x.k_head) + (i0 + tok) * src_step;
        for (int e = in_team; e < chunks || early; e += team) {
            const Pieces p = pieces_of<N>(e, D, half, interleaved);
            Raw<T, N> a[kTok], b[kTok];
            bool some[kTok];
#pragma unroll
            for (int u = 0; u < kTok; u++) {
                some[u] = tok + u < n && e < chunks && (early || (queries ? w.position[tok + u] >= 0 : w.at[tok + u] >= 0));
                some[u] = some[u] && GR_WITHIN(queries ? A.in_q : values ? A.in_v : A.in_k, src + u * src_step + p.c0, N * sizeof(T))
                          && GR_WITHIN(queries ? A.in_q : values ? A.in_v : A.in_k, src + u * src_step + p.c1, N * sizeof(T));
                if (some[u]) { a[u] = load_raw<T, N>(src + u * src_step + p.c0); b[u] = load_raw<T, N>(src + u * src_step + p.c1); }
            }
            if (early) {
                before();
                early = false;
                if (live) some[0] = some[0] && (queries ? w.position[tok] >= 0 : w.at[tok] >= 0);
            }
#pragma unroll
            for (int u = 0; u < kTok; u++) {
                if (!some[u]) continue;
                float x[N], y[N];
                unpack(x, a[u]); unpack(y, b[u]);
                if (half > 0 && !GR_WITHIN(shared_span(cs), cs + (tok + u) * step, step * sizeof(float2))) continue;
                turn_pieces<N>(x, y, p, cs + (tok + u) * step, half, interleaved);
                if (queries) {
                    T* to = (T*)A.x.q_out + (long long)head * A.x.out_head + (i0 + tok + u) * A.x.out_token;
                    if (GR_WITHIN(A.out_q, to + p.c0, N * sizeof(T)) && GR_WITHIN(A.out_q, to + p.c1, N * sizeof(T))) { store_n<T, N>(to + p.c0, x); store_n<T, N>(to + p.c1, y); }
                } else {
                    C* to = (C*)(values ? A.values : A.keys) + (long long)head * A.head_stride + w.at[tok + u];
                    if (GR_WITHIN(values ? A.held_v : A.held_k, to + p.c0, N * sizeof(C)) && GR_WITHIN(values ? A.held_v : A.held_k, to + p.c1, N * sizeof(C))) {
                        store_n<C, N>(to + p.c0, x); store_n<C, N>(to + p.c1, y);
                    }
                }
            }
        }
        tok += kTok * by_tok; row += by_row;
        if (row >= per) { row -= per; tok += kTok; }
    } while (tok < n);
}

// Rows of one kind (keys, values or queries) of a window of many tokens, two tokens of a head at a time by a team.
template <typename T, typename C, int N, bool kCache, bool kTurn>
__device__ __forceinline__ void append_kind(const CacheArgs& A, const Tokens& w, const float2* cs, int i0, int n, int part, const T* src, int src_token, int src_head,
                                            C* dst, long long dst_token, long long dst_head, int heads, int by_pair, float of_heads)
{
    const int D = A.dim, chunks = D / (2 * N), team = A.team, in_team = threadIdx.x & (team - 1), teams = kCacheThreads / team, stride = A.split * teams;
    const int half = kTurn ? A.half : 0, step = angle_step(half);
    const bool interleaved = kTurn && A.interleaved;
    const int by_head = stride - by_pair * heads;
    int head = part * teams + threadIdx.x / team, tok = (int)(((float)head + 0.5f) * of_heads);
    head -= tok * heads;
    tok *= 2;
    for (; tok < n; tok += 2 * by_pair, head += by_head) {
        if (head >= heads) { head -= heads; tok += 2; if (tok >= n) break; }
        const T* from = src + (long long)head * src_head + (long long)(i0 + tok) * src_token;
        C* to = dst + (long long)head * dst_head;
        for (int e = in_team; e < chunks; e += team) {
            const Pieces p = pieces_of<N>(e, D, half, interleaved);
            Raw<T, N> a[2], b[2];
            bool some[2];
            long long at[2];
#pragma unroll
            for (int u = 0; u < 2; u++) {
                some[u] = tok + u < n;
                if (some[u]) {
                    at[u] = kCache ? w.at[tok + u] : (long long)(i0 + tok + u) * dst_token;
                    some[u] = kCache ? at[u] >= 0 : w.position[tok + u] >= 0;
                }
                some[u] = some[u] && GR_WITHIN(kCache ? (kTurn ? A.in_k : A.in_v) : A.in_q, from + u * src_token + p.c0, N * sizeof(T))
                          && GR_WITHIN(kCache ? (kTurn ? A.in_k : A.in_v) : A.in_q, from + u * src_token + p.c1, N * sizeof(T));
                if (some[u]) { a[u] = load_raw<T, N>(from + u * src_token + p.c0); b[u] = load_raw<T, N>(from + u * src_token + p.c1); }
            }
#pragma unroll
            for (int u = 0; u < 2; u++) {
                if (!some[u]) continue;
                float x[N], y[N];
                unpack(x, a[u]); unpack(y, b[u]);
                if (half > 0 && !GR_WITHIN(shared_span(cs), cs + (tok + u) * step, step * sizeof(float2))) continue;
                if (kTurn) turn_pieces<N>(x, y, p, cs + (tok + u) * step, half, interleaved);
                if (GR_WITHIN(kCache ? (kTurn ? A.held_k : A.held_v) : A.out_q, to + at[u] + p.c0, N * sizeof(C))
                    && GR_WITHIN(kCache ? (kTurn ? A.held_k : A.held_v) : A.out_q, to + at[u] + p.c1, N * sizeof(C))) {
                    store_n<C, N>(to + at[u] + p.c0, x); store_n<C, N>(to + at[u] + p.c1, y);
                }
            }
        }
    }
}

template <typename T, typename C, int N, bool kFew>
__global__ void __launch_bounds__(kCacheThreads, 4)
append_kernel(const __grid_constant__ CacheArgs A)
{
    extern __shared__ __align__(16) float2 cs[];
    __shared__ Tokens w;
    pdl_wait();
    const int i0 = blockIdx.x * A.window, n = min(A.window, A.tokens - i0);
    auto prologue = [&] { window_tokens(A, w, i0, n); window_angles(A, w, cs, 0, n); };
    if (!kFew) {
        prologue();
        const gr_cache_tokens& x = A.x;
        append_kind<T, C, N, true, true>(A, w, cs, i0, n, blockIdx.y, (const T*)x.k, (int)x.k_token, (int)x.k_head, (C*)A.keys, 0, A.head_stride, A.heads, A.by_heads, A.of_heads);
        append_kind<T, C, N, true, false>(A, w, cs, i0, n, blockIdx.y, (const T*)x.v, (int)x.v_token, (int)x.v_head, (C*)A.values, 0, A.head_stride, A.heads, A.by_heads, A.of_heads);
        if (x.q_heads > 0)
            append_kind<T, T, N, false, true>(A, w, cs, i0, n, blockIdx.y, (const T*)x.q, (int)x.q_token, (int)x.q_head, (T*)x.q_out, x.out_token, x.out_head, x.q_heads, A.by_queries, A.of_queries);
    } else append_rows<T, C, N, false, true>(A, w, cs, i0, n, blockIdx.y, prologue);
}

// ---------------------------------------------------------------- a 4-bit cache

// The runs that begin in a window of n tokens, of m that are looked at: tokens i, i + 1, ... that lie one after another in one octet, i the
// window's first where the one before has no such run.
__device__ __forceinline__ void window_runs(const CacheArgs& A, Tokens& w, int i0, int n, int m)
{
    if (threadIdx.x < 32) {
        const int t = threadIdx.x;
        bool begins = false;
        int size = 0;
        if (t < n && w.at[t] >= 0) {
            const long long slot = w.slot[t];
            const int in = (int)(slot & 7);
            begins = in == 0 || (t > 0 ? w.slot[t - 1] != slot - 1 : i0 == 0 || A.slots[i0 - 1] != slot - 1);
            size = 1;
            while (size < 8 - in && t + size < m && w.slot[t + size] == slot + size) size++;
        }
        const unsigned mask = __ballot_sync(0xffffffffu, begins);
        if (begins) {
            const int k = __popc(mask & ((1u << t) - 1u));
            w.first[k] = t; w.size[k] = size;
        }
        if (t == 0) w.runs = __popc(mask);
    }
    __syncthreads();
}

// The word of codes of eight dims x (as pairs) of a group of four lanes, and the group's scale: that of the element of largest magnitude
// (the positive one of two), for which the code is 0, that is -8, as fp16.  A group with a NaN or an infinity gets the scale NaN.
__device__ __forceinline__ unsigned quantise(const unsigned long long (&x)[4], unsigned& scale)
{
    // (a NaN stays the largest; magnitudes order as their bits, the sign goes below them)
    float hi = f_lo(x[0]), lo = hi;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(hi) : "f"(f_lo(x[i])), "f"(f_hi(x[i])));
        asm("min.f32 %0, %0, %1, %2;" : "+f"(lo) : "f"(f_lo(x[i])), "f"(f_hi(x[i])));
    }
    const float peak = -lo > hi ? lo : hi;
    unsigned most = __funnelshift_l(~__float_as_uint(peak), __float_as_uint(peak), 1);
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const bool met = most >= 0xff000000u;
    const __half h = __float2half_rn(fminf(__uint_as_float(most >> 1) * 0.125f, 65504.f));
    scale = met ? 0x7fffu : (unsigned)__half_as_ushort(h) | (most & 1) << 15;
    if (met || (scale & 0x7fffu) == 0) return 0x88888888u;
    const float s = __half2float(__ushort_as_half((unsigned short)scale));
    float inverse;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(s));
    // The whole number w nearest to x / s by the approximate quotient (8 is added in units of the sum's last place), or one next to that: x - w s is
    // exact in one fused operation, and where it is more than half of s, or half of it and w odd, its sign says which.
    const float magic = 12582912.f + 8.f, half = 0.5f * fabsf(s);
    const unsigned long long inverse2 = f_pack(inverse, inverse), magic2 = f_pack(magic, magic), s2 = f_pack(-s, -s), back2 = f_pack(-magic, -magic);
    constexpr int kZero = 0x4b400000, kZeros = (int)(0x4b400000u * 0x11111111u);      // the bits of 12582912, in code and in eight of them
    int code[8];                               // and kZero
    unsigned long long left[4];
    float most_left = 0.f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned long long y = fma2(x[i], inverse2, magic2);
        left[i] = fma2(add2(y, back2), s2, x[i]);
        asm("max.abs.f32 %0, %0, %1, %2;" : "+f"(most_left) : "f"(f_lo(left[i])), "f"(f_hi(left[i])));
        code[2 * i] = (int)(unsigned)y;
        code[2 * i + 1] = (int)(unsigned)(y >> 32);
    }
    // (fp16 scales below 2^-14 are so coarse that quotients below -8 come up, and where the scale is clamped they are as small as elements are large)
    if (most_left >= half || (scale & 0x7c00u) == 0 || (scale & 0x7fffu) == 0x7bffu) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float r = i & 1 ? f_hi(left[i / 2]) : f_lo(left[i / 2]);
            if (fabsf(r) > half || (fabsf(r) == half && (code[i] & 1))) code[i] += (r < 0.f) != (s < 0.f) ? -1 : 1;
            code[i] = max(code[i], kZero);
        }
    }
    unsigned w = (unsigned)min(code[7], kZero + 15);
#pragma unroll
    for (int i = 6; i >= 0; i--) w = w * 16u + (unsigned)min(code[i], kZero + 15);
    return w - (unsigned)kZeros;
}

// x cos + y sin of two elements next to one another and their partners (sin of the sign that the elements' side of the pairs has), each product and sum
// rounded by itself.  (Not in packed arithmetic: the assembler joins mul.rn.f32x2 and add.rn.f32x2 to one operation that rounds once.)
__device__ __forceinline__ unsigned long long turned2(unsigned long long x, unsigned long long y, float c0, float s0, float c1, float s1)
{
    return f_pack(__fadd_rn(__fmul_rn(f_lo(x), c0), __fmul_rn(f_lo(y), s0)), __fadd_rn(__fmul_rn(f_hi(x), c1), __fmul_rn(f_hi(y), s1)));
}

template <typename T, bool kVec>
__global__ void __launch_bounds__(kCacheThreads, 4)
append4_kernel(const __grid_constant__ CacheArgs A)
{
    extern __shared__ __align__(16) float2 cs[];
    __shared__ Tokens w;
    pdl_wait();
    const int w0 = blockIdx.x * A.window, wn = min(A.window, A.tokens - w0), wm = min(A.window + 7, A.tokens - w0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = A.dim, J = D / 32, half = A.half;
    window_tokens(A, w, w0, wm);
    window_runs(A, w, w0, wn, wm);
    // (the tokens of the runs, and of the queries)
    if (w.runs > 0 || A.x.q_heads > 0) {
        const int last = w.runs > 0 ? w.first[w.runs - 1] + w.size[w.runs - 1] : 0;
        window_angles(A, w, cs, A.x.q_heads > 0 ? 0 : w.first[0], A.x.q_heads > 0 ? max(last, wn) : last);
    }
    const long long head_bytes = (long long)(A.block >> 3) * octet_bytes(D);
    // Of each run a head's keys or values by warps, a pair of the octet's places by each of four, a token of the pair by half a warp, eight dims
    // by a lane: a word of keys; of values two half words, of which the two tokens' lanes exchange one, so that each writes a word.
    const int mine = lane >> 4, l = lane & 15, o0 = 2 * (warp & 3);
    for (int run = 0; run < w.runs; run++) {
        const int tok = w.first[run], n = w.size[run], first = (int)(w.slot[tok] & 7), at = tok + o0 - first + mine;      // at: this half warp's token in the window
        if (o0 + 1 < first || o0 >= first + n) continue;
        const bool has = o0 + mine >= first && o0 + mine < first + n, both = o0 >= first && o0 + 1 < first + n;
        const float2* angle = cs + at * angle_step(half);
        const int every = 2 * A.split, from = 2 * blockIdx.y + (warp >> 2);
        for (int c0 = 0; c0 < D; c0 += 128) {
            const int c = c0 + 8 * l, j = c >> 5, t = l & 3;
            const bool in = c < D && has;
            // ---- keys
            {
                const T* row = (const T*)A.x.k + (long long)from * A.x.k_head + (long long)(w0 + at) * A.x.k_token;
                char* octet = A.keys + w.at[tok] + from * head_bytes;
                const bool turns = in && c < 2 * half, two = c >= half, pairs = turns && kVec && !A.interleaved;
                const int other = two ? c - half : c + half;
                const float sign = two ? 1.f : -1.f;
                Raw<T, 8> x_next, y_next;
                if (kVec && in && from < A.heads) { if (GR_WITHIN(A.in_k, row + c, 8 * sizeof(T))) x_next = load_raw<T, 8>(row + c); if (pairs && GR_WITHIN(A.in_k, row + other, 8 * sizeof(T))) y_next = load_raw<T, 8>(row + other); }
                for (int head = from; head < A.heads; head += every) {
                    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    unsigned long long x2[4];
                    const T* here = row;
                    row += (long long)every * A.x.k_head;
                    if (in && (kVec || GR_WITHIN(A.in_k, here, D * sizeof(T))) && (half == 0 || GR_WITHIN(shared_span(cs), angle, angle_step(half) * sizeof(float2)))) {
                        if (kVec) {
                            // (a head ahead)
                            const Raw<T, 8> x_raw = x_next, y_raw = y_next;
                            if (head + every < A.heads) { if (GR_WITHIN(A.in_k, row + c, 8 * sizeof(T))) x_next = load_raw<T, 8>(row + c); if (pairs && GR_WITHIN(A.in_k, row + other, 8 * sizeof(T))) y_next = load_raw<T, 8>(row + other); }
                            unpack(x, x_raw);
                            if (pairs) {
                                // (the eight are on one side of their pairs: a difference is a sum with a number of the other sign)
                                float y[8];
                                unpack(y, y_raw);
                                const float4* z = reinterpret_cast<const float4*>(angle + angle_at(two ? c - half : c));
#pragma unroll
                                for (int i = 0; i < 8; i += 2) {
                                    const float4 q = z[i / 2];
                                    const unsigned long long r = turned2(f_pack(x[i], x[i + 1]), mul2(f_pack(y[i], y[i + 1]), f_pack(sign, sign)), q.x, q.y, q.z, q.w);
                                    x[i] = f_lo(r); x[i + 1] = f_hi(r);
                                }
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; i++) x[i] = to_f32(here[c + i]);
                        }
                        if (turns && A.interleaved) {
#pragma unroll
                            for (int i = 0; i < 8; i += 2) {
                                if (c + i >= 2 * half) continue;
                                const float2 z = angle[angle_at((c + i) >> 1)];
                                const float a = x[i], b = x[i + 1];
                                x[i] = turned(a, b, z, false); x[i + 1] = turned(b, a, z, true);
                            }
                        } else if (turns && !kVec) {
#pragma unroll
                            for (int i = 0; i < 8; i++) {
                                const int d = c + i;
                                if (d < 2 * half) x[i] = turned(x[i], to_f32(here[d < half ? d + half : d - half]), angle[angle_at(d >= half ? d - half : d)], d >= half);
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) x2[i] = f_pack(x[2 * i], x[2 * i + 1]);
                    unsigned scale;
                    const unsigned code = quantise(x2, scale);
                    if (in && GR_WITHIN(A.held_k, octet, octet_bytes(D))) {
                        *(unsigned*)(octet + (o0 + mine) * (D / 2) + (t * J + j) * 4) = code;
                        if (t == 0) *(unsigned short*)(octet + octet_kscale(D) + ((o0 + mine) * J + j) * 2) = (unsigned short)scale;
                    }
                    octet += every * head_bytes;
                }
            }
            // ---- values
            {
                const T* row = (const T*)A.x.v + (long long)from * A.x.v_head + (long long)(w0 + at) * A.x.v_token;
                char* octet = A.keys + w.at[tok] + from * head_bytes;
                Raw<T, 8> x_next;
                if (kVec && in && from < A.heads && GR_WITHIN(A.in_v, row + c, 8 * sizeof(T))) x_next = load_raw<T, 8>(row + c);
                for (int head = from; head < A.heads; head += every) {
                    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    const T* here = row;
                    row += (long long)every * A.x.v_head;
                    if (in && (kVec || GR_WITHIN(A.in_v, here, D * sizeof(T)))) {
                        if (kVec) {
                            const Raw<T, 8> x_raw = x_next;
                            if (head + every < A.heads && GR_WITHIN(A.in_v, row + c, 8 * sizeof(T))) x_next = load_raw<T, 8>(row + c);
                            unpack(x, x_raw);
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; i++) x[i] = to_f32(here[c + i]);
                        }
                    }
                    unsigned long long x2[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) x2[i] = f_pack(x[2 * i], x[2 * i + 1]);
                    unsigned scale;
                    const unsigned code = quantise(x2, scale), other = __shfl_xor_sync(0xffffffffu, code, 16);
                    // half words 2 t and 2 t + 1 of this token: the first token's lane writes the former of both, the second's the latter
                    char* to = octet + octet_vcode(D) + (((2 * t + mine) * 4 + (o0 >> 1)) * J + j) * 4;
                    const bool writes = in && GR_WITHIN(A.held_k, octet, octet_bytes(D));
                    if (both) {
                        if (writes) *(unsigned*)to = mine ? __byte_perm(other, code, 0x7632) : __byte_perm(code, other, 0x5410);
                    } else if (writes) {
                        char* own = octet + octet_vcode(D) + ((2 * t * 4 + (o0 >> 1)) * J + j) * 4 + 2 * mine;
                        *(unsigned short*)own = (unsigned short)code;
                        *(unsigned short*)(own + 16 * J) = (unsigned short)(code >> 16);
                    }
                    if (writes && t == 0) *(unsigned short*)(octet + octet_vscale(D) + ((o0 >> 1) * J + j) * 4 + 2 * mine) = (unsigned short)scale;
                    octet += every * head_bytes;
                }
            }
        }
    }
    if (A.x.q_heads > 0) {
        if (A.queries_vec) append_rows<T, T, 4, true, false>(A, w, cs, w0, wn, blockIdx.y, [] {});
        else append_rows<T, T, 1, true, false>(A, w, cs, w0, wn, blockIdx.y, [] {});
    }
}

// ---------------------------------------------------------------- reading

struct ReadArgs {
    CacheArgs c;                               // the cache, tokens, window, split, slots, team
    void* k; void* v;
    long long k_token, k_head, v_token, v_head;
};

template <typename C, typename T, int N>
__global__ void __launch_bounds__(kCacheThreads)
read_kernel(const __grid_constant__ ReadArgs R)
{
    constexpr int kRows = 4;
    __shared__ Tokens w;
    const CacheArgs& A = R.c;
    pdl_wait();
    const int i0 = blockIdx.x * A.window, n = min(A.window, A.tokens - i0), D = A.dim;
    const int chunks = D / N, team = A.team, in_team = threadIdx.x & (team - 1), teams = kCacheThreads / team, per = 2 * A.heads, total = n * per;
    window_tokens(A, w, i0, n);
    const float by_per = 1.f / (float)per;
    for (int r0 = blockIdx.y * teams + threadIdx.x / team; r0 < total; r0 += kRows * A.split * teams) {
        const C* src[kRows];
        T* dst[kRows];
        bool second[kRows];
#pragma unroll
        for (int u = 0; u < kRows; u++) {
            const int r = r0 + u * A.split * teams;
            src[u] = nullptr; dst[u] = nullptr; second[u] = false;
            if (r >= total) continue;
            const int tok = (int)(((float)r + 0.5f) * by_per), row = r - tok * per;
            second[u] = row >= A.heads;
            const int head = second[u] ? row - A.heads : row;
            const long long i = i0 + tok;
            dst[u] = second[u] ? (T*)R.v + i * R.v_token + head * R.v_head : (T*)R.k + i * R.k_token + head * R.k_head;
            if (w.at[tok] >= 0) src[u] = (const C*)(second[u] ? A.values : A.keys) + w.at[tok] + head * A.head_stride;
        }
        for (int e = in_team; e < chunks; e += team) {
            Raw<C, N> x[kRows];
#pragma unroll
            for (int u = 0; u < kRows; u++)
                if (src[u] && (GR_WITHIN(second[u] ? A.held_v : A.held_k, src[u] + e * N, N * sizeof(C)))) x[u] = load_raw<C, N>(src[u] + e * N);
#pragma unroll
            for (int u = 0; u < kRows; u++) {
                if (!dst[u]) continue;
                float y[N];
                unpack(y, x[u]);
#pragma unroll
                for (int i = 0; i < N; i++) y[i] = src[u] ? y[i] : 0.f;
                if (GR_WITHIN(second[u] ? A.in_v : A.in_k, dst[u] + e * N, N * sizeof(T))) store_n<T, N>(dst[u] + e * N, y);
            }
        }
    }
}

template <int J, typename W>
__device__ __forceinline__ void load_run(W (&w)[J], const W* p)        // J words, aligned to all of them as far as J is even
{
    constexpr int N = J % 4 == 0 ? 4 : J % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < J; i += N) {
        const Pack<W, N> v = *reinterpret_cast<const Pack<W, N>*>(p + i);
#pragma unroll
        for (int z = 0; z < N; z++) w[i + z] = v.x[z];
    }
}

// Of a run of an octet a warp takes a head: a lane the words of token lane / 4 (keys) and of a pair of tokens (values).  s (u - 8) is
// 16 s (1 + u / 16) - 24 s, u put into the fraction of 1: exact before its one rounding.
template <typename T, int J, bool kVec>
__device__ __forceinline__ void read_octet(const char* octet, T* k, T* v, long long k_step, long long v_step, int first, int n, int lane)
{
    constexpr int D = 32 * J;
    const int g = lane >> 2, t = lane & 3;
    unsigned kw[J], vw[J], vs[J];
    unsigned short ks[J];
    load_run<J>(kw, (const unsigned*)octet + lane * J);
    load_run<J>(vw, (const unsigned*)(octet + octet_vcode(D)) + lane * J);
    load_run<J>(ks, (const unsigned short*)(octet + octet_kscale(D)) + g * J);
    load_run<J>(vs, (const unsigned*)(octet + octet_vscale(D)) + t * J);
    auto number = [](unsigned word, int place, float s16, float s24) {       // the code at bits `place` .. + 3
        const unsigned b = place < 19 ? word << (19 - place) : word >> (place - 19);
        return fmaf(__uint_as_float(b & 0x00780000u | 0x3f800000u), s16, s24);
    };
    if (g >= first && g < first + n) {
        T* to = k + (long long)(g - first) * k_step + 8 * t;
#pragma unroll
        for (int j = 0; j < J; j++) {
            const float s = __half2float(__ushort_as_half(ks[j])), s16 = 16.f * s, s24 = -24.f * s;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = number(kw[j], 4 * i, s16, s24);
            if (kVec) store_n<T, 8>(to + 32 * j, x);
            else {
#pragma unroll
                for (int i = 0; i < 8; i++) to[32 * j + i] = from_f32<T>(x[i]);
            }
        }
    }
#pragma unroll
    for (int z = 0; z < 2; z++) {
        const int tok = 2 * t + z;
        if (tok < first || tok >= first + n) continue;
        T* to = v + (long long)(tok - first) * v_step + 4 * g;
#pragma unroll
        for (int j = 0; j < J; j++) {
            const float s = __half2float(__ushort_as_half((unsigned short)(vs[j] >> (16 * z)))), s16 = 16.f * s, s24 = -24.f * s;
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; i++) x[i] = number(vw[j], 16 * z + 4 * i, s16, s24);
            if (kVec) store_n<T, 4>(to + 32 * j, x);
            else {
#pragma unroll
                for (int i = 0; i < 4; i++) to[32 * j + i] = from_f32<T>(x[i]);
            }
        }
    }
}

template <typename T, int J, bool kVec>
__global__ void __launch_bounds__(kCacheThreads)
read4_kernel(const __grid_constant__ ReadArgs R)
{
    const CacheArgs& A = R.c;
    __shared__ Tokens w;
    pdl_wait();
    const int w0 = blockIdx.x * A.window, wn = min(A.window, A.tokens - w0), wm = min(A.window + 7, A.tokens - w0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int D = 32 * J;
    window_tokens(A, w, w0, wm);
    window_runs(A, w, w0, wn, wm);
    const long long head_bytes = (long long)(A.block >> 3) * octet_bytes(D);
    for (int item = blockIdx.y * kCacheWarps + warp; item < w.runs * A.heads; item += A.split * kCacheWarps) {
        const int run = item / A.heads, head = item - run * A.heads, tok = w.first[run];
        const long long i = w0 + tok;
        if (!GR_WITHIN(A.held_k, A.keys + w.at[tok] + head * head_bytes, octet_bytes(D))) continue;
        if (!GR_WITHIN(A.in_k, (T*)R.k + i * R.k_token + head * R.k_head, ((w.size[run] - 1) * R.k_token + D) * sizeof(T))) continue;
        if (!GR_WITHIN(A.in_v, (T*)R.v + i * R.v_token + head * R.v_head, ((w.size[run] - 1) * R.v_token + D) * sizeof(T))) continue;
        read_octet<T, J, kVec>(A.keys + w.at[tok] + head * head_bytes, (T*)R.k + i * R.k_token + head * R.k_head, (T*)R.v + i * R.v_token + head * R.v_head,
                               R.k_token, R.v_token, (int)(w.slot[tok] & 7), w.size[run], lane);
    }
    // (no place: zeros)
    const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int tok = 0; tok < wn; tok++) {
        if (w.at[tok] >= 0) continue;
        const long long i = w0 + tok;
        for (int row = blockIdx.y * kCacheWarps + warp; row < 2 * A.heads; row += A.split * kCacheWarps) {
            T* to = row < A.heads ? (T*)R.k + i * R.k_token + row * R.k_head : (T*)R.v + i * R.v_token + (row - A.heads) * R.v_head;
            if (!GR_WITHIN(row < A.heads ? A.in_k : A.in_v, to, D * sizeof(T))) continue;
            if (kVec) { if (8 * lane < D) store_n<T, 8>(to + 8 * lane, none); }
            else for (int d = lane; d < D; d += 32) to[d] = from_f32<T>(0.f);
        }
    }
}

// ---------------------------------------------------------------- host

int check_cache(const void* keys, const void* values, const gr_cache_layout* layout)
{
    if (!layout) return GR_E_NULL;
    const gr_cache_layout& L = *layout;
    const bool four = L.format == GR_Q4;
    if (!four && !known_type(L.format)) return GR_E_INVALID;
    if (L.heads < 1 || L.heads > GR_MAX_HEADS || L.block_size < 1 || L.num_blocks < 0) return GR_E_INVALID;
    if (L.dim < 2 || L.dim % 2 || L.dim > GR_MAX_DIM) return GR_E_INVALID;
    if (four) {
        if (L.dim % 32 || L.dim > GR_MAX_DIM_Q4 || L.block_size % 8) return GR_E_INVALID;
        const long long size = (long long)L.heads * (L.block_size / 8) * octet_bytes(L.dim);
        if (L.block_stride < size || L.block_stride % 16 || L.block_stride > (1ll << 58) / std::max(1, L.num_blocks)) return GR_E_INVALID;
    } else {
        const long long step[3] = {L.block_stride, L.token_stride, L.head_stride}, size[3] = {L.num_blocks, L.block_size, L.heads};
        if (!apart(L.dim, step, size, 3)) return GR_E_INVALID;
    }
    if (L.num_blocks == 0) return GR_OK;
    if (!keys || (!four && !values)) return GR_E_NULL;
    const uintptr_t mask = four ? 15 : type_size(L.format) - 1;
    if (((uintptr_t)keys & mask) || (!four && ((uintptr_t)values & mask))) return GR_E_ALIGN;
    return GR_OK;
}

// How a call's tokens are dealt out: windows of one token where there are few, with the heads in several CTAs until an SM has two; of `most`
// where that leaves every SM `each`, else of eight.  (4 bits, 8 heads of 128 dims, 8 and 16 tokens, us: append 12000 39 and 41, 20000 66 and 69, 40000
// 125 and 120, 65536 201 and 189: a CTA's time is its last wave's; read 9600 12.5 and 12.7, 20000 26.5 and 24.6, 65536 72 and 66.)
static void deal(CacheArgs& A, int rows_of_token, int most, int each)
{
    A.window = A.tokens >= each * kSms * most ? most : A.tokens >= kCacheMany ? 8 : 1;
    const int windows = (A.tokens + A.window - 1) / A.window;
    A.split = std::max(1, std::min((2 * kSms + windows - 1) / windows, (rows_of_token + kCacheWarps - 1) / kCacheWarps));
}

// (after the team is known)
static void quotients(CacheArgs& A)
{
    const int stride = A.split * (kCacheThreads / A.team), half = std::max(1, A.half), queries = std::max(1, A.x.q_heads);
    A.by_half = kCacheThreads / half; A.by_heads = stride / A.heads; A.by_queries = stride / queries;
    A.of_half = 1.f / (float)half; A.of_heads = 1.f / (float)A.heads; A.of_queries = 1.f / (float)queries;
}

template <class Args>
static void launch_cache(void (*kernel)(Args), const Args& args, const CacheArgs& A, int smem, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)((A.tokens + A.window - 1) / A.window), (unsigned)A.split);
    cfg.blockDim = dim3(kCacheThreads); cfg.dynamicSmemBytes = (size_t)smem; cfg.stream = st; cfg.attrs = &at; cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kernel, args);
}

static int pow2_up(int n) { int p = 1; while (p < n) p *= 2; return std::min(p, 32); }

template <typename T, typename C, bool kFew>
static void launch_append_of(CacheArgs& A, int n, int smem, cudaStream_t st)
{
    A.team = pow2_up(A.dim / (2 * n));
    quotients(A);
    if (sizeof(T) == 2 && sizeof(C) == 2 && n == 8) launch_cache(append_kernel<T, C, sizeof(T) == 2 && sizeof(C) == 2 ? 8 : 4, kFew>, A, A, smem, st);
    else if (n == 4) launch_cache(append_kernel<T, C, 4, kFew>, A, A, smem, st);
    else launch_cache(append_kernel<T, C, 1, kFew>, A, A, smem, st);
}
template <typename T, typename C>
static void launch_append(CacheArgs& A, int n, int smem, cudaStream_t st)
{
    if (A.window == 1) launch_append_of<T, C, true>(A, n, smem, st); else launch_append_of<T, C, false>(A, n, smem, st);
}
template <typename T>
static void launch_append_to(CacheArgs& A, int format, int n, int smem, cudaStream_t st)
{
    if (format == GR_F32) launch_append<T, float>(A, n, smem, st);
    else if (format == GR_BF16) launch_append<T, __nv_bfloat16>(A, n, smem, st);
    else launch_append<T, __half>(A, n, smem, st);
}
template <typename T>
static void launch_append4(CacheArgs& A, bool vec, int n, int smem, cudaStream_t st)
{
    A.queries_vec = n >= 4;
    A.team = pow2_up(A.dim / (2 * (n >= 4 ? 4 : 1)));
    quotients(A);
    if (vec) launch_cache(append4_kernel<T, true>, A, A, smem, st);
    else launch_cache(append4_kernel<T, false>, A, A, smem, st);
}

template <typename C, typename T>
static void launch_read(ReadArgs& R, int n, cudaStream_t st)
{
    R.c.team = pow2_up(R.c.dim / n);
    if (sizeof(T) == 2 && sizeof(C) == 2 && n == 8) launch_cache(read_kernel<C, T, sizeof(T) == 2 && sizeof(C) == 2 ? 8 : 4>, R, R.c, 0, st);
    else if (n == 4) launch_cache(read_kernel<C, T, 4>, R, R.c, 0, st);
    else launch_cache(read_kernel<C, T, 1>, R, R.c, 0, st);
}
template <typename C>
static void launch_read_to(ReadArgs& R, int dtype, int n, cudaStream_t st)
{
    if (dtype == GR_F32) launch_read<C, float>(R, n, st);
    else if (dtype == GR_BF16) launch_read<C, __nv_bfloat16>(R, n, st);
    else launch_read<C, __half>(R, n, st);
}
template <typename T, bool kVec>
static void launch_read4_of(ReadArgs& R, cudaStream_t st)
{
    switch (R.c.dim / 32) {
        case 1: launch_cache(read4_kernel<T, 1, kVec>, R, R.c, 0, st); break;
        case 2: launch_cache(read4_kernel<T, 2, kVec>, R, R.c, 0, st); break;
        case 3: launch_cache(read4_kernel<T, 3, kVec>, R, R.c, 0, st); break;
        case 4: launch_cache(read4_kernel<T, 4, kVec>, R, R.c, 0, st); break;
        case 5: launch_cache(read4_kernel<T, 5, kVec>, R, R.c, 0, st); break;
        case 6: launch_cache(read4_kernel<T, 6, kVec>, R, R.c, 0, st); break;
        case 7: launch_cache(read4_kernel<T, 7, kVec>, R, R.c, 0, st); break;
        default: launch_cache(read4_kernel<T, 8, kVec>, R, R.c, 0, st); break;
    }
}
template <typename T>
static void launch_read4(ReadArgs& R, bool vec, cudaStream_t st)
{
    if (vec) launch_read4_of<T, true>(R, st); else launch_read4_of<T, false>(R, st);
}

}  // namespace gr

extern "C" {

#ifdef GR_CHECK
int gr_cache_check(void) { return gr::span_check(); }
#endif

int gr_cache_append(void* keys, void* values, const gr_cache_layout* layout, const gr_cache_tokens* in, int tokens,
                    const long long* slots, const int* positions, const double* frequencies, int rot, int interleaved, void* stream)
{
    if (!in) return GR_E_NULL;
    const int rc = gr::check_cache(keys, values, layout);
    if (rc != GR_OK) return rc;
    const gr_cache_layout& L = *layout;
    const gr_cache_tokens& X = *in;
    if (tokens < 0 || !gr::known_type(X.dtype)) return GR_E_INVALID;
    if (rot < 0 || rot % 2 || rot > L.dim || X.q_heads < 0 || X.q_heads > GR_MAX_HEADS) return GR_E_INVALID;
    const int e = gr::type_size(X.dtype);
    if (!gr::counted(X.k_token, X.k_head, tokens, L.heads) || !gr::counted(X.v_token, X.v_head, tokens, L.heads)) return GR_E_INVALID;
    const bool queries = X.q_heads > 0;
    if (queries) {
        const long long step[2] = {X.out_token, X.out_head}, size[2] = {tokens, X.q_heads};
        if (!gr::counted(X.q_token, X.q_head, tokens, X.q_heads) || !gr::apart(L.dim, step, size, 2)) return GR_E_INVALID;
        if (X.q == X.q_out && ((tokens > 1 && X.q_token != X.out_token) || (X.q_heads > 1 && X.q_head != X.out_head))) return GR_E_INVALID;
    }
    if (tokens == 0) return GR_OK;
    if (!X.k || !X.v || (queries && (!X.q || !X.q_out))) return GR_E_NULL;
    const uintptr_t unit = (uintptr_t)(e - 1);
    if (((uintptr_t)X.k & unit) || ((uintptr_t)X.v & unit) || (queries && (((uintptr_t)X.q & unit) || ((uintptr_t)X.q_out & unit)))) return GR_E_ALIGN;
    // (queries may lie among keys and values, as in one projection's output, and be rotated there; the cache lies apart from all of them)
    const gr::Span rows[4] = {gr::rows_span(X.k, e, L.dim, X.k_token, X.k_head, tokens, L.heads), gr::rows_span(X.v, e, L.dim, X.v_token, X.v_head, tokens, L.heads),
                              gr::rows_span(X.q, e, L.dim, X.q_token, X.q_head, tokens, X.q_heads), gr::rows_span(X.q_out, e, L.dim, X.out_token, X.out_head, tokens, X.q_heads)};
    const gr::Span held[2] = {gr::cache_span(keys, L), L.format == GR_Q4 ? gr::Span{0, 0} : gr::cache_span(values, L)};
    for (const gr::Span& a : held) for (const gr::Span& b : rows) if (gr::meet(a, b)) return GR_E_INVALID;
    if (L.format != GR_Q4 && gr::meet(gr::cache_places(keys, L), gr::cache_places(values, L))) return GR_E_INVALID;
    const gr::Places out = gr::rows_places(X.q_out, e, L.dim, X.out_token, X.out_head, tokens, X.q_heads);
    if (queries) {
        const gr::Places in[3] = {gr::rows_places(X.k, e, L.dim, X.k_token, X.k_head, tokens, L.heads), gr::rows_places(X.v, e, L.dim, X.v_token, X.v_head, tokens, L.heads),
                                  gr::rows_places(X.q, e, L.dim, X.q_token, X.q_head, tokens, X.q_heads)};
        for (int i = 0; i < (X.q == X.q_out ? 2 : 3); i++) if (gr::meet(in[i], out)) return GR_E_INVALID;
    }
    if (!slots || (rot > 0 && (!positions || !frequencies))) return GR_E_NULL;
    if (((uintptr_t)slots & 7) || ((uintptr_t)positions & 3) || (rot > 0 && ((uintptr_t)frequencies & 7))) return GR_E_ALIGN;
    const struct { const void* p; long long bytes; } lists[3] = {{slots, 8ll * tokens}, {positions, 4ll * tokens}, {rot > 0 ? frequencies : nullptr, 4ll * rot}};
    for (const auto& l : lists) {
        if (!l.p) continue;
        const gr::Span span = {(uintptr_t)l.p, (uintptr_t)l.p + (uintptr_t)l.bytes};
        if (gr::meet(held[0], span) || gr::meet(held[1], span) || (queries && gr::meet(out, gr::bytes_at(l.p, l.bytes)))) return GR_E_INVALID;
    }
    gr::CacheArgs A = {};
    A.keys = (char*)keys; A.values = (char*)values;
    A.block_stride = L.block_stride; A.token_stride = L.token_stride; A.head_stride = L.head_stride;
    A.heads = L.heads; A.dim = L.dim; A.block = L.block_size; A.num_blocks = L.num_blocks;
    A.x = X; A.tokens = tokens; A.slots = slots; A.positions = positions; A.freq = frequencies;
    A.half = rot / 2; A.interleaved = interleaved != 0;
    GR_SET_SPAN(A.in_k, rows[0]); GR_SET_SPAN(A.in_v, rows[1]); GR_SET_SPAN(A.in_q, rows[2]); GR_SET_SPAN(A.out_q, rows[3]); GR_SET_SPAN(A.held_k, held[0]); GR_SET_SPAN(A.held_v, held[1]);
    const bool four = L.format == GR_Q4;
    gr::Align kv, q, c;
    kv.add(X.k, e, {X.k_token, X.k_head}); kv.add(X.v, e, {X.v_token, X.v_head});
    if (queries) { q.add(X.q, e, {X.q_token, X.q_head}); q.add(X.q_out, e, {X.out_token, X.out_head}); }
    if (!four) {
        const int ce = gr::type_size(L.format);
        c.add(keys, ce, {L.block_stride, L.token_stride, L.head_stride}); c.add(values, ce, {L.block_stride, L.token_stride, L.head_stride});
    }
    // pieces of N elements: both halves of the rotated dims and of the others are whole numbers of them
    auto fits = [&](int n, unsigned long long own, unsigned long long cache) {
        const int ce = four ? 1 : gr::type_size(L.format);
        return own % (unsigned long long)(n * e) == 0 && (four || cache % (unsigned long long)(n * ce) == 0) && L.dim % (2 * n) == 0
               && (interleaved ? true : (rot / 2) % n == 0 && (L.dim - rot) / 2 % n == 0);
    };
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_cache_append");
    if (four) {
        const bool vec = kv.bits % 16 == 0 && (interleaved || (rot / 2) % 8 == 0);
        const int n = fits(4, q.bits, 0) ? 4 : 1;
        A.four = 1;
        gr::deal(A, 8 * L.heads + (X.q_heads + 3) / 4, 16, 16);
        const int smem = (A.window + 7) * gr::angle_step(A.half) * (int)sizeof(float2);
        if (X.dtype == GR_F32) gr::launch_append4<float>(A, vec, n, smem, st);
        else if (X.dtype == GR_BF16) gr::launch_append4<__nv_bfloat16>(A, vec, n, smem, st);
        else gr::launch_append4<__half>(A, vec, n, smem, st);
    } else {
        const unsigned long long own = kv.bits | q.bits;
        const int n = e == 2 && gr::type_size(L.format) == 2 && fits(8, own, c.bits) ? 8 : fits(4, own, c.bits) ? 4 : 1;
        gr::deal(A, (2 * L.heads + X.q_heads + 3) / 4, 8, 4);
        const int smem = A.window * gr::angle_step(A.half) * (int)sizeof(float2);
        if (X.dtype == GR_F32) gr::launch_append_to<float>(A, L.format, n, smem, st);
        else if (X.dtype == GR_BF16) gr::launch_append_to<__nv_bfloat16>(A, L.format, n, smem, st);
        else gr::launch_append_to<__half>(A, L.format, n, smem, st);
    }
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

int gr_cache_read(const void* keys, const void* values, const gr_cache_layout* layout, const long long* slots, int tokens, int dtype,
                  void* k, long long k_token, long long k_head, void* v, long long v_token, long long v_head, void* stream)
{
    const int rc = gr::check_cache(keys, values, layout);
    if (rc != GR_OK) return rc;
    const gr_cache_layout& L = *layout;
    if (tokens < 0 || !gr::known_type(dtype)) return GR_E_INVALID;
    const long long ks[2] = {k_token, k_head}, vs[2] = {v_token, v_head}, size[2] = {tokens, L.heads};
    if (!gr::apart(L.dim, ks, size, 2) || !gr::apart(L.dim, vs, size, 2)) return GR_E_INVALID;
    if (tokens == 0) return GR_OK;
    if (!k || !v) return GR_E_NULL;
    const int e = gr::type_size(dtype);
    if (((uintptr_t)k & (uintptr_t)(e - 1)) || ((uintptr_t)v & (uintptr_t)(e - 1))) return GR_E_ALIGN;
    const gr::Places out_k = gr::rows_places(k, e, L.dim, k_token, k_head, tokens, L.heads), out_v = gr::rows_places(v, e, L.dim, v_token, v_head, tokens, L.heads);
    if (gr::meet(out_k, out_v)) return GR_E_INVALID;
    const gr::Span written[2] = {gr::rows_span(k, e, L.dim, k_token, k_head, tokens, L.heads), gr::rows_span(v, e, L.dim, v_token, v_head, tokens, L.heads)};
    const gr::Span held[2] = {gr::cache_span(keys, L), L.format == GR_Q4 ? gr::Span{0, 0} : gr::cache_span(values, L)};
    for (const gr::Span& a : held) for (const gr::Span& b : written) if (gr::meet(a, b)) return GR_E_INVALID;
    if (!slots) return GR_E_NULL;
    if ((uintptr_t)slots & 7) return GR_E_ALIGN;
    const gr::Places read = gr::bytes_at(slots, 8ll * tokens);
    if (gr::meet(out_k, read) || gr::meet(out_v, read)) return GR_E_INVALID;
    gr::ReadArgs R = {};
    gr::CacheArgs& A = R.c;
    A.keys = (char*)keys; A.values = (char*)values;
    A.block_stride = L.block_stride; A.token_stride = L.token_stride; A.head_stride = L.head_stride;
    A.heads = L.heads; A.dim = L.dim; A.block = L.block_size; A.num_blocks = L.num_blocks;
    A.tokens = tokens; A.slots = slots;
    GR_SET_SPAN(A.in_k, written[0]); GR_SET_SPAN(A.in_v, written[1]); GR_SET_SPAN(A.held_k, held[0]); GR_SET_SPAN(A.held_v, held[1]);
    R.k = k; R.v = v; R.k_token = k_token; R.k_head = k_head; R.v_token = v_token; R.v_head = v_head;
    gr::Align out, c;
    out.add(k, e, {k_token, k_head}); out.add(v, e, {v_token, v_head});
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_cache_read");
    if (L.format == GR_Q4) {
        A.four = 1;
        gr::deal(A, L.heads, 16, 4);
        const bool vec = out.bits % (unsigned long long)(8 * e) == 0;
        if (dtype == GR_F32) gr::launch_read4<float>(R, vec, st);
        else if (dtype == GR_BF16) gr::launch_read4<__nv_bfloat16>(R, vec, st);
        else gr::launch_read4<__half>(R, vec, st);
    } else {
        const int ce = gr::type_size(L.format);
        c.add(keys, ce, {L.block_stride, L.token_stride, L.head_stride}); c.add(values, ce, {L.block_stride, L.token_stride, L.head_stride});
        auto fits = [&](int n) { return out.bits % (unsigned long long)(n * e) == 0 && c.bits % (unsigned long long)(n * ce) == 0 && L.dim % n == 0; };
        const int n = e == 2 && ce == 2 && fits(8) ? 8 : fits(4) ? 4 : 1;
        gr::deal(A, (2 * L.heads + 3) / 4, 8, 4);
        if (L.format == GR_F32) gr::launch_read_to<float>(R, dtype, n, st);
        else if (L.format == GR_BF16) gr::launch_read_to<__nv_bfloat16>(R, dtype, n, st);
        else gr::launch_read_to<__half>(R, dtype, n, st);
    }
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
