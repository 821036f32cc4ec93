// gr_cache_append and gr_cache_read: new tokens' keys and values into a paged cache, rotated by their positions on the way, and out again.
//
// Both move bytes.  A CTA takes the tokens of one window (one token where there are few, for latency; eight otherwise) and all their
// heads, so that a token's angles are worked out once: position x frequency in fp64, brought to [-pi / 4, pi / 4] in fp64 (far
// positions lose nothing), sine and cosine by their Taylor series, rounded to fp32 once.  The rotation takes fp32 products and sums
// without contraction, each rounded, so that what is held follows from the formula whatever computes it; an angle's two
// numbers cost 30 fp64 operations, shared by all heads.
// In a 4-bit cache the unit is the octet: a run of a call's tokens that lie one after another in one octet is taken by one CTA, the
// one whose window its first token is in, so that a prompt's octets are written whole.
#include <math.h>
#include <algorithm>
#include "gr_host.h"
#include "gr_cache.cuh"

namespace gr {

constexpr int kCacheThreads = 256, kCacheWarps = kCacheThreads / 32;
constexpr int kCacheWindow = 8;                // tokens of a CTA where there are many
constexpr int kCacheMany = 16 * kSms;          // from so many tokens on

struct CacheArgs {
    char* keys; char* values;
    long long block_stride, token_stride, head_stride;     // elements of the cache (4 bits: bytes, the first only)
    int heads, dim, block, num_blocks;
    gr_cache_tokens x;
    int tokens, window, split;                 // split: CTAs that share a window's rows
    const long long* slots; const int* positions; const double* freq;
    int half, interleaved;                     // half: pairs of dims that are rotated
    int team, queries_vec;                     // team: threads of a row
};

// ---------------------------------------------------------------- angles

// sine and cosine of a, rounded to fp32
__device__ __forceinline__ float2 cos_sin(double a)
{
    const double k = rint(a * 0.63661977236758134308);                     // 2 / pi
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
    const int quadrant = (int)((long long)k & 3);
    const double cq = quadrant & 1 ? s : c, sq = quadrant & 1 ? c : s;
    return make_float2((float)(quadrant == 1 || quadrant == 2 ? -cq : cq), (float)(quadrant >= 2 ? -sq : sq));
}

// (cos, sin) of the pairs of `n` tokens from `i0` on into cs[n][half]
__device__ __forceinline__ void fill_angles(const CacheArgs& A, float2* cs, int i0, int n)
{
    for (int e = threadIdx.x; e < n * A.half; e += kCacheThreads) {
        const int tok = e / A.half, f = e - tok * A.half;
        cs[e] = cos_sin((double)A.positions[i0 + tok] * A.freq[f]);
    }
    if (A.half > 0) __syncthreads();
}

// a rotated number: x the element itself, y the other of its pair
__device__ __forceinline__ float turned(float x, float y, float2 cs, bool second)
{
    const float p = __fmul_rn(x, cs.x), q = __fmul_rn(y, cs.y);
    return second ? __fadd_rn(p, q) : __fsub_rn(p, q);
}

template <typename T, int N>
__device__ __forceinline__ void load_n(float (&x)[N], const T* p)
{
    const Pack<T, N> v = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = to_f32(v.x[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&x)[N])
{
    Pack<T, N> v;
#pragma unroll
    for (int i = 0; i < N; i++) v.x[i] = from_f32<T>(x[i]);
    *reinterpret_cast<Pack<T, N>*>(p) = v;
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

template <int N>
__device__ __forceinline__ void turn_pieces(float (&a)[N], float (&b)[N], const Pieces& p, const float2* cs, int half, bool interleaved)
{
    if (p.turn == 1) {
        const int f = interleaved ? p.c0 / 2 : p.c0;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float2 t = cs[f + i];
            const float x = a[i], y = b[i];
            a[i] = turned(x, y, t, false); b[i] = turned(y, x, t, true);
        }
    } else if (p.turn == 2) {
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            if (p.c0 + i < 2 * half) {
                const float2 t = cs[(p.c0 + i) / 2];
                const float x = a[i], y = a[i + 1];
                a[i] = turned(x, y, t, false); a[i + 1] = turned(y, x, t, true);
            }
            if (p.c1 + i < 2 * half) {
                const float2 t = cs[(p.c1 + i) / 2];
                const float x = b[i], y = b[i + 1];
                b[i] = turned(x, y, t, false); b[i + 1] = turned(y, x, t, true);
            }
        }
    }
}

// The rows of a window's tokens: keys and values (but for a 4-bit cache, whose queries alone come here), queries.
template <typename T, typename C, int N, bool kQueries>
__device__ __forceinline__ void append_rows(const CacheArgs& A, const float2* cs, int i0, int n, int part)
{
    constexpr int kRows = 2;                               // in flight for each team
    const int D = A.dim, chunks = D / (2 * N), team = A.team, in_team = threadIdx.x & (team - 1);
    const int per = (kQueries ? 0 : 2 * A.heads) + A.x.q_heads, total = n * per, teams = kCacheThreads / team;
    const long long places = (long long)A.num_blocks * A.block;
    for (int r0 = part * teams + threadIdx.x / team; r0 < total; r0 += kRows * A.split * teams) {
        const T* src[kRows];
        void* dst[kRows];
        int tok[kRows], kind[kRows];                       // kind: 0 nothing, 1 keys, 2 values, 3 queries
#pragma unroll
        for (int u = 0; u < kRows; u++) {
            const int r = r0 + u * A.split * teams;
            kind[u] = 0; src[u] = nullptr; dst[u] = nullptr; tok[u] = 0;
            if (r >= total) continue;
            tok[u] = r / per;
            int row = r - tok[u] * per;
            const long long i = i0 + tok[u];
            if (!kQueries && row < 2 * A.heads) {
                const bool second = row >= A.heads;
                if (second) row -= A.heads;
                const long long slot = A.slots[i];
                if (slot >= 0 && slot < places) {
                    const long long block = slot / A.block, at = slot - block * A.block;
                    const long long to = block * A.block_stride + at * A.token_stride + row * A.head_stride;
                    kind[u] = second ? 2 : 1;
                    src[u] = second ? (const T*)A.x.v + i * A.x.v_token + row * A.x.v_head : (const T*)A.x.k + i * A.x.k_token + row * A.x.k_head;
                    dst[u] = (C*)(second ? A.values : A.keys) + to;
                }
            } else {
                if (!kQueries) row -= 2 * A.heads;
                if (!A.positions || A.positions[i] >= 0) {
                    kind[u] = 3;
                    src[u] = (const T*)A.x.q + i * A.x.q_token + row * A.x.q_head;
                    dst[u] = (T*)A.x.q_out + i * A.x.out_token + row * A.x.out_head;
                }
            }
        }
        for (int e = in_team; e < chunks; e += team) {
            const Pieces turn = pieces_of<N>(e, D, A.half, A.interleaved), plain = pieces_of<N>(e, D, 0, false);
            float a[kRows][N], b[kRows][N];
#pragma unroll
            for (int u = 0; u < kRows; u++) {
                const Pieces& p = kind[u] == 2 ? plain : turn;
                if (kind[u]) { load_n<T, N>(a[u], src[u] + p.c0); load_n<T, N>(b[u], src[u] + p.c1); }
            }
#pragma unroll
            for (int u = 0; u < kRows; u++) {
                if (!kind[u]) continue;
                const Pieces& p = kind[u] == 2 ? plain : turn;
                if (kind[u] != 2) turn_pieces<N>(a[u], b[u], p, cs + tok[u] * A.half, A.half, A.interleaved);
                if (kind[u] == 3) { store_n<T, N>((T*)dst[u] + p.c0, a[u]); store_n<T, N>((T*)dst[u] + p.c1, b[u]); }
                else { store_n<C, N>((C*)dst[u] + p.c0, a[u]); store_n<C, N>((C*)dst[u] + p.c1, b[u]); }
            }
        }
    }
}

template <typename T, typename C, int N>
__global__ void __launch_bounds__(kCacheThreads)
append_kernel(const __grid_constant__ CacheArgs A)
{
    extern __shared__ float2 cs[];
    pdl_wait();
    const int i0 = blockIdx.x * A.window, n = min(A.window, A.tokens - i0);
    fill_angles(A, cs, i0, n);
    append_rows<T, C, N, false>(A, cs, i0, n, blockIdx.y);
}

// ---------------------------------------------------------------- a 4-bit cache

// The run of tokens that begins at i, if one does: tokens i, i + 1, ... that lie one after another in one octet.  0: the token before
// has it, or it has no place.
__device__ __forceinline__ int run_at(const CacheArgs& A, int i, long long& slot)
{
    const long long places = (long long)A.num_blocks * A.block;
    slot = A.slots[i];
    if (slot < 0 || slot >= places) return 0;
    if ((slot & 7) != 0 && i > 0 && A.slots[i - 1] == slot - 1) return 0;
    int n = 1;
    while (n < 8 - (int)(slot & 7) && i + n < A.tokens && A.slots[i + n] == slot + n) n++;
    return n;
}

// Code of x, in units of s: the whole number nearest to x / s from -8 to 7 (ties to even), decided by the sign of x - (m + 1/2) s,
// which one fused operation gives exactly; then + 8.
__device__ __forceinline__ unsigned code_of(float x, float s, float inverse)
{
    const float m = floorf(fminf(fmaxf(x * inverse, -9.f), 8.f));
    const float d = fmaf(-(m + 0.5f), s, x), up = s < 0.f ? -d : d;
    const int w = (int)m;
    return (unsigned)(min(max(w + (up > 0.f || (up == 0.f && (w & 1)) ? 1 : 0), -8), 7) + 8);
}

// The half word of codes of four dims x of a group of eight lanes, and the group's scale: that of the element of largest magnitude
// (the positive one of two), for which the code is 0, that is -8, as fp16.  A group with a NaN or an infinity gets the scale NaN.
__device__ __forceinline__ unsigned short quantise(const float (&x)[4], unsigned short& scale)
{
    float hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    const bool bad = !(fabsf(x[0]) < INFINITY && fabsf(x[1]) < INFINITY && fabsf(x[2]) < INFINITY && fabsf(x[3]) < INFINITY);
#pragma unroll
    for (int o = 1; o < 8; o *= 2) {
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    const unsigned met = __ballot_sync(0xffffffffu, bad) >> (threadIdx.x & 24) & 0xffu;
    const __half h = __float2half_rn(fminf(fmaxf((hi >= -lo ? hi : lo) * -0.125f, -65504.f), 65504.f));
    const float s = __half2float(h), inverse = 1.f / s;
    scale = met ? 0x7fffu : __half_as_ushort(h);
    if (met || s == 0.f) return 0x8888u;
    return (unsigned short)(code_of(x[0], s, inverse) | code_of(x[1], s, inverse) << 4 | code_of(x[2], s, inverse) << 8 | code_of(x[3], s, inverse) << 12);
}

// four elements from c on of a row, rotated
template <typename T, bool kVec>
__device__ __forceinline__ void load_four(float (&x)[4], const T* row, int c)
{
    if (kVec) load_n<T, 4>(x, row + c);
    else {
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = to_f32(row[c + i]);
    }
}
template <typename T, bool kVec>
__device__ __forceinline__ void load_partners(float (&y)[4], const float (&x)[4], const T* row, int c, int half, bool interleaved)
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; i++) y[i] = x[i ^ 1];
    } else if (kVec) {
        if (c < 2 * half) load_n<T, 4>(y, row + (c < half ? c + half : c - half));
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) if (c + i < 2 * half) y[i] = to_f32(row[c + i < half ? c + i + half : c + i - half]);
    }
}

template <typename T, bool kVec>
__global__ void __launch_bounds__(kCacheThreads)
append4_kernel(const __grid_constant__ CacheArgs A)
{
    extern __shared__ float2 cs[];
    pdl_wait();
    const int w0 = blockIdx.x * A.window, wn = min(A.window, A.tokens - w0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = A.dim, J = D / 32, half = A.half;
    for (int i0 = w0; i0 < w0 + wn; i0++) {
        long long slot;
        const int n = run_at(A, i0, slot);
        if (n == 0) continue;                              // (the same for all threads)
        const int first = (int)(slot & 7);
        if (i0 > w0) __syncthreads();                      // (the angles of the run before are done with)
        fill_angles(A, cs, i0, n);
        const long long block = slot / A.block;
        char* base = A.keys + block * A.block_stride + (long long)((int)(slot - block * A.block) >> 3) * octet_bytes(D);
        const long long head_bytes = (long long)(A.block >> 3) * octet_bytes(D);
        // (head, keys or values) by warps; a lane has four dims, half a word of keys, a half word of values
        for (int e = blockIdx.y * kCacheWarps + warp; e < 2 * A.heads; e += A.split * kCacheWarps) {
            const bool second = e >= A.heads;
            const int head = second ? e - A.heads : e;
            char* octet = base + head * head_bytes;
            const T* row = second ? (const T*)A.x.v + i0 * A.x.v_token + head * A.x.v_head : (const T*)A.x.k + i0 * A.x.k_token + head * A.x.k_head;
            const long long step = second ? A.x.v_token : A.x.k_token;
            for (int c0 = 0; c0 < D; c0 += 128) {
                const int c = c0 + 4 * lane, j = c >> 5, r = lane & 7;
                const bool in = c < D;
#pragma unroll 1
                for (int o0 = first & 4; o0 < first + n; o0 += 4) {      // four of the octet's places at a time
                    float x[4][4], y[4][4];
                    bool some[4];
#pragma unroll
                    for (int u = 0; u < 4; u++) {
                        const int t = o0 + u - first;
                        some[u] = t >= 0 && t < n;
#pragma unroll
                        for (int i = 0; i < 4; i++) { x[u][i] = 0.f; y[u][i] = 0.f; }
                        if (some[u] && in) {
                            load_four<T, kVec>(x[u], row + t * step, c);
                            if (!second && c < 2 * half) load_partners<T, kVec>(y[u], x[u], row + t * step, c, half, A.interleaved);
                        }
                    }
                    unsigned short code[4], scale[4];
#pragma unroll
                    for (int u = 0; u < 4; u++) {
                        if (!second && some[u]) {
                            const float2* at = cs + (o0 + u - first) * half;
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                const int d = c + i;
                                if (d >= 2 * half) continue;
                                const bool two = A.interleaved ? d & 1 : d >= half;
                                x[u][i] = turned(x[u][i], y[u][i], at[A.interleaved ? d >> 1 : two ? d - half : d], two);
                            }
                        }
                        code[u] = quantise(x[u], scale[u]);
                    }
                    if (!in) continue;
                    if (!second) {
#pragma unroll
                        for (int u = 0; u < 4; u++) {
                            if (!some[u]) continue;
                            *(unsigned short*)(octet + (o0 + u) * (D / 2) + ((r >> 1) * J + j) * 4 + (r & 1) * 2) = code[u];
                            if (r == 0) *(unsigned short*)(octet + octet_kscale(D) + ((o0 + u) * J + j) * 2) = scale[u];
                        }
                    } else {
#pragma unroll
                        for (int u = 0; u < 4; u += 2) {
                            const int pair = (o0 + u) >> 1;
                            char* at = octet + octet_vcode(D) + ((r * 4 + pair) * J + j) * 4;
                            char* sc = octet + octet_vscale(D) + (pair * J + j) * 4;
                            if (some[u] && some[u + 1]) {
                                *(unsigned*)at = code[u] | (unsigned)code[u + 1] << 16;
                                if (r == 0) *(unsigned*)sc = scale[u] | (unsigned)scale[u + 1] << 16;
                            } else {
#pragma unroll
                                for (int z = 0; z < 2; z++) {
                                    if (!some[u + z]) continue;
                                    *(unsigned short*)(at + 2 * z) = code[u + z];
                                    if (r == 0) *(unsigned short*)(sc + 2 * z) = scale[u + z];
                                }
                            }
                        }
                    }
                }
            }
        }
    }
    if (A.x.q_heads > 0) {
        __syncthreads();
        fill_angles(A, cs, w0, wn);
        if (A.queries_vec) append_rows<T, T, 4, true>(A, cs, w0, wn, blockIdx.y);
        else append_rows<T, T, 1, true>(A, cs, w0, wn, blockIdx.y);
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
    const CacheArgs& A = R.c;
    pdl_wait();
    const int i0 = blockIdx.x * A.window, n = min(A.window, A.tokens - i0), D = A.dim;
    const int chunks = D / N, team = A.team, in_team = threadIdx.x & (team - 1), teams = kCacheThreads / team, total = n * 2 * A.heads;
    const long long places = (long long)A.num_blocks * A.block;
    for (int r0 = blockIdx.y * teams + threadIdx.x / team; r0 < total; r0 += kRows * A.split * teams) {
        const C* src[kRows];
        T* dst[kRows];
#pragma unroll
        for (int u = 0; u < kRows; u++) {
            const int r = r0 + u * A.split * teams;
            src[u] = nullptr; dst[u] = nullptr;
            if (r >= total) continue;
            const int tok = r / (2 * A.heads), row = r - tok * 2 * A.heads;
            const bool second = row >= A.heads;
            const int head = second ? row - A.heads : row;
            const long long i = i0 + tok, slot = A.slots[i];
            dst[u] = second ? (T*)R.v + i * R.v_token + head * R.v_head : (T*)R.k + i * R.k_token + head * R.k_head;
            if (slot >= 0 && slot < places) {
                const long long block = slot / A.block, at = slot - block * A.block;
                src[u] = (const C*)(second ? A.values : A.keys) + block * A.block_stride + at * A.token_stride + head * A.head_stride;
            }
        }
        for (int e = in_team; e < chunks; e += team) {
            float x[kRows][N];
#pragma unroll
            for (int u = 0; u < kRows; u++) {
#pragma unroll
                for (int i = 0; i < N; i++) x[u][i] = 0.f;
                if (src[u]) load_n<C, N>(x[u], src[u] + e * N);
            }
#pragma unroll
            for (int u = 0; u < kRows; u++) if (dst[u]) store_n<T, N>(dst[u] + e * N, x[u]);
        }
    }
}

// Of a run of an octet a warp takes (head, keys or values): a lane the words of token lane / 4 (keys), of a pair of tokens (values).
template <typename T, int J, bool kVec>
__device__ __forceinline__ void read_octet(const char* octet, bool second, T* out, long long step, int first, int n, int lane)
{
    constexpr int D = 32 * J, kWords = J % 4 == 0 ? 4 : J % 2 == 0 ? 2 : 1;
    const int g = lane >> 2, t = lane & 3;
    unsigned w[J];
    const unsigned* code = (const unsigned*)(octet + (second ? octet_vcode(D) : 0)) + lane * J;
#pragma unroll
    for (int i = 0; i < J; i += kWords) {
        const Pack<unsigned, kWords> p = *reinterpret_cast<const Pack<unsigned, kWords>*>(code + i);
#pragma unroll
        for (int z = 0; z < kWords; z++) w[i + z] = p.x[z];
    }
    if (!second) {
        if (g < first || g >= first + n) return;
        const __half* scale = (const __half*)(octet + octet_kscale(D)) + g * J;
        T* to = out + (long long)(g - first) * step + 8 * t;
#pragma unroll
        for (int j = 0; j < J; j++) {
            const float s = __half2float(scale[j]);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = (float)((int)(w[j] >> (4 * i) & 15u) - 8) * s;
            if (kVec) store_n<T, 8>(to + 32 * j, x);
            else {
#pragma unroll
                for (int i = 0; i < 8; i++) to[32 * j + i] = from_f32<T>(x[i]);
            }
        }
    } else {
        const __half2* scale = (const __half2*)(octet + octet_vscale(D)) + t * J;
#pragma unroll
        for (int z = 0; z < 2; z++) {
            const int tok = 2 * t + z;
            if (tok < first || tok >= first + n) continue;
            T* to = out + (long long)(tok - first) * step + 4 * g;
#pragma unroll
            for (int j = 0; j < J; j++) {
                const __half2 h = scale[j];
                const float s = z ? __high2float(h) : __low2float(h);
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; i++) x[i] = (float)((int)(w[j] >> (16 * z + 4 * i) & 15u) - 8) * s;
                if (kVec) store_n<T, 4>(to + 32 * j, x);
                else {
#pragma unroll
                    for (int i = 0; i < 4; i++) to[32 * j + i] = from_f32<T>(x[i]);
                }
            }
        }
    }
}

template <typename T, int J, bool kVec>
__global__ void __launch_bounds__(kCacheThreads)
read4_kernel(const __grid_constant__ ReadArgs R)
{
    const CacheArgs& A = R.c;
    pdl_wait();
    const int w0 = blockIdx.x * A.window, wn = min(A.window, A.tokens - w0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int D = 32 * J;
    const long long places = (long long)A.num_blocks * A.block, head_bytes = (long long)(A.block >> 3) * octet_bytes(D);
    for (int i0 = w0; i0 < w0 + wn; i0++) {
        long long slot;
        const int n = run_at(A, i0, slot);
        if (n == 0) {
            if (slot >= 0 && slot < places) continue;
            // (no place: zeros)
            for (int e = blockIdx.y * kCacheThreads + threadIdx.x; e < 2 * A.heads * D; e += A.split * kCacheThreads) {
                const int row = e / D, d = e - row * D;
                if (row < A.heads) ((T*)R.k)[i0 * R.k_token + row * R.k_head + d] = from_f32<T>(0.f);
                else ((T*)R.v)[i0 * R.v_token + (row - A.heads) * R.v_head + d] = from_f32<T>(0.f);
            }
            continue;
        }
        const long long block = slot / A.block;
        const char* base = A.keys + block * A.block_stride + (long long)((int)(slot - block * A.block) >> 3) * octet_bytes(D);
        for (int e = blockIdx.y * kCacheWarps + warp; e < 2 * A.heads; e += A.split * kCacheWarps) {
            const int head = e >> 1;
            const bool second = e & 1;
            T* out = second ? (T*)R.v + i0 * R.v_token + head * R.v_head : (T*)R.k + i0 * R.k_token + head * R.k_head;
            read_octet<T, J, kVec>(base + head * head_bytes, second, out, second ? R.v_token : R.k_token, (int)(slot & 7), n, lane);
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

// How a call's tokens are dealt out: windows of one token where there are few, with the heads in several CTAs until an SM has two.
static void deal(CacheArgs& A, int rows_of_token)
{
    A.window = A.tokens >= kCacheMany ? kCacheWindow : 1;
    const int windows = (A.tokens + A.window - 1) / A.window;
    A.split = std::max(1, std::min((2 * kSms + windows - 1) / windows, (rows_of_token + kCacheWarps - 1) / kCacheWarps));
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

template <typename T, typename C>
static void launch_append(CacheArgs& A, int n, int smem, cudaStream_t st)
{
    A.team = pow2_up(A.dim / (2 * n));
    if (sizeof(T) == 2 && sizeof(C) == 2 && n == 8) launch_cache(append_kernel<T, C, sizeof(T) == 2 && sizeof(C) == 2 ? 8 : 4>, A, A, smem, st);
    else if (n == 4) launch_cache(append_kernel<T, C, 4>, A, A, smem, st);
    else launch_cache(append_kernel<T, C, 1>, A, A, smem, st);
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
    if (!X.k || !X.v || !slots || (rot > 0 && (!positions || !frequencies)) || (queries && (!X.q || !X.q_out))) return GR_E_NULL;
    const uintptr_t unit = (uintptr_t)(e - 1);
    if (((uintptr_t)X.k & unit) || ((uintptr_t)X.v & unit) || (queries && (((uintptr_t)X.q & unit) || ((uintptr_t)X.q_out & unit)))) return GR_E_ALIGN;
    // (queries may lie among keys and values, as in one projection's output, and be rotated there; the cache lies apart from all of them)
    const gr::Span rows[4] = {gr::rows_span(X.k, e, L.dim, X.k_token, X.k_head, tokens, L.heads), gr::rows_span(X.v, e, L.dim, X.v_token, X.v_head, tokens, L.heads),
                              gr::rows_span(X.q, e, L.dim, X.q_token, X.q_head, tokens, X.q_heads), gr::rows_span(X.q_out, e, L.dim, X.out_token, X.out_head, tokens, X.q_heads)};
    const gr::Span held[2] = {gr::cache_span(keys, L), L.format == GR_Q4 ? gr::Span{0, 0} : gr::cache_span(values, L)};
    for (const gr::Span& a : held) for (const gr::Span& b : rows) if (gr::meet(a, b)) return GR_E_INVALID;
    if (L.format != GR_Q4 && keys == values && L.num_blocks > 0) return GR_E_INVALID;
    gr::CacheArgs A = {};
    A.keys = (char*)keys; A.values = (char*)values;
    A.block_stride = L.block_stride; A.token_stride = L.token_stride; A.head_stride = L.head_stride;
    A.heads = L.heads; A.dim = L.dim; A.block = L.block_size; A.num_blocks = L.num_blocks;
    A.x = X; A.tokens = tokens; A.slots = slots; A.positions = positions; A.freq = frequencies;
    A.half = rot / 2; A.interleaved = interleaved != 0;
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
        const bool vec = kv.bits % (unsigned long long)(4 * e) == 0 && (interleaved || (rot / 2) % 4 == 0);
        const int n = fits(4, q.bits, 0) ? 4 : 1;
        gr::deal(A, 2 * L.heads + (X.q_heads + 3) / 4);
        const int smem = gr::kCacheWindow * A.half * (int)sizeof(float2);
        if (X.dtype == GR_F32) gr::launch_append4<float>(A, vec, n, smem, st);
        else if (X.dtype == GR_BF16) gr::launch_append4<__nv_bfloat16>(A, vec, n, smem, st);
        else gr::launch_append4<__half>(A, vec, n, smem, st);
    } else {
        const unsigned long long own = kv.bits | q.bits;
        const int n = e == 2 && gr::type_size(L.format) == 2 && fits(8, own, c.bits) ? 8 : fits(4, own, c.bits) ? 4 : 1;
        gr::deal(A, (2 * L.heads + X.q_heads + 3) / 4);
        const int smem = A.window * A.half * (int)sizeof(float2);
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
    if (!slots || !k || !v) return GR_E_NULL;
    if (k == v) return GR_E_INVALID;
    const int e = gr::type_size(dtype);
    if (((uintptr_t)k & (uintptr_t)(e - 1)) || ((uintptr_t)v & (uintptr_t)(e - 1))) return GR_E_ALIGN;
    const gr::Span written[2] = {gr::rows_span(k, e, L.dim, k_token, k_head, tokens, L.heads), gr::rows_span(v, e, L.dim, v_token, v_head, tokens, L.heads)};
    const gr::Span held[2] = {gr::cache_span(keys, L), L.format == GR_Q4 ? gr::Span{0, 0} : gr::cache_span(values, L)};
    for (const gr::Span& a : held) for (const gr::Span& b : written) if (gr::meet(a, b)) return GR_E_INVALID;
    gr::ReadArgs R = {};
    gr::CacheArgs& A = R.c;
    A.keys = (char*)keys; A.values = (char*)values;
    A.block_stride = L.block_stride; A.token_stride = L.token_stride; A.head_stride = L.head_stride;
    A.heads = L.heads; A.dim = L.dim; A.block = L.block_size; A.num_blocks = L.num_blocks;
    A.tokens = tokens; A.slots = slots;
    R.k = k; R.v = v; R.k_token = k_token; R.k_head = k_head; R.v_token = v_token; R.v_head = v_head;
    gr::Align out, c;
    out.add(k, e, {k_token, k_head}); out.add(v, e, {v_token, v_head});
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_cache_read");
    if (L.format == GR_Q4) {
        gr::deal(A, 2 * L.heads);
        const bool vec = out.bits % (unsigned long long)(8 * e) == 0;
        if (dtype == GR_F32) gr::launch_read4<float>(R, vec, st);
        else if (dtype == GR_BF16) gr::launch_read4<__nv_bfloat16>(R, vec, st);
        else gr::launch_read4<__half>(R, vec, st);
    } else {
        const int ce = gr::type_size(L.format);
        c.add(keys, ce, {L.block_stride, L.token_stride, L.head_stride}); c.add(values, ce, {L.block_stride, L.token_stride, L.head_stride});
        auto fits = [&](int n) { return out.bits % (unsigned long long)(n * e) == 0 && c.bits % (unsigned long long)(n * ce) == 0 && L.dim % n == 0; };
        const int n = e == 2 && ce == 2 && fits(8) ? 8 : fits(4) ? 4 : 1;
        gr::deal(A, (2 * L.heads + 3) / 4);
        if (L.format == GR_F32) gr::launch_read_to<float>(R, dtype, n, st);
        else if (L.format == GR_BF16) gr::launch_read_to<__nv_bfloat16>(R, dtype, n, st);
        else gr::launch_read_to<__half>(R, dtype, n, st);
    }
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
