// The 4-bit paged cache: where an octet (eight tokens of a head) keeps what.  With J = dim / 32 groups of 32 dims,
//   keys' codes    [8 tokens][4][J] words     word (t, j) of a token: dims 32 j + 8 t .. + 7, the first in its lowest bits
//   keys' scales   [8 tokens][J] fp16
//   values' codes  [8][4 pairs][J][2 tokens] half words    half word (g, pair, j, token): dims 32 j + 4 g .. + 3
//   values' scales [4 pairs][J][2 tokens] fp16
// so that lane (g, t) of a warp finds its share of the operands of a 16 x 8 x 16 product, of a tile whose first eight rows (keys:
// tokens, values: depth) are this octet's, in J consecutive words at place 4 g + t, codes and scales alike; a token's bytes are its own.
#pragma once
#include <algorithm>
#include <initializer_list>
#include "gr_common.cuh"

namespace gr {

__host__ __device__ constexpr int octet_bytes(int dim) { return 9 * dim; }
__host__ __device__ constexpr int octet_kscale(int dim) { return 4 * dim; }
__host__ __device__ constexpr int octet_vcode(int dim) { return 4 * dim + dim / 2; }
__host__ __device__ constexpr int octet_vscale(int dim) { return 8 * dim + dim / 2; }

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// N elements of a type as one access, on an address aligned to all of them
template <typename T, int N> struct __align__(sizeof(T) * N) Pack { T x[N]; };

__host__ inline bool known_type(int t) { return t == GR_F32 || t == GR_BF16 || t == GR_F16; }
__host__ inline int type_size(int t) { return t == GR_F32 ? 4 : 2; }

// The bounds-checked build (gr_common.cuh) in the kernels of caches and attention: GR_WITHIN(span, p, n) says whether n bytes at p lie in a span that the
// arguments carry there, GR_IN_SHARED(p, n) whether in the launch's shared memory; an access elsewhere is skipped, and met by the next call of gr_cache_check
// or gr_attend_check.  In the regular build both are true.
struct Span { uintptr_t lo, hi; };
#ifdef GR_CHECK
static __device__ int g_span_check;
__device__ __noinline__ inline bool within(Span s, const void* p, long long n)
{
    const uintptr_t a = (uintptr_t)p;
    if (a >= s.lo && a + (uintptr_t)n <= s.hi) return true;
    g_span_check = 1;
    return false;
}
__device__ inline Span shared_span(const void* p)
{
    unsigned n;
    asm("mov.u32 %0, %dynamic_smem_size;" : "=r"(n));
    return {(uintptr_t)p, (uintptr_t)p + n};
}
// whether an access was skipped since the last call of this (-1: it cannot be read)
static int span_check()
{
    int met = -1, none = 0;
    if (cudaMemcpyFromSymbol(&met, g_span_check, sizeof(int)) != cudaSuccess || cudaMemcpyToSymbol(g_span_check, &none, sizeof(int)) != cudaSuccess) return -1;
    return met;
}
#define GR_SPAN(name) ::gr::Span name
#define GR_SET_SPAN(name, ...) ((void)((name) = __VA_ARGS__))
#define GR_WITHIN(span, p, n) ::gr::within(span, p, n)
#else
#define GR_SPAN(name) static_assert(true, "")
#define GR_SET_SPAN(name, ...) ((void)0)
#define GR_WITHIN(span, p, n) true
#endif

// Whether places of `count` strided dimensions lie apart, each `unit` elements long.
inline bool apart(long long unit, const long long* step, const long long* size, int count)
{
    int order[3] = {0, 1, 2};
    std::sort(order, order + count, [&](int a, int b) { return step[a] < step[b]; });
    long long span = unit;
    for (int i = 0; i < count; i++) {
        const long long s = step[order[i]], n = size[order[i]];
        if (n <= 1) continue;
        if (s < span || s > (1ll << 58) / n) return false;
        span += s * (n - 1);
    }
    return true;
}

// Whether strides of what is read are ones (31 bits; that of a single token or head is not looked at).
inline bool counted(long long token, long long head, int tokens, int heads)
{
    return (tokens <= 1 || (token >= 0 && token < (1ll << 31) && token <= (1ll << 58) / tokens)) && (heads <= 1 || (head >= 0 && head < (1ll << 31)));
}

// First byte and the one behind the last of strided places.
inline Span span_of(const void* p, long long unit, const long long* step, const long long* size, int count)
{
    for (int i = 0; i < count; i++) { if (size[i] <= 0) return {0, 0}; unit += step[i] * (size[i] - 1); }
    return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)unit};
}
inline bool meet(Span a, Span b) { return a.lo < b.hi && b.lo < a.hi; }

// Where the pieces of a strided array lie, `unit` bytes each, the level of the largest step first; nowhere: unit 0.
struct Places { uintptr_t at; long long unit; int levels; long long step[3], size[3]; };
inline Places places_of(const void* p, long long unit, const long long* step, const long long* size, int count)
{
    Places a = {(uintptr_t)p, unit, 0, {}, {}};
    for (int i = 0; i < count; i++) {
        if (size[i] <= 0) a.unit = 0;
        if (size[i] <= 1 || step[i] == 0) continue;
        int at = a.levels++;
        for (; at > 0 && a.step[at - 1] < step[i]; at--) { a.step[at] = a.step[at - 1]; a.size[at] = a.size[at - 1]; }
        a.step[at] = step[i]; a.size[at] = size[i];
    }
    return a;
}
// Whether a piece of b meets one of a, by the levels from i and j on, b's beginning d bytes behind a's.  Levels of one step are looked at together (only differences
// of about d / step leave the levels within anything to do), others piece by piece; `left`: how many more of these.
inline bool pieces_meet(const Places& a, int i, const Places& b, int j, long long d, int& left)
{
    auto span = [](const Places& p, int from) { long long n = p.unit; for (int l = from; l < p.levels; l++) n += p.step[l] * (p.size[l] - 1); return n; };
    if (d >= span(a, i) || -d >= span(b, j)) return false;
    if (i == a.levels && j == b.levels) return true;
    if (--left < 0) return true;
    auto down = [](long long x, long long s) { return x >= 0 ? x / s : -((-x + s - 1) / s); };
    const bool both = i < a.levels && j < b.levels && a.step[i] == b.step[j], of_a = both || j == b.levels || (i < a.levels && a.step[i] > b.step[j]);
    const long long s = of_a ? a.step[i] : b.step[j];
    // pieces c of a (less those of b): d - c s below what is left of a, above minus what is left of b
    const long long in_a = span(a, of_a ? i + 1 : i), in_b = span(b, both || !of_a ? j + 1 : j);
    long long from = down(d - in_a, s) + 1, to = down(d + in_b - 1, s);
    from = std::max(from, both || !of_a ? 1 - b.size[j] : 0ll); to = std::min(to, of_a ? a.size[i] - 1 : 0ll);
    for (long long c = from; c <= to; c++) if (pieces_meet(a, of_a ? i + 1 : i, b, both || !of_a ? j + 1 : j, d - c * s, left)) return true;
    return false;
}
// (those within one another at different strides, of more than 2^20 pieces, are taken for it)
inline bool meet(const Places& a, const Places& b)
{
    int left = 1 << 20;
    return a.unit > 0 && b.unit > 0 && pieces_meet(a, 0, b, 0, (long long)(b.at - a.at), left);
}
inline Places cache_places(const void* p, const gr_cache_layout& L)       // (not of 4 bits)
{
    const int e = type_size(L.format);
    const long long step[3] = {L.block_stride * e, L.token_stride * e, L.head_stride * e}, size[3] = {L.num_blocks, L.block_size, L.heads};
    return places_of(p, (long long)L.dim * e, step, size, 3);
}
inline Places bytes_at(const void* p, long long bytes) { return places_of(p, bytes, nullptr, nullptr, 0); }
inline Places rows_places(const void* p, int e, int dim, long long token, long long head, int tokens, int heads)
{
    const long long step[2] = {token * e, head * e}, size[2] = {tokens, heads};
    return places_of(p, (long long)dim * e, step, size, 2);
}
inline Span cache_span(const void* p, const gr_cache_layout& L)
{
    if (L.format == GR_Q4) {
        const long long step[1] = {L.block_stride}, size[1] = {L.num_blocks};
        return span_of(p, (long long)L.heads * (L.block_size / 8) * octet_bytes(L.dim), step, size, 1);
    }
    const int e = type_size(L.format);
    const long long step[3] = {L.block_stride * e, L.token_stride * e, L.head_stride * e}, size[3] = {L.num_blocks, L.block_size, L.heads};
    return span_of(p, (long long)L.dim * e, step, size, 3);
}
inline Span rows_span(const void* p, int e, int dim, long long token, long long head, int tokens, int heads)
{
    const long long step[2] = {token * e, head * e}, size[2] = {tokens, heads};
    return span_of(p, (long long)dim * e, step, size, 2);
}

// The elements that pointers and strides (of `e` bytes an element) let an access take: 8 (16 bytes), 4 or 1.
struct Align {
    unsigned long long bits = 0;
    void add(const void* p, int e, std::initializer_list<long long> strides) {
        bits |= (unsigned long long)(uintptr_t)p;
        for (long long s : strides) bits |= (unsigned long long)s * (unsigned long long)e;
    }
};

// What a layout has to satisfy (`keys` aligned as its format asks for); GR_OK or the GR_E_* code.
int check_cache(const void* keys, const void* values, const gr_cache_layout* layout);

}  // namespace gr
