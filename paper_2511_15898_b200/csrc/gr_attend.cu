// gr_cache_attend: attention of each row's last tokens over the row's tokens in a 4-bit paged cache.
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(x_t - m),  x_t = scale log2(e) q . k_t,  m a number at or a little above the largest x met,
// in one pass over the row's octets.  Codes are whole numbers u, values s (u - 8), so with a scale per 32 dims
//   q . k = sum_j s_j (sum_d q_d u_d - 8 sum_d q_d),     sum_t p_t v_t = sum_t (p_t s_tj) u_td - 8 sum_t p_t s_tj,
// and the matrix instructions take the codes as they are: four bits in the low end of an fp16 number are u 2^-24, the next four 16 u 2^-24
// (subnormal numbers, exact in the products), so a word of eight codes becomes operands by one shift and four ANDs; the 16 goes into
// the queries, or into the result.  Queries are scaled by a power of two that brings a row's largest to 2^13 .. 2^14: exact.
// Keys and values are the 16-row operand (tokens, and depth), query rows the 8 columns: a decode step of eight query heads or
// tokens to a key head wastes nothing.  Rounded to fewer bits: p and p s, to fp16 before the second product, as codes are there: 2^-12 of themselves each,
// against an output of 8 or 11 bits, as long as they are normal fp16 numbers.  So p is held as 2^lift p (kLift), and what is not a normal number
// then is off by 2^-35 of the largest weight: thousands of tokens that share a part of the weight keep it, whatever another token takes, with values
// of 0.05 as with ones of 5 (a lift of 0 lost such parts).  x, m, sums of p and both products are fp32; weights come from x - m, so scores beyond
// what fp32 resolves keep their order.
//
// Work.  A unit is 128 tokens of a (row, head, tile of query rows), or 64; the units of the call in that order are cut into equal shares, one to
// a CTA, however ragged the rows are.  Up to 16 query rows: a CTA of four warps, each takes 32 of a unit's tokens for all of them and brings them
// itself, the next ones while it works on these (cp.async.bulk into a ring of its own).  More: a CTA of up to eight warps, which
// make the operands of 64 tokens together and each take all of them for eight query rows.  What a CTA does not finish it leaves
// as (m, sum, f, product) in the workspace; a second kernel joins the pieces in the order of the tokens, so results do not depend on which CTA was first.
//
// What bounds it.  64 rows of 6000 tokens, 8 heads of 128 dims, 4 query heads each: 108 us, 63 % of the copy rate; 81 without the arithmetic.  16
// tokens of a head take 320 warp instructions (80 of them the shifts and ANDs of their 256 words, 20 matrix instructions), which the
// SMs issue at half of their rate, 16 warps of 128 registers each; three CTAs of 168 registers are as fast, five of 96 spill (149 us).  36 query rows
// (nine tokens of four heads): 127 us where the bytes take 18; matrix instructions of this kind at their full rate would take 30, and it has the same
// half of the issue slots, barriers between making operands and using them among them (four warps that each made their own for 16 query rows: 163).
// One request of 900 tokens: 12 us, two launches and the chains of loads (offsets, positions, table, octets) before the first product.
#include <math.h>
#include <algorithm>
#include "gr_host.h"
#include "gr_cache.cuh"

namespace gr {

constexpr int kEaters = 4;                     // warps of a CTA that takes up to 16 query rows
constexpr int kMostWarps = 8;                  // of one that takes more, 8 each
constexpr int kBite = 32;                      // tokens that a warp takes at a time
// How far above the largest x met the reference is put (p stays at or below 1): at 0 it has to follow every few tokens (36 query rows 141 -> 136 us, a
// decode batch 115 -> 111).
constexpr float kHeadroom = 4.f;
// Weights are held as 2^lift p, lift 14 for scales of values up to 2 (values up to 16) and one less for each power of two that a query row's scales go beyond, so
// that weights and their products with scales are at the upper end of fp16 numbers.  The largest weight is held as 2^10 at least; what is below 2^-14
// is off by 2^-25, that is by 2^-35 of it.  (Looked at for all 32 tokens by one word or two to a lane: a decode batch 110 -> 111 us, drafts 126 -> 128.)
constexpr float kLift = 14.f;
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;
constexpr unsigned long long kWaitNs = 2000000000ull;      // longest wait for a copy

struct AttendArgs {
    const void* q; void* out;
    long long q_token, q_head, out_token, out_head;
    const char* cache; long long block_stride, head_bytes;
    const int* table; const int* offsets; const int* positions; int* status;
    int dtype, q_vec, out_vec, tokens, heads, group, octets, num_blocks, width, rows, window, most;     // octets: of a block; most: tokens that a table's row has room for
    unsigned by_octets; int shift;             // quotients by octets
    int tile_rows;                             // query rows of an item
    float scale;                               // with log2(e)
    char* ws; int ctas;
    GR_SPAN(in_q); GR_SPAN(out_q); GR_SPAN(held); GR_SPAN(blocks); GR_SPAN(starts); GR_SPAN(places); GR_SPAN(states); GR_SPAN(room);
};

// What a CTA says of the piece that it began and did not finish.
struct __align__(32) AttendNote { int valid, token, row, rows, head, last, failed, pad; };     // rows from flat row `row` of the tokens from `token` on; last: the CTA with the end
static_assert(sizeof(AttendNote) == 32, "workspace layout");

template <int J, int NT, bool kRows>
struct Shape {
    static constexpr int D = 32 * J, kOctet = octet_bytes(D), kWarps = kRows ? kMostWarps : kEaters;
    static constexpr int kTile = kRows ? 64 : kBite * kEaters;             // tokens of a unit
    static constexpr int kStage = (kRows ? kTile : kBite) / 8 * kOctet;    // bytes of a place in a ring
    static constexpr int kRings = kRows ? 1 : kEaters;
    static constexpr int kStep = D + 4;        // floats from one row of the joined results to the next: threads of a quarter warp meet all banks
    static constexpr int kJoin = kRows ? 0 : 2 * 8 * NT * kStep * 4;
    static constexpr int kOperands = kRows ? kTile / 16 * J * 2 * 1024 : 0;  // a unit's keys and values as operands
    // resident CTAs per SM, by registers (128, 168 or 255 a thread); of many query rows as many as there is room for
    static constexpr int kCtas = kRows ? (J <= 4 ? 2 : 1) : NT == 1 ? (J <= 4 ? 4 : J <= 6 ? 3 : 2) : (J <= 1 ? 4 : J <= 3 ? 3 : 2);
    static constexpr int kRoom = 227 * 1024 / kCtas - 2560 - kJoin - kOperands;
    static constexpr int kStages = kRows ? 2 : kRoom / (kRings * kStage) < 4 ? kRoom / (kRings * kStage) : 4;
    static constexpr int kSmem = kStages * kRings * kStage + kJoin + kOperands;
    static_assert(kStages >= 2 && kRoom >= kStages * kRings * kStage, "a ring");
    static int ctas(int warps) { return kRows ? std::max(1, std::min((J <= 4 ? 16 : 8) / warps, 227 * 1024 / (kSmem + 2560))) : kCtas; }
};
constexpr int kMaxStages = 4;
__host__ __device__ inline size_t piece_floats(int tile_rows, int dim) { return (size_t)tile_rows * (dim + 3); }      // m, l, f, product

// ---------------------------------------------------------------- instructions

__device__ __forceinline__ unsigned smem_addr(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(unsigned bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity)
{
    unsigned done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
__device__ __forceinline__ unsigned long long now_ns() { unsigned long long t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
// false: it did not happen within kWaitNs
__device__ __noinline__ bool bar_wait_long(unsigned bar, unsigned parity)
{
    const unsigned long long from = now_ns();
    while (!bar_try(bar, parity)) if (now_ns() - from > kWaitNs) return false;
    return true;
}
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity)
{
    return bar_try(bar, parity) || bar_wait_long(bar, parity);
}
__device__ __forceinline__ void bulk_load(unsigned to, const void* from, unsigned bytes, unsigned bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1, float c0, float c1, float c2, float c3)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void mma(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    mma(d, a0, a1, a2, a3, b0, b1, d[0], d[1], d[2], d[3]);
}
__device__ __forceinline__ void mma8(float (&d)[4], unsigned a0, unsigned a1, unsigned b)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(b));
}
__device__ __forceinline__ unsigned transposed(unsigned v)
{
    unsigned r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float exp2_of(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ unsigned pack_h2(float lo, float hi) { const __half2 h = __floats2half2_rn(lo, hi); return *reinterpret_cast<const unsigned*>(&h); }
__device__ __forceinline__ unsigned mul_h2(unsigned a, unsigned b)
{
    const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const unsigned*>(&h);
}
template <int J>
__device__ __forceinline__ void load_words(unsigned (&w)[J], const char* p)        // J words, aligned to 4 J bytes
{
    constexpr int W = J % 4 == 0 ? 4 : J % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < J; i += W) {
        const Pack<unsigned, W> v = *reinterpret_cast<const Pack<unsigned, W>*>(p + 4 * i);
#pragma unroll
        for (int z = 0; z < W; z++) w[i + z] = v.x[z];
    }
}

// J fp16 numbers, two to a word, aligned to 2 J bytes
template <int J>
__device__ __forceinline__ void load_halves(unsigned (&w)[(J + 1) / 2], const char* p)
{
    if constexpr (J % 2 == 0) load_words<J / 2>(w, p);
    else {
#pragma unroll
        for (int i = 0; i < J; i++) {
            const unsigned h = *reinterpret_cast<const unsigned short*>(p + 2 * i);
            w[i / 2] = i & 1 ? w[i / 2] | h << 16 : h;
        }
    }
}
__device__ __forceinline__ float half_of(const unsigned* w, int i)
{
    const __half2 h = *reinterpret_cast<const __half2*>(w + i / 2);
    return i & 1 ? __high2float(h) : __low2float(h);
}

// ---------------------------------------------------------------- the order of the work

// A place in the call's units: an item is (row, head, tile of query rows), of `count` units of which `at` are behind.  (kTile: tokens of a unit.)
struct Walk {
    int r, token, n, p0;                       // row; its first query token, their number, the first one's position
    int h, y, lo, hi, first, count, at;        // first: the item's first unit of the row's; [lo, hi): tokens that any of its query rows sees
};
__device__ __forceinline__ void walk_row(Walk& w, const AttendArgs& A)
{
    if (!GR_WITHIN(A.starts, A.offsets + w.r, 8)) { w.token = w.n = 0; w.p0 = -1; return; }
    w.token = min(max(A.offsets[w.r], 0), A.tokens);
    w.n = min(max(A.offsets[w.r + 1], w.token), A.tokens) - w.token;
    w.p0 = w.n > 0 && GR_WITHIN(A.places, A.positions + w.token, 4) ? A.positions[w.token] : -1;
}
template <int kTile>
__device__ __forceinline__ void walk_item(Walk& w, const AttendArgs& A)
{
    const int first = w.y * A.tile_rows / A.group, last = (min(w.n * A.group, (w.y + 1) * A.tile_rows) - 1) / A.group;
    w.hi = w.p0 < 0 ? 0 : (int)min((long long)w.p0 + last + 1, (long long)A.most);
    w.lo = A.window > 0 ? (int)max((long long)w.p0 + first - A.window + 1, 0ll) : 0;
    w.lo = min(w.lo, w.hi);
    w.first = w.lo / kTile;
    w.count = w.hi > w.lo ? (w.hi + kTile - 1) / kTile - w.first : 1;        // (a row that sees nothing: a unit of nothing, which writes its zeros)
}
// units of a head of row w.r (64 bits: a prompt of 2^21 tokens has more than 2^31)
template <int kTile>
__device__ __forceinline__ long long row_units(Walk& w, const AttendArgs& A)
{
    long long sum = 0;
    for (w.y = 0; w.y * A.tile_rows < w.n * A.group; w.y++) { walk_item<kTile>(w, A); sum += w.count; }
    return sum;
}
template <int kTile>
__device__ __forceinline__ void walk_next(Walk& w, const AttendArgs& A)
{
    w.at = 0;
    if (++w.y * A.tile_rows >= w.n * A.group) {
        w.y = 0;
        if (++w.h == A.heads) {
            w.h = 0;
            do { if (++w.r >= A.rows) return; walk_row(w, A); } while (w.n == 0);
        }
    }
    walk_item<kTile>(w, A);
}

// where share i of `parts` of the units begins (32 bits divide in a fraction of the time)
__device__ __forceinline__ long long share_of(long long total, int i, long long parts)
{
    return total < (1 << 20) ? (long long)((unsigned)total * (unsigned)i / (unsigned)parts) : total * i / parts;
}

extern __shared__ __align__(128) char attend_rings[];

// ---------------------------------------------------------------- a warp's share

template <int J, int NT>
struct State {
    uint4 q[NT][J];                            // the queries as operands, scaled
    unsigned sum[NT][(J + 3) / 4];             // -8 2^-24 times the queries' sums by groups, in two fp16 parts, as operands (group t, t + 4)
    float f[NT][2];                            // from products to x, positive
    float m[NT][2], ref[NT][2], l[NT][2];      // m: no product is above it; ref: `lift` below m, or 0 where there is none
    float o[NT][2 * J][4], off[NT][4];
};

// Whether one of this lane's share of the scales of four octets' values, of those that are there, is 2 or more in magnitude (fp16 numbers that have
// the highest bit of their exponent), or none.
template <int J>
__device__ __forceinline__ bool large_scales(const char* at, unsigned have, int lane)
{
    constexpr int D = 32 * J;
    const char* from = at + (lane >> 3) * octet_bytes(D) + octet_vscale(D);
    unsigned share = 0u;
    if constexpr (J % 2 == 0) {
        unsigned z[J / 2];
        load_words<J / 2>(z, from + 2 * J * (lane & 7));
#pragma unroll
        for (int i = 0; i < J / 2; i++) share |= z[i];
    } else {
#pragma unroll
        for (int i = 0; i < (J + 1) / 2; i++)
            if (8 * i + (lane & 7) < 4 * J) share |= *(const unsigned*)(from + 4 * (8 * i + (lane & 7)));
    }
    return (share & 0x40004000u) && have >> (lane >> 3) & 1;
}
// the lift for scales up to `top` (fp16, a number)
__device__ __forceinline__ float lift_for(unsigned top)
{
    const unsigned bits = __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
    return fminf(kLift, kLift + 1.f + 127.f - (float)((bits + 0x7fffffu) >> 23));
}

// Query rows from flat row `row` on of the item's tokens.  lifts: their headroom and lift, in units of products, in shared memory.
template <int J, int NT>
__device__ __forceinline__ void load_queries(State<J, NT>& s, float2* lifts, const AttendArgs& A, const Walk& w, int row, int lane)
{
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int x = 0; x < NT; x++) {
        const int i = row + 8 * x + g;
        const bool in = i < w.n * A.group;
        const int tok = i / A.group;
        const unsigned short* p = (const unsigned short*)A.q + (in ? (w.token + tok) * A.q_token + (long long)(w.h * A.group + i - tok * A.group) * A.q_head : 0) + 8 * t;
        float v[J][8];
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < J; j++) {
            unsigned d[4] = {0, 0, 0, 0};
            if (in && GR_WITHIN(A.in_q, p + 32 * j, 16)) {
                if (A.q_vec) { const uint4 z = *reinterpret_cast<const uint4*>(p + 32 * j); d[0] = z.x; d[1] = z.y; d[2] = z.z; d[3] = z.w; }
                else {
#pragma unroll
                    for (int e = 0; e < 8; e++) d[e >> 1] |= (unsigned)p[32 * j + e] << (16 * (e & 1));
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (A.dtype == GR_BF16) { v[j][2 * e] = __uint_as_float(d[e] << 16); v[j][2 * e + 1] = __uint_as_float(d[e] & 0xffff0000u); }
                else { const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&d[e])); v[j][2 * e] = z.x; v[j][2 * e + 1] = z.y; }
                most = fmaxf(most, fmaxf(fabsf(v[j][2 * e]), fabsf(v[j][2 * e + 1])));
            }
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        int up = 140 - (int)(__float_as_uint(most) >> 23) + 127;             // exponent field of 2^(13 - exponent of most)
        up = most > 0.f && most < INFINITY ? min(max(up, 1), 253) : 127;
        const float by = copysignf(__uint_as_float((unsigned)up << 23), A.scale);        // (a negative scale turns the queries around)
        // (2^24 / by goes onto the scale from the side on which nothing overflows that is not beyond 2^100.  From there on, products that differ at all,
        // which they do by 2^-72 at least, are so far apart that the largest alone has weight, as at 2^100; below 1e-30 no two are told apart)
        const float size = fabsf(A.scale), inverse = __uint_as_float((unsigned)(254 - up) << 23);
        const float back = fminf(fmaxf(up < 127 ? size * 16777216.f * inverse : size * (16777216.f * inverse), 1e-30f), 1.267650600e30f);
        if (t == 0) lifts[8 * x + g] = make_float2(kHeadroom / back, kLift / back);
        s.f[x][0] = __shfl_sync(0xffffffffu, back, 8 * t); s.f[x][1] = __shfl_sync(0xffffffffu, back, 8 * t + 4);
#pragma unroll
        for (int j = 0; j < J; j += 4) s.sum[x][j / 4] = 0u;
#pragma unroll
        for (int j = 0; j < J; j++) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) { v[j][e] *= by; sum += v[j][e]; }
            s.q[x][j] = make_uint4(pack_h2(v[j][0], v[j][4]), pack_h2(v[j][1] * 0.0625f, v[j][5] * 0.0625f),
                                   pack_h2(v[j][2], v[j][6]), pack_h2(v[j][3] * 0.0625f, v[j][7] * 0.0625f));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            // (below 2^-2; what the second part leaves is at most 2^-25, an eighth of a unit of the largest of the 32 products)
            sum *= -8.f / 16777216.f;
            const float high = __half2float(__float2half_rn(sum));
            if (t == (j & 3)) s.sum[x][j / 4] = pack_h2(high, sum - high);
        }
#pragma unroll
        for (int z = 0; z < 2; z++) { s.m[x][z] = -INFINITY; s.ref[x][z] = 0.f; s.l[x][z] = 0.f; }
#pragma unroll
        for (int z = 0; z < 4; z++) {
            s.off[x][z] = 0.f;
#pragma unroll
            for (int j = 0; j < 2 * J; j++) s.o[x][j][z] = 0.f;
        }
    }
    __syncwarp();                              // (lifts)
}

// Operands out of two octets' words: of keys rows are tokens, four dims of eight to a step; of values rows are dims.
__device__ __forceinline__ uint4 key_operand(unsigned w0, unsigned w1) { return make_uint4(w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u); }
__device__ __forceinline__ uint4 value_operand(unsigned w0, unsigned w1) { return make_uint4(w0 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x000f000fu, w1 & 0x00f000f0u); }

// 16 tokens' keys or values as operands: to[J][2][32 lanes]
template <int J>
__device__ __forceinline__ void make_operands(uint4* to, const char* at, bool values, int lane)
{
    constexpr int D = 32 * J, kOctet = octet_bytes(D);
    unsigned w0[J], w1[J];
    if (!GR_WITHIN(shared_span(attend_rings), at, 2 * kOctet) || !GR_WITHIN(shared_span(attend_rings), to, J * 1024)) return;
    at += (values ? octet_vcode(D) : 0) + 4 * J * lane;
    load_words<J>(w0, at);
    load_words<J>(w1, at + kOctet);
#pragma unroll
    for (int j = 0; j < J; j++) {
        to[2 * j * 32 + lane] = values ? value_operand(w0[j], w1[j]) : key_operand(w0[j], w1[j]);
        to[(2 * j + 1) * 32 + lane] = values ? value_operand(w0[j] >> 8, w1[j] >> 8) : key_operand(w0[j] >> 8, w1[j] >> 8);
    }
}

// 32 tokens from `token` on, four octets at `at`.  kAll: every query row sees them all.  Else `have` says which of the octets
// are there, and each query row's own range which of the tokens it sees; what it does not see stays out whatever is held there.
// kReady: `ready` holds the two halves' keys and values as operands (else they are made here).
template <int J, int NT, bool kAll, bool kReady>
__device__ __forceinline__ void eat(State<J, NT>& s, float2* lifts, const uint4* ready, const char* at, int lane, const AttendArgs& A, const Walk& w, int row, int token, unsigned have)
{
    constexpr int D = 32 * J, kOctet = octet_bytes(D);
    const int g = lane >> 2, t = lane & 3;
    float x[NT][2][4];
    if (!GR_WITHIN(shared_span(attend_rings), at, 4 * kOctet) || (kReady && !GR_WITHIN(shared_span(attend_rings), ready, J * 4096))) return;
    {
        // what 8 is taken off for: group by group the scale times the queries' sum
#pragma unroll
        for (int b = 0; b < 2; b++) {
            const char* from = at + 2 * b * kOctet + octet_kscale(D) + 2 * J * g;
#pragma unroll
            for (int j = 0; j < J; j += 4) {
                const unsigned short h0 = j + t < J ? *(const unsigned short*)(from + 2 * (j + t)) : (unsigned short)0;
                const unsigned short h1 = j + t < J ? *(const unsigned short*)(from + kOctet + 2 * (j + t)) : (unsigned short)0;
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    if (j == 0) x[n][b][0] = x[n][b][1] = x[n][b][2] = x[n][b][3] = 0.f;
                    mma8(x[n][b], h0 * 0x10001u, h1 * 0x10001u, s.sum[n][j / 4]);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < 2; b++) {
            unsigned k[2][J], sc[2][(J + 1) / 2];
#pragma unroll
            for (int o = 0; o < 2; o++) {
                const char* from = at + (2 * b + o) * kOctet;
                if (!kReady) load_words<J>(k[o], from + 4 * J * lane);
                load_halves<J>(sc[o], from + octet_kscale(D) + 2 * J * g);
            }
#pragma unroll
            for (int j = 0; j < J; j++) {
                const float c = half_of(sc[0], j), e = half_of(sc[1], j);
                uint4 a0, a1;
                if (kReady) { a0 = ready[((b * 2 * J + j) * 2) * 32 + lane]; a1 = ready[((b * 2 * J + j) * 2 + 1) * 32 + lane]; }
                else { a0 = key_operand(k[0][j], k[1][j]); a1 = key_operand(k[0][j] >> 8, k[1][j] >> 8); }
#pragma unroll
                for (int n = 0; n < NT; n++) {
                    float d[4], (&y)[4] = x[n][b];
                    mma(d, a0.x, a0.y, a0.z, a0.w, s.q[n][j].x, s.q[n][j].y, 0.f, 0.f, 0.f, 0.f);
                    mma(d, a1.x, a1.y, a1.z, a1.w, s.q[n][j].z, s.q[n][j].w);
                    y[0] = fmaf(c, d[0], y[0]); y[1] = fmaf(c, d[1], y[1]); y[2] = fmaf(e, d[2], y[2]); y[3] = fmaf(e, d[3], y[3]);
                }
            }
        }
    }
    // (looked at here, where nothing waits for it)
    const bool large = large_scales<J>(at, kAll ? 15u : have, lane);
    bool more = large;
#pragma unroll
    for (int n = 0; n < NT; n++) {
        if (!kAll) {
#pragma unroll
            for (int z = 0; z < 2; z++) {
                const int i = row + 8 * n + 2 * t + z;
                const long long p = (long long)w.p0 + i / A.group;
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const int tok = token + g + 8 * y;
                    const bool sees = (have >> y & 1) && i < w.n * A.group && w.p0 >= 0 && tok <= p && tok < A.most && (A.window <= 0 || tok > p - A.window);
                    if (!sees) x[n][y >> 1][(y & 1) * 2 + z] = -INFINITY;
                }
            }
        }
        more |= fmaxf(fmaxf(x[n][0][0], x[n][0][2]), fmaxf(x[n][1][0], x[n][1][2])) > s.m[n][0]
                || fmaxf(fmaxf(x[n][0][1], x[n][0][3]), fmaxf(x[n][1][1], x[n][1][3])) > s.m[n][1];
    }
    if (__any_sync(0xffffffffu, more)) {
        // a product is above the reference: that moves above it, by some more, and what has been added up moves along
        // (a scale is 2 or more: the lift of the query rows that see it becomes what fits it)
        const bool larger = __any_sync(0xffffffffu, large);
        if (larger) {
            // the largest scales of tokens g + 8 y, numbers only (a row sees those whose x is not -infinity)
            unsigned most[4];
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const char* from = at + y * kOctet + octet_vscale(D) + 4 * J * (g >> 1) + 2 * (g & 1);
                most[y] = 0u;
#pragma unroll
                for (int j = 0; j < J; j++) {
                    const unsigned h = *(const unsigned short*)(from + 4 * j) & 0x7fffu;
                    most[y] = max(most[y], h < 0x7c00u ? h : 0u);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; n++)
#pragma unroll
                for (int z = 0; z < 2; z++) {
                    unsigned top = 0u;
#pragma unroll
                    for (int y = 0; y < 4; y++) top = max(top, x[n][y >> 1][(y & 1) * 2 + z] == -INFINITY ? 0u : most[y]);
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                    if (g == 0) lifts[8 * n + 2 * t + z].y = fminf(lifts[8 * n + 2 * t + z].y, lift_for(top) / s.f[n][z]);
                }
            __syncwarp();
        }
#pragma unroll
        for (int n = 0; n < NT; n++) {
            float by[2];
#pragma unroll
            for (int z = 0; z < 2; z++) {
                float m = fmaxf(fmaxf(x[n][0][z], x[n][0][z + 2]), fmaxf(x[n][1][z], x[n][1][z + 2]));
#pragma unroll
                for (int o = 4; o < 32; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                const float2 lift = lifts[8 * n + 2 * t + z];
                m = m > s.m[n][z] ? m + lift.x : s.m[n][z];
                const float ref = m == -INFINITY ? 0.f : __fsub_ru(m, lift.y);       // (up: no weight passes 2^lift)
                by[z] = s.m[n][z] == -INFINITY ? 1.f : exp2_of((s.ref[n][z] - ref) * s.f[n][z]);       // (nothing has been added up)
                s.m[n][z] = m;
                s.ref[n][z] = ref;
                s.l[n][z] *= by[z];
            }
#pragma unroll
            for (int z = 0; z < 4; z++) {
                s.off[n][z] *= by[z & 1];
#pragma unroll
                for (int j = 0; j < 2 * J; j++) s.o[n][j][z] *= by[z & 1];
            }
        }
    }
    unsigned p[NT][2][2];
#pragma unroll
    for (int n = 0; n < NT; n++) {
        const unsigned long long down = f_pack(-s.ref[n][0], -s.ref[n][1]), f = f_pack(s.f[n][0], s.f[n][1]);
#pragma unroll
        for (int b = 0; b < 2; b++) {
            float e[4];
#pragma unroll
            for (int z = 0; z < 4; z += 2) {
                // (the difference first, which is exact where it tells: scores that 32 bits do not resolve keep their order, and equal ones their weight)
                const unsigned long long y = mul2(add2(f_pack(x[n][b][z], x[n][b][z + 1]), down), f);
                e[z] = exp2_of(f_lo(y)); e[z + 1] = exp2_of(f_hi(y));
                s.l[n][0] += e[z]; s.l[n][1] += e[z + 1];
            }
            p[n][b][0] = transposed(pack_h2(e[0], e[1]));
            p[n][b][1] = transposed(pack_h2(e[2], e[3]));
        }
    }
#pragma unroll
    for (int b = 0; b < 2; b++) {
        const char* v = at + 2 * b * kOctet + octet_vcode(D);
        const char* sc = at + 2 * b * kOctet + octet_vscale(D);
        unsigned v0[J], v1[J], z0[J], z1[J];
        if (!kReady) {
            load_words<J>(v0, v + 4 * J * lane);
            load_words<J>(v1, v + kOctet + 4 * J * lane);
        }
        load_words<J>(z0, sc + 4 * J * t);
        load_words<J>(z1, sc + kOctet + 4 * J * t);
#pragma unroll
        for (int j = 0; j < J; j++) {
            uint4 a0, a1;
            if (kReady) { a0 = ready[((b * 2 * J + J + j) * 2) * 32 + lane]; a1 = ready[((b * 2 * J + J + j) * 2 + 1) * 32 + lane]; }
            else { a0 = value_operand(v0[j], v1[j]); a1 = value_operand(v0[j] >> 8, v1[j] >> 8); }
#pragma unroll
            for (int n = 0; n < NT; n++) {
                unsigned b0 = mul_h2(p[n][b][0], z0[j]), b1 = mul_h2(p[n][b][1], z1[j]);
                if (!kAll) {
                    // (0 stays 0 whatever the scale is)
                    b0 &= __hneu2_mask(*reinterpret_cast<const __half2*>(&p[n][b][0]), __half2half2(__ushort_as_half(0)));
                    b1 &= __hneu2_mask(*reinterpret_cast<const __half2*>(&p[n][b][1]), __half2half2(__ushort_as_half(0)));
                }
                // (row j: the sums of group j, of the same rounded numbers that the codes are multiplied by, so that a rounding's error is taken u - 8 times)
                const unsigned one = g == j ? 0x3c003c00u : 0u;
                mma(s.off[n], one, 0u, one, 0u, b0, b1);
                mma(s.o[n][2 * j], a0.x, a0.y, a0.z, a0.w, b0, b1);
                mma(s.o[n][2 * j + 1], a1.x, a1.y, a1.z, a1.w, b0, b1);
            }
        }
    }
}

// The products become results, before the division by the sum: o[x][2 j][z], o[x][2 j][z + 2], o[x][2 j + 1][z], o[x][2 j + 1][z + 2] the dims
// 32 j + 4 g .. + 3 of query row 2 t + z of tile x; sums of p over all lanes.
template <int J, int NT>
__device__ __forceinline__ void results(State<J, NT>& s, int lane)
{
#pragma unroll
    for (int x = 0; x < NT; x++)
#pragma unroll
        for (int z = 0; z < 2; z++) {
#pragma unroll
            for (int o = 4; o < 32; o *= 2) s.l[x][z] += __shfl_xor_sync(0xffffffffu, s.l[x][z], o);
#pragma unroll
            for (int j = 0; j < J; j++) {
                const float down = -8.f * __shfl_sync(0xffffffffu, s.off[x][z], 4 * j + (lane & 3));
                s.o[x][2 * j][z] = fmaf(s.o[x][2 * j][z], 16777216.f, down); s.o[x][2 * j][z + 2] = fmaf(s.o[x][2 * j][z + 2], 1048576.f, down);
                s.o[x][2 * j + 1][z] = fmaf(s.o[x][2 * j + 1][z], 16777216.f, down); s.o[x][2 * j + 1][z + 2] = fmaf(s.o[x][2 * j + 1][z + 2], 1048576.f, down);
            }
        }
}
template <int J, int NT>
__device__ __forceinline__ void times(State<J, NT>& s, int x, int z, float by)
{
#pragma unroll
    for (int j = 0; j < 2 * J; j++) { s.o[x][j][z] *= by; s.o[x][j][z + 2] *= by; }
}

__device__ __forceinline__ void store_out(const AttendArgs& A, long long at, const float (&v)[4])
{
    unsigned short* p = (unsigned short*)A.out + at;
    if (!GR_WITHIN(A.out_q, p, 8)) return;
    unsigned d[2];
    if (A.dtype == GR_BF16) {
#pragma unroll
        for (int z = 0; z < 2; z++) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * z], v[2 * z + 1]); d[z] = *reinterpret_cast<const unsigned*>(&h); }
    } else { d[0] = pack_h2(v[0], v[1]); d[1] = pack_h2(v[2], v[3]); }
    if (A.out_vec) *reinterpret_cast<uint2*>(p) = make_uint2(d[0], d[1]);
    else {
#pragma unroll
        for (int z = 0; z < 4; z++) p[z] = (unsigned short)(d[z >> 1] >> (16 * (z & 1)));
    }
}
// (flat row i of the tokens from `token` on)
__device__ __forceinline__ long long out_at(const AttendArgs& A, int token, int i, int head)
{
    const int tok = i / A.group;
    return (long long)(token + tok) * A.out_token + (long long)(head * A.group + i - tok * A.group) * A.out_head;
}

// ---------------------------------------------------------------- first kernel

// Brings octets into a ring, ahead of what is eaten.  An octet of the next 32 is each lane's: where they are is looked up once for several units.  The
// place in the units is in shared memory, for registers.
struct FeedItem {
    const char* head;                          // the cache from the item's head on
    const int* row;                            // the table's row
    int hi, lo, units, token;                  // tokens that are wanted; units of the item; the first token to look up next
    unsigned mask;                             // which of the 32 octets are wanted and there
};
template <int J, int NT, bool kRows>
struct Feeder {
    using S = Shape<J, NT, kRows>;
    static constexpr int kOctets = S::kStage / S::kOctet, kUnits = 32 / kOctets;
    const char* from;                          // this lane's octet, if a copy begins there
    int bytes, fed;                            // of that copy, or 0; units of the item that have been brought

    __device__ __forceinline__ void begin(FeedItem& f, const AttendArgs& A, const Walk& w, int units, int skip, int lane)
    {
        if (lane == 0)
            f = FeedItem{A.cache + (long long)w.h * A.head_bytes, A.table + (long long)w.r * A.width, w.hi, w.lo, min(w.count - w.at, units), (w.first + w.at) * S::kTile + skip, 0u};
        fed = 0;
        __syncwarp();
        look(f, A, lane);
    }
    // (octets next to one another in a block and a unit by one copy: the instruction takes one address a warp, lanes with one each go through it in turn)
    __device__ __forceinline__ void look(FeedItem& f, const AttendArgs& A, int lane)
    {
        // (may pass 2^31 in the units behind the last)
        const unsigned token = (unsigned)f.token + (unsigned)(lane / kOctets * S::kTile + 8 * (lane % kOctets));
        int id = -1, in = 0;
        if (token < (unsigned)f.hi && (int)token + 8 > f.lo) {
            // (blocks of a multiple of eight tokens; the quotient by a product with the reciprocal, rounded up)
            const unsigned octet = token >> 3, block = A.octets == 1 ? octet : __umulhi(octet, A.by_octets) >> A.shift;
            in = (int)(octet - block * (unsigned)A.octets);
            if ((int)block < A.width && GR_WITHIN(A.blocks, f.row + block, 4)) id = f.row[block];
        }
        const bool want = id >= 0 && id < A.num_blocks;
        const unsigned mask = __ballot_sync(0xffffffffu, want);
        const bool start = want && (lane % kOctets == 0 || in == 0 || !(mask >> ((lane - 1) & 31) & 1));
        // up to the next start, or the first that is not wanted
        const unsigned stop = (__ballot_sync(0xffffffffu, start) | ~mask) & ~((2u << lane) - 1u);
        from = f.head + (start ? id * A.block_stride + (long long)in * S::kOctet : 0);
        bytes = start ? ((stop ? __ffs(stop) - 1 : 32) - lane) * S::kOctet : 0;
        __syncwarp();
        if (lane == 0) { f.mask = mask; f.token = (int)((unsigned)f.token + kUnits * S::kTile); }
        __syncwarp();
    }
    // The next unit into place `place` of the ring; `have`: which octets it will hold.  Whether that was the item's last.
    __device__ __forceinline__ bool bring(const FeedItem& f, const AttendArgs& A, char* place, unsigned long long* full, unsigned* have, int lane)
    {
        const int at = fed & (kUnits - 1);
        const unsigned bar = smem_addr(full);
        if (lane == 0) {
            const unsigned here = f.mask >> (at * kOctets) & ((1u << kOctets) - 1u);
            *have = here;
            bar_expect(bar, __popc(here) * S::kOctet);
        }
        __syncwarp();
        if (lane / kOctets == at && bytes > 0 && GR_WITHIN(A.held, from, bytes) && GR_WITHIN(shared_span(attend_rings), place + lane % kOctets * S::kOctet, bytes)) bulk_load(smem_addr(place) + lane % kOctets * S::kOctet, from, bytes, bar);
        return ++fed == f.units;
    }
};

template <int J, int NT, bool kRows>
__global__ void __launch_bounds__(32 * Shape<J, NT, kRows>::kWarps, Shape<J, NT, kRows>::kCtas)
attend_kernel(const __grid_constant__ AttendArgs A)
{
    using S = Shape<J, NT, kRows>;
    constexpr int D = S::D, kStages = S::kStages, kTile = S::kTile, kWarps = S::kWarps;
    const int tile_rows = A.tile_rows, warps = kRows ? blockDim.x >> 5 : kEaters, threads = 32 * warps;
    char* rings = attend_rings;
    __shared__ __align__(8) unsigned long long s_full[S::kRings][kMaxStages];
    __shared__ unsigned s_have[S::kRings][kMaxStages];
    __shared__ float s_m[kEaters][8 * NT], s_l[kEaters][8 * NT];
    __shared__ float2 s_lift[kWarps][8 * NT];
    __shared__ long long s_scan[kWarps], s_from, s_to, s_total, s_ctas;
    __shared__ Walk s_eat[kWarps], s_feed[kWarps];         // each warp's own
    __shared__ FeedItem s_item[kWarps];
    __shared__ int s_failed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < kStages; i++) for (int r = 0; r < S::kRings; r++) bar_init(smem_addr(&s_full[r][i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_failed = 0;
    }
    pdl_wait();
    // ---- this CTA's share of the units
    {
        const int per = (A.rows + threads - 1) / threads;
        long long mine = 0;
        Walk w;
        for (int r = tid * per; r < min((tid + 1) * per, A.rows); r++) {
            w.r = r;
            walk_row(w, A);
            mine += row_units<kTile>(w, A) * A.heads;
        }
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) { const long long z = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += z; }
        if (lane == 31) s_scan[warp] = upto;
        __syncthreads();
        long long total = 0;
#pragma unroll
        for (int i = 0; i < kWarps; i++) if (i < warps) { if (i < warp) upto += s_scan[i]; total += s_scan[i]; }
        const long long ctas = min((long long)A.ctas, total);
        const bool works = blockIdx.x < ctas;
        const long long from = works ? share_of(total, blockIdx.x, ctas) : 0, to = works ? share_of(total, blockIdx.x + 1, ctas) : 0;
        if (tid == 0) { s_from = from; s_to = to; s_total = total; s_ctas = ctas; }
        if (from < to && upto - mine <= from && from < upto) {
            // (one thread's rows hold the share's first unit)
            long long left = from - (upto - mine);
            for (int r = tid * per;; r++) {
                w.r = r;
                walk_row(w, A);
                const long long units = row_units<kTile>(w, A);
                if (left >= units * A.heads) { left -= units * A.heads; continue; }
                w.h = (left | units) >> 32 ? (int)(left / units) : (int)((unsigned)left / (unsigned)units);
                left -= w.h * units;
                for (w.y = 0;; w.y++) {
                    walk_item<kTile>(w, A);
                    if (left < w.count) break;
                    left -= w.count;
                }
                w.at = (int)left;
                break;
            }
#pragma unroll
            for (int i = 0; i < kWarps; i++) { s_eat[i] = w; s_feed[i] = w; }
        }
    }
    __syncthreads();
    const long long from = s_from;
    const int total = (int)(s_to - from);      // (a share of 2^31 units would take hours)
    AttendNote* note = reinterpret_cast<AttendNote*>(A.ws) + blockIdx.x;
    if (!GR_WITHIN(A.room, note, sizeof(AttendNote))) return;
    if (total <= 0) {
        if (tid == 0) *note = AttendNote{0, 0, 0, 0, 0, 0, 0, 0};
        return;
    }
    bool ok = true;                            // (false: a wait ran out; from there on nothing is waited for or brought, and the call says so)
    const bool feeds = !kRows || warp == 0;
    char* ring = rings + (kRows ? 0 : warp * kStages * S::kStage);
    unsigned long long* full = s_full[kRows ? 0 : warp];
    unsigned* held = s_have[kRows ? 0 : warp];
    Feeder<J, NT, kRows> feeder;
    // unit `next` of the share
    auto feed = [&](int next) {
        const int place = next % kStages;
        const bool end = feeder.bring(s_item[warp], A, ring + place * S::kStage, full + place, held + place, lane);
        if (next + 1 == total) return;
        if (end) {
            Walk w = s_feed[warp];
            __syncwarp();
            walk_next<kTile>(w, A);
            if (lane == 0) s_feed[warp] = w;
            feeder.begin(s_item[warp], A, w, total - next - 1, kRows ? 0 : kBite * warp, lane);
        } else if ((feeder.fed & (Feeder<J, NT, kRows>::kUnits - 1)) == 0) feeder.look(s_item[warp], A, lane);
    };
    if (feeds) {
        feeder.begin(s_item[warp], A, s_feed[warp], total, kRows ? 0 : kBite * warp, lane);
        for (int i = 0; i < kStages && i < total; i++) feed(i);
    }

    State<J, NT> s;
    AttendNote left = {0, 0, 0, 0, 0, 0, 0, 0};
    float* pieces = reinterpret_cast<float*>(A.ws + (size_t)A.ctas * sizeof(AttendNote));
    const Walk& w = s_eat[warp];
    int done = 0;
    while (done < total) {
        const int row = w.y * tile_rows + (kRows ? warp * 8 * NT : 0);         // this warp's first query row
        load_queries<J, NT>(s, s_lift[warp], A, w, row, lane);
        const int item_rows = min(tile_rows, w.n * A.group - w.y * tile_rows), last_row = w.y * tile_rows + item_rows - 1;
        const bool idle = kRows && row > last_row;
        // tokens that all of the item's query rows see
        const int all_hi = w.p0 < 0 ? 0 : (int)min((long long)w.p0 + w.y * tile_rows / A.group + 1, (long long)A.most);
        const int all_lo = A.window > 0 ? (int)min(max((long long)w.p0 + last_row / A.group - A.window + 1, 0ll), (long long)A.most) : 0;
        const int begin = w.at, count = w.count, upto = min(count, begin + total - done);
        int token = (w.first + begin) * kTile + (kRows ? 0 : kBite * warp);
        for (int at = begin; at < upto; at++, done++, token += kTile) {
            const int stage = done % kStages;
            if (ok) ok = __all_sync(0xffffffffu, bar_wait(smem_addr(full + stage), (done / kStages) & 1));
            const unsigned have = ok ? held[stage] : 0u;
            const char* octets = ring + stage * S::kStage;
            if (kRows) {
                // the warps make the operands together, then all take all of them
                // (of octets that are not there too: whatever the codes are they are numbers, and 0 times them is 0)
                uint4* ready = reinterpret_cast<uint4*>(rings + S::kRings * kStages * S::kStage + S::kJoin);
                for (int i = warp; i < kTile / 8; i += warps) make_operands<J>(ready + i * J * 64, octets + (i & ~1) * S::kOctet, i & 1, lane);
                __syncthreads();
                if (!idle) {
#pragma unroll 1
                    for (int b = 0; b < kTile / kBite; b++) {
                        const unsigned four = have >> (4 * b) & 15;
                        const uint4* from = ready + b * J * 256;
                        if (four == 15 && token + kBite * b >= all_lo && token + kBite * (b + 1) <= all_hi)
                            eat<J, NT, true, true>(s, s_lift[warp], from, octets + 4 * b * S::kOctet, lane, A, w, row, token + kBite * b, four);
                        else if (four) eat<J, NT, false, true>(s, s_lift[warp], from, octets + 4 * b * S::kOctet, lane, A, w, row, token + kBite * b, four);
                    }
                }
                __syncthreads();
                if (feeds && ok && done + kStages < total) feed(done + kStages);
            } else {
                if (have == 15 && token >= all_lo && token + kBite <= all_hi) eat<J, NT, true, false>(s, s_lift[warp], nullptr, octets, lane, A, w, row, token, have);
                else if (have) eat<J, NT, false, false>(s, s_lift[warp], nullptr, octets, lane, A, w, row, token, have);
                __syncwarp();
                if (ok && done + kStages < total) feed(done + kStages);
            }
        }
        // ---- the item's end, or this CTA's
        const bool complete = begin == 0 && upto == count;
        float* piece = pieces + (2 * (size_t)blockIdx.x + (begin == 0 ? 1 : 0)) * piece_floats(tile_rows, D);
        const int g = lane >> 2, t = lane & 3;
        results<J, NT>(s, lane);
        if (!kRows) {
            // the warps' results to the first one's: half of them to the others, twice
            if (g == 0) {
#pragma unroll
                for (int x = 0; x < NT; x++)
#pragma unroll
                    for (int z = 0; z < 2; z++) {
                        s_m[warp][8 * x + 2 * t + z] = s.m[x][z] == -INFINITY ? -INFINITY : s.ref[x][z];
                        s_l[warp][8 * x + 2 * t + z] = s.l[x][z];
                    }
            }
            __syncthreads();
            float* join = reinterpret_cast<float*>(rings + S::kRings * kStages * S::kStage);
            float* mine = join + (warp & 1) * 8 * NT * S::kStep;
#pragma unroll
            for (int x = 0; x < NT; x++)
#pragma unroll
                for (int z = 0; z < 2; z++) {
                    const int i = 8 * x + 2 * t + z;
                    float m = -INFINITY, l = 0.f;
#pragma unroll
                    for (int k = 0; k < kEaters; k++) m = fmaxf(m, s_m[k][i]);
#pragma unroll
                    for (int k = 0; k < kEaters; k++) l += s_m[k][i] == -INFINITY ? s_l[k][i] : s_l[k][i] * exp2_of((s_m[k][i] - m) * s.f[x][z]);      // (0, or NaN)
                    if (s.m[x][z] != -INFINITY) times(s, x, z, exp2_of((s.ref[x][z] - m) * s.f[x][z]));
                    s.m[x][z] = m; s.l[x][z] = l;
                }
#pragma unroll
            for (int step = 2; step > 0; step >>= 1) {
                if (warp >= step && warp < 2 * step) {
                    float* to = step == 1 ? join : mine;
#pragma unroll
                    for (int x = 0; x < NT; x++)
#pragma unroll
                        for (int z = 0; z < 2; z++)
#pragma unroll
                            for (int j = 0; j < J; j++)
                                if (GR_WITHIN(shared_span(attend_rings), to + (8 * x + 2 * t + z) * S::kStep + 32 * j + 4 * g, 16))
                                    *reinterpret_cast<float4*>(to + (8 * x + 2 * t + z) * S::kStep + 32 * j + 4 * g) =
                                        make_float4(s.o[x][2 * j][z], s.o[x][2 * j][z + 2], s.o[x][2 * j + 1][z], s.o[x][2 * j + 1][z + 2]);
                }
                __syncthreads();
                if (warp < step) {
#pragma unroll
                    for (int x = 0; x < NT; x++)
#pragma unroll
                        for (int z = 0; z < 2; z++)
#pragma unroll
                            for (int j = 0; j < J; j++) {
                                const float4 v = *reinterpret_cast<const float4*>(mine + (8 * x + 2 * t + z) * S::kStep + 32 * j + 4 * g);
                                s.o[x][2 * j][z] += v.x; s.o[x][2 * j][z + 2] += v.y; s.o[x][2 * j + 1][z] += v.z; s.o[x][2 * j + 1][z + 2] += v.w;
                            }
                }
                __syncthreads();
            }
        }
        if (kRows || warp == 0) {
#pragma unroll
            for (int x = 0; x < NT; x++)
#pragma unroll
                for (int z = 0; z < 2; z++) {
                    const int i = (kRows ? warp * 8 * NT : 0) + 8 * x + 2 * t + z;
                    if (i >= item_rows) continue;
                    if (!complete) {
                        if (!GR_WITHIN(A.room, piece, piece_floats(tile_rows, D) * sizeof(float))) continue;
                        if (g == 0) { piece[i] = kRows && s.m[x][z] != -INFINITY ? s.ref[x][z] : s.m[x][z]; piece[tile_rows + i] = s.l[x][z]; piece[2 * tile_rows + i] = s.f[x][z]; }
#pragma unroll
                        for (int j = 0; j < J; j++)
                            *reinterpret_cast<float4*>(piece + 3 * tile_rows + i * D + 32 * j + 4 * g) =
                                make_float4(s.o[x][2 * j][z], s.o[x][2 * j][z + 2], s.o[x][2 * j + 1][z], s.o[x][2 * j + 1][z + 2]);
                        continue;
                    }
                    const float by = s.l[x][z] == 0.f ? 0.f : 1.f / s.l[x][z];
                    const long long to = out_at(A, w.token, w.y * tile_rows + i, w.h) + 4 * g;
#pragma unroll
                    for (int j = 0; j < J; j++) {
                        const float v[4] = {s.o[x][2 * j][z] * by, s.o[x][2 * j][z + 2] * by, s.o[x][2 * j + 1][z] * by, s.o[x][2 * j + 1][z + 2] * by};
                        store_out(A, to + 32 * j, v);
                    }
                }
        }
        if (begin == 0 && !complete) {
            // the CTA with the item's last unit
            const long long end = from + done - upto + count - 1, all = s_total, ctas = s_ctas;
            long long c = end * ctas / all;
            while (share_of(all, (int)c + 1, ctas) <= end) c++;
            left = AttendNote{1, w.token, w.y * tile_rows, item_rows, w.h, (int)c, 0, 0};
        }
        if (upto == count && done < total) {
            Walk next = w;
            __syncwarp();
            walk_next<kTile>(next, A);
            if (lane == 0) s_eat[warp] = next;
            __syncwarp();
        }
    }
    if (feeds) {
        // (its copies end before it does, whether or not they were waited for)
        for (int i = max(0, total - kStages); i < total; i++) ok &= bar_wait(smem_addr(full + i % kStages), (i / kStages) & 1);
    }
    if (!ok && lane == 0) *(volatile int*)&s_failed = 1;
    __syncthreads();
    if (tid == 0) { left.failed = *(volatile int*)&s_failed; *note = left; }
}

// ---------------------------------------------------------------- second kernel

// Joins the pieces of the item that CTA blockIdx.x began and did not finish, a query row to a warp, in the order of the tokens.  kWide, where
// there are few items of many pieces: of the blockIdx.x-th such item, query row blockIdx.y, every eighth piece to a warp.  The last
// blockIdx.y says of every row of the call whether its positions and block ids are ones.
template <int V, bool kWide>                   // V: vectors of a query row to a lane
__global__ void __launch_bounds__(kJoinThreads)
attend_join_kernel(const __grid_constant__ AttendArgs A, int tile_rows, int dim)
{
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const AttendNote* notes = reinterpret_cast<const AttendNote*>(A.ws);
    if (blockIdx.y + 1 < gridDim.y) {
        __shared__ int s_first, s_count[kJoinWarps];
        __shared__ float4 s_sum[kWide ? kJoinWarps : 1][kWide ? 32 * V : 1];
        int first = blockIdx.x;
        if (kWide) {
            // the blockIdx.x-th of the CTAs that began an item and did not finish it
            if (tid == 0) s_first = -1;
            int before = 0;
            for (int c0 = 0; c0 < A.ctas; c0 += kJoinThreads) {
                const int c = c0 + tid;
                const bool valid = c < A.ctas && notes[c].valid;
                const unsigned mask = __ballot_sync(0xffffffffu, valid);
                if (lane == 0) s_count[warp] = __popc(mask);
                __syncthreads();
                int at = before + __popc(mask & ((1u << lane) - 1u));
                for (int k = 0; k < kJoinWarps; k++) { if (k < warp) at += s_count[k]; before += s_count[k]; }
                if (valid && at == (int)blockIdx.x) s_first = c;
                __syncthreads();
            }
            first = s_first;
            if (first < 0) return;
        }
        const AttendNote note = notes[first];
        const int i = kWide ? (int)blockIdx.y : (int)blockIdx.y * kJoinWarps + warp;
        if (!note.valid || i >= note.rows) return;
        const float* pieces = reinterpret_cast<const float*>(A.ws + (size_t)A.ctas * sizeof(AttendNote));
        const size_t size = piece_floats(tile_rows, dim);
        const int all = note.last - first + 1, member = kWide ? warp : 0, every = kWide ? kJoinWarps : 1, count = (all - member + every - 1) / every;
        // (of the k-th of this warp's:) of the item's first CTA the one it began, of the k-th behind it the one it went on with
        auto piece = [&](int n) { const int k = member + n * every; return pieces + (k == 0 ? 2 * (size_t)first + 1 : 2 * ((size_t)first + k)) * size; };
        constexpr int kAhead = 8 / V;          // pieces on their way at a time
        float4 v[kAhead][V];
        auto load = [&](int k0) {
#pragma unroll
            for (int u = 0; u < kAhead; u++)
#pragma unroll
                for (int z = 0; z < V; z++)
                    if (k0 + u < count && GR_WITHIN(A.room, piece(k0 + u), size * sizeof(float))) v[u][z] = *reinterpret_cast<const float4*>(piece(k0 + u) + 3 * tile_rows + i * dim + min(4 * (lane + 32 * z), dim - 4));
        };
        load(0);
        const float f = pieces[(2 * (size_t)first + 1) * size + 2 * tile_rows + i];
        float m = -INFINITY, l = 0.f;
        float4 sum[V];
#pragma unroll
        for (int z = 0; z < V; z++) sum[z] = make_float4(0.f, 0.f, 0.f, 0.f);
        // (the largest of up to 32 pieces at a time: what has been added up moves there)
        for (int k0 = 0; k0 < count; k0 += 32) {
            float pm = -INFINITY, pl = 0.f;
            if (k0 + lane < count && GR_WITHIN(A.room, piece(k0 + lane), size * sizeof(float))) { const float* p = piece(k0 + lane); pm = p[i]; pl = p[tile_rows + i]; }
            float top = pm;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            top = fmaxf(top, m);
            const float down = m == -INFINITY ? 1.f : exp2_of((m - top) * f), by = pm == -INFINITY ? 1.f : exp2_of((pm - top) * f);      // (0 or NaN throughout where m is -infinity)
            pl *= by;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) pl += __shfl_xor_sync(0xffffffffu, pl, o);
            l = fmaf(l, down, pl);
            m = top;
#pragma unroll
            for (int z = 0; z < V; z++) { sum[z].x *= down; sum[z].y *= down; sum[z].z *= down; sum[z].w *= down; }
#pragma unroll 1
            for (int k1 = k0; k1 < min(k0 + 32, count); k1 += kAhead) {
                if (k1 > 0) load(k1);
#pragma unroll
                for (int u = 0; u < kAhead; u++) {
                    const float w = __shfl_sync(0xffffffffu, by, (k1 - k0 + u) & 31);
                    if (k1 + u >= count) continue;
#pragma unroll
                    for (int z = 0; z < V; z++) {
                        sum[z].x = fmaf(v[u][z].x, w, sum[z].x); sum[z].y = fmaf(v[u][z].y, w, sum[z].y);
                        sum[z].z = fmaf(v[u][z].z, w, sum[z].z); sum[z].w = fmaf(v[u][z].w, w, sum[z].w);
                    }
                }
            }
        }
        if (kWide) {
            // the warps' shares, in their order
            __shared__ float s_m[kJoinWarps], s_l[kJoinWarps];
            if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
            for (int z = 0; z < V; z++) s_sum[warp][lane + 32 * z] = sum[z];
            __syncthreads();
            if (warp > 0) return;
            float top = m;
            for (int k = 1; k < kJoinWarps; k++) top = fmaxf(top, s_m[k]);
            l = 0.f;
#pragma unroll
            for (int z = 0; z < V; z++) sum[z] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < kJoinWarps; k++) {
                const float by = s_m[k] == -INFINITY ? 1.f : exp2_of((s_m[k] - top) * f);
                l = fmaf(s_l[k], by, l);
#pragma unroll
                for (int z = 0; z < V; z++) {
                    const float4 v = s_sum[k][lane + 32 * z];
                    sum[z].x = fmaf(v.x, by, sum[z].x); sum[z].y = fmaf(v.y, by, sum[z].y); sum[z].z = fmaf(v.z, by, sum[z].z); sum[z].w = fmaf(v.w, by, sum[z].w);
                }
            }
        }
        const float by = l == 0.f ? 0.f : 1.f / l;
        const long long at = out_at(A, note.token, note.row + i, note.head);
#pragma unroll
        for (int z = 0; z < V; z++) {
            const int d = 4 * (lane + 32 * z);
            const float o[4] = {sum[z].x * by, sum[z].y * by, sum[z].z * by, sum[z].w * by};
            if (d < dim) store_out(A, at + d, o);
        }
        return;
    }
    bool failed = false;
    for (int c = tid; c < A.ctas; c += kJoinThreads) failed |= notes[c].failed != 0;
    failed = __syncthreads_or(failed);
    for (int r = blockIdx.x; r < A.rows; r += gridDim.x) {
        Walk w;
        w.r = r;
        walk_row(w, A);
        bool bad = A.offsets[r] < 0 || A.offsets[r] > A.tokens || A.offsets[r + 1] < A.offsets[r] || A.offsets[r + 1] > A.tokens;
        if (w.n > 0 && w.p0 >= 0) {
            const long long end = (long long)w.p0 + w.n;
            bad |= end > A.most;
            const int size = 8 * A.octets, hi = (int)min(end, (long long)A.most);
            const int lo = A.window > 0 ? (int)min(max((long long)w.p0 - A.window + 1, 0ll), (long long)hi) : 0;
            const int last = (hi + size - 1) / size;
#pragma unroll 4
            for (int b = lo / size + tid; b < last; b += kJoinThreads) {
                if (!GR_WITHIN(A.blocks, A.table + (long long)r * A.width + b, 4)) continue;
                const int id = A.table[(long long)r * A.width + b];
                bad |= id < 0 || id >= A.num_blocks;
            }
        }
        bad = __syncthreads_or(bad);
        if (tid == 0 && GR_WITHIN(A.states, A.status + r, 4)) A.status[r] = failed ? GR_CHECK_FAILED : bad ? GR_BAD_ROW : GR_OK;
    }
}

// ---------------------------------------------------------------- host

// The kernel for a call, by a key head's query rows (a row's tokens times its group, on average): up to 8 in one tile, up to 16 in two (with heads of more
// than 128 dims there are no registers for two); beyond, a warp for each 8.  (17 to 64 by tiles of 8 that each read the row again: 136 us for 126 at 36.)
// The average is all that the host knows, and `tokens` counts the room behind the last row's: 64 decode rows take 105 us, with room for 64 tokens behind them
// too, with room for 1024 383; 63 of them and a prompt of 1000 tokens in one call 670, in two 103 and 113.
struct Choice { int nt; bool rows; int warps; };
static Choice choose(int dim, int group, int rows, int tokens)
{
    const double each = (double)tokens / std::max(1, rows) * group;
    if (each > 16 || (dim > 128 && each > 8)) return {1, true, std::max(2, std::min(kMostWarps, (int)std::min((each + 7) / 8, 100.0)))};
    return {each > 8 ? 2 : 1, false, kEaters};
}
template <int J, int NT, bool kRows> struct Pick { using S = Shape<J, NT, kRows>; };
template <class F>
static auto with_shape(int dim, Choice c, F f)
{
#define GR_ATTEND_J(J) case J: if (c.rows) return f(Pick<J, 1, true>()); if (c.nt == 2) return f(Pick<J, J <= 4 ? 2 : 1, false>()); return f(Pick<J, 1, false>());
    switch (dim / 32) {
        GR_ATTEND_J(1) GR_ATTEND_J(2) GR_ATTEND_J(3) GR_ATTEND_J(4) GR_ATTEND_J(5) GR_ATTEND_J(6) GR_ATTEND_J(7)
        default: if (c.rows) return f(Pick<8, 1, true>()); return f(Pick<8, 1, false>());
    }
#undef GR_ATTEND_J
}
template <int J, int NT, bool kRows> static auto attend_of(Pick<J, NT, kRows>) { return &attend_kernel<J, NT, kRows>; }

static bool attend_shape_ok(int heads, int q_heads, int dim, int rows, int tokens)
{
    return heads >= 1 && heads <= GR_MAX_HEADS && q_heads >= 1 && q_heads <= GR_MAX_HEADS && q_heads % heads == 0 && dim >= 32 && dim <= GR_MAX_DIM_Q4
           && dim % 32 == 0 && rows >= 0 && rows <= (1 << 20) && tokens >= 0 && (long long)tokens * (q_heads / std::max(1, heads)) < (1ll << 31) - 256;
}

}  // namespace gr

extern "C" {

#ifdef GR_CHECK
int gr_attend_check(void) { return gr::span_check(); }
#endif

size_t gr_attend_workspace_bytes(int heads, int q_heads, int dim, int rows, int tokens)
{
    if (!gr::attend_shape_ok(heads, q_heads, dim, rows, tokens)) return 0;
    const gr::Choice c = gr::choose(dim, q_heads / heads, rows, tokens);
    return gr::with_shape(dim, c, [&](auto pick) {
        const size_t ctas = (size_t)gr::kSms * decltype(pick)::S::ctas(c.warps);
        return ctas * (sizeof(gr::AttendNote) + 2 * sizeof(float) * gr::piece_floats(c.rows ? 8 * c.warps : 8 * c.nt, dim));
    });
}

int gr_cache_attend(const void* q, int dtype, int q_heads, long long q_token, long long q_head, const void* cache, const gr_cache_layout* layout,
                    const int* table, int width, int rows, const int* offsets, const int* positions, int tokens, float scale, int window,
                    void* workspace, void* out, long long out_token, long long out_head, int* status, void* stream)
{
    if (!layout) return GR_E_NULL;
    if (layout->format != GR_Q4) return GR_E_INVALID;
    const int rc = gr::check_cache(cache, nullptr, layout);
    if (rc != GR_OK) return rc;
    const gr_cache_layout& L = *layout;
    if ((dtype != GR_BF16 && dtype != GR_F16) || !gr::attend_shape_ok(L.heads, q_heads, L.dim, rows, tokens)) return GR_E_INVALID;
    if (width < 0 || (long long)width * L.block_size >= (1ll << 31) - 256 || (long long)rows * std::max(1, width) >= (1ll << 31)) return GR_E_INVALID;
    if (window < 0 || !(fabsf(scale) < 1.7e38f)) return GR_E_INVALID;        // (with log2(e) still a number)
    if (!gr::counted(q_token, q_head, tokens, q_heads)) return GR_E_INVALID;
    const long long step[2] = {out_token, out_head}, size[2] = {tokens, q_heads};
    if (!gr::apart(L.dim, step, size, 2)) return GR_E_INVALID;
    if (rows == 0) return GR_OK;
    if (!offsets || !workspace || (tokens > 0 && (!q || !out || !positions)) || (width > 0 && !table)) return GR_E_NULL;
    if (((uintptr_t)q & 1) || ((uintptr_t)out & 1) || ((uintptr_t)workspace & 31)) return GR_E_ALIGN;
    if (((uintptr_t)table | (uintptr_t)offsets | (uintptr_t)positions | (uintptr_t)status) & 3) return GR_E_ALIGN;
    const gr::Span written = gr::rows_span(out, 2, L.dim, out_token, out_head, tokens, q_heads);
    if (gr::meet(written, gr::cache_span(cache, L))) return GR_E_INVALID;
    if (gr::meet(written, gr::rows_span(q, 2, L.dim, q_token, q_head, tokens, q_heads))) return GR_E_INVALID;
    // (workspace and status lie apart from all, the lists from what is written; the status is looked at last)
    const gr::Places result = gr::rows_places(out, 2, L.dim, out_token, out_head, tokens, q_heads), in = gr::rows_places(q, 2, L.dim, q_token, q_head, tokens, q_heads);
    const gr::Places lists[3] = {gr::bytes_at(table, 4ll * rows * width), gr::bytes_at(offsets, 4ll * rows + 4), gr::bytes_at(positions, 4ll * tokens)};
    const gr::Places own[2] = {gr::bytes_at(workspace, (long long)gr_attend_workspace_bytes(L.heads, q_heads, L.dim, rows, tokens)), gr::bytes_at(status, 4ll * rows)};
    const gr::Span held = gr::cache_span(cache, L);
    for (const gr::Places& l : lists) if (gr::meet(result, l)) return GR_E_INVALID;
    for (int i = 0; i < 2; i++) {
        if (i == 1 && !status) return GR_E_NULL;
        const gr::Places& o = own[i];
        for (const gr::Places& l : lists) if (gr::meet(o, l)) return GR_E_INVALID;
        if (gr::meet(o, result) || gr::meet(o, in) || gr::meet(held, {o.at, o.at + (uintptr_t)o.unit}) || (i == 1 && gr::meet(o, own[0]))) return GR_E_INVALID;
    }
    gr::AttendArgs A = {};
    A.q = q; A.out = out; A.q_token = q_token; A.q_head = q_head; A.out_token = out_token; A.out_head = out_head;
    A.octets = L.block_size / 8; A.num_blocks = L.num_blocks; A.block_stride = L.block_stride;
    A.cache = (const char*)cache; A.head_bytes = (long long)A.octets * gr::octet_bytes(L.dim);
    A.table = table; A.offsets = offsets; A.positions = positions; A.status = status;
    A.dtype = dtype; A.tokens = tokens; A.heads = L.heads; A.group = q_heads / L.heads; A.width = width; A.rows = rows; A.window = window;
    A.most = width * L.block_size;
    // n / octets for n < 2^28: ceil(2^(32 + shift) / octets) n / 2^(32 + shift), with 2^shift the power of two at or above half of octets
    while (A.octets > 2 << A.shift) A.shift++;
    A.by_octets = A.octets > 1 ? (unsigned)(((1ull << (32 + A.shift)) + (unsigned)A.octets - 1) / (unsigned)A.octets) : 0u;
    A.scale = scale * 1.44269504088896340736f;
    GR_SET_SPAN(A.in_q, gr::rows_span(q, 2, L.dim, q_token, q_head, tokens, q_heads)); GR_SET_SPAN(A.out_q, written); GR_SET_SPAN(A.held, gr::cache_span(cache, L));
    GR_SET_SPAN(A.blocks, {(uintptr_t)table, (uintptr_t)(table + (size_t)rows * width)}); GR_SET_SPAN(A.starts, {(uintptr_t)offsets, (uintptr_t)(offsets + rows + 1)});
    GR_SET_SPAN(A.places, {(uintptr_t)positions, (uintptr_t)(positions + tokens)}); GR_SET_SPAN(A.states, {(uintptr_t)status, (uintptr_t)(status + rows)});
    GR_SET_SPAN(A.room, {(uintptr_t)workspace, (uintptr_t)workspace + gr_attend_workspace_bytes(L.heads, q_heads, L.dim, rows, tokens)});
    A.ws = (char*)workspace;
    gr::Align from, to;
    from.add(q, 2, {tokens > 1 ? q_token : 0, q_heads > 1 ? q_head : 0});
    to.add(out, 2, {tokens > 1 ? out_token : 0, q_heads > 1 ? out_head : 0});
    A.q_vec = from.bits % 16 == 0; A.out_vec = to.bits % 8 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_cache_attend");
    const gr::Choice c = gr::choose(L.dim, A.group, rows, tokens);
    A.tile_rows = c.rows ? 8 * c.warps : 8 * c.nt;
    const int done = gr::with_shape(L.dim, c, [&](auto pick) {
        using S = typename decltype(pick)::S;
        A.ctas = gr::kSms * S::ctas(c.warps);
        const auto kernel = gr::attend_of(pick);
        static bool set[gr::kMaxDevices] = {};
        int device = 0;
        if (cudaGetDevice(&device) != cudaSuccess) return GR_E_LAUNCH;
        if (device >= gr::kMaxDevices || !set[device]) {
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) return GR_E_LAUNCH;
            if (device < gr::kMaxDevices) set[device] = true;
        }
        if (gr::launch_pdl(kernel, A.ctas, 32 * c.warps, S::kSmem, st, A) != cudaSuccess) return GR_E_LAUNCH;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at = {};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        // items that may be: few, and each has many pieces
        const long long items = (long long)A.heads * ((long long)tokens * A.group / A.tile_rows + rows);
        const bool wide = 4 * items <= A.ctas;
        cfg.gridDim = wide ? dim3((unsigned)items, 1u + (unsigned)A.tile_rows) : dim3((unsigned)A.ctas, 1u + (unsigned)((A.tile_rows + gr::kJoinWarps - 1) / gr::kJoinWarps));
        cfg.blockDim = dim3(gr::kJoinThreads); cfg.stream = st; cfg.attrs = &at; cfg.numAttrs = 1;
        const auto join = L.dim > 128 ? (wide ? &gr::attend_join_kernel<2, true> : &gr::attend_join_kernel<2, false>)
                                     : (wide ? &gr::attend_join_kernel<1, true> : &gr::attend_join_kernel<1, false>);
        return cudaLaunchKernelEx(&cfg, join, A, A.tile_rows, L.dim) == cudaSuccess ? GR_OK : GR_E_LAUNCH;
    });
    if (done != GR_OK || cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
