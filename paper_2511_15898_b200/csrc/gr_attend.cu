// gr_cache_attend: attention of each row's last tokens over the row's tokens in a 4-bit paged cache.
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(x_t - m),  x_t = scale log2(e) q . k_t,  m the largest x met,
// in one pass over the row's octets.  Codes are whole numbers u, values s (u - 8), so with a scale per 32 dims
//   q . k = sum_j s_j (sum_d q_d u_d - 8 sum_d q_d),     sum_t p_t v_t = sum_t (p_t s_tj) u_td - 8 sum_t p_t s_tj,
// and the matrix instructions take the codes as they are: four bits in the low end of an fp16 number are u 2^-24, the next four 16 u 2^-24
// (subnormal numbers, exact in the products), so a word of eight codes becomes operands by one shift and four ANDs; the 16 goes into
// the queries, or into the result.  Queries are scaled by a power of two that brings a row's largest to 2^13 .. 2^14: exact.
// Keys and values are the 16-row operand (tokens, and depth), query rows the 8 columns: a decode step of eight query heads or
// tokens to a key head wastes nothing.  Rounded to fewer bits: p (11 bits) and p s (11 bits) before the second product; both are relative to
// themselves, 2^-12 each, against an output of 8 or 11 bits.  x, m, sums of p and both products are fp32.
//
// Work.  A unit is 64 tokens of a (row, head, tile of query rows); the units of the call in that order are cut into equal shares, one to a CTA,
// however ragged the rows are.  A warp brings a unit's octets into a ring in shared memory (cp.async.bulk, one per octet), four warps
// take 16 tokens each (or, where there are many query rows, the same 64 tokens for 16 query rows each).  What a CTA does not finish it
// leaves as (m, sum, product) in the workspace; a second kernel joins the pieces in the order of the tokens, so results do not depend
// on which CTA was first.
#include <math.h>
#include <algorithm>
#include "gr_host.h"
#include "gr_cache.cuh"

namespace gr {

constexpr int kTile = 64;                      // tokens of a unit
constexpr int kEaters = 4;                     // warps that compute; one more brings the octets
constexpr int kAttendThreads = 32 * (kEaters + 1);
constexpr int kJoinThreads = 256;
constexpr unsigned long long kWaitNs = 2000000000ull;      // longest wait for a copy or a free place in the ring

struct AttendArgs {
    const void* q; void* out;
    long long q_token, q_head, out_token, out_head;
    const char* cache; long long block_stride, head_bytes;
    const int* table; const int* offsets; const int* positions; int* status;
    int dtype, q_vec, out_vec, tokens, heads, group, octets, num_blocks, width, rows, window, most;     // octets: of a block; most: tokens that a table's row has room for
    float scale;                               // with log2(e)
    char* ws; int ctas;
};

// What a CTA says of the piece that it began and did not finish.
struct __align__(32) AttendNote { int valid, token, row, rows, head, last, failed, pad; };     // rows from flat row `row` of the tokens from `token` on; last: the CTA with the end
static_assert(sizeof(AttendNote) == 32, "workspace layout");

template <int J, int NT, bool kRows>
struct Shape {
    static constexpr int D = 32 * J, kTileRows = 8 * NT * (kRows ? kEaters : 1), kOctet = octet_bytes(D), kUnit = kTile / 8 * kOctet;
    static constexpr int kStep = D + 4;        // floats from one row of the joined results to the next: threads of a quarter warp meet all banks
    static constexpr int kJoin = kRows ? 0 : kEaters * 8 * NT * kStep * 4;
    static constexpr int kCtas = NT == 1 ? (J <= 2 ? 4 : J <= 4 ? 3 : 2) : (J <= 2 ? 3 : 2);      // resident per SM, by registers
    static constexpr int kRoom = 227 * 1024 / kCtas - 2048 - kJoin;
    static constexpr int kStages = kRoom / kUnit < 8 ? kRoom / kUnit : 8;
    static constexpr int kSmem = kStages * kUnit + kJoin;
    static_assert(kStages >= 2, "a ring");
};
constexpr int kMaxStages = 8;
__host__ __device__ inline size_t piece_floats(int tile_rows, int dim) { return (size_t)tile_rows * (dim + 2); }

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
#pragma unroll 1
    for (int i = 0; i < 32; i++) if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity);
}
__device__ __forceinline__ void bulk_load(unsigned to, const void* from, unsigned bytes, unsigned bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void eaters_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kEaters) : "memory"); }
__device__ __forceinline__ void mma(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

// ---------------------------------------------------------------- the order of the work

// A place in the call's units: an item is (row, head, tile of query rows), of `count` units of which `at` are behind.
struct Walk {
    int r, token, n, p0;                       // row; its first query token, their number, the first one's position
    int h, y, lo, hi, first, count, at;        // first: the item's first unit of 64 tokens; [lo, hi): tokens that any of its query rows sees
};
__device__ __forceinline__ void walk_row(Walk& w, const AttendArgs& A)
{
    w.token = min(max(A.offsets[w.r], 0), A.tokens);
    w.n = min(max(A.offsets[w.r + 1], w.token), A.tokens) - w.token;
    w.p0 = w.n > 0 ? A.positions[w.token] : -1;
}
template <int kTileRows>
__device__ __forceinline__ void walk_item(Walk& w, const AttendArgs& A)
{
    const int first = w.y * kTileRows / A.group, last = (min(w.n * A.group, (w.y + 1) * kTileRows) - 1) / A.group;
    w.hi = w.p0 < 0 ? 0 : (int)min((long long)w.p0 + last + 1, (long long)A.most);
    w.lo = A.window > 0 ? (int)max((long long)w.p0 + first - A.window + 1, 0ll) : 0;
    w.lo = min(w.lo, w.hi);
    w.first = w.lo / kTile;
    w.count = w.hi > w.lo ? (w.hi + kTile - 1) / kTile - w.first : 1;        // (a row that sees nothing: a unit of nothing, which writes its zeros)
}
// units of a head of row w.r
template <int kTileRows>
__device__ __forceinline__ int row_units(Walk& w, const AttendArgs& A)
{
    int sum = 0;
    for (w.y = 0; w.y * kTileRows < w.n * A.group; w.y++) { walk_item<kTileRows>(w, A); sum += w.count; }
    return sum;
}
template <int kTileRows>
__device__ __forceinline__ void walk_next(Walk& w, const AttendArgs& A)
{
    w.at = 0;
    if (++w.y * kTileRows >= w.n * A.group) {
        w.y = 0;
        if (++w.h == A.heads) {
            w.h = 0;
            do { if (++w.r >= A.rows) return; walk_row(w, A); } while (w.n == 0);
        }
    }
    walk_item<kTileRows>(w, A);
}

// ---------------------------------------------------------------- a warp's share

template <int J, int NT>
struct State {
    unsigned q[NT][J][4];                      // the queries as operands, scaled
    float down[NT][J][2];                      // -8 2^-24 times the queries' sums
    float f[NT][2];                            // from products to x
    float m[NT][2], ref[NT][2], l[NT][2];      // ref: m, or 0 where that is -infinity
    float o[NT][2 * J][4], off[NT][4];
};

// Query rows from flat row `row` on of the item's tokens.
template <int J, int NT>
__device__ __forceinline__ void load_queries(State<J, NT>& s, const AttendArgs& A, const Walk& w, int row, int lane)
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
            if (in) {
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
        up = most > 0.f && most < INFINITY ? min(max(up, 1), 254) : 127;
        const float by = __uint_as_float((unsigned)up << 23);
        const float back = A.scale * 16777216.f / by;
        s.f[x][0] = __shfl_sync(0xffffffffu, back, 8 * t); s.f[x][1] = __shfl_sync(0xffffffffu, back, 8 * t + 4);
#pragma unroll
        for (int j = 0; j < J; j++) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) { v[j][e] *= by; sum += v[j][e]; }
#pragma unroll
            for (int z = 0; z < 2; z++) {
                s.q[x][j][2 * z] = pack_h2(v[j][2 * z], v[j][2 * z + 4]);
                s.q[x][j][2 * z + 1] = pack_h2(v[j][2 * z + 1] * 0.0625f, v[j][2 * z + 5] * 0.0625f);
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            sum *= -8.f / 16777216.f;
            s.down[x][j][0] = __shfl_sync(0xffffffffu, sum, 8 * t); s.down[x][j][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
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
}

// 16 tokens from `token` on, two octets at `at`.  kAll: every query row sees them all.  Else `have` says which of the two octets
// are there, and each query row's own range which of the tokens it sees; what it does not see stays out whatever is held there.
template <int J, int NT, bool kAll>
__device__ __forceinline__ void eat(State<J, NT>& s, const char* at, int lane, const AttendArgs& A, const Walk& w, int row, int token, unsigned have)
{
    constexpr int D = 32 * J, kOctet = octet_bytes(D);
    const int g = lane >> 2, t = lane & 3;
    float x[NT][4];
    {
        unsigned k0[J], k1[J];
        load_words<J>(k0, at + 4 * J * lane);
        load_words<J>(k1, at + kOctet + 4 * J * lane);
        const __half* s0 = (const __half*)(at + octet_kscale(D)) + g * J;
        const __half* s1 = (const __half*)(at + kOctet + octet_kscale(D)) + g * J;
#pragma unroll
        for (int n = 0; n < NT; n++) { x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f; }
#pragma unroll
        for (int j = 0; j < J; j++) {
            const float a = __half2float(s0[j]), b = __half2float(s1[j]);
            const unsigned u0 = k0[j] >> 8, u1 = k1[j] >> 8;
#pragma unroll
            for (int n = 0; n < NT; n++) {
                float d[4] = {s.down[n][j][0], s.down[n][j][1], s.down[n][j][0], s.down[n][j][1]};
                mma(d, k0[j] & 0x000f000fu, k1[j] & 0x000f000fu, k0[j] & 0x00f000f0u, k1[j] & 0x00f000f0u, s.q[n][j][0], s.q[n][j][1]);
                mma(d, u0 & 0x000f000fu, u1 & 0x000f000fu, u0 & 0x00f000f0u, u1 & 0x00f000f0u, s.q[n][j][2], s.q[n][j][3]);
                x[n][0] = fmaf(a, d[0], x[n][0]); x[n][1] = fmaf(a, d[1], x[n][1]);
                x[n][2] = fmaf(b, d[2], x[n][2]); x[n][3] = fmaf(b, d[3], x[n][3]);
            }
        }
    }
    bool more = false;
#pragma unroll
    for (int n = 0; n < NT; n++) {
#pragma unroll
        for (int z = 0; z < 4; z++) {
            x[n][z] *= s.f[n][z & 1];
            if (!kAll) {
                const int i = row + 8 * n + 2 * t + (z & 1), tok = token + g + 8 * (z >> 1);
                const long long p = (long long)w.p0 + i / A.group;
                const bool sees = (have >> (z >> 1) & 1) && i < w.n * A.group && w.p0 >= 0 && tok <= p && tok < A.most && (A.window <= 0 || tok > p - A.window);
                if (!sees) x[n][z] = -INFINITY;
            }
        }
        more |= fmaxf(x[n][0], x[n][2]) > s.m[n][0] || fmaxf(x[n][1], x[n][3]) > s.m[n][1];
    }
    if (__any_sync(0xffffffffu, more)) {
        // the largest x has grown: what has been added up moves to the new one
#pragma unroll
        for (int n = 0; n < NT; n++) {
            float by[2];
#pragma unroll
            for (int z = 0; z < 2; z++) {
                float m = fmaxf(x[n][z], x[n][z + 2]);
#pragma unroll
                for (int o = 4; o < 32; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                m = fmaxf(m, s.m[n][z]);
                by[z] = s.m[n][z] == -INFINITY ? 1.f : exp2_of(s.m[n][z] - m);       // (nothing has been added up)
                s.m[n][z] = m;
                s.ref[n][z] = m == -INFINITY ? 0.f : m;
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
    unsigned p0[NT], p1[NT];
#pragma unroll
    for (int n = 0; n < NT; n++) {
        float p[4];
#pragma unroll
        for (int z = 0; z < 4; z++) p[z] = exp2_of(x[n][z] - s.ref[n][z & 1]);
        s.l[n][0] += p[0] + p[2];
        s.l[n][1] += p[1] + p[3];
        p0[n] = transposed(pack_h2(p[0], p[1]));
        p1[n] = transposed(pack_h2(p[2], p[3]));
    }
    const char* v = at + octet_vcode(D);
    unsigned v0[J], v1[J], z0[J], z1[J];
    load_words<J>(v0, v + 4 * J * lane);
    load_words<J>(v1, v + kOctet + 4 * J * lane);
    const char* sc = at + octet_vscale(D);
    load_words<J>(z0, sc + 4 * J * t);
    load_words<J>(z1, sc + kOctet + 4 * J * t);
    if (kAll) {
        // row j of the operand: group j's scales
        const unsigned a0 = g < J ? *(const unsigned*)(sc + 4 * (J * t + g)) : 0u, a2 = g < J ? *(const unsigned*)(sc + kOctet + 4 * (J * t + g)) : 0u;
#pragma unroll
        for (int n = 0; n < NT; n++) mma(s.off[n], a0, 0u, a2, 0u, p0[n], p1[n]);
    }
#pragma unroll
    for (int j = 0; j < J; j++) {
        const unsigned u0 = v0[j] >> 8, u1 = v1[j] >> 8;
#pragma unroll
        for (int n = 0; n < NT; n++) {
            unsigned b0 = mul_h2(p0[n], z0[j]), b1 = mul_h2(p1[n], z1[j]);
            if (!kAll) {
                // (0 stays 0 whatever the scale is)
                b0 &= __hneu2_mask(*reinterpret_cast<const __half2*>(&p0[n]), __half2half2(__ushort_as_half(0)));
                b1 &= __hneu2_mask(*reinterpret_cast<const __half2*>(&p1[n]), __half2half2(__ushort_as_half(0)));
                const unsigned one = g == j ? 0x3c003c00u : 0u;
                mma(s.off[n], one, 0u, one, 0u, b0, b1);
            }
            mma(s.o[n][2 * j], v0[j] & 0x000f000fu, v0[j] & 0x00f000f0u, v1[j] & 0x000f000fu, v1[j] & 0x00f000f0u, b0, b1);
            mma(s.o[n][2 * j + 1], u0 & 0x000f000fu, u0 & 0x00f000f0u, u1 & 0x000f000fu, u1 & 0x00f000f0u, b0, b1);
        }
    }
}

// dims 32 j + 4 g .. + 3 of query row 2 t + z of tile x, before the division by the sum
template <int J, int NT>
__device__ __forceinline__ void result(const State<J, NT>& s, int x, int j, int z, int lane, float (&v)[4])
{
    const float down = -8.f * __shfl_sync(0xffffffffu, s.off[x][z], 4 * j + (lane & 3));
    v[0] = fmaf(s.o[x][2 * j][z], 16777216.f, down); v[1] = fmaf(s.o[x][2 * j][z + 2], 1048576.f, down);
    v[2] = fmaf(s.o[x][2 * j + 1][z], 16777216.f, down); v[3] = fmaf(s.o[x][2 * j + 1][z + 2], 1048576.f, down);
}

__device__ __forceinline__ void store_out(const AttendArgs& A, long long at, const float (&v)[4])
{
    unsigned short* p = (unsigned short*)A.out + at;
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

template <int J, int NT, bool kRows>
__global__ void __launch_bounds__(kAttendThreads, Shape<J, NT, kRows>::kCtas)
attend_kernel(const __grid_constant__ AttendArgs A)
{
    using S = Shape<J, NT, kRows>;
    constexpr int D = S::D, kTileRows = S::kTileRows, kStages = S::kStages, kOctet = S::kOctet;
    extern __shared__ __align__(128) char ring[];
    __shared__ __align__(8) unsigned long long s_full[kMaxStages], s_free[kMaxStages];
    __shared__ unsigned s_have[kMaxStages];
    __shared__ float s_m[kEaters][8 * NT], s_l[kEaters][8 * NT];
    __shared__ long long s_scan[kEaters + 1], s_from, s_to, s_total, s_ctas;
    __shared__ Walk s_walk;
    __shared__ int s_failed;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < kStages; i++) { bar_init(smem_addr(&s_full[i]), 1); bar_init(smem_addr(&s_free[i]), kEaters); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_failed = 0;
    }
    pdl_wait();
    // ---- this CTA's share of the units
    {
        const int per = (A.rows + kAttendThreads - 1) / kAttendThreads;
        long long mine = 0;
        Walk w;
        for (int r = tid * per; r < min((tid + 1) * per, A.rows); r++) {
            w.r = r;
            walk_row(w, A);
            mine += (long long)row_units<kTileRows>(w, A) * A.heads;
        }
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) { const long long z = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += z; }
        if (lane == 31) s_scan[warp] = upto;
        __syncthreads();
        long long total = 0;
#pragma unroll
        for (int i = 0; i <= kEaters; i++) { if (i < warp) upto += s_scan[i]; total += s_scan[i]; }
        const long long ctas = min((long long)A.ctas, total);
        const long long from = ctas > 0 && blockIdx.x < ctas ? total * blockIdx.x / ctas : 0, to = ctas > 0 && blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : 0;
        if (tid == 0) { s_from = from; s_to = to; s_total = total; s_ctas = ctas; }
        if (from < to && upto - mine <= from && from < upto) {
            // (one thread's rows hold the share's first unit)
            long long left = from - (upto - mine);
            for (int r = tid * per;; r++) {
                w.r = r;
                walk_row(w, A);
                const int units = row_units<kTileRows>(w, A);
                if (left >= (long long)units * A.heads) { left -= (long long)units * A.heads; continue; }
                w.h = (int)(left / units);
                left -= (long long)w.h * units;
                for (w.y = 0;; w.y++) {
                    walk_item<kTileRows>(w, A);
                    if (left < w.count) break;
                    left -= w.count;
                }
                w.at = (int)left;
                break;
            }
            s_walk = w;
        }
    }
    __syncthreads();
    const long long from = s_from, to = s_to;
    AttendNote* note = reinterpret_cast<AttendNote*>(A.ws) + blockIdx.x;
    if (from >= to) {
        if (tid == 0) *note = AttendNote{0, 0, 0, 0, 0, 0, 0, 0};
        return;
    }
    Walk w = s_walk;
    bool ok = true;                            // (false: a wait ran out; from there on nothing is waited for, nothing is brought, and the call says so)

    if (warp == kEaters) {
        // ---- brings the octets
        int held = -1, row_of = -1, blocks_from = 0;
        long long u = from;
        int issued = 0;
        while (u < to && ok) {
            const int upto = (int)min((long long)w.count, (long long)w.at + (to - u));
            for (; w.at < upto && ok; w.at++, u++, issued++) {
                const int stage = issued % kStages, turn = issued / kStages;
                const int token = (w.first + w.at) * kTile + 8 * lane;
                bool want = lane < kTile / 8 && token < w.hi && token + 8 > w.lo;
                const int octet = token >> 3, block = octet / A.octets;
                // block ids of the row, 32 at a time
                const int first = __shfl_sync(0xffffffffu, block, 0), last = min(__shfl_sync(0xffffffffu, block, kTile / 8 - 1), A.width - 1);
                if (w.r != row_of || first < blocks_from || last >= blocks_from + 32) {
                    row_of = w.r; blocks_from = first;
                    held = first + lane < A.width ? A.table[(long long)w.r * A.width + first + lane] : -1;
                }
                const int id = __shfl_sync(0xffffffffu, held, min(max(block - blocks_from, 0), 31));
                want = want && block < A.width && id >= 0 && id < A.num_blocks;
                const unsigned have = __ballot_sync(0xffffffffu, want);
                if (turn > 0) ok = bar_wait(smem_addr(&s_free[stage]), (turn - 1) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const unsigned bar = smem_addr(&s_full[stage]);
                if (lane == 0) {
                    s_have[stage] = have;
                    bar_expect(bar, __popc(have) * kOctet);
                }
                __syncwarp();
                if (want)
                    bulk_load(smem_addr(ring) + stage * S::kUnit + lane * kOctet,
                              A.cache + id * A.block_stride + w.h * A.head_bytes + (long long)(octet - block * A.octets) * kOctet, kOctet, bar);
            }
            if (w.at == w.count && u < to) walk_next<kTileRows>(w, A);
        }
        // (its copies end before it does, whether or not they were waited for)
        for (int i = max(0, issued - kStages); i < issued; i++) ok &= bar_wait(smem_addr(&s_full[i % kStages]), (i / kStages) & 1);
        if (!ok && lane == 0) *(volatile int*)&s_failed = 1;
    } else {
        State<J, NT> s;
        long long u = from;
        int eaten = 0;
        AttendNote left = {0, 0, 0, 0, 0, 0, 0, 0};
        float* pieces = reinterpret_cast<float*>(A.ws + (size_t)A.ctas * sizeof(AttendNote));
        while (u < to) {
            const int row = w.y * kTileRows + (kRows ? warp * 8 * NT : 0);     // this warp's first query row
            load_queries<J, NT>(s, A, w, row, lane);
            // tokens that all of the item's query rows see
            const int last_row = min(w.n * A.group, (w.y + 1) * kTileRows) - 1;
            const int all_hi = w.p0 < 0 ? 0 : (int)min((long long)w.p0 + w.y * kTileRows / A.group + 1, (long long)A.most);
            const int all_lo = A.window > 0 ? (int)min(max((long long)w.p0 + last_row / A.group - A.window + 1, 0ll), (long long)A.most) : 0;
            const int begin = w.at, upto = (int)min((long long)w.count, (long long)w.at + (to - u));
            for (; w.at < upto; w.at++, u++, eaten++) {
                const int stage = eaten % kStages;
                if (ok) ok = __all_sync(0xffffffffu, bar_wait(smem_addr(&s_full[stage]), (eaten / kStages) & 1));
                if (ok) {
                    const unsigned have = s_have[stage];
#pragma unroll 1
                    for (int sub = kRows ? 0 : warp; sub < (kRows ? kTile / 16 : warp + 1); sub++) {
                        const unsigned both = have >> (2 * sub) & 3;
                        const int token = (w.first + w.at) * kTile + 16 * sub;
                        const char* at = ring + stage * S::kUnit + 2 * sub * kOctet;
                        if (kRows && row > last_row) break;
                        if (both == 3 && token >= all_lo && token + 16 <= all_hi) eat<J, NT, true>(s, at, lane, A, w, row, token, both);
                        else if (both) eat<J, NT, false>(s, at, lane, A, w, row, token, both);
                    }
                }
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&s_free[stage]));
            }
            // ---- the item's end, or this CTA's
            const bool complete = begin == 0 && upto == w.count;
            const int rows = min(kTileRows, w.n * A.group - w.y * kTileRows);
            float* piece = pieces + (2 * (size_t)blockIdx.x + (begin == 0 ? 1 : 0)) * piece_floats(kTileRows, D);
#pragma unroll
            for (int x = 0; x < NT; x++)
#pragma unroll
                for (int z = 0; z < 2; z++)
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) s.l[x][z] += __shfl_xor_sync(0xffffffffu, s.l[x][z], o);
            const int g = lane >> 2, t = lane & 3;
            if (kRows) {
#pragma unroll
                for (int x = 0; x < NT; x++)
#pragma unroll
                    for (int z = 0; z < 2; z++) {
                        const int i = warp * 8 * NT + 8 * x + 2 * t + z;
                        const float by = !complete ? 1.f : s.l[x][z] == 0.f ? 0.f : 1.f / s.l[x][z];
                        if (!complete && i < rows && g == 0) { piece[i] = s.m[x][z]; piece[kTileRows + i] = s.l[x][z]; }
                        const long long at = complete && i < rows ? out_at(A, w.token, w.y * kTileRows + i, w.h) : 0;
#pragma unroll
                        for (int j = 0; j < J; j++) {
                            float v[4];
                            result<J, NT>(s, x, j, z, lane, v);
                            if (i >= rows) continue;
#pragma unroll
                            for (int e = 0; e < 4; e++) v[e] *= by;
                            if (complete) store_out(A, at + 32 * j + 4 * g, v);
                            else *reinterpret_cast<float4*>(piece + 2 * kTileRows + i * D + 32 * j + 4 * g) = make_float4(v[0], v[1], v[2], v[3]);
                        }
                    }
            } else {
                if (g == 0) {
#pragma unroll
                    for (int x = 0; x < NT; x++)
#pragma unroll
                        for (int z = 0; z < 2; z++) { s_m[warp][8 * x + 2 * t + z] = s.m[x][z]; s_l[warp][8 * x + 2 * t + z] = s.l[x][z]; }
                }
                eaters_sync();
                float* join = reinterpret_cast<float*>(ring + kStages * S::kUnit);
#pragma unroll
                for (int x = 0; x < NT; x++)
#pragma unroll
                    for (int z = 0; z < 2; z++) {
                        const int i = 8 * x + 2 * t + z;
                        float m = -INFINITY;
#pragma unroll
                        for (int k = 0; k < kEaters; k++) m = fmaxf(m, s_m[k][i]);
                        const float by = s.m[x][z] == -INFINITY ? (s.l[x][z] == 0.f ? 0.f : 1.f) : exp2_of(s.m[x][z] - m);
#pragma unroll
                        for (int j = 0; j < J; j++) {
                            float v[4];
                            result<J, NT>(s, x, j, z, lane, v);
                            *reinterpret_cast<float4*>(join + (warp * 8 * NT + i) * S::kStep + 32 * j + 4 * g) = make_float4(v[0] * by, v[1] * by, v[2] * by, v[3] * by);
                        }
                    }
                eaters_sync();
                for (int e = tid; e < rows * (D / 4); e += 32 * kEaters) {
                    const int i = e / (D / 4), c = 4 * (e - i * (D / 4));
                    float m = -INFINITY, l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < kEaters; k++) m = fmaxf(m, s_m[k][i]);
#pragma unroll
                    for (int k = 0; k < kEaters; k++) {
                        l += s_m[k][i] == -INFINITY ? s_l[k][i] : s_l[k][i] * exp2_of(s_m[k][i] - m);      // (0, or NaN)
                        const float4 z = *reinterpret_cast<const float4*>(join + (k * 8 * NT + i) * S::kStep + c);
                        v[0] += z.x; v[1] += z.y; v[2] += z.z; v[3] += z.w;
                    }
                    if (complete) {
                        const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                        for (int z = 0; z < 4; z++) v[z] *= by;
                        store_out(A, out_at(A, w.token, w.y * kTileRows + i, w.h) + c, v);
                    } else {
                        if (c == 0) { piece[i] = m; piece[kTileRows + i] = l; }
                        *reinterpret_cast<float4*>(piece + 2 * kTileRows + i * D + c) = make_float4(v[0], v[1], v[2], v[3]);
                    }
                }
                eaters_sync();
            }
            if (begin == 0 && !complete) {
                // the CTA with the item's last unit
                const long long end = u - upto + w.count - 1, total = s_total, ctas = s_ctas;
                long long c = end * ctas / total;
                while (total * (c + 1) / ctas <= end) c++;
                left = AttendNote{1, w.token, w.y * kTileRows, rows, w.h, (int)c, 0, 0};
            }
            if (w.at == w.count && u < to) walk_next<kTileRows>(w, A);
        }
        if (!ok && lane == 0) *(volatile int*)&s_failed = 1;
        eaters_sync();
        if (tid == 0) { left.failed = *(volatile int*)&s_failed; *note = left; }
    }
}

// ---------------------------------------------------------------- second kernel

// Joins the pieces of the item that CTA blockIdx.x began and did not finish, a warp per query row; and says of every row whether its
// positions and block ids are ones.
__global__ void __launch_bounds__(kJoinThreads)
attend_join_kernel(const __grid_constant__ AttendArgs A, int tile_rows, int dim)
{
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const AttendNote* notes = reinterpret_cast<const AttendNote*>(A.ws);
    if (blockIdx.x < A.ctas) {
        const AttendNote note = notes[blockIdx.x];
        if (note.valid) {
            const float* pieces = reinterpret_cast<const float*>(A.ws + (size_t)A.ctas * sizeof(AttendNote));
            const size_t size = piece_floats(tile_rows, dim);
            const int count = note.last - (int)blockIdx.x + 1;
            // piece k: of this CTA the one it began, of the k-th behind it the one it went on with
            auto piece = [&](int k) { return pieces + (k == 0 ? 2 * (size_t)blockIdx.x + 1 : 2 * ((size_t)blockIdx.x + k)) * size; };
            for (int i = warp; i < note.rows; i += kJoinThreads / 32) {
                float m = -INFINITY, l = 0.f;
                for (int k = lane; k < count; k += 32) m = fmaxf(m, piece(k)[i]);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                for (int k = 0; k < count; k++) {
                    const float* p = piece(k);
                    const float by = p[i] == -INFINITY ? 1.f : exp2_of(p[i] - m);        // (0 or NaN throughout where p[i] is -infinity)
                    l = fmaf(p[tile_rows + i], by, l);
#pragma unroll
                    for (int z = 0; z < 8; z++) if (32 * z < dim) v[z] = fmaf(p[2 * tile_rows + i * dim + 32 * z + lane], by, v[z]);
                }
                const float by = l == 0.f ? 0.f : 1.f / l;
                const long long at = out_at(A, note.token, note.row + i, note.head);
#pragma unroll
                for (int z = 0; z < 8; z++) {
                    if (32 * z >= dim) continue;
                    if (A.dtype == GR_BF16) ((__nv_bfloat16*)A.out)[at + 32 * z + lane] = __float2bfloat16_rn(v[z] * by);
                    else ((__half*)A.out)[at + 32 * z + lane] = __float2half_rn(v[z] * by);
                }
            }
        }
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
            for (int b = lo / size + tid; b * (long long)size < hi; b += kJoinThreads) {
                const int id = A.table[(long long)r * A.width + b];
                bad |= id < 0 || id >= A.num_blocks;
            }
        }
        bad = __syncthreads_or(bad);
        if (tid == 0) A.status[r] = failed ? GR_CHECK_FAILED : bad ? GR_BAD_ROW : GR_OK;
    }
}

// ---------------------------------------------------------------- host

// The kernel for a call: whether a key head's query rows (a row's tokens times its group, on average) fill more than 8 of the products' columns, more than 16.
struct Choice { int nt; bool rows; };
static Choice choose(int dim, int group, int rows, int tokens)
{
    const double each = (double)tokens / std::max(1, rows) * group;
    if (dim > 128) return {1, each > 8};
    return {each > 8 ? 2 : 1, each > 16};
}
template <int J, int NT, bool kRows> struct Pick { using S = Shape<J, NT, kRows>; };
template <class F>
static auto with_shape(int dim, Choice c, F f)
{
#define GR_ATTEND_J(J) case J: if (c.rows) return f(Pick<J, J <= 4 ? 2 : 1, true>()); if (c.nt == 2) return f(Pick<J, J <= 4 ? 2 : 1, false>()); return f(Pick<J, 1, false>());
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

size_t gr_attend_workspace_bytes(int heads, int q_heads, int dim, int rows, int tokens)
{
    if (!gr::attend_shape_ok(heads, q_heads, dim, rows, tokens)) return 0;
    return gr::with_shape(dim, gr::choose(dim, q_heads / heads, rows, tokens), [&](auto pick) {
        using S = typename decltype(pick)::S;
        const size_t ctas = (size_t)gr::kSms * S::kCtas;
        return ctas * (sizeof(gr::AttendNote) + 2 * sizeof(float) * gr::piece_floats(S::kTileRows, dim));
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
    if (window < 0 || !isfinite(scale)) return GR_E_INVALID;
    if (!gr::counted(q_token, q_head, tokens, q_heads)) return GR_E_INVALID;
    const long long step[2] = {out_token, out_head}, size[2] = {tokens, q_heads};
    if (!gr::apart(L.dim, step, size, 2)) return GR_E_INVALID;
    if (rows == 0) return GR_OK;
    if (!offsets || !status || !workspace || (tokens > 0 && (!q || !out || !positions)) || (width > 0 && !table)) return GR_E_NULL;
    if (((uintptr_t)q & 1) || ((uintptr_t)out & 1) || ((uintptr_t)workspace & 31)) return GR_E_ALIGN;
    const gr::Span written = gr::rows_span(out, 2, L.dim, out_token, out_head, tokens, q_heads);
    if (gr::meet(written, gr::cache_span(cache, L))) return GR_E_INVALID;
    if (gr::meet(written, gr::rows_span(q, 2, L.dim, q_token, q_head, tokens, q_heads))) return GR_E_INVALID;
    gr::AttendArgs A = {};
    A.q = q; A.out = out; A.q_token = q_token; A.q_head = q_head; A.out_token = out_token; A.out_head = out_head;
    A.octets = L.block_size / 8; A.num_blocks = L.num_blocks; A.block_stride = L.block_stride;
    A.cache = (const char*)cache; A.head_bytes = (long long)A.octets * gr::octet_bytes(L.dim);
    A.table = table; A.offsets = offsets; A.positions = positions; A.status = status;
    A.dtype = dtype; A.tokens = tokens; A.heads = L.heads; A.group = q_heads / L.heads; A.width = width; A.rows = rows; A.window = window;
    A.most = width * L.block_size;
    A.scale = scale * 1.44269504088896340736f;
    A.ws = (char*)workspace;
    gr::Align in, to;
    in.add(q, 2, {tokens > 1 ? q_token : 0, q_heads > 1 ? q_head : 0});
    to.add(out, 2, {tokens > 1 ? out_token : 0, q_heads > 1 ? out_head : 0});
    A.q_vec = in.bits % 16 == 0; A.out_vec = to.bits % 8 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_cache_attend");
    const int done = gr::with_shape(L.dim, gr::choose(L.dim, A.group, rows, tokens), [&](auto pick) {
        using S = typename decltype(pick)::S;
        A.ctas = gr::kSms * S::kCtas;
        const auto kernel = gr::attend_of(pick);
        static bool set[gr::kMaxDevices] = {};
        int device = 0;
        if (cudaGetDevice(&device) != cudaSuccess) return GR_E_LAUNCH;
        if (device >= gr::kMaxDevices || !set[device]) {
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem) != cudaSuccess) return GR_E_LAUNCH;
            if (device < gr::kMaxDevices) set[device] = true;
        }
        if (gr::launch_pdl(kernel, A.ctas, gr::kAttendThreads, S::kSmem, st, A) != cudaSuccess) return GR_E_LAUNCH;
        if (gr::launch_pdl(gr::attend_join_kernel, A.ctas, gr::kJoinThreads, 0, st, A, S::kTileRows, L.dim) != cudaSuccess) return GR_E_LAUNCH;
        return GR_OK;
    });
    if (done != GR_OK || cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
