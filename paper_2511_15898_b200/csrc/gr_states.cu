// What models keep per hypothesis follows the hypotheses: gr_reorder_states (dense states, in place or into other
// tensors) and gr_copy_blocks (blocks of a paged cache that two rows shared until one of them writes).  Both are bound by HBM:
// 1 GB of caches for four beams in 160 us (the measured copy rate; sixteen beams 197 us for 1.2 GB, 252 where the states lie a power
// of two apart), 512 blocks of 32 KB in 16 caches in 90 us (92 %).
#include <algorithm>
#include <memory>
#include <new>
#include <type_traits>
#include "gr_host.h"

namespace gr {

constexpr int kStatesPerLaunch = 128;      // pointers that travel as kernel arguments
constexpr int kCopyThreads = 256;
static_assert(kCopyThreads == 1 << 8, "a team of all threads");
constexpr int kCopyColumns = 4;            // vectors of a block per thread
constexpr int kMostTeams = 16;             // teams of a CTA

// Bounds-checked build: an access outside a tensor's first and last bytes, or across a piece's end, is skipped and noted in a word that
// gr_states_check reads (these operators have no status).
#ifdef GR_CHECK
__device__ int g_states_check;
__device__ __forceinline__ bool within(const char* p, long long n, const char* base, long long span, long long column, long long piece)
{
    if (p >= base && p + n <= base + span && column >= 0 && column + n <= piece) return true;
    g_states_check = 1;
    return false;
}
#define GR_WITHIN(...) within(__VA_ARGS__)
#else
#define GR_WITHIN(...) true
#endif

struct ReorderArgs {
    const char* src[kStatesPerLaunch];
    char* dst[kStatesPerLaunch];
    long long src_span, dst_span;          // bytes from a tensor's first to its last
    gr_state_layout at;
    int in_place, team_shift;              // threads of a team: 1 << team_shift
    long long tokens;                      // of a piece (with lengths)
};

// the first n bytes of a vector
__device__ __forceinline__ void store_bytes(char* to, const uint4& v, int n)
{
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16; i++) if (i < n) to[i] = (char)(w[i / 4] >> (8 * (i % 4)));
}
__device__ __forceinline__ void store_bytes(char* to, const uint2& v, int n)
{
#pragma unroll
    for (int i = 0; i < 8; i++) if (i < n) to[i] = (char)((i < 4 ? v.x : v.y) >> (8 * (i % 4)));
}
__device__ __forceinline__ void store_bytes(char* to, unsigned v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; i++) if (i < n) to[i] = (char)(v >> (8 * i));
}

// One thread owns a column of kVec bytes of every state of a group: it reads, for each state that changes, the parent's
// column, all of them before it writes the first.  So a group reorders in place whatever the mapping (no second buffer, no
// order among the copies), a parent of several states is read from memory once (the other reads meet it in the first-level
// cache), and states that stay are not touched.
// A CTA takes C * kCopyThreads neighbouring columns of one piece; what is copied from where is worked out once for it, in
// shared memory (by every thread for itself, the chain of look-ups for 16 states cost as much as the copies).
template <int W, typename Vec, int C>
__global__ void __launch_bounds__(kCopyThreads)
reorder_kernel(const __grid_constant__ ReorderArgs A, const int* __restrict__ parents, const int* __restrict__ lengths)
{
    constexpr int kVec = (int)sizeof(Vec), kStep = kCopyThreads * kVec;
    __shared__ const char* s_from[W];
    __shared__ int s_left[W];                  // bytes that are copied from the CTA's first column on (0: none, or the state stays)
    pdl_wait();
    const gr_state_layout& L = A.at;
    const int tid = threadIdx.x;
    const unsigned pieces = (unsigned)L.parts * (unsigned)L.batch;           // (below 2^31; the one after next may lie beyond)
    const long long start = (long long)blockIdx.x * C * kStep;
#pragma unroll 1
    for (unsigned piece = blockIdx.y; piece < pieces; piece += gridDim.y) {
        const int b = (int)piece / L.parts, part = (int)piece - b * L.parts, s = blockIdx.z;
        bool any = false;
        if (tid < W) {
            int left = 0;
            const char* from = nullptr;
            if (tid < L.beams_out) {
                const int p = __ldg(parents + (size_t)b * L.beams_out + tid);
                if (p >= 0 && p < L.beams_in && !(A.in_place && p == tid)) {
                    long long used = L.part_bytes;
                    if (lengths) used = min(A.tokens, (long long)max(0, __ldg(lengths + (size_t)b * L.beams_in + p))) * L.token_bytes;
                    left = (int)min(max(used - start, 0ll), 1ll << 30);
                    from = A.src[s] + b * L.src_group + p * L.src_beam + part * L.src_part + start;
                }
            }
            s_left[tid] = left; s_from[tid] = from;
            any = left > 0;
        }
        if (__syncthreads_or(any)) {
            char* dst = A.dst[s] + b * L.dst_group + part * L.dst_part + start + tid * kVec;
            Vec v[C][W];
#pragma unroll
            for (int j = 0; j < W; j++) {
#pragma unroll
                for (int c = 0; c < C; c++) {
                    // (a vector that holds the last used byte is read whole: pieces are a multiple of kVec long)
                    if (tid * kVec + c * kStep < s_left[j] && GR_WITHIN(s_from[j] + tid * kVec + c * kStep, kVec, A.src[s], A.src_span, start + tid * kVec + c * kStep, L.part_bytes)) v[c][j] = *reinterpret_cast<const Vec*>(s_from[j] + tid * kVec + c * kStep);
                }
            }
#pragma unroll
            for (int j = 0; j < W; j++) {
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const int more = s_left[j] - tid * kVec - c * kStep;
                    char* to = dst + j * L.dst_beam + c * kStep;
                    if (more > 0 && !GR_WITHIN(to, min(more, kVec), A.dst[s], A.dst_span, start + tid * kVec + c * kStep, L.part_bytes)) continue;
                    if (more >= kVec) *reinterpret_cast<Vec*>(to) = v[c][j];
                    else if (more > 0) store_bytes(to, v[c][j], more);
                }
            }
        }
        if (piece + gridDim.y < pieces) __syncthreads();
    }
}

// The same for pieces that are short: a CTA takes several of them, a team of threads for each.  (A kernel of its own: strides that
// are not constants cost odd widths 60 us for 43.)
template <int W, typename Vec, int C>
__global__ void __launch_bounds__(kCopyThreads)
reorder_short_kernel(const __grid_constant__ ReorderArgs A, const int* __restrict__ parents, const int* __restrict__ lengths)
{
    constexpr int kVec = (int)sizeof(Vec);
    __shared__ const char* s_from[kMostTeams][W];
    __shared__ int s_left[kMostTeams][W];      // bytes that are copied from the team's first column on (0: none, or the state stays)
    pdl_wait();
    const gr_state_layout& L = A.at;
    const int shift = A.team_shift;
    const int tid = threadIdx.x, team = tid >> shift, at = tid & ((1 << shift) - 1);
    const int teams = kCopyThreads >> shift, step = kVec << shift;
    const unsigned pieces = (unsigned)L.parts * (unsigned)L.batch, s = blockIdx.z;
    const long long start = (long long)blockIdx.x * C * step;
#pragma unroll 1
    for (unsigned piece0 = blockIdx.y * teams; piece0 < pieces; piece0 += gridDim.y * teams) {
        bool any = false;
        for (int e = tid; e < teams * W; e += kCopyThreads) {
            const int t = e / W, j = e % W;
            const unsigned piece = piece0 + t;
            int left = 0;
            const char* from = nullptr;
            if (j < L.beams_out && piece < pieces) {
                const int b = (int)piece / L.parts, part = (int)piece - b * L.parts;
                const int p = __ldg(parents + (size_t)b * L.beams_out + j);
                if (p >= 0 && p < L.beams_in && !(A.in_place && p == j)) {
                    long long used = L.part_bytes;
                    if (lengths) used = min(A.tokens, (long long)max(0, __ldg(lengths + (size_t)b * L.beams_in + p))) * L.token_bytes;
                    left = (int)min(max(used - start, 0ll), 1ll << 30);
                    from = A.src[s] + b * L.src_group + p * L.src_beam + part * L.src_part + start;
                }
            }
            s_left[t][j] = left; s_from[t][j] = from;
            any |= left > 0;
        }
        if (__syncthreads_or(any)) {
            // (a team beyond the last piece has nothing to copy)
            const int piece = (int)min(piece0 + team, pieces - 1), b = piece / L.parts, part = piece - b * L.parts;
            char* dst = A.dst[s] + b * L.dst_group + part * L.dst_part + start + at * kVec;
            Vec v[C][W];
#pragma unroll
            for (int j = 0; j < W; j++) {
#pragma unroll
                for (int c = 0; c < C; c++) {
                    // (a vector that holds the last used byte is read whole: pieces are a multiple of kVec long)
                    if (at * kVec + c * step < s_left[team][j] && GR_WITHIN(s_from[team][j] + at * kVec + c * step, kVec, A.src[s], A.src_span, start + at * kVec + c * step, L.part_bytes)) v[c][j] = *reinterpret_cast<const Vec*>(s_from[team][j] + at * kVec + c * step);
                }
            }
#pragma unroll
            for (int j = 0; j < W; j++) {
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const int more = s_left[team][j] - at * kVec - c * step;
                    char* to = dst + j * L.dst_beam + c * step;
                    if (more > 0 && !GR_WITHIN(to, min(more, kVec), A.dst[s], A.dst_span, start + at * kVec + c * step, L.part_bytes)) continue;
                    if (more >= kVec) *reinterpret_cast<Vec*>(to) = v[c][j];
                    else if (more > 0) store_bytes(to, v[c][j], more);
                }
            }
        }
        if (piece0 + gridDim.y * teams < pieces) __syncthreads();
    }
}

struct CopyArgs {
    char* cache[kStatesPerLaunch];
    const int* src; const int* dst;
    long long stride, bytes;
    int num_blocks, pairs, chunks, team_shift;         // chunks of a block; threads of a team: 1 << team_shift
};

// Each CTA takes a segment of the pair list, keeps the pairs that copy something (in their order, which is then the same in
// all CTAs of the segment), and takes its share of (pair, chunk) in one cache, a team of threads
// for each (all threads, but for short blocks).
template <typename Vec>
__global__ void __launch_bounds__(kCopyThreads)
copy_blocks_kernel(const __grid_constant__ CopyArgs A)
{
    constexpr int kVec = (int)sizeof(Vec), C = kCopyColumns;
    __shared__ int s_src[kCopyThreads], s_dst[kCopyThreads], s_warp[kCopyThreads / 32];
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i = blockIdx.y * kCopyThreads + tid;
    int from = -1, to = -1;
    if (i < A.pairs) { from = A.src[i]; to = A.dst[i]; }
    const bool copies = from >= 0 && from < A.num_blocks && to >= 0 && to < A.num_blocks && from != to;
    const unsigned mask = __ballot_sync(0xffffffffu, copies);
    if (lane == 0) s_warp[warp] = __popc(mask);
    __syncthreads();
    int at = __popc(mask & ((1u << lane) - 1u)), n = 0;
    for (int w = 0; w < kCopyThreads / 32; w++) { if (w < warp) at += s_warp[w]; n += s_warp[w]; }
    if (copies) { s_src[at] = from; s_dst[at] = to; }
    __syncthreads();
    char* cache = A.cache[blockIdx.z];
    const int units = A.chunks * n, team = tid >> A.team_shift, at_vec = tid & ((1 << A.team_shift) - 1);
    const int teams = kCopyThreads >> A.team_shift, step = kVec << A.team_shift;
#pragma unroll 1
    for (int u = blockIdx.x * teams + team; u < units; u += gridDim.x * teams) {
        const int k = u / A.chunks;
        const long long first = (long long)(u - k * A.chunks) * C * step + at_vec * kVec;
        const char* in = cache + s_src[k] * A.stride + first;
        char* out = cache + s_dst[k] * A.stride + first;
        Vec v[C];
#pragma unroll
        for (int c = 0; c < C; c++) if (first + c * step < A.bytes && GR_WITHIN(in + c * step, kVec, cache, A.stride * (A.num_blocks - 1) + A.bytes, first + c * step, A.bytes)) v[c] = *reinterpret_cast<const Vec*>(in + c * step);
#pragma unroll
        for (int c = 0; c < C; c++) if (first + c * step < A.bytes && GR_WITHIN(out + c * step, kVec, cache, A.stride * (A.num_blocks - 1) + A.bytes, first + c * step, A.bytes)) *reinterpret_cast<Vec*>(out + c * step) = v[c];
    }
}

// largest power of two up to 16 that divides everything or-ed into `bits`
static int vec_of(unsigned long long bits) {
    int v = 16;
    while (bits & (unsigned long long)(v - 1)) v >>= 1;
    return v;
}

constexpr long long kMaxBytes = 1ll << 46;        // beyond any device's memory: keeps the sums of strides in range

// Bytes that size[i] pieces at stride[i] apart, i = 0 .. 2, of `bytes` bytes each span; 0 where that leaves the address range
// or (with `apart`) where the pieces do not lie clear of one another (by nesting: each stride spans all that lies within it).
static long long span_of(long long bytes, const long long* stride, const int* size, bool apart)
{
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
    if (bytes > kMaxBytes) return 0;
    __int128 span = bytes;
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (apart && stride[i] < span) return 0;
        span += (__int128)stride[i] * (size[i] - 1);
        if (span > kMaxBytes) return 0;
    }
    return (long long)span;
}

// Whether any of p[i] .. p[i] + a meets any of q[j] .. q[j] + b
static bool meet(const void* const* p, long long a, void* const* q, long long b, int count)
{
    uintptr_t p0 = UINTPTR_MAX, p1 = 0, q0 = UINTPTR_MAX, q1 = 0;
    for (int i = 0; i < count; i++) {
        p0 = std::min(p0, (uintptr_t)p[i]); p1 = std::max(p1, (uintptr_t)p[i] + (uintptr_t)a);
        q0 = std::min(q0, (uintptr_t)q[i]); q1 = std::max(q1, (uintptr_t)q[i] + (uintptr_t)b);
    }
    if (p1 <= q0 || q1 <= p0) return false;
    for (int i = 0; i < count; i++) {
        for (int j = 0; j < count; j++) {
            if ((uintptr_t)p[i] < (uintptr_t)q[j] + (uintptr_t)b && (uintptr_t)q[j] < (uintptr_t)p[i] + (uintptr_t)a) return true;
        }
    }
    return false;
}

// Where the pieces of a tensor lie: `bytes` each, size[i] of them stride[i] apart, i = 0 .. 2, innermost first; span[i]: what the levels
// before i span.  (Clear of one another: stride[i] >= span[i].)
struct Lattice {
    long long bytes, stride[3], span[4];
    int size[3];
};
static Lattice lattice_of(long long bytes, const long long* stride, const int* size)
{
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
    Lattice t;
    t.bytes = bytes; t.span[0] = bytes;
    for (int i = 0; i < 3; i++) {
        t.size[i] = size[order[i]];
        t.stride[i] = t.size[i] > 1 ? stride[order[i]] : 0;
        t.span[i + 1] = t.span[i] + t.stride[i] * (t.size[i] - 1);
    }
    return t;
}

// Whether a piece of one tensor meets a piece of another that lies `d` bytes behind it, by the first `levels` levels: of the outermost
// one's differences only the two around d / stride leave the levels within anything to do.
static bool pieces_meet(const Lattice& t, int levels, long long d)
{
    while (levels > 0 && t.size[levels - 1] == 1) levels--;
    if (d >= t.span[levels] || -d >= t.span[levels]) return false;
    if (levels == 0) return true;
    const long long s = t.stride[levels - 1], k = d >= 0 ? d / s : -((-d + s - 1) / s);
    for (long long c = k; c <= k + 1; c++) if (c > -t.size[levels - 1] && c < t.size[levels - 1] && pieces_meet(t, levels - 1, d - c * s)) return true;
    return false;
}

// GR_OK where no two tensors of this layout share a byte.  Tensors beside one another are told by their first and last bytes, tensors
// within one another mostly by the place of their pieces between two steps of a stride, the others pair by pair.
static int check_apart(const void* const* p, int count, const Lattice& t)
{
    std::unique_ptr<uintptr_t[]> at(new (std::nothrow) uintptr_t[count]);
    if (!at) return GR_E_TOO_LARGE;
    auto fill = [&](unsigned long long modulus) {
        for (int i = 0; i < count; i++) at[i] = modulus ? (uintptr_t)p[i] % modulus : (uintptr_t)p[i];
        std::sort(at.get(), at.get() + count);
    };
    auto apart = [&](long long bytes) {
        for (int i = 1; i < count; i++) if (at[i] - at[i - 1] < (uintptr_t)bytes) return false;
        return true;
    };
    fill(0);
    if (apart(t.span[3])) return GR_OK;
    if (!apart(t.bytes)) return GR_E_INVALID;
    for (int i = 2; i >= 0; i--) {
        // (modulo stride i, which divides all larger ones, a tensor is span[i] bytes in a row, round the end)
        const long long s = t.stride[i];
        bool divides = s > 0;
        for (int j = i + 1; j < 3 && divides; j++) divides = t.stride[j] % s == 0;
        if (!divides) continue;
        fill((unsigned long long)s);
        if (apart(t.span[i]) && at[0] + (uintptr_t)s - at[count - 1] >= (uintptr_t)t.span[i]) return GR_OK;
    }
    fill(0);
    for (int i = 0; i < count; i++) {
        for (int j = i + 1; j < count && at[j] - at[i] < (uintptr_t)t.span[3]; j++) if (pieces_meet(t, 3, (long long)(at[j] - at[i]))) return GR_E_INVALID;
    }
    return GR_OK;
}

template <int W>
static void launch_reorder(const ReorderArgs& A, int count, int vec, const int* parents, const int* lengths, cudaStream_t st)
{
    const gr_state_layout& L = A.at;
    auto go = [&](auto whole, auto shorts, int bytes, int columns) {
        ReorderArgs B = A;
        B.team_shift = 8;
        while (B.team_shift > 4 && L.part_bytes <= (long long)bytes * columns << (B.team_shift - 1)) B.team_shift--;
        const long long per = (long long)bytes * columns << B.team_shift;
        const int teams = kCopyThreads >> B.team_shift, rows = (L.parts * L.batch - 1) / teams + 1;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at = {};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((unsigned)((L.part_bytes + per - 1) / per), (unsigned)std::min(rows, 65535), (unsigned)count);
        cfg.blockDim = dim3(kCopyThreads); cfg.stream = st; cfg.attrs = &at; cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, teams > 1 ? shorts : whole, B, parents, lengths);
    };
    // Columns of 16 bytes where they fit, two per thread up to four states (1 GB of caches 186 -> 157 us), of 8 bytes beyond 16 states,
    // whose wider ones leave one CTA an SM its registers (20 states 55 -> 44 us, 31 168 -> 142).  Narrow columns: several of them
    // per thread, so that as many bytes are in flight.
    constexpr int N4 = W <= 4 ? 8 : W <= 8 ? 4 : 2, kWide = W <= 4 ? 2 : 1;
    using Wide = std::conditional_t<(W <= 16), uint4, uint2>;
    switch (vec) {
        case 16: go(reorder_kernel<W, Wide, kWide>, reorder_short_kernel<W, Wide, kWide>, (int)sizeof(Wide), kWide); break;
        case 8: go(reorder_kernel<W, uint2, kWide>, reorder_short_kernel<W, uint2, kWide>, 8, kWide); break;
        case 4: go(reorder_kernel<W, unsigned, N4>, reorder_short_kernel<W, unsigned, N4>, 4, N4); break;
        case 2: go(reorder_kernel<W, unsigned short, N4>, reorder_short_kernel<W, unsigned short, N4>, 2, N4); break;
        default: go(reorder_kernel<W, unsigned char, N4>, reorder_short_kernel<W, unsigned char, N4>, 1, N4); break;
    }
}

}  // namespace gr

extern "C" {

#ifdef GR_CHECK
// whether an access was skipped since the last call of this (-1: it cannot be read)
int gr_states_check(void)
{
    int met = -1, none = 0;
    if (cudaMemcpyFromSymbol(&met, gr::g_states_check, sizeof(int)) != cudaSuccess || cudaMemcpyToSymbol(gr::g_states_check, &none, sizeof(int)) != cudaSuccess) return -1;
    return met;
}
#endif

int gr_reorder_states(const void* const* src, void* const* dst, int count, const gr_state_layout* layout,
                      const int* parents, const int* lengths, void* stream)
{
    if (!layout) return GR_E_NULL;
    const gr_state_layout L = *layout;
    if (count < 0 || L.batch < 0 || L.parts < 0 || L.part_bytes < 0) return GR_E_INVALID;
    if (L.beams_in < 1 || L.beams_in > GR_MAX_BEAMS || L.beams_out < 1 || L.beams_out > GR_MAX_BEAMS) return GR_E_INVALID;
    if (L.src_group < 0 || L.src_beam < 0 || L.src_part < 0 || L.dst_group < 0 || L.dst_beam < 0 || L.dst_part < 0) return GR_E_INVALID;
    if ((long long)L.batch * L.parts >= (1ll << 31)) return GR_E_INVALID;
    if (lengths && (L.token_bytes < 1 || L.part_bytes % L.token_bytes)) return GR_E_INVALID;
    if (count == 0 || L.batch == 0 || L.parts == 0 || L.part_bytes == 0) return GR_OK;
    if (!src || !dst) return GR_E_NULL;
    for (int i = 0; i < count; i++) if (!src[i] || !dst[i]) return GR_E_NULL;
    const bool in_place = src[0] == dst[0];
    for (int i = 1; i < count; i++) if ((src[i] == dst[i]) != in_place) return GR_E_INVALID;
    if (in_place && (L.beams_out > L.beams_in || L.src_group != L.dst_group || L.src_beam != L.dst_beam || L.src_part != L.dst_part))
        return GR_E_INVALID;
    const long long to[3] = {L.dst_group, L.dst_beam, L.dst_part}, from[3] = {L.src_group, L.src_beam, L.src_part};
    const int to_size[3] = {L.batch, in_place ? L.beams_in : L.beams_out, L.parts}, from_size[3] = {L.batch, L.beams_in, L.parts};
    const long long to_span = gr::span_of(L.part_bytes, to, to_size, true), from_span = gr::span_of(L.part_bytes, from, from_size, false);
    if (to_span == 0 || from_span == 0) return GR_E_INVALID;
    if (!in_place && gr::meet(src, from_span, dst, to_span, count)) return GR_E_INVALID;
    const int apart = count > 1 ? gr::check_apart(dst, count, gr::lattice_of(L.part_bytes, to, to_size)) : GR_OK;
    if (apart != GR_OK) return apart;
    if (!parents) return GR_E_NULL;                        // (last: without them a call looks at the rest and launches nothing)
    unsigned long long bits = (unsigned long long)L.part_bytes;
    if (L.batch > 1) bits |= (unsigned long long)(L.src_group | L.dst_group);
    if (L.beams_in > 1) bits |= (unsigned long long)L.src_beam;
    if (L.beams_out > 1) bits |= (unsigned long long)L.dst_beam;
    if (L.parts > 1) bits |= (unsigned long long)(L.src_part | L.dst_part);
    for (int i = 0; i < count; i++) bits |= (unsigned long long)(uintptr_t)src[i] | (unsigned long long)(uintptr_t)dst[i];
    const int vec = gr::vec_of(bits);
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_reorder_states");
    for (int lo = 0; lo < count; lo += gr::kStatesPerLaunch) {
        gr::ReorderArgs A;
        A.at = L; A.in_place = in_place;
        A.src_span = from_span; A.dst_span = to_span;
        A.tokens = lengths ? L.part_bytes / L.token_bytes : 0;
        const int n = std::min(count - lo, gr::kStatesPerLaunch);
        for (int i = 0; i < n; i++) { A.src[i] = (const char*)src[lo + i]; A.dst[i] = (char*)dst[lo + i]; }
        if (L.beams_out <= 4) gr::launch_reorder<4>(A, n, vec, parents, lengths, st);
        else if (L.beams_out <= 8) gr::launch_reorder<8>(A, n, vec, parents, lengths, st);
        else if (L.beams_out <= 16) gr::launch_reorder<16>(A, n, vec, parents, lengths, st);
        else gr::launch_reorder<32>(A, n, vec, parents, lengths, st);
    }
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

int gr_copy_blocks(void* const* caches, int count, int num_blocks, long long block_stride, long long block_bytes,
                   const int* copy_src, const int* copy_dst, int pairs, void* stream)
{
    if (count < 0 || num_blocks < 0 || pairs < 0 || block_bytes < 0 || block_stride < block_bytes) return GR_E_INVALID;
    if (num_blocks > 0 && block_stride > gr::kMaxBytes / num_blocks) return GR_E_INVALID;
    if (count == 0 || num_blocks == 0 || pairs == 0 || block_bytes == 0) return GR_OK;
    if (!caches) return GR_E_NULL;
    for (int i = 0; i < count; i++) if (!caches[i]) return GR_E_NULL;
    const long long steps[3] = {block_stride, 0, 0};
    const int sizes[3] = {num_blocks, 1, 1};
    const int apart = count > 1 ? gr::check_apart(caches, count, gr::lattice_of(block_bytes, steps, sizes)) : GR_OK;
    if (apart != GR_OK) return apart;
    unsigned long long bits = (unsigned long long)(block_stride | block_bytes);
    for (int i = 0; i < count; i++) bits |= (unsigned long long)(uintptr_t)caches[i];
    const int vec = gr::vec_of(bits);
    const int segments = (int)(((long long)pairs + gr::kCopyThreads - 1) / gr::kCopyThreads);
    int team_shift = 8;
    while (team_shift > 5 && block_bytes <= (long long)vec * gr::kCopyColumns << (team_shift - 1)) team_shift--;
    const long long per = (long long)vec * gr::kCopyColumns << team_shift, chunks = (block_bytes + per - 1) / per;
    if (segments > 65535 || chunks > (1 << 22)) return GR_E_TOO_LARGE;
    if (!copy_src || !copy_dst) return GR_E_NULL;          // (last, as above)
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_copy_blocks");
    for (int lo = 0; lo < count; lo += gr::kStatesPerLaunch) {
        gr::CopyArgs A;
        A.src = copy_src; A.dst = copy_dst; A.stride = block_stride; A.bytes = block_bytes;
        A.num_blocks = num_blocks; A.pairs = pairs;
        A.chunks = (int)chunks; A.team_shift = team_shift;
        const int n = std::min(count - lo, gr::kStatesPerLaunch);
        for (int i = 0; i < n; i++) A.cache[i] = (char*)caches[lo + i];
        const dim3 grid(std::max(1, 8 * gr::kSms / (segments * n)), segments, n);
        auto go = [&](auto kernel) {
            cudaLaunchConfig_t cfg = {};
            cudaLaunchAttribute at = {};
            at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
            at.val.programmaticStreamSerializationAllowed = 1;
            cfg.gridDim = grid; cfg.blockDim = dim3(gr::kCopyThreads); cfg.stream = st; cfg.attrs = &at; cfg.numAttrs = 1;
            cudaLaunchKernelEx(&cfg, kernel, A);
        };
        switch (vec) {
            case 16: go(gr::copy_blocks_kernel<uint4>); break;
            case 8: go(gr::copy_blocks_kernel<uint2>); break;
            case 4: go(gr::copy_blocks_kernel<unsigned>); break;
            case 2: go(gr::copy_blocks_kernel<unsigned short>); break;
            default: go(gr::copy_blocks_kernel<unsigned char>); break;
        }
    }
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
