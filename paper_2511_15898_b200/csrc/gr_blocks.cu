// gr_block_plan: block tables, reference counts and slots of a paged cache for the next step.
//
// Rows and blocks depend on one another through sums only: how many rows hold a block, how many of the holders are about to
// write to it, how many blocks the rows before need, how many of the blocks before are free.  One cluster of CTAs goes through
// the phases between those sums, separated by cluster barriers, instead of a chain of launches.  Around it two kernels for all
// SMs, where there is work for them: tables that follow parents (before), and slot maps of many tokens (after).
// Latency bounds all of it: 256 rows of a pool of 32768 blocks, a token each, 17 k cycles (9.2 us replayed; with 1024 threads per
// CTA and rows in global memory between the phases 23.7), 48 prompts of 8000 tokens 14.2 (slots by the cluster alone: 56), 64 x 8
// forked rows 16.0 (forked by the cluster: 24).
#include <limits.h>
#include <algorithm>
#include "gr_host.h"

namespace gr {

constexpr int kPlanThreads = 512;
constexpr int kPlanNear = 1024;            // rows that every CTA holds in shared memory
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kPlanCluster = 8;
constexpr int kSlotThreads = 256;
constexpr int kForkThreads = 256;
constexpr int kForkSplits = 16;
constexpr int kSlotsAlone = 32768;          // slot maps beyond this are written by a kernel of their own

// a row between the phases
struct __align__(16) PlanRow {
    int base, ask;            // tokens kept; tokens asked for (0 where the row is full or bad)
    int before, kept;         // blocks held before the call; blocks that the kept tokens lie in
    int last;                 // the partly filled block that is about to be written to, or -1
    int need, copies;         // blocks needed, one of them for a copy
    int status;
    int parent;               // row of the table it goes on from, or -1
    int first_token;          // number of its first token
    int start;                // number of its first new block among all needed
    int pad;
};
static_assert(sizeof(PlanRow) == 48, "workspace layout");

struct PlanArgs {
    int* table; int* lengths; int* refs;
    const int* parents; const int* keep; const int* append;
    long long* slots; int* positions; int* offsets; int* copy_src; int* copy_dst; int* status;
    PlanRow* row;
    unsigned long long* best; int* writers;     // per block: the writer with the most tokens in it; number of writers
    int* fresh;                                  // each CTA's free blocks, by id, from the number of its first block on
    int* part;                                   // how many free blocks each CTA has
    unsigned char* bad;                          // per part of a group's columns and row: a held id outside the pool was met
    int rows, width, beams, block, num_blocks, max_tokens;
    int wide, split;                             // refs, slots and positions lie on 16 bytes; slots by a kernel of their own
    int splits;                                  // parts of a group's columns
};

__host__ __device__ inline int div_up(int a, int b) { return a / b + (a % b != 0 ? 1 : 0); }

// Exclusive sum over the CTA's threads, in their order; the total in `total`.  (s_part: one entry per warp and one more.)
__device__ __forceinline__ long long cta_scan(long long v, GR_PTR(long long) s_part, long long& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) s_part[warp] = x;
    __syncthreads();
    if (warp == 0) {
        long long w = lane < kPlanWarps ? s_part[lane] : 0, z = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, z, o);
            if (lane >= o) z += y;
        }
        if (lane < kPlanWarps) s_part[lane] = z - w;
        if (lane == 31) s_part[kPlanWarps] = z;
    }
    __syncthreads();
    total = s_part[kPlanWarps];
    return s_part[warp] + x - v;
}

// a count of block b, where there is such a block
__device__ __forceinline__ void count_add(int* counts, int n, int b, int v) { if (b >= 0 && b < n) atomicAdd(counts + b, v); }

// which of the blocks i .. i + 3 are free, as bits
__device__ __forceinline__ unsigned free_of(GR_PTR(int) refs, long long i, int n, bool wide)
{
    unsigned m = 0;
#ifndef GR_CHECK
    if (wide && i + 4 <= n) {
        const int4 v = *reinterpret_cast<const int4*>(refs + i);
        return (v.x == 0 ? 1u : 0u) | (v.y == 0 ? 2u : 0u) | (v.z == 0 ? 4u : 0u) | (v.w == 0 ? 8u : 0u);
    }
#endif
    for (int k = 0; k < 4; k++) if (i + k < n && refs[i + k] == 0) m |= 1u << k;
    return m;
}

__device__ __forceinline__ void plan_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void plan_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void plan_barrier() { plan_arrive(); plan_wait(); }

__host__ __device__ inline int plan_hash_size(int rows) { int n = 32; while (n < 2 * rows) n *= 2; return n; }

// place of block b in the table of shared blocks, which it enters if it is not there (there is room for every row's)
__device__ __forceinline__ int plan_find(GR_PTR(int) h_block, int size, int b)
{
    int at = (int)(((unsigned)b * 2654435761u) >> 7) & (size - 1);
    for (int k = 0; k < size; k++, at = (at + 1) & (size - 1)) {
        const int was = atomicCAS(&h_block[at], -1, b);
        if (was == -1 || was == b) return at;
    }
    return 0;
}

// What row r keeps: its numbers that depend on no other row's.
struct PlanKeep { int status, parent, base, before, kept; };
__device__ __forceinline__ PlanKeep plan_keep(const PlanArgs& A, int r, int* check)
{
    GR_PTR(const int) lengths = GR_MKPTR(const int, A.lengths, A.rows, check);
    GR_PTR(const int) keeps = GR_MKPTR(const int, A.keep, A.rows, check);
    GR_PTR(const int) parents = GR_MKPTR(const int, A.parents, A.rows, check);
    const long long most = (long long)A.width * A.block;
    const long long own = lengths[r];
    const int keep = A.keep ? max(0, keeps[r]) : INT_MAX;
    PlanKeep k;
    k.status = GR_OK;
    k.parent = r;
    long long len = own;
    if (A.parents) {
        const int p = parents[r];
        if (p < -1 || p >= A.beams) k.status = GR_BAD_ROW;
        k.parent = p >= 0 && p < A.beams ? r / A.beams * A.beams + p : -1;
        len = k.parent >= 0 ? lengths[k.parent] : 0;
    }
    if (len < 0 || len > most) { k.status = GR_BAD_ROW; len = min(max(len, 0ll), most); }
    k.base = min((int)len, keep);
    k.before = div_up((int)min(max(own, 0ll), most), A.block);
    k.kept = div_up(k.base, A.block);
    return k;
}

// The tables follow the parents and the counts follow the tables: a group per CTA, or part of its columns.  A lane owns a
// column of the group's tables and reads all of its entries before it writes one.
template <int W>
__global__ void __launch_bounds__(kForkThreads)
fork_kernel(const __grid_constant__ PlanArgs A)
{
    __shared__ PlanKeep s_row[W];
    __shared__ int s_bad[W], s_any;
    pdl_wait();
    GR_CHECK_FLAG_DECL;
    GR_CHECK_FLAG_INIT;
    GR_PTR(int) table = GR_MKPTR(int, A.table, (long long)A.rows * A.width, GR_CHECK_FLAG);
    GR_PTR(unsigned char) bad = GR_MKPTR(unsigned char, A.bad, (long long)A.splits * A.rows, GR_CHECK_FLAG);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = A.beams, N = A.num_blocks;
    const int r0 = blockIdx.x * G;
    if (tid == 0) s_any = 0;
    __syncthreads();
    if (tid < G) {
        const PlanKeep k = plan_keep(A, r0 + tid, GR_CHECK_FLAG);
        s_row[tid] = k;
        s_bad[tid] = 0;
        // (the columns that there is anything to do in: of a row that goes on from itself, those it releases)
        const int upto = k.parent == r0 + tid ? (k.before > k.kept ? k.before : 0) : max(k.before, k.kept);
        atomicMax(&s_any, upto);
    }
    __syncthreads();
    const int upto = s_any;
#pragma unroll 1
    for (int c = ((int)blockIdx.y * (kForkThreads / 32) + warp) * 32 + lane; c < upto; c += (int)gridDim.y * kForkThreads) {
        int now[W], was[W];
#pragma unroll
        for (int j = 0; j < W; j++) {
            now[j] = was[j] = -1;
            if (j < G && c < s_row[j].kept) now[j] = table[(long long)s_row[j].parent * A.width + c];
            if (j < G && c < s_row[j].before) was[j] = table[(long long)(r0 + j) * A.width + c];
        }
#pragma unroll
        for (int j = 0; j < W; j++) {
            if (j >= G) break;
            const bool held = c < s_row[j].before, holds = c < s_row[j].kept;
            // (only of a row that goes on from another: how much of the others' is looked at depends on their neighbours)
            if (holds && s_row[j].parent != r0 + j && (now[j] < 0 || now[j] >= N)) s_bad[j] = 1;
            if (held ? was[j] == now[j] : !holds) continue;
            if (held) count_add(A.refs, N, was[j], -1);
            if (holds) count_add(A.refs, N, now[j], 1);
            table[(long long)(r0 + j) * A.width + c] = now[j];
        }
    }
    __syncthreads();
    // (bit 1: the bounds-checked build skipped an access)
    if (tid < G) bad[(long long)blockIdx.y * A.rows + r0 + tid] = (unsigned char)(s_bad[tid] | (GR_CHECK_VALUE ? 2 : 0));
}

// blocks that a CTA looks through
__host__ __device__ inline int plan_share(int num_blocks) { return (div_up(num_blocks, kPlanCluster * kPlanThreads) + 3) & ~3; }
// the k-th free block by id, out of the CTAs' lists
__device__ __forceinline__ int fresh_at(GR_PTR(int) fresh, const int* count, int share, int k)
{
    long long from = 0;
#pragma unroll 1
    for (int i = 0; i < kPlanCluster - 1 && k >= count[i]; i++) { k -= count[i]; from += (long long)kPlanThreads * share; }
    return fresh[from + k];
}

// a writer of a shared block that is about to be written to: by its tokens in the block, then the lowest row
__device__ __forceinline__ unsigned long long writer_rank(int tokens, int r) { return ((unsigned long long)tokens << 32) | (0xffffffffu - (unsigned)r); }

// Slots of the appended tokens, K neighbouring ones per thread (four where there are many: one search for the row, one store of
// each kind for them).
// `fresh(k)`: the k-th free block; `first(r)`: number of row r's first token; `at(r)`: the row.
template <int K, class Block, class First, class Row>
__device__ __forceinline__ void write_slots(const PlanArgs& A, Block fresh, int total, long long thread, long long threads, First first, Row at, int* check)
{
    GR_PTR(long long) slots = GR_MKPTR(long long, A.slots, A.max_tokens, check);
    GR_PTR(int) positions = GR_MKPTR(int, A.positions, A.max_tokens, check);
    const int bs = A.block, R = A.rows;
    for (long long i0 = K * thread; i0 < A.max_tokens; i0 += K * threads) {
        long long slot[K];
        int position[K];
        int r = 0, next = 0, block = 0, within = 0;          // tokens up to `next` are row r's
        bool entered = false;                                // block and within are the last token's
        PlanRow q = {};
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int i = (int)i0 + k;
            slot[k] = -1; position[k] = -1;
            if (i0 + k >= total) continue;
            if (i >= next) {
                // the last row that begins at or before token i (rows without tokens begin where the next one does)
                int lo = r, hi = R - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (first(mid) <= i) lo = mid; else hi = mid - 1;
                }
                r = lo; entered = false;
                next = r + 1 < R ? first(r + 1) : total;
                q = at(r);
            }
            const int t = i - q.first_token;
            if (t >= q.ask) continue;
            position[k] = q.base + t;
            if (entered && within + 1 < bs) within++;
            else {
                const int c = position[k] / bs;
                within = position[k] - c * bs;
                if (c >= q.kept) block = fresh(q.start + q.copies + c - q.kept);
                else block = q.copies ? fresh(q.start) : q.last;
                entered = true;
            }
            slot[k] = (long long)block * bs + within;
        }
#ifndef GR_CHECK
        if (K == 4 && A.wide && i0 + K <= A.max_tokens) {
            *reinterpret_cast<longlong2*>(A.slots + i0) = make_longlong2(slot[0], slot[K / 4]);
            *reinterpret_cast<longlong2*>(A.slots + i0 + 2) = make_longlong2(slot[K / 2], slot[K - 1]);
            *reinterpret_cast<int4*>(A.positions + i0) = make_int4(position[0], position[K / 4], position[K / 2], position[K - 1]);
            continue;
        }
#endif
#pragma unroll
        for (int k = 0; k < K; k++) if (i0 + k < A.max_tokens) { slots[i0 + k] = slot[k]; positions[i0 + k] = position[k]; }
    }
}

// kNear: up to kPlanNear rows.  Every CTA then works all rows out for itself, in its shared memory, and the CTAs wait for one
// another only where tables and counts have changed and where free blocks are numbered.  With more rows each CTA has a share of
// them and the others' in the workspace.
template <bool kNear>
__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const __grid_constant__ PlanArgs A)
{
    extern __shared__ __align__(16) unsigned char s_dyn[];
    __shared__ long long s_part_raw[kPlanWarps + 1];
    __shared__ int s_free[kPlanCluster];
    pdl_wait();
    GR_CHECK_FLAG_DECL;
    GR_CHECK_FLAG_INIT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ctas = gridDim.x, me = blockIdx.x;
    const int R = A.rows, bs = A.block, N = A.num_blocks;
    const long long most = (long long)A.width * bs;
    GR_PTR(long long) s_part = GR_MKPTR(long long, s_part_raw, kPlanWarps + 1, GR_CHECK_FLAG);
    GR_PTR(int) table = GR_MKPTR(int, A.table, (long long)A.rows * A.width, GR_CHECK_FLAG);
    GR_PTR(int) refs = GR_MKPTR(int, A.refs, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(PlanRow) row = GR_MKPTR(PlanRow, kNear ? reinterpret_cast<PlanRow*>(s_dyn) : A.row, A.rows, GR_CHECK_FLAG);
    GR_PTR(unsigned long long) best = GR_MKPTR(unsigned long long, A.best, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(int) writers = GR_MKPTR(int, A.writers, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(int) fresh = GR_MKPTR(int, A.fresh, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(unsigned char) bad = GR_MKPTR(unsigned char, A.bad, (long long)A.splits * A.rows, GR_CHECK_FLAG);
    // near: the shared blocks that are written to, by open addressing (hash_size a power of two, twice the rows at least)
    const int hash_size = kNear ? plan_hash_size(R) : 1;
    GR_PTR(unsigned long long) h_best = GR_MKPTR(unsigned long long, reinterpret_cast<unsigned long long*>(s_dyn + sizeof(PlanRow) * (kNear ? R : 0)), hash_size, GR_CHECK_FLAG);
    GR_PTR(int) h_block = GR_MKPTR(int, reinterpret_cast<int*>(s_dyn + sizeof(PlanRow) * (kNear ? R : 0) + 8 * (size_t)hash_size), hash_size, GR_CHECK_FLAG);
    GR_PTR(int) h_count = GR_MKPTR(int, reinterpret_cast<int*>(s_dyn + sizeof(PlanRow) * (kNear ? R : 0) + 12 * (size_t)hash_size), hash_size, GR_CHECK_FLAG);
    // far: this CTA's rows are me, me + ctas, ...; near: all
    auto mine = [&](int r) { return kNear || r % ctas == me; };

    // ---- A: what each row keeps and asks for.  Every CTA sums the rows' tokens for itself; a thread has neighbouring rows.
    const int per = div_up(R, kPlanThreads), lo = min(R, tid * per), hi = min(R, lo + per);
    long long total;
    bool released = false;
    {
        if (kNear) for (int i = tid; i < hash_size; i += kPlanThreads) { h_best[i] = 0ull; h_block[i] = -1; h_count[i] = 0; }
        long long sum = 0;
        for (int r = lo; r < hi; r++) sum += max(0, A.append[r]);
        // (a thread with one row: its loads do not wait for the sum)
        const bool ahead = kNear && per == 1;
        PlanKeep k;
        if (ahead && lo < hi) k = plan_keep(A, lo, GR_CHECK_FLAG);
        long long at = cta_scan(sum, s_part, total);
        for (int r = lo; r < hi; r++) {
            const int want = A.append[r];
            const long long from = at;
            at += max(0, want);
            if (!mine(r)) continue;
            if (!ahead) k = plan_keep(A, r, GR_CHECK_FLAG);
            PlanRow q;
            q.status = want < 0 ? GR_BAD_ROW : k.status;
            q.parent = k.parent; q.base = k.base; q.before = k.before; q.kept = k.kept;
            q.ask = max(0, want);
            if (q.status == GR_OK && ((long long)q.base + q.ask > most || at > A.max_tokens)) q.status = GR_ROW_FULL;
            if (q.status != GR_OK) q.ask = 0;
            q.first_token = (int)min(from, (long long)A.max_tokens);
            q.last = -1; q.need = 0; q.copies = 0; q.start = 0; q.pad = 0;
            row[r] = q;
            released |= q.kept < q.before;
            if (r % ctas == me) A.offsets[r] = q.first_token;
        }
        if (me == 0 && tid == 0) A.offsets[R] = (int)min(total, (long long)A.max_tokens);
    }
    // (near: every CTA sees all rows, and whether any of them releases a block)
    bool releases = true;
    if (kNear) releases = __syncthreads_or(released) != 0; else plan_barrier();

    // ---- B: without parents a row only releases what it does not keep, mostly nothing (a warp per row)
    if (!A.parents && releases) {
        for (int r = me + ctas * warp; r < R; r += ctas * kPlanWarps) {
            const int before = row[r].before;
            for (int c = row[r].kept + lane; c < before; c += 32) {
                const long long at = (long long)r * A.width + c;
                count_add(A.refs, N, table[at], -1);
                table[at] = -1;
            }
        }
        plan_barrier();
    }

    // ---- C: who writes to a shared block, what each row needs; how many blocks are free
    const int share = plan_share(N);
    const long long b0 = ((long long)me * kPlanThreads + tid) * share;
    // (a thread's first row: its last block's id is on the way while the counts are looked through)
    auto writes_within = [&](const PlanRow& q) { return q.status == GR_OK && q.ask > 0 && q.base % bs != 0; };
    int first_last = -1;
    if (lo < hi && mine(lo)) {
        const PlanRow q = row[lo];
        if (writes_within(q)) first_last = table[(long long)lo * A.width + q.base / bs];
    }
    int free_here = 0;
    unsigned free_bits = 0;                                  // the first 32 of the thread's blocks
    for (int i = 0; i < share; i += 4) {
        const unsigned m = free_of(refs, b0 + i, N, A.wide);
        free_here += __popc(m);
        if (i < 32) free_bits |= m << i;
    }
    for (int r = lo; r < hi; r++) {
        if (!mine(r)) continue;
        PlanRow q = row[r];
        if (A.parents) {
            for (int y = 0; y < A.splits; y++) {
                const int met = bad[(long long)y * R + r];
                if (met & 1) q.status = GR_BAD_ROW;
#ifdef GR_CHECK
                if (met & 2) *GR_CHECK_FLAG = 1;
#endif
            }
        }
        if (writes_within(q)) {
            const int b = r == lo ? first_last : table[(long long)r * A.width + q.base / bs];
            if (b < 0 || b >= N) q.status = GR_BAD_ROW;
            else {
                q.last = b;
                q.need = refs[b];                            // (for now: the block's holders)
                if (!kNear && q.need > 1) { best[b] = 0ull; writers[b] = 0; }
            }
        }
        if (q.status != GR_OK) q.ask = 0;
        row[r] = q;
        if (kNear && q.need > 1) {
            const int at = plan_find(h_block, hash_size, q.last);
            atomicAdd(&h_count[at], 1);
            atomicMax(&h_best[at], writer_rank(q.base % bs, r));
        }
    }
    long long cta_free;
    const long long free_before = cta_scan(free_here, s_part, cta_free);     // (a barrier too)
    if (tid == 0) A.part[me] = (int)cta_free;
    if (!kNear) {
        plan_barrier();
        for (int r = lo; r < hi; r++) {
            if (!mine(r) || row[r].need <= 1) continue;
            count_add(A.writers, N, row[r].last, 1);
            atomicMax(A.best + row[r].last, writer_rank(row[r].base % bs, r));
        }
        plan_barrier();
    }
    long long sum = 0;
    for (int r = lo; r < hi; r++) {
        if (!mine(r)) continue;
        PlanRow q = row[r];
        if (q.need > 1) {
            // (every holder writes, and this one has the most tokens in the block: it keeps it)
            const int at = kNear ? plan_find(h_block, hash_size, q.last) : q.last;
            const int writing = kNear ? h_count[at] : writers[at];
            const unsigned long long first = kNear ? h_best[at] : best[at];
            q.copies = writing == q.need && (unsigned)first == 0xffffffffu - (unsigned)r ? 0 : 1;
        }
        q.need = q.ask > 0 ? q.copies + div_up(q.base + q.ask, bs) - q.kept : 0;
        sum += q.need;
        row[r] = q;
    }
    // ---- D: the free blocks by id, each CTA its own (no more than are needed, where that is known); the rows' places among the
    // needed blocks
    long long needed = N, place = 0;
    if (kNear) place = cta_scan(sum, s_part, needed);
    {
        long long k = free_before;
        const long long mine0 = (long long)me * kPlanThreads * share;
        for (int i = 0; i < share && free_here > 0 && k < needed; i += 4) {
            for (unsigned m = i < 32 ? free_bits >> i & 15u : free_of(refs, b0 + i, N, A.wide); m && k < needed; m &= m - 1) fresh[mine0 + k++] = (int)(b0 + i) + __ffs(m) - 1;
        }
    }
    plan_barrier();
    if (tid < kPlanCluster) s_free[tid] = A.part[tid];
    __syncthreads();
    if (!kNear) {
        sum = 0;
        for (int r = lo; r < hi; r++) sum += row[r].need;
        place = cta_scan(sum, s_part, needed);
    }
    long long avail = 0;
    for (int i = 0; i < kPlanCluster; i++) avail += s_free[i];
    for (int r = lo; r < hi; r++) {
        const int n = row[r].need;
        const long long from = place;
        place += n;
        if (!mine(r)) continue;
        if (n > 0 && place > avail) { row[r].status = GR_NO_BLOCKS; row[r].ask = 0; row[r].copies = 0; row[r].start = 0; }
        else row[r].start = (int)from;
    }
    // (near: nothing that another CTA changes from here on is read again)
    if (kNear) __syncthreads(); else plan_barrier();
    auto block_at = [&](int k) { return fresh_at(fresh, s_free, share, k); };

    // ---- E: rows take their blocks, a warp for each; tokens get their slots
    for (int r = me + ctas * warp; r < R; r += ctas * kPlanWarps) {
        const PlanRow q = row[r];
        const long long line = (long long)r * A.width;
        const int after = div_up(q.base + q.ask, bs);
        for (int c = q.kept + lane; c < after; c += 32) {
            const int b = block_at(q.start + q.copies + c - q.kept);
            table[line + c] = b;
            refs[b] = 1;
        }
        if (lane == 0) {
            int src = -1, dst = -1;
            if (q.copies) {
                src = q.last; dst = block_at(q.start);
                count_add(A.refs, N, src, -1);
                refs[dst] = 1;
                table[line + q.base / bs] = dst;
            }
            A.copy_src[r] = src; A.copy_dst[r] = dst;
            A.lengths[r] = q.base + q.ask;
            A.status[r] = q.status;
#ifdef GR_CHECK
            if (GR_CHECK_VALUE) A.status[r] = GR_CHECK_FAILED;
#endif
            if (kNear && A.split) A.row[r] = q;
        }
    }
    if (!A.split) {
        const int end = (int)min(total, (long long)A.max_tokens);
        const long long thread = (long long)me + (long long)ctas * tid, threads = (long long)ctas * kPlanThreads;
        auto first = [&](int r) { return row[r].first_token; };
        auto at = [&](int r) { return (PlanRow)row[r]; };
        if (A.max_tokens <= 2 * threads) write_slots<1>(A, block_at, end, thread, threads, first, at, GR_CHECK_FLAG);
        else write_slots<4>(A, block_at, end, thread, threads, first, at, GR_CHECK_FLAG);
    }
#ifdef GR_CHECK
    plan_barrier();
    if (tid == 0 && GR_CHECK_VALUE && R > 0) A.status[0] = GR_CHECK_FAILED;
#endif
}

// the slots of many tokens, by all SMs
__global__ void __launch_bounds__(kSlotThreads)
slots_kernel(const __grid_constant__ PlanArgs A)
{
    __shared__ int s_first[kPlanNear], s_free[kPlanCluster];
    pdl_wait();
    GR_CHECK_FLAG_DECL;
    GR_CHECK_FLAG_INIT;
    const bool near = A.rows <= kPlanNear;
    GR_PTR(PlanRow) row = GR_MKPTR(PlanRow, A.row, A.rows, GR_CHECK_FLAG);
    GR_PTR(int) fresh = GR_MKPTR(int, A.fresh, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(int) firsts = GR_MKPTR(int, s_first, kPlanNear, GR_CHECK_FLAG);
    if (threadIdx.x < kPlanCluster) s_free[threadIdx.x] = A.part[threadIdx.x];
    if (near) for (int r = threadIdx.x; r < A.rows; r += kSlotThreads) firsts[r] = row[r].first_token;
    __syncthreads();
    const int share = plan_share(A.num_blocks);
    auto first = [&](int r) { return near ? (int)firsts[r] : row[r].first_token; };
    auto at = [&](int r) { return (PlanRow)row[r]; };
    write_slots<4>(A, [&](int k) { return fresh_at(fresh, s_free, share, k); }, A.offsets[A.rows], (long long)blockIdx.x * kSlotThreads + threadIdx.x, (long long)gridDim.x * kSlotThreads,
                   first, at, GR_CHECK_FLAG);
#ifdef GR_CHECK
    __syncthreads();
    if (threadIdx.x == 0 && GR_CHECK_VALUE && A.rows > 0) A.status[0] = GR_CHECK_FAILED;
#endif
}

static size_t plan_layout(int rows, int num_blocks, char* ws, PlanArgs* A)
{
    size_t at = 0;
    auto take = [&](size_t bytes) { char* p = ws + at; at += (bytes + 15) & ~(size_t)15; return p; };
    char* row = take(sizeof(PlanRow) * (size_t)rows);
    char* best = take(8 * (size_t)num_blocks);
    char* writers = take(4 * (size_t)num_blocks);
    char* fresh = take(4 * (size_t)num_blocks);
    char* part = take(4 * (size_t)kPlanCluster);
    char* bad = take((size_t)kForkSplits * (size_t)rows);
    if (A) A->bad = (unsigned char*)bad;
    if (A) { A->row = (PlanRow*)row; A->best = (unsigned long long*)best; A->writers = (int*)writers; A->fresh = (int*)fresh; A->part = (int*)part; }
    return at;
}

template <bool kNear>
static int launch_plan(const PlanArgs& A, cudaStream_t st)
{
    // (near: the rows and the table of shared blocks)
    const int smem = kNear ? (int)sizeof(PlanRow) * A.rows + 16 * plan_hash_size(A.rows) : 0;
    if (smem > 40 * 1024) {
        constexpr int kMost = (int)sizeof(PlanRow) * kPlanNear + 16 * 2 * kPlanNear;
        static bool raised[kMaxDevices] = {false};
        int dev = -1;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return GR_E_LAUNCH; }
        if (!raised[dev]) {
            if (cudaFuncSetAttribute(plan_kernel<kNear>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) != cudaSuccess) {
                cudaGetLastError();
                return GR_E_LAUNCH;
            }
            raised[dev] = true;
        }
    }
    launch_pdl_cluster(kPlanCluster, plan_kernel<kNear>, kPlanCluster, kPlanThreads, smem, st, A);
    return GR_OK;
}

static void launch_fork(const PlanArgs& A, cudaStream_t st)
{
    const int groups = A.rows / A.beams;
    if (groups == 0) return;
    auto go = [&](auto kernel) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at = {};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3(groups, A.splits); cfg.blockDim = dim3(kForkThreads); cfg.stream = st; cfg.attrs = &at; cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, kernel, A);
    };
    if (A.beams <= 4) go(fork_kernel<4>);
    else if (A.beams <= 8) go(fork_kernel<8>);
    else if (A.beams <= 16) go(fork_kernel<16>);
    else go(fork_kernel<32>);
}

static bool plan_shape_ok(int rows, int num_blocks) { return rows >= 0 && rows <= (1 << 20) && num_blocks >= 0 && num_blocks <= (1 << 26); }

}  // namespace gr

extern "C" {

size_t gr_block_workspace_bytes(int rows, int num_blocks)
{
    if (!gr::plan_shape_ok(rows, num_blocks)) return 0;
    return gr::plan_layout(rows, num_blocks, nullptr, nullptr);
}

int gr_block_plan(int* table, int rows, int width, int beams, int block_size, int* lengths, int* refs, int num_blocks,
                  const int* parents, const int* keep, const int* append, int max_tokens, void* workspace,
                  long long* slots, int* positions, int* offsets, int* copy_src, int* copy_dst, int* status,
                  void* stream)
{
    if (!gr::plan_shape_ok(rows, num_blocks) || width < 0 || block_size < 1 || max_tokens < 0) return GR_E_INVALID;
    if (beams < 1 || beams > GR_MAX_BEAMS || rows % beams) return GR_E_INVALID;
    if ((long long)rows * width >= (1ll << 31) || (long long)width * block_size >= (1ll << 31)) return GR_E_INVALID;
    if (rows == 0 && max_tokens == 0) return GR_OK;
    if (!offsets || !workspace || (max_tokens > 0 && (!slots || !positions))) return GR_E_NULL;
    if (rows > 0 && ((width > 0 && !table) || !lengths || !append || !copy_src || !copy_dst || !status)) return GR_E_NULL;
    if (num_blocks > 0 && !refs) return GR_E_NULL;
    if ((uintptr_t)workspace & 15) return GR_E_ALIGN;
    gr::PlanArgs A;
    gr::plan_layout(rows, num_blocks, (char*)workspace, &A);
    A.table = table; A.lengths = lengths; A.refs = refs; A.parents = parents; A.keep = keep; A.append = append;
    A.slots = slots; A.positions = positions; A.offsets = offsets; A.copy_src = copy_src; A.copy_dst = copy_dst;
    A.status = status; A.rows = rows; A.width = width; A.beams = beams; A.block = block_size;
    A.num_blocks = num_blocks; A.max_tokens = max_tokens;
    A.wide = (((uintptr_t)refs | (uintptr_t)slots | (uintptr_t)positions) & 15) == 0;
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_block_plan");
    A.split = max_tokens > gr::kSlotsAlone;
    A.splits = 0;
    if (parents && rows > 0) {
        // (few groups: several CTAs to the columns of one)
        const int segs = gr::div_up(width, gr::kForkThreads), room = 2 * gr::kSms / (rows / beams);
        A.splits = std::max(1, std::min(std::min(segs, room), gr::kForkSplits));
        gr::launch_fork(A, st);
    }
    const int rc = rows <= gr::kPlanNear ? gr::launch_plan<true>(A, st) : gr::launch_plan<false>(A, st);
    if (rc != GR_OK) return rc;
    if (A.split) gr::launch_pdl(gr::slots_kernel, (int)std::min<long long>(4 * gr::kSms, ((long long)max_tokens + 4 * gr::kSlotThreads - 1) / (4 * gr::kSlotThreads)), gr::kSlotThreads, 0, st, A);
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
