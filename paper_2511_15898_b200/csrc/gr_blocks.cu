// gr_block_plan: block tables, reference counts and slots of a paged cache for the next step, in one launch of one cluster.
//
// Rows and blocks depend on one another through sums only: how many rows hold a block, how many of the holders are about to
// write to it, how many blocks the rows before need, how many of the blocks before are free.  The phases between those
// sums are separated by cluster barriers, so that a step is one launch instead of a chain of them; what a phase hands to the
// next lies in the workspace.
#include "gr_host.h"

namespace gr {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kPlanCluster = 8;

// a row between the phases
struct __align__(16) PlanRow {
    int base, ask;            // tokens kept; tokens asked for (0 where the row is full or bad)
    int before, kept;         // blocks held before the call; blocks that the kept tokens lie in
    int last;                 // the partly filled block that is about to be written to, or -1
    int need, copies;         // blocks needed, one of them for a copy
    int status;
    int parent;               // row of the table it goes on from, or -1
    int bad;                  // a held id outside the pool was met
    int first_token;          // number of its first token
    int start;                // number of its first new block among all needed
};
static_assert(sizeof(PlanRow) == 48, "workspace layout");

struct PlanArgs {
    int* table; int* lengths; int* refs;
    const int* parents; const int* keep; const int* append;
    long long* slots; int* positions; int* offsets; int* copy_src; int* copy_dst; int* status;
    PlanRow* row;
    unsigned long long* best; int* writers;     // per block: the writer with the most tokens in it; number of writers
    int* fresh;                                  // the free blocks with the smallest ids, as many as are needed
    int* part;                                   // free blocks by CTA
    int rows, width, beams, block, num_blocks, max_tokens;
};

__host__ __device__ inline int div_up(int a, int b) { return (int)(((long long)a + b - 1) / b); }

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
        s_part[lane] = z - w;
        if (lane == 31) s_part[kPlanWarps] = z;
    }
    __syncthreads();
    total = s_part[kPlanWarps];
    return s_part[warp] + x - v;
}

// a count of block b, where there is such a block
__device__ __forceinline__ void count_add(int* counts, int n, int b, int v) { if (b >= 0 && b < n) atomicAdd(counts + b, v); }

__device__ __forceinline__ void plan_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// W: room for a group's entries of a column
template <int W>
__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const __grid_constant__ PlanArgs A)
{
    __shared__ long long s_part_raw[kPlanWarps + 1];
    pdl_wait();
    GR_CHECK_FLAG_DECL;
    GR_CHECK_FLAG_INIT;
    GR_PTR(long long) s_part = GR_MKPTR(long long, s_part_raw, kPlanWarps + 1, GR_CHECK_FLAG);
    GR_PTR(int) table = GR_MKPTR(int, A.table, (long long)A.rows * A.width, GR_CHECK_FLAG);
    GR_PTR(int) lengths = GR_MKPTR(int, A.lengths, A.rows, GR_CHECK_FLAG);
    GR_PTR(int) refs = GR_MKPTR(int, A.refs, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(PlanRow) row = GR_MKPTR(PlanRow, A.row, A.rows, GR_CHECK_FLAG);
    GR_PTR(unsigned long long) best = GR_MKPTR(unsigned long long, A.best, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(int) writers = GR_MKPTR(int, A.writers, A.num_blocks, GR_CHECK_FLAG);
    GR_PTR(int) fresh = GR_MKPTR(int, A.fresh, A.num_blocks, GR_CHECK_FLAG);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ctas = gridDim.x, me = blockIdx.x;
    const int R = A.rows, bs = A.block, N = A.num_blocks;
    const int G = A.parents ? A.beams : 1;        // (without parents a row's table depends on its own alone)
    const long long most = (long long)A.width * bs;

    // ---- A: what each row keeps and asks for.  Every CTA sums the rows' tokens for itself; a thread has neighbouring rows.
    {
        const int per = div_up(R, kPlanThreads), lo = min(R, tid * per), hi = min(R, lo + per);
        long long sum = 0, total;
        for (int r = lo; r < hi; r++) sum += max(0, A.append[r]);
        long long at = cta_scan(sum, s_part, total);
        for (int r = lo; r < hi; r++) {
            const int want = A.append[r];
            const long long from = at;
            at += max(0, want);
            if (r % ctas != me) continue;
            PlanRow q;
            q.status = want < 0 ? GR_BAD_ROW : GR_OK;
            q.parent = r;
            if (A.parents) {
                const int p = A.parents[r];
                if (p < -1 || p >= A.beams) q.status = GR_BAD_ROW;
                q.parent = p >= 0 && p < A.beams ? r / A.beams * A.beams + p : -1;
            }
            long long len = q.parent >= 0 ? lengths[q.parent] : 0;
            if (len < 0 || len > most) { q.status = GR_BAD_ROW; len = min(max(len, 0ll), most); }
            q.base = (int)len;
            if (A.keep) q.base = min(q.base, max(0, A.keep[r]));
            q.before = div_up((int)min(max((long long)lengths[r], 0ll), most), bs);
            q.kept = div_up(q.base, bs);
            q.ask = max(0, want);
            if (q.status == GR_OK && ((long long)q.base + q.ask > most || at > A.max_tokens)) q.status = GR_ROW_FULL;
            if (q.status != GR_OK) q.ask = 0;
            q.first_token = (int)min(from, (long long)A.max_tokens);
            q.last = -1; q.need = 0; q.copies = 0; q.bad = 0; q.start = 0;
            if (q.ask > 0 && q.base % bs != 0) {
                const int b = table[(long long)q.parent * A.width + q.base / bs];
                if (b >= 0 && b < N) { q.last = b; best[b] = 0ull; writers[b] = 0; }
            }
            row[r] = q;
            A.offsets[r] = q.first_token;
        }
        if (me == 0 && tid == 0) A.offsets[R] = (int)min(total, (long long)A.max_tokens);
    }
    plan_barrier();

    // ---- B: the tables follow the parents, the counts follow the tables; who writes to which block.
    // A lane owns a column of its group's tables and reads all the entries it needs before it writes one.
    {
        const int segs = div_up(A.width, 32);
        const long long units = (long long)(R / G) * segs;
#pragma unroll 1
        for (long long u = (long long)me * kPlanWarps + warp; u < units; u += (long long)ctas * kPlanWarps) {
            const int r0 = (int)(u / segs) * G, c = (int)(u % segs) * 32 + lane;
            if (c >= A.width) continue;
            int now[W];
#pragma unroll
            for (int j = 0; j < W; j++) {
                now[j] = -1;
                if (j < G && c < row[r0 + j].kept) now[j] = table[(long long)row[r0 + j].parent * A.width + c];
            }
#pragma unroll
            for (int j = 0; j < W; j++) {
                if (j >= G) break;
                const bool held = c < row[r0 + j].before, holds = c < row[r0 + j].kept;
                if (holds && (now[j] < 0 || now[j] >= N)) row[r0 + j].bad = 1;
                if (!held && !holds) continue;
                const long long at = (long long)(r0 + j) * A.width + c;
                const int old = held ? table[at] : -1;
                if (held && old == now[j]) continue;
                if (held) count_add(A.refs, N, old, -1);
                if (holds) count_add(A.refs, N, now[j], 1);
                table[at] = now[j];
            }
        }
        for (int r = me * kPlanThreads + tid; r < R; r += ctas * kPlanThreads) {
            const int b = row[r].last;
            if (b < 0) continue;
            count_add(A.writers, N, b, 1);
            atomicMax(A.best + b, ((unsigned long long)(row[r].base % bs) << 32) | (0xffffffffu - (unsigned)r));
        }
    }
    plan_barrier();

    // ---- C: what each row needs; how many blocks are free
    for (int r = me * kPlanThreads + tid; r < R; r += ctas * kPlanThreads) {
        PlanRow q = row[r];
        if (q.bad) q.status = GR_BAD_ROW;
        // (a writer without a valid last block has met an id outside the pool)
        if (q.status == GR_OK && q.ask > 0) {
            if (q.last >= 0 && refs[q.last] > 1) {
                const bool keeps = writers[q.last] == refs[q.last] && (unsigned)best[q.last] == 0xffffffffu - (unsigned)r;
                q.copies = keeps ? 0 : 1;
            }
            q.need = q.copies + div_up(q.base + q.ask, bs) - q.kept;
        } else q.ask = 0;
        row[r] = q;
    }
    const int share = (div_up(N, ctas * kPlanThreads) + 3) & ~3;
    const long long b0 = ((long long)me * kPlanThreads + tid) * share;
    int free_here = 0;
    for (int i = 0; i < share; i++) if (b0 + i < N && refs[b0 + i] == 0) free_here++;
    long long cta_free;
    const long long free_before = cta_scan(free_here, s_part, cta_free);
    if (tid == 0) A.part[me] = (int)cta_free;
    plan_barrier();

    // ---- D: the rows' places among the needed blocks; the free blocks by number
    long long avail = 0, ahead = 0;
    for (int i = 0; i < ctas; i++) { const int f = A.part[i]; if (i < me) ahead += f; avail += f; }
    long long needed;
    {
        const int per = div_up(R, kPlanThreads), lo = min(R, tid * per), hi = min(R, lo + per);
        long long sum = 0;
        for (int r = lo; r < hi; r++) sum += row[r].need;
        long long at = cta_scan(sum, s_part, needed);
        for (int r = lo; r < hi; r++) {
            const int n = row[r].need;
            const long long from = at;
            at += n;
            if (r % ctas != me) continue;
            if (n > 0 && at > avail) { row[r].status = GR_NO_BLOCKS; row[r].ask = 0; row[r].copies = 0; row[r].start = 0; }
            else row[r].start = (int)from;
        }
    }
    {
        long long k = ahead + free_before;
        const long long upto = min(needed, avail);
        for (int i = 0; i < share && k < upto; i++)
            if (b0 + i < N && refs[b0 + i] == 0) fresh[k++] = (int)(b0 + i);
    }
    plan_barrier();

    // ---- E: rows take their blocks (a warp per row); tokens get their slots
    for (int r = me * kPlanWarps + warp; r < R; r += ctas * kPlanWarps) {
        const PlanRow q = row[r];
        const int after = div_up(q.base + q.ask, bs);
        const long long mine = (long long)r * A.width;
        if (lane == 0) {
            int from = -1, to = -1;
            if (q.copies) {
                from = q.last; to = fresh[q.start];
                count_add(A.refs, N, from, -1);
                refs[to] = 1;
                table[mine + q.base / bs] = to;
            }
            A.copy_src[r] = from; A.copy_dst[r] = to;
            lengths[r] = q.base + q.ask;
            A.status[r] = q.status;
#ifdef GR_CHECK
            if (GR_CHECK_VALUE) A.status[r] = GR_CHECK_FAILED;
#endif
        }
        for (int c = q.kept + lane; c < after; c += 32) {
            const int b = fresh[q.start + q.copies + c - q.kept];
            table[mine + c] = b;
            refs[b] = 1;
        }
    }
    const int total = A.offsets[R];
    for (int i = me * kPlanThreads + tid; i < A.max_tokens; i += ctas * kPlanThreads) {
        long long slot = -1;
        int position = -1;
        if (i < total) {
            // the last row that begins at or before token i (rows without tokens begin where the next one does)
            int lo = 0, hi = R - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (row[mid].first_token <= i) lo = mid; else hi = mid - 1;
            }
            const PlanRow q = row[lo];
            const int k = i - q.first_token;
            if (k < q.ask) {
                position = q.base + k;
                const int c = position / bs;
                int b;
                if (c >= q.kept) b = fresh[q.start + q.copies + c - q.kept];
                else b = q.copies ? fresh[q.start] : q.last;
                slot = (long long)b * bs + position % bs;
            }
        }
        A.slots[i] = slot;
        A.positions[i] = position;
    }
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
    if (A) { A->row = (PlanRow*)row; A->best = (unsigned long long*)best; A->writers = (int*)writers; A->fresh = (int*)fresh; A->part = (int*)part; }
    return at;
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
    cudaStream_t st = (cudaStream_t)stream;
    gr::NvtxRange whole("gr_block_plan");
    const int ctas = gr::kPlanCluster;
    auto go = [&](auto kernel) { gr::launch_pdl_cluster(ctas, kernel, ctas, gr::kPlanThreads, 0, st, A); };
    const int group = parents ? beams : 1;
    if (group == 1) go(gr::plan_kernel<1>);
    else if (group <= 4) go(gr::plan_kernel<4>);
    else if (group <= 8) go(gr::plan_kernel<8>);
    else if (group <= 16) go(gr::plan_kernel<16>);
    else go(gr::plan_kernel<32>);
    if (cudaPeekAtLastError() != cudaSuccess) { cudaGetLastError(); return GR_E_LAUNCH; }
    return GR_OK;
}

}  // extern "C"
