// Pages of the cache: forking, extending (with a copy where a shared page is written), freeing and compacting sequences.
//
// The state is the caller's: one reference count per page (0: free), the block table and the sequence lengths, all on the device, so
// that a captured decode loop can allocate.  Everything is decided by whole numbers in a fixed order (free pages are taken lowest
// number first, sequences and slots in ascending order), so that the same state gives the same result; counts change by atomic
// additions, whose order does not matter.
//
// What bounds these: pages_fork and pages_free are a launch and two dependent loads; pages_plan_* read the reference counts with one
// CTA of 1024 threads (16 counts a thread and round, all loads of a round in flight); pages_copy_kernel moves whole pages and is
// bound by HBM where there are many (an extend has a CTA for a sequence and KV head, whatever the page size: one copy of 1024 tokens
// and 8 heads takes 78 us, 0.1 TB/s).  Measured: fork, extend (two launches) and free of four children of 4099 tokens 17 us, of 128 children with their
// copies 27; compaction of 27 900 pages of 16 tokens, 11 500 of them moved, 290 us (5.2 TB/s; 4, 8 pieces of a thread in flight and
// 8, 16 CTAs a SM: 290, 361, 306).  None of them lets the kernels behind it start early: they write sequence lengths, which others
// read before their own wait (the rules are in ha_common.cuh).
#include "ha_common.cuh"

namespace ha {

constexpr int kP_Threads = 256;          // per forked or freed sequence
constexpr int kP_Plan = 1024;
constexpr int kP_Counts = 16;            // counts of a thread and round
constexpr int kP_Copy = 128;             // threads of a copying CTA
constexpr int kP_Batch = 4;              // 16-byte pieces of a thread in flight

struct PageState {
    int32_t *seq_lens, *table, *ref;
    long long bt_sb;
    int B, width, n_pages, shift;
    uint32_t *status;
};
struct PagePools {
    TensorView K, V;
    uint32_t *codes;                     // NULL: no signatures
    long long c_page, c_head;
    int heads;
};
// Lists of a plan, in the workspace: what the copying kernel does.
struct PagePlan {
    int32_t *n_copies;                   // [0] copies, [1] a call's second number
    int32_t *first;                      // [B + 1] first new page of each sequence (extend)
    int32_t *list;                       // [n_pages] free pages, or holes
    int32_t *src, *dst;                  // copies
};

__device__ __forceinline__ int pages_of(long long n, int shift) { return (int)((n + (1LL << shift) - 1) >> shift); }
__device__ __forceinline__ void flag(uint32_t *status, uint32_t bit) { atomicOr(status, bit); }

// ---- fork: the children's rows become their parents', every page counts one more holder
__global__ void __launch_bounds__(kP_Threads) pages_fork_kernel(const PageState p, const int32_t *__restrict__ parents,
                                                               const int32_t *__restrict__ children, int n) {
    pdl_wait();
    const int i = blockIdx.x, parent = __ldcg(parents + i), child = __ldcg(children + i);
    bool bad = parent < 0 || parent >= p.B || child < 0 || child >= p.B;
    for (int j = threadIdx.x; j < n; j += kP_Threads) {
        const int c = __ldcg(children + j);
        bad |= (c == child && j < i) || c == parent;   // a child twice: the first counts; no sequence is child and parent
    }
    int len = 0, pages = 0;
    if (!bad) {
        len = __ldcg(p.seq_lens + parent);
        pages = pages_of(len > 0 ? len : 0, p.shift);
        bad = __ldcg(p.seq_lens + child) != 0 || len < 0 || pages > p.width;
    }
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) flag(p.status, HA_DEV_BAD_INDEX);
        return;
    }
    const int32_t *from = p.table + (long long)parent * p.bt_sb;
    int32_t *to = p.table + (long long)child * p.bt_sb;
    for (int s = threadIdx.x; s < pages; s += kP_Threads) {
        const int page = __ldcg(from + s);
        to[s] = page;
        if ((unsigned)page < (unsigned)p.n_pages) atomicAdd(p.ref + page, 1);
        else flag(p.status, HA_DEV_BAD_INDEX);
    }
    if (threadIdx.x == 0) {                            // every thread has read it: behind the barrier above
        p.seq_lens[child] = len;
        __threadfence();                               // kernels behind read it before their wait
    }
}

// ---- free: every page of the sequence counts one holder less
__global__ void __launch_bounds__(kP_Threads) pages_free_kernel(const PageState p, const int32_t *__restrict__ seqs, int n) {
    pdl_wait();
    const int i = blockIdx.x, seq = __ldcg(seqs + i);
    if (seq < 0 || seq >= p.B) {
        if (threadIdx.x == 0) flag(p.status, HA_DEV_BAD_INDEX);
        return;
    }
    bool again = false;
    for (int j = threadIdx.x; j < i; j += kP_Threads) again |= __ldcg(seqs + j) == seq;
    if (__syncthreads_or(again)) return;               // listed before
    const int len = __ldcg(p.seq_lens + seq);
    int pages = pages_of(len > 0 ? len : 0, p.shift);
    if (pages > p.width) {
        if (threadIdx.x == 0) flag(p.status, HA_DEV_BAD_INDEX);
        pages = p.width;
    }
    for (int s = threadIdx.x; s < pages; s += kP_Threads) {
        const int page = __ldcg(p.table + (long long)seq * p.bt_sb + s);
        bool ok = (unsigned)page < (unsigned)p.n_pages;
        if (ok && atomicSub(p.ref + page, 1) <= 0) {   // nobody holds it: the count goes back to what it was
            atomicAdd(p.ref + page, 1);
            ok = false;
        }
        if (!ok) flag(p.status, HA_DEV_BAD_INDEX);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        p.seq_lens[seq] = 0;
        __threadfence();                               // kernels behind read it before their wait
    }
}

// exclusive sum over the CTA and the whole sum
template <typename T>
__device__ __forceinline__ T block_before(T v, T *sums, T &all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        T y = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const T z = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) y += z;
        }
        sums[lane] = y;
    }
    __syncthreads();
    all = sums[kP_Plan / 32 - 1];
    return (warp ? sums[warp - 1] : T(0)) + x - v;
}
// this thread's 16 counts of a round; those behind the last page read as -1 (neither free nor held)
__device__ __forceinline__ void load_counts(const int32_t *ref, int n_pages, long long first, int (&r)[kP_Counts]) {
    const long long at = first + (long long)threadIdx.x * kP_Counts;
    if (at + kP_Counts <= n_pages && (reinterpret_cast<uintptr_t>(ref) & 15) == 0) {
#pragma unroll
        for (int q = 0; q < kP_Counts / 4; ++q) {
            const int4 v = __ldcg(reinterpret_cast<const int4 *>(ref + at) + q);
            r[4 * q] = v.x; r[4 * q + 1] = v.y; r[4 * q + 2] = v.z; r[4 * q + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kP_Counts; ++i) r[i] = at + i < n_pages ? __ldcg(ref + at + i) : -1;
    }
}

// ---- extend, first kernel: how many pages each sequence needs, which ones it gets; all or nothing
__global__ void __launch_bounds__(kP_Plan, 1) pages_plan_extend_kernel(const PageState p, const int32_t *__restrict__ n_new, const PagePlan plan) {
    __shared__ long long needs[32];
    __shared__ int sums[32];
    __shared__ int s_copies;
    pdl_wait();
    const int tid = threadIdx.x;
    if (tid == 0) s_copies = 0;
    long long total = 0;
    uint32_t wrong = 0;
    // (first[b] keeps the number of pages in front of sequence b's; the sign bit marks one whose last page is copied)
    for (int b0 = 0; b0 < p.B; b0 += kP_Plan) {
        const int b = b0 + tid;
        int need = 0;
        bool copy = false;
        if (b < p.B) {
            const int add = __ldcg(n_new + b), len = __ldcg(p.seq_lens + b);
            if (add < 0 || len < 0) wrong |= HA_DEV_BAD_INDEX;
            else if (add > 0) {
                const int have = pages_of(len, p.shift), want = pages_of((long long)len + add, p.shift);
                if ((long long)len + add > 0x7fffffff || want > p.width) wrong |= HA_DEV_NO_PAGE;
                else {
                    if (len & ((1 << p.shift) - 1)) {
                        const int page = __ldcg(p.table + (long long)b * p.bt_sb + have - 1);
                        if ((unsigned)page >= (unsigned)p.n_pages) wrong |= HA_DEV_BAD_INDEX;
                        else copy = __ldcg(p.ref + page) > 1;
                    }
                    need = want - have + (copy ? 1 : 0);
                }
            }
        }
        long long all;
        const long long before = block_before((long long)need, needs, all);
        // a sum past the pages there are is cut there: it is refused below
        const long long f = total + before;
        if (b < p.B) plan.first[b] = (int)(f < p.n_pages ? f : p.n_pages) | (copy ? (int)0x80000000 : 0);
        total += all;
        if (total > p.n_pages) wrong |= HA_DEV_NO_PAGE;
    }
    // (the appends of the tokens that there is no room for learn of it: their places are other tokens' now)
    auto refuse = [&](uint32_t bit) {
        if (tid == 0) {
            flag(p.status, bit);
            p.status[kRefusedWord] = 1u;
            plan.n_copies[0] = 0;
        }
    };
    if (__syncthreads_or((int)(wrong & HA_DEV_BAD_INDEX))) {
        refuse(HA_DEV_BAD_INDEX);
        return;
    }
    if (__syncthreads_or((int)wrong)) {
        refuse(HA_DEV_NO_PAGE);
        return;
    }
    const int need = (int)total;
    int found = 0;
    for (long long first = 0; found < need && first < p.n_pages; first += kP_Plan * kP_Counts) {
        int r[kP_Counts], mine = 0;
        load_counts(p.ref, p.n_pages, first, r);
#pragma unroll
        for (int i = 0; i < kP_Counts; ++i) mine += r[i] == 0;
        int all;
        int at = found + block_before(mine, sums, all);
#pragma unroll
        for (int i = 0; i < kP_Counts; ++i)
            if (r[i] == 0) {
                if (at < need) plan.list[at] = (int)(first + (long long)tid * kP_Counts + i);
                ++at;
            }
        found += all;
    }
    if (found < need) {                                // uniform
        refuse(HA_DEV_NO_PAGE);
        return;
    }
    __syncthreads();
    // ---- nothing is refused any more: hand them out.  New page r belongs to the last sequence whose first is at or before r
    for (int r = tid; r < need; r += kP_Plan) {
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if ((plan.first[mid] & 0x7fffffff) <= r) lo = mid;
            else hi = mid - 1;
        }
        const int b = lo, f = plan.first[b];
        const bool copy = f < 0;
        const int len = __ldcg(p.seq_lens + b), slot = pages_of(len, p.shift) - (copy ? 1 : 0) + r - (f & 0x7fffffff), page = plan.list[r];
        int32_t *entry = p.table + (long long)b * p.bt_sb + slot;
        if (copy && r == (f & 0x7fffffff)) {
            const int k = atomicAdd(&s_copies, 1), old = __ldcg(entry);   // (the order of the list does not matter)
            plan.src[k] = old;
            plan.dst[k] = page;
            atomicSub(p.ref + old, 1);
        }
        *entry = page;
        p.ref[page] = 1;
    }
    __syncthreads();
    for (int b = tid; b < p.B; b += kP_Plan) p.seq_lens[b] = __ldcg(p.seq_lens + b) + __ldcg(n_new + b);
    if (tid == 0) {
        plan.n_copies[0] = s_copies;
        p.status[kRefusedWord] = 0u;
    }
}

// ---- compact, first kernel: pages in use at or above their number U move into the holes below it, in order
__global__ void __launch_bounds__(kP_Plan, 1) pages_plan_compact_kernel(const PageState p, int32_t *__restrict__ page_map,
                                                                       int32_t *__restrict__ n_used, const PagePlan plan) {
    __shared__ int sums[32];
    pdl_wait();
    const int tid = threadIdx.x;
    int used = 0;
    for (long long first = 0; first < p.n_pages; first += kP_Plan * kP_Counts) {
        int r[kP_Counts];
        load_counts(p.ref, p.n_pages, first, r);
#pragma unroll
        for (int i = 0; i < kP_Counts; ++i) used += r[i] > 0;
    }
    int U;
    block_before(used, sums, U);
    int done = 0, holes = 0;                           // pages in use in front of the round; holes below U of this thread
    for (long long first = 0; first < p.n_pages; first += kP_Plan * kP_Counts) {
        int r[kP_Counts], mine = 0;
        load_counts(p.ref, p.n_pages, first, r);
#pragma unroll
        for (int i = 0; i < kP_Counts; ++i) mine += r[i] > 0;
        int all;
        int before = done + block_before(mine, sums, all);
#pragma unroll
        for (int i = 0; i < kP_Counts; ++i) {
            const long long page = first + (long long)tid * kP_Counts + i;
            if (page >= p.n_pages) continue;
            if (r[i] > 0) {
                if (page >= U) plan.src[before] = (int)page;           // copy (before - number in use below U)
                else page_map[page] = (int)page;
                ++before;
            } else {
                page_map[page] = -1;
                if (page < U) {
                    plan.dst[page - before] = (int)page;
                    ++holes;
                }
            }
        }
        done += all;
    }
    int moves;
    block_before(holes, sums, moves);                  // as many as pages in use at or above U
    for (int m = tid; m < moves; m += kP_Plan) page_map[plan.src[U - moves + m]] = plan.dst[m];
    if (tid == 0) {
        plan.n_copies[0] = moves;
        plan.n_copies[1] = U - moves;
        n_used[0] = U;
    }
}

// ---- whole pages from src to dst: K, V and signatures
struct CompactTail {                     // compact: block table and counts follow
    const int32_t *page_map, *table, *ref;
    int32_t *table_out, *ref_out;
    long long out_sb;
};
template <bool kCompact>
__global__ void __launch_bounds__(kP_Copy) pages_copy_kernel(const PageState p, const PagePools pools, const PagePlan plan, const CompactTail t) {
    pdl_wait();
    const int n = plan.n_copies[0], tid = threadIdx.x;
    const int32_t *src = plan.src + (kCompact ? plan.n_copies[1] : 0), *dst = plan.dst;
    if (kCompact) {
        const long long stride = (long long)gridDim.x * kP_Copy, at = (long long)blockIdx.x * kP_Copy + tid;
        const long long entries = (long long)p.B * p.width;
        for (long long e = at; e < entries; e += stride) {
            const int b = (int)(e / p.width), s = (int)(e % p.width);
            const int len = __ldcg(p.seq_lens + b);
            int page = __ldcg(t.table + (long long)b * p.bt_sb + s);
            if (s < pages_of(len > 0 ? len : 0, p.shift)) {
                if ((unsigned)page < (unsigned)p.n_pages) page = __ldcg(t.page_map + page);
                else flag(p.status, HA_DEV_BAD_INDEX);
            }
            t.table_out[(long long)b * t.out_sb + s] = page;
        }
        // counts: a moved page's goes with it and leaves 0; every count is read and written by one thread
        const int U = n + plan.n_copies[1];
        for (long long e = at; e < p.n_pages; e += stride) {
            const int to = __ldcg(t.page_map + e);
            if (to == (int)e) t.ref_out[e] = __ldcg(t.ref + e);
            else if (e >= U && to < 0) t.ref_out[e] = 0;
        }
        for (long long m = at; m < n; m += stride) {
            const int v = __ldcg(t.ref + src[m]);
            t.ref_out[src[m]] = 0;
            t.ref_out[dst[m]] = v;
        }
    }
    // rows of 256 bytes in the order (copy, head, K / V, slot): sixteen lanes a row, kP_Batch rows of a lane in flight
    const unsigned heads = pools.heads, mask = (1u << p.shift) - 1;
    const long long rows = ((long long)n * heads * 2) << p.shift;
    constexpr int kAtOnce = kP_Copy / 16;
    for (long long r0 = (long long)blockIdx.x * kAtOnce * kP_Batch; r0 < rows; r0 += (long long)gridDim.x * kAtOnce * kP_Batch) {
        uint4 v[kP_Batch];
        uint16_t *to[kP_Batch];
#pragma unroll
        for (int u = 0; u < kP_Batch; ++u) {
            const long long r = r0 + u * kAtOnce + (tid >> 4);
            to[u] = nullptr;
            if (r >= rows) continue;
            const unsigned long long pair = (unsigned long long)r >> p.shift;
            const unsigned long long mh = pair >> 1;
            const long long m = mh <= 0xffffffffu ? (unsigned)mh / heads : mh / heads;
            const long long h = (long long)mh - m * heads;
            const TensorView &T = pair & 1 ? pools.V : pools.K;
            const uint16_t *base = T.ptr + h * T.sh + (long long)(r & mask) * T.sn + (tid & 15) * 8;
            v[u] = __ldcs(reinterpret_cast<const uint4 *>(base + (long long)src[m] * T.sb));
            to[u] = const_cast<uint16_t *>(base) + (long long)dst[m] * T.sb;
        }
#pragma unroll
        for (int u = 0; u < kP_Batch; ++u)
            if (to[u]) *reinterpret_cast<uint4 *>(to[u]) = v[u];
    }
    if (pools.codes) {                   // words in the order (copy, head, slot)
        const long long words = ((long long)n * heads) << p.shift;
        for (long long w = (long long)blockIdx.x * kP_Copy + tid; w < words; w += (long long)gridDim.x * kP_Copy) {
            const unsigned long long mh = (unsigned long long)w >> p.shift;
            const long long m = mh <= 0xffffffffu ? (unsigned)mh / heads : mh / heads;
            uint32_t *c = pools.codes + ((long long)mh - m * heads) * pools.c_head + (w & mask);
            c[(long long)dst[m] * pools.c_page] = c[(long long)src[m] * pools.c_page];
        }
    }
}

// ---- workspace: front, numbers, then the lists
struct PagesLayout {
    size_t off_numbers, off_first, off_list, off_src, off_dst, total;
};
static PagesLayout pages_layout(int n_pages, int B) {
    PagesLayout L;
    size_t o = kWorkspaceFront;
    L.off_numbers = o; o += 256;
    L.off_first = o;   o = align_up(o + ((size_t)B + 1) * 4, 256);
    L.off_list = o;    o = align_up(o + (size_t)n_pages * 4, 256);
    const size_t copies = (size_t)(n_pages > B ? n_pages : B);
    L.off_src = o;     o = align_up(o + copies * 4, 256);
    L.off_dst = o;     o = align_up(o + copies * 4, 256);
    L.total = o;
    return L;
}
size_t pages_workspace_bytes(int n_pages, int B) { return pages_layout(n_pages, B).total; }

static PagePlan plan_in(void *workspace, int n_pages, int B) {
    const PagesLayout L = pages_layout(n_pages, B);
    char *ws = reinterpret_cast<char *>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<int32_t *>(ws + off); };
    return PagePlan{at(L.off_numbers), at(L.off_first), at(L.off_list), at(L.off_src), at(L.off_dst)};
}
static PageState state_of(const PagesView &v, void *workspace) {
    return PageState{v.seq_lens, v.table, v.ref, v.bt_sb, v.B, v.width, v.n_pages, v.shift, reinterpret_cast<uint32_t *>(workspace)};
}

cudaError_t launch_pages_fork(const PagesView &v, const int32_t *parents, const int32_t *children, int n, void *workspace, cudaStream_t st) {
    const cudaError_t e = launch_pdl(pages_fork_kernel, dim3(n), dim3(kP_Threads), 0, st, state_of(v, workspace), parents, children, n);
    if (e != cudaSuccess) return e;
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_pages_free(const PagesView &v, const int32_t *seqs, int n, void *workspace, cudaStream_t st) {
    const cudaError_t e = launch_pdl(pages_free_kernel, dim3(n), dim3(kP_Threads), 0, st, state_of(v, workspace), seqs, n);
    if (e != cudaSuccess) return e;
    count_launch();
    return cudaGetLastError();
}

static PagePools pools_of(TensorView K, TensorView V, int heads, uint32_t *codes, long long c_page, long long c_head) {
    return PagePools{K, V, codes, c_page, c_head, heads};
}

cudaError_t launch_pages_extend(const PagesView &v, const int32_t *n_new, TensorView K, TensorView V, int heads, uint32_t *codes,
                                long long c_page, long long c_head, void *workspace, cudaStream_t st) {
    const PageState s = state_of(v, workspace);
    const PagePlan plan = plan_in(workspace, v.n_pages, v.B);
    cudaError_t e = launch_pdl(pages_plan_extend_kernel, dim3(1), dim3(kP_Plan), 0, st, s, n_new, plan);
    if (e != cudaSuccess) return e;
    long long grid = (long long)v.B * heads;             // at most one page of each sequence is copied
    if (grid > 8LL * sm_count()) grid = 8LL * sm_count();
    e = launch_pdl(pages_copy_kernel<false>, dim3((unsigned)grid), dim3(kP_Copy), 0, st, s, pools_of(K, V, heads, codes, c_page, c_head), plan,
                   CompactTail{});
    if (e != cudaSuccess) return e;
    count_launch(2);
    return cudaGetLastError();
}

cudaError_t launch_pages_compact(const PagesView &v, TensorView K, TensorView V, int heads, uint32_t *codes, long long c_page,
                                 long long c_head, int32_t *table_out, long long out_sb, int32_t *ref_out, int32_t *page_map,
                                 int32_t *n_used, void *workspace, cudaStream_t st) {
    const PageState s = state_of(v, workspace);
    const PagePlan plan = plan_in(workspace, v.n_pages, v.B);
    cudaError_t e = launch_pdl(pages_plan_compact_kernel, dim3(1), dim3(kP_Plan), 0, st, s, page_map, n_used, plan);
    if (e != cudaSuccess) return e;
    const CompactTail t{page_map, v.table, v.ref, table_out, ref_out, out_sb};
    e = launch_pdl(pages_copy_kernel<true>, dim3((unsigned)(8 * sm_count())), dim3(kP_Copy), 0, st, s,
                   pools_of(K, V, heads, codes, c_page, c_head), plan, t);
    if (e != cudaSuccess) return e;
    count_launch(2);
    return cudaGetLastError();
}

} // namespace ha
