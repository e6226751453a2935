// The ledger of a paged cache (page table, lengths, counts): room for new tokens, forks, ends, compaction. Whole
// numbers only; what a call allots does not depend on the order in which its threads run.
//
// A call is one launch: a CTA, or a cluster of eight where the ledger is large, so that its phases (what is needed
// and what is free; the decision; the pages; the table) are parted by the cluster's barrier instead of by
// launches. Every thread owns a run of consecutive slots and one of consecutive pages; prefix sums over the threads give each
// its place among the pages taken, in ascending order. Bound by latency: the loads of one phase and three or four barriers.
#include "serve_common.cuh"
#include "warp_common.cuh"

namespace stream {
namespace {

constexpr int kThreads = 1024;
constexpr int kMaxCtas = 8;

struct Args {
    CacheGeom c;
    const int32_t *in;  // n_new, parent or done: one per slot
    int32_t *pairs, *info;
    int32_t *slot_at;   // workspace [n_slots]: a slot's first place among the pages taken
    int32_t *page_at;   // workspace [n_pages]: the pages taken, in order; compaction: a page's new number
};

struct Shared {
    int warp_sums[3][32];
    int cta_sums[3];   // read by the cluster's other CTAs
};

// All threads of all CTAs; what they wrote before, in global and in shared memory, is there behind it.
__device__ __forceinline__ void sync_all() {
    if (wp::cluster_size() == 1) {
        __syncthreads();
        return;
    }
    wp::cluster_arrive();
    wp::cluster_wait();
}
// before[i]: the sum of x[i] over the threads in front of this one, all CTAs counted; total[i]: over all.
template <int n>
__device__ void scan(Shared &sh, const int (&x)[n], int (&before)[n], int (&total)[n]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl[n];
#pragma unroll
    for (int i = 0; i < n; ++i) {
        incl[i] = x[i];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl[i], d);
            if (lane >= d) incl[i] += y;
        }
        if (lane == 31) sh.warp_sums[i][warp] = incl[i];
    }
    __syncthreads();
    if (warp == 0) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int own = sh.warp_sums[i][lane];
            int s = own;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, s, d);
                if (lane >= d) s += y;
            }
            sh.warp_sums[i][lane] = s - own;
            if (lane == 31) sh.cta_sums[i] = s;
        }
    }
    sync_all();
    const unsigned ctas = wp::cluster_size(), rank = wp::cluster_rank();
#pragma unroll
    for (int i = 0; i < n; ++i) {
        before[i] = sh.warp_sums[i][warp] + incl[i] - x[i];
        total[i] = 0;
        for (unsigned r = 0; r < ctas; ++r) {
            const int s = ctas == 1 ? sh.cta_sums[i] : __float_as_int(wp::load_in_cluster(reinterpret_cast<const float *>(&sh.cta_sums[i]), r));
            if (r < rank) before[i] += s;
            total[i] += s;
        }
    }
    sync_all();  // (the sums may be written again, and a CTA may leave)
}

struct Run { int first, end; };
// This thread's run of n things.
__device__ __forceinline__ Run own_run(int n) {
    const int threads = (int)wp::cluster_size() * kThreads, per = (n + threads - 1) / threads;
    const long long me = (long long)wp::cluster_rank() * kThreads + threadIdx.x;
    return {(int)min((long long)n, me * per), (int)min((long long)n, (me + 1) * per)};
}
__device__ __forceinline__ int free_in(const CacheGeom &c, Run r) {
    int n = 0;
    for (int p = r.first; p < r.end; ++p) n += c.count[p] == 0 ? 1 : 0;
    return n;
}
__device__ __forceinline__ bool in_cache(const CacheGeom &c, int page) { return (unsigned)page < (unsigned)c.n_pages; }
__device__ __forceinline__ void say(const Args &a, int done, int moved, int free, int bad) {
    if (threadIdx.x == 0 && wp::cluster_rank() == 0) *reinterpret_cast<int4 *>(a.info) = make_int4(done, moved, free, bad);
}
// The free pages of this thread's run, the first of them being the before-th of all, take their places among the `total` taken ones.
__device__ __forceinline__ void take_pages(const Args &a, Run r, int before, int total) {
    for (int p = r.first; p < r.end && before < total; ++p)
        if (a.c.count[p] == 0) {
            a.page_at[before++] = p;
            a.c.count[p] = 1;
        }
}
// Warps of all CTAs take the slots in turn.
struct Warps { int first, step; };
__device__ __forceinline__ Warps all_warps() { return {(int)(wp::cluster_rank() * (kThreads / 32) + (threadIdx.x >> 5)), (int)wp::cluster_size() * (kThreads / 32)}; }

__global__ void __launch_bounds__(kThreads, 1) reserve_kernel(Args a) {
    __shared__ Shared sh;
    const CacheGeom &c = a.c;
    after_previous_kernel();
    const Run slots = own_run(c.n_slots), pages = own_run(c.n_pages);
    auto need_of = [&](int s, int &have, int &bad) -> int {
        const int n = a.in[s], len = c.len[s];
        const long long after = ((long long)len + n + c.page - 1) / c.page;
        bad = n < 0 || len < 0 || after > c.max_pages ? 1 : 0;
        have = bad ? 0 : ceil_div(len, c.page);
        return bad ? 0 : (int)after - have;
    };
    int x[3] = {0, free_in(c, pages), 0}, before[3], total[3], have, bad;
    for (int s = slots.first; s < slots.end; ++s) {
        x[0] += need_of(s, have, bad);
        x[2] += bad;
    }
    scan(sh, x, before, total);
    if (total[2] > 0 || total[0] > total[1]) {
        say(a, 0, total[0], total[1], total[2]);
        return;
    }
    say(a, 1, total[0], total[1] - total[0], 0);
    int at = before[0];
    for (int s = slots.first; s < slots.end; ++s) {
        a.slot_at[s] = at;
        at += need_of(s, have, bad);
    }
    take_pages(a, pages, before[1], total[0]);
    sync_all();
    const Warps w = all_warps();
    const int lane = threadIdx.x & 31;
    for (int s = w.first; s < c.n_slots; s += w.step) {
        const int need = need_of(s, have, bad);
        for (int i = lane; i < need; i += 32) c.table[(long long)s * c.max_pages + have + i] = a.page_at[a.slot_at[s] + i];
        __syncwarp();  // (every lane has read the length)
        if (lane == 0) c.len[s] += a.in[s];
    }
}

__global__ void __launch_bounds__(kThreads, 1) fork_kernel(Args a) {
    __shared__ Shared sh;
    const CacheGeom &c = a.c;
    after_previous_kernel();
    const Run slots = own_run(c.n_slots), pages = own_run(c.n_pages);
    // whether slot s becomes a copy that takes a page (its last one is not full); bad: it cannot become one
    auto needs = [&](int s, int &bad) -> int {
        bad = 0;
        const int p = a.in[s];
        if (p < 0) return 0;
        if (p >= c.n_slots || a.in[p] >= 0 || c.len[s] != 0) { bad = 1; return 0; }
        const int n = c.len[p];
        if (n < 0 || n > c.max_pages * c.page) { bad = 1; return 0; }
        return n % c.page != 0 ? 1 : 0;
    };
    int x[3] = {0, free_in(c, pages), 0}, before[3], total[3], bad;
    for (int s = slots.first; s < slots.end; ++s) {
        x[0] += needs(s, bad);
        x[2] += bad;
    }
    scan(sh, x, before, total);
    const bool done = total[2] == 0 && total[0] <= total[1];
    say(a, done ? 1 : 0, total[0], total[1] - (done ? total[0] : 0), total[2]);
    for (int i = slots.first; i < slots.end; ++i)
        if (!done || i >= total[0]) *reinterpret_cast<int2 *>(a.pairs + 2ll * i) = make_int2(-1, -1);
    if (!done) return;
    int at = before[0];
    for (int s = slots.first; s < slots.end; ++s) {
        a.slot_at[s] = at;
        at += needs(s, bad);
    }
    take_pages(a, pages, before[1], total[0]);
    sync_all();
    const Warps w = all_warps();
    const int lane = threadIdx.x & 31;
    for (int s = w.first; s < c.n_slots; s += w.step) {
        const int p = a.in[s];
        if (p < 0) continue;
        const int n = c.len[p], entries = ceil_div(n, c.page), full = n / c.page;  // (nobody writes a parent's length)
        for (int j = lane; j < entries; j += 32) {
            int page = c.table[(long long)p * c.max_pages + j];
            if (j < full) {
                if (in_cache(c, page)) atomicAdd(&c.count[page], 1);
            } else {
                const int fresh = a.page_at[a.slot_at[s]];
                *reinterpret_cast<int2 *>(a.pairs + 2ll * a.slot_at[s]) = make_int2(page, fresh);
                page = fresh;
            }
            c.table[(long long)s * c.max_pages + j] = page;
        }
        if (lane == 0) c.len[s] = n;
    }
}

__global__ void __launch_bounds__(kThreads, 1) free_kernel(Args a) {
    __shared__ Shared sh;
    const CacheGeom &c = a.c;
    after_previous_kernel();
    const Warps w = all_warps();
    const int lane = threadIdx.x & 31;
    int x[3] = {0, 0, 0}, before[3], total[3];
    for (int s = w.first; s < c.n_slots; s += w.step) {
        if (a.in[s] == 0) continue;
        const int tokens = tokens_of(c, s), entries = ceil_div(tokens, c.page);
        if (lane == 0 && c.len[s] != tokens) ++x[2];
        for (int j = lane; j < c.max_pages; j += 32) {
            int32_t *const e = c.table + (long long)s * c.max_pages + j;
            if (j < entries) {
                const int page = *e;
                if (!in_cache(c, page)) {
                    ++x[2];
                } else {
                    const int was = atomicSub(&c.count[page], 1);
                    if (was == 1) ++x[0];
                    if (was <= 0) { atomicAdd(&c.count[page], 1); ++x[2]; }
                }
            }
            *e = -1;
        }
        __syncwarp();
        if (lane == 0) c.len[s] = 0;
    }
    sync_all();
    x[1] = free_in(c, own_run(c.n_pages));
    scan(sh, x, before, total);
    say(a, 1, total[0], total[1], total[2]);
}

__global__ void __launch_bounds__(kThreads, 1) compact_kernel(Args a) {
    __shared__ Shared sh;
    const CacheGeom &c = a.c;
    after_previous_kernel();
    const Run pages = own_run(c.n_pages);
    int free[1] = {free_in(c, pages)}, before[1], n_free[1];
    scan(sh, free, before, n_free);
    const int n_used = c.n_pages - n_free[0];
    // used pages from n_used on, and free ones below it: as many of one as of the other
    int x[2] = {0, 0}, at[2], n[2];
    for (int p = pages.first; p < pages.end; ++p) {
        const bool is_free = c.count[p] == 0;
        if (!is_free && p >= n_used) ++x[0];
        if (is_free && p < n_used) ++x[1];
        a.page_at[p] = p;
    }
    scan(sh, x, at, n);
    const int moves = n[0];
    say(a, 1, moves, n_free[0], 0);
    for (int p = pages.first; p < pages.end; ++p) {
        const bool is_free = c.count[p] == 0;
        if (!is_free && p >= n_used) a.pairs[2ll * at[0]++] = p;
        if (is_free && p < n_used) a.pairs[2ll * at[1]++ + 1] = p;
    }
    const int threads = (int)wp::cluster_size() * kThreads, me = (int)wp::cluster_rank() * kThreads + threadIdx.x;
    for (int i = moves + me; i < c.n_pages / 2; i += threads) *reinterpret_cast<int2 *>(a.pairs + 2ll * i) = make_int2(-1, -1);
    sync_all();
    for (int i = me; i < moves; i += threads) {
        const int2 pr = *reinterpret_cast<const int2 *>(a.pairs + 2ll * i);
        a.page_at[pr.x] = pr.y;
        c.count[pr.y] = c.count[pr.x];
        c.count[pr.x] = 0;
    }
    sync_all();
    const long long entries = (long long)c.n_slots * c.max_pages;
    for (long long i = me; i < entries; i += threads) {
        const int page = c.table[i];
        if (in_cache(c, page) && page >= n_used) c.table[i] = a.page_at[page];
    }
}

stream_status launch(void (*kern)(Args), const CacheGeom &c, const int32_t *in, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st, const char *what) {
    Args a = {};
    a.c = c; a.in = in; a.pairs = pairs; a.info = info;
    a.slot_at = (int32_t *)ws;
    a.page_at = a.slot_at + ((c.n_slots + 63) & ~63);
    const long long size = (long long)c.n_slots * c.max_pages + c.n_pages;
    const unsigned ctas = size > 16 * kThreads ? kMaxCtas : 1;
    const cudaError_t e = ctas == 1 ? launch_early(kern, 1, kThreads, 0, st, a) : launch_clusters(kern, ctas, kThreads, 0, st, ctas, a);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, what);
}

}  // namespace

size_t ledger_workspace_bytes(const CacheGeom &c) {
    return ((size_t)((c.n_slots + 63) & ~63) + (size_t)((c.n_pages + 63) & ~63)) * sizeof(int32_t);
}

stream_status launch_reserve(const CacheGeom &c, const int32_t *n_new, int32_t *info, void *ws, cudaStream_t st) {
    return launch(reserve_kernel, c, n_new, nullptr, info, ws, st, "cache reserve launch");
}
stream_status launch_fork(const CacheGeom &c, const int32_t *parent, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st) {
    return launch(fork_kernel, c, parent, pairs, info, ws, st, "cache fork launch");
}
stream_status launch_free(const CacheGeom &c, const int32_t *done, int32_t *info, void *ws, cudaStream_t st) {
    return launch(free_kernel, c, done, nullptr, info, ws, st, "cache free launch");
}
stream_status launch_compact(const CacheGeom &c, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st) {
    return launch(compact_kernel, c, nullptr, pairs, info, ws, st, "cache compact launch");
}

}  // namespace stream
