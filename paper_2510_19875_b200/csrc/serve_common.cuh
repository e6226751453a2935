// Shared by the dense-attention and cache kernels: geometry, launches, sequence bounds.
#pragma once
#include <math_constants.h>

#include <atomic>

#include "common.cuh"

namespace stream {

// Packed prompts as the kernels see them. Rows of a kv head's queries are counted token by token, query head by query
// head within one: row r of a sequence is token r / hpg, head g * hpg + r % hpg.
struct PromptGeom {
    int n_seqs, H, G, hpg, d, causal;
    int total_q, total_k;
    long long qs_t, qs_h, ks_t, ks_h;
    const int32_t *cu_q, *cu_k;
    float scale_log2;  // logit scale times log2(e)
    void *out;
    float *lse;
};

// A paged cache and the ledger.
struct CacheGeom {
    int n_slots, n_pages, page, max_pages, G, d, n_layers;
    long long s_l, s_p, s_t, s_h;
    int32_t *table, *len, *count;
};

constexpr float kLn2 = 0.6931471805599453f;

// Entries s and s + 1 of an ascending list of offsets, whatever it holds, within 0 .. total.
struct Span { int first, n; };
__device__ __forceinline__ Span span_of(const int32_t *cu, int s, int total) {
    const int a = min(max(cu[s], 0), total), b = min(max(cu[s + 1], a), total);
    return {a, b - a};
}
// Tokens of a slot.
__device__ __forceinline__ int tokens_of(const CacheGeom &c, int s) { return min(max(c.len[s], 0), c.max_pages * c.page); }
__host__ __device__ __forceinline__ int ceil_div(int a, int b) { return (int)(((long long)a + b - 1) / b); }

// The kernels that give every tile of `rows` rows of a kv head's queries a CTA: which sequence the nth one lies in, and its number
// there. By a whole warp. seq < 0: there are fewer.
struct RowTile { int seq, nth; };
__device__ __forceinline__ RowTile row_tile(const PromptGeom &g, int nth, int rows, int lane) {
    long long sum = 0;  // (offsets that fall make sequences overlap: more tiles than 32 bits count)
    for (int s0 = 0; s0 < g.n_seqs; s0 += 32) {
        const int s = s0 + lane;
        const long long tiles = s < g.n_seqs ? ((long long)span_of(g.cu_q, s, g.total_q).n * g.hpg + rows - 1) / rows : 0;
        long long incl = tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, nth < sum + incl);
        if (past != 0) {
            const int at = __ffs(past) - 1;
            return {s0 + at, (int)(nth - sum - __shfl_sync(0xffffffffu, incl - tiles, at))};
        }
        sum += __shfl_sync(0xffffffffu, incl, 31);
    }
    return {-1, 0};
}
// No more tiles than this, of all kv heads, however the rows are dealt to the sequences.
inline long long most_row_tiles(const PromptGeom &g, int rows) {
    return ((long long)g.total_q * g.hpg / rows + (g.n_seqs < g.total_q ? g.n_seqs : g.total_q)) * g.G;
}

// A programmatic dependent (see after_previous_kernel), and clusters of CTAs.
template <class... K, class... A>
cudaError_t launch_early(void (*kern)(K...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A &&...args) {
    return launch_kernel(kern, grid, threads, smem, st, 1u, std::forward<A>(args)...);
}
template <class... K, class... A>
cudaError_t launch_clusters(void (*kern)(K...), unsigned grid, unsigned threads, size_t smem, cudaStream_t st, unsigned cluster, A &&...args) {
    return launch_kernel(kern, grid, threads, smem, st, cluster, std::forward<A>(args)...);
}

// What a short call need not ask the runtime every time, by device (a process may use several, and they may differ).
constexpr int kMaxDevices = 64;
inline int current_device() {
    int dev = -1;
    if (cudaGetDevice(&dev) == cudaSuccess) return dev;
    (void)cudaGetLastError();
    return -1;
}
inline int current_sm_count() {
    static std::atomic<int> known[kMaxDevices];
    const int dev = current_device();
    if (dev < 0) return 0;
    int n = dev < kMaxDevices ? known[dev].load(std::memory_order_relaxed) : 0;
    if (n > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (dev < kMaxDevices) known[dev].store(n, std::memory_order_relaxed);
    return n;
}
// Dynamic shared memory of a kernel beyond 48 KB, asked for once a device; `done`: of that kernel.
typedef std::atomic<unsigned long long> DeviceFlags;
template <class... K>
cudaError_t allow_smem_once(void (*kern)(K...), int bytes, DeviceFlags &done) {
    const int dev = current_device();
    const unsigned long long bit = dev >= 0 && dev < kMaxDevices ? 1ull << dev : 0ull;
    if ((done.load(std::memory_order_relaxed) & bit) != 0) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

bool prompt_tc_supported(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v);
stream_status launch_prompt_tc(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st);
bool prompt_mma_supported(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v);
stream_status launch_prompt_mma(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st);
bool prompt_f32_supported(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v);
stream_status launch_prompt_f32(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st);
stream_status launch_prompt_generic(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v, cudaStream_t st);

struct DecodeCall {
    CacheGeom c;
    int H, hpg;
    long long qs_s, qs_h;
    const void *q, *k, *v;  // k, v: of the layer
    float scale_log2;
    void *out;
    float *lse;
};
size_t decode_workspace_bytes(const CacheGeom &c);
stream_status launch_decode(const DecodeCall &a, int dtype, void *workspace, cudaStream_t st);

size_t ledger_workspace_bytes(const CacheGeom &c);
stream_status launch_reserve(const CacheGeom &c, const int32_t *n_new, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_fork(const CacheGeom &c, const int32_t *parent, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_free(const CacheGeom &c, const int32_t *done, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_compact(const CacheGeom &c, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_copy_pages(const CacheGeom &c, int elem, void *k, void *v, const int32_t *pairs, const int32_t *count, int n_pairs, cudaStream_t st);
stream_status launch_write(const CacheGeom &c, int elem, const void *k, const void *v, int total, long long s_t, long long s_h,
                           const int32_t *cu_new, const int32_t *done, void *k_pages, void *v_pages, cudaStream_t st);

}  // namespace stream
