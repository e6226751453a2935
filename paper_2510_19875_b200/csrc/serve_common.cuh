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
    int window, sinks; // window > 0: a query at position p sees the keys j <= p with j > p - window or j < sinks
};

// What a tile of rows walks of the keys where there is a window: those of the sinks, in whole units, and behind a gap all from the first key that the
// first row's window has. Tiles are cut from the keys as they are counted without the gap. (Positions below 0 see nothing.)
struct Walked {
    int sink_keys, gap;  // keys in front of the gap, a multiple of the unit; keys of the gap
    __device__ __forceinline__ int key(int walked) const { return walked < sink_keys ? walked : walked + gap; }
};
__device__ __forceinline__ Walked walked_keys(const PromptGeom &g, int unit, int first_pos, int n_keys) {
    const int low = max(0, max(first_pos, 0) - g.window + 1), sinks = (min(g.sinks, n_keys) + unit - 1) / unit * unit;
    return {sinks, max(0, low - sinks)};
}
// The first key of a position's window.
__device__ __forceinline__ int window_begin(const PromptGeom &g, int pos) { return max(0, max(pos, 0) - g.window + 1); }

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
// The slot whose packed rows hold row t, if any does: the last one that begins at or before it (32 candidates a step). By a whole warp.
__device__ __forceinline__ int slot_of_row(const int32_t *cu, int n_slots, long long t, int lane) {
    int lo = 0, hi = n_slots;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const long long at = lo + (long long)lane * step;
        const unsigned below = __ballot_sync(0xffffffffu, at < hi && cu[at] <= t);
        const int last = below != 0 ? 31 - __clz(below) : 0;
        lo += last * step;
        hi = min(hi, lo + step);
    }
    return lo;
}
// Tokens of a slot.
__device__ __forceinline__ int tokens_of(const CacheGeom &c, int s) { return min(max(c.len[s], 0), c.max_pages * c.page); }
// a >= 0, b > 0. (A division of 64 bits is hundreds of cycles.)
__host__ __device__ __forceinline__ int ceil_div(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

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
// Division of numbers below 2^31: n / d = (n + (n m >> 32)) >> s with 2^(s-1) < d <= 2^s and m = 2^32 (2^s - d) / d, rounded down, and 1.
struct Divisor {
    unsigned m, d;
    int s;
    __device__ __forceinline__ unsigned quotient(unsigned n) const { return (__umulhi(n, m) + n) >> s; }
};
inline Divisor make_divisor(int d) {
    Divisor r = {0, (unsigned)d, 0};
    while ((1ll << r.s) < d) ++r.s;
    r.m = (unsigned)((((1ull << r.s) - (unsigned long long)d) << 32) / (unsigned long long)d + 1);
    return r;
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
    int window, sinks;     // as in PromptGeom
};
// The scales of a cache in 8 bits: of the layer.
struct Scales {
    const float *k, *v;
    long long s_p, s_b, s_h;  // page, block, head
    int block;                // tokens
};
size_t decode_workspace_bytes(const CacheGeom &c);
stream_status launch_decode(const DecodeCall &a, int dtype, void *workspace, cudaStream_t st);
stream_status launch_decode8(const DecodeCall &a, const Scales &sc, int dtype, void *workspace, cudaStream_t st);

size_t ledger_workspace_bytes(const CacheGeom &c);
stream_status launch_reserve(const CacheGeom &c, const int32_t *n_new, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_fork(const CacheGeom &c, const int32_t *parent, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_free(const CacheGeom &c, const int32_t *done, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_compact(const CacheGeom &c, int32_t *pairs, int32_t *info, void *ws, cudaStream_t st);
stream_status launch_copy_pages(const CacheGeom &c, int elem, void *k, void *v, const int32_t *pairs, const int32_t *count, int n_pairs, cudaStream_t st);
stream_status launch_write(const CacheGeom &c, int elem, const void *k, const void *v, int total, long long s_t, long long s_h,
                           const int32_t *cu_new, const int32_t *done, void *k_pages, void *v_pages, cudaStream_t st);
stream_status launch_read(const CacheGeom &c, int elem, const void *k_pages, const void *v_pages, const int32_t *cu, int total, void *k_out, void *v_out, cudaStream_t st);
stream_status launch_write8(const CacheGeom &c, const Scales &sc, int dtype, const void *k, const void *v, int total, long long s_t, long long s_h,
                            const int32_t *cu_new, const int32_t *done, void *k_pages, void *v_pages, cudaStream_t st);
stream_status launch_read8(const CacheGeom &c, const Scales &sc, int dtype, const void *k_pages, const void *v_pages, const int32_t *cu, int total,
                           void *k_out, void *v_out, cudaStream_t st);

}  // namespace stream
