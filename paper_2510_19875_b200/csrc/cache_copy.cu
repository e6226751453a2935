// The bytes of a paged cache: whole pages copied in all layers, and new tokens' keys and values written to their pages. Both
// move every byte once and are bound by HBM; threads move 16 bytes at a time (8, 4 or 2 where a stride or an address asks for it),
// eight loads before the first store.
#include "serve_common.cuh"

#include <initializer_list>

namespace stream {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 8;  // loads in flight a thread
// CTAs an SM of a grid, at most. us with 8, 16, 64 of them, and with 64 and four loads ahead: pages of 28 layers forked, freed and compacted, 1.29 GB moved,
// 237, 224, 220, 225; 18566 new tokens, 152 MB, 36.3, 35.1, 35.1, 35.2; pages of four layers, 100 MB, 27.8, 28.0, 27.9, 28.8; small calls the same with all.
constexpr int kCtas = 64;

// ----------------------------------------------------------------------------------------------
// Pages: runs of `run` units (a whole page where it is one piece of memory, else a token or a head's row)
// ----------------------------------------------------------------------------------------------
struct CopyArgs {
    char *base[2];               // K, V
    const int32_t *pairs, *count;
    int n_pairs, n_pages, n_layers;
    long long s_l, s_p;          // bytes
    int n_outer, n_inner;        // runs of a page: n_outer x n_inner
    long long s_outer, s_inner;  // bytes
    int run;                     // units of a run
    int per_page;                // units of a page
    int pieces;                  // of a page, kThreads * kAhead units each
};

// kFlat: a page is one run.
template <class Unit, bool kFlat>
__global__ void __launch_bounds__(kThreads) copy_pages_kernel(const __grid_constant__ CopyArgs a) {
    after_previous_kernel();
    const int n = min(max(*a.count, 0), a.n_pairs);
    const long long items = (long long)n * a.n_layers * 2 * a.pieces;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int piece = (int)(it % a.pieces);
        const long long x = it / a.pieces;
        const int kv = (int)(x & 1), layer = (int)((x >> 1) % a.n_layers), i = (int)((x >> 1) / a.n_layers);
        const int from = a.pairs[2ll * i], to = a.pairs[2ll * i + 1];
        if ((unsigned)from >= (unsigned)a.n_pages || (unsigned)to >= (unsigned)a.n_pages) continue;
        const char *src = a.base[kv] + layer * a.s_l + from * a.s_p;
        char *dst = a.base[kv] + layer * a.s_l + to * a.s_p;
        auto at = [&](int e) -> long long {
            if (kFlat) return (long long)e * (int)sizeof(Unit);
            const int k = e / a.run, outer = k / a.n_inner;
            return outer * a.s_outer + (k - outer * a.n_inner) * a.s_inner + (long long)(e - k * a.run) * (int)sizeof(Unit);
        };
        const int e0 = piece * kAhead * kThreads + (int)threadIdx.x;
        Unit r[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (e0 + u * kThreads < a.per_page) r[u] = *reinterpret_cast<const Unit *>(src + at(e0 + u * kThreads));
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (e0 + u * kThreads < a.per_page) *reinterpret_cast<Unit *>(dst + at(e0 + u * kThreads)) = r[u];
    }
}

// ----------------------------------------------------------------------------------------------
// New tokens: a warp a token
// ----------------------------------------------------------------------------------------------
struct WriteArgs {
    CacheGeom c;
    const char *k, *v;
    char *k_pages, *v_pages;
    const int32_t *cu, *done;
    int total, elem;
    long long s_t, s_h;          // bytes, of k and v
    int run, per_token;          // units of a head's row (of all heads where they lie side by side on both sides); of a token
};

template <class Unit>
__global__ void __launch_bounds__(kThreads) write_kernel(const __grid_constant__ WriteArgs a) {
    after_previous_kernel();
    const CacheGeom &c = a.c;
    if (a.done != nullptr && *a.done == 0) return;
    const int lane = threadIdx.x & 31;
    for (long long t = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < a.total; t += (long long)gridDim.x * (kThreads / 32)) {
        const int lo = slot_of_row(a.cu, c.n_slots, t, lane);
        const Span sp = span_of(a.cu, lo, a.total);
        const int len = tokens_of(c, lo);
        const long long pos = (long long)len - sp.n + (t - sp.first);
        if (t < sp.first || t >= (long long)sp.first + sp.n || pos < 0) continue;
        const int page = c.table[(long long)lo * c.max_pages + (int)pos / c.page];
        if ((unsigned)page >= (unsigned)c.n_pages) continue;
        const long long to = (page * c.s_p + ((int)pos % c.page) * c.s_t) * a.elem, from = t * a.s_t;
        for (int u = lane; u < a.per_token; u += 32) {
            const int h = u / a.run;
            const long long x = (long long)(u - h * a.run) * (int)sizeof(Unit);
            const Unit k = *reinterpret_cast<const Unit *>(a.k + from + h * a.s_h + x), v = *reinterpret_cast<const Unit *>(a.v + from + h * a.s_h + x);
            *reinterpret_cast<Unit *>(a.k_pages + to + h * c.s_h * a.elem + x) = k;
            *reinterpret_cast<Unit *>(a.v_pages + to + h * c.s_h * a.elem + x) = v;
        }
    }
}

// The way back: packed rows out of the pages, zeros where there is no page. (29558 tokens of 8 heads, d = 128: bf16 43 us, 242 MB at 86 % of the copy rate,
// 6556 GB/s; fp32 80, 92 %.)
struct ReadArgs {
    CacheGeom c;
    const char *k_pages, *v_pages;
    char *k, *v;
    const int32_t *cu;
    int total, elem;
    int run, per_token;          // as in WriteArgs
};

template <class Unit>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ ReadArgs a) {
    after_previous_kernel();
    const CacheGeom &c = a.c;
    const int lane = threadIdx.x & 31;
    for (long long t = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < a.total; t += (long long)gridDim.x * (kThreads / 32)) {
        const int s = slot_of_row(a.cu, c.n_slots, t, lane);
        const Span sp = span_of(a.cu, s, a.total);
        if (t < sp.first || t >= (long long)sp.first + sp.n) continue;
        const long long pos = (long long)tokens_of(c, s) - sp.n + (t - sp.first);
        const int page = pos >= 0 ? c.table[(long long)s * c.max_pages + (int)pos / c.page] : -1;
        const bool there = (unsigned)page < (unsigned)c.n_pages;
        const long long from = there ? (page * c.s_p + ((int)pos % c.page) * c.s_t) * a.elem : 0, to = t * a.per_token * (long long)sizeof(Unit);
        for (int u = lane; u < a.per_token; u += 32) {
            const int h = u / a.run;
            const long long x = h * c.s_h * a.elem + (long long)(u - h * a.run) * (int)sizeof(Unit);
            Unit k = {}, v = {};
            if (there) {
                k = *reinterpret_cast<const Unit *>(a.k_pages + from + x);
                v = *reinterpret_cast<const Unit *>(a.v_pages + from + x);
            }
            *reinterpret_cast<Unit *>(a.k + to + u * (long long)sizeof(Unit)) = k;
            *reinterpret_cast<Unit *>(a.v + to + u * (long long)sizeof(Unit)) = v;
        }
    }
}

// The widest unit that all of these are multiples of: 16, 8, 4, 2 bytes or one.
int unit_of(std::initializer_list<long long> bytes) {
    unsigned long long any = 16;
    for (long long b : bytes) any |= (unsigned long long)b;
    return (int)(any & (~any + 1));
}

template <class A>
cudaError_t launch_unit(int unit, void (*k16)(A), void (*k8)(A), void (*k4)(A), void (*k2)(A), unsigned grid, cudaStream_t st, const A &a, void (*k1)(A) = nullptr) {
    return launch_early(unit == 16 ? k16 : unit == 8 ? k8 : unit == 4 ? k4 : unit == 2 ? k2 : k1, grid, kThreads, 0, st, a);
}

}  // namespace

stream_status launch_copy_pages(const CacheGeom &c, int elem, void *k, void *v, const int32_t *pairs, const int32_t *count, int n_pairs, cudaStream_t st) {
    CopyArgs a = {};
    a.base[0] = (char *)k; a.base[1] = (char *)v;
    a.pairs = pairs; a.count = count; a.n_pairs = n_pairs; a.n_pages = c.n_pages; a.n_layers = c.n_layers;
    a.s_l = c.s_l * elem; a.s_p = c.s_p * elem;
    // tokens outside, heads inside, or the other way round: whichever has the smaller stride is inside; what lies side by side is one run
    const bool token_outside = c.s_t >= c.s_h;
    int n_out = token_outside ? c.page : c.G, n_in = token_outside ? c.G : c.page;
    long long s_out = (token_outside ? c.s_t : c.s_h) * elem, s_in = (token_outside ? c.s_h : c.s_t) * elem, run = (long long)c.d * elem;
    if (n_in == 1 || s_in == run) { run *= n_in; n_in = 1; s_in = 0; }
    if (n_in == 1 && (n_out == 1 || s_out == run)) { run *= n_out; n_out = 1; s_out = 0; }
    a.n_outer = n_out; a.n_inner = n_in; a.s_outer = s_out; a.s_inner = s_in;
    const int unit = unit_of({(long long)(uintptr_t)k, (long long)(uintptr_t)v, a.s_l, a.s_p, s_out, s_in, run});
    a.run = (int)(run / unit);
    a.per_page = a.run * n_out * n_in;
    a.pieces = (a.per_page + kThreads * kAhead - 1) / (kThreads * kAhead);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    const long long items = (long long)n_pairs * c.n_layers * 2 * a.pieces, most = (long long)n_sm * kCtas;
    const unsigned grid = (unsigned)(items < most ? items : most);
    const cudaError_t e = n_in == 1 && n_out == 1
        ? launch_unit<CopyArgs>(unit, copy_pages_kernel<uint4, true>, copy_pages_kernel<uint2, true>, copy_pages_kernel<unsigned, true>, copy_pages_kernel<unsigned short, true>, grid, st, a, copy_pages_kernel<unsigned char, true>)
        : launch_unit<CopyArgs>(unit, copy_pages_kernel<uint4, false>, copy_pages_kernel<uint2, false>, copy_pages_kernel<unsigned, false>, copy_pages_kernel<unsigned short, false>, grid, st, a, copy_pages_kernel<unsigned char, false>);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, "cache copy launch");
}

stream_status launch_write(const CacheGeom &c, int elem, const void *k, const void *v, int total, long long s_t, long long s_h,
                           const int32_t *cu_new, const int32_t *done, void *k_pages, void *v_pages, cudaStream_t st) {
    WriteArgs a = {};
    a.c = c; a.k = (const char *)k; a.v = (const char *)v; a.k_pages = (char *)k_pages; a.v_pages = (char *)v_pages;
    a.cu = cu_new; a.done = done; a.total = total; a.elem = elem; a.s_t = s_t * elem; a.s_h = s_h * elem;
    const long long row = (long long)c.d * elem, all = row * c.G;
    const bool side_by_side = c.G == 1 || (s_h == c.d && c.s_h == c.d);
    const int unit = unit_of({(long long)(uintptr_t)k, (long long)(uintptr_t)v, (long long)(uintptr_t)k_pages, (long long)(uintptr_t)v_pages,
                              a.s_t, a.s_h, c.s_p * elem, c.s_t * elem, c.s_h * elem, row});
    a.per_token = (int)(all / unit);
    a.run = side_by_side ? a.per_token : (int)(row / unit);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    const long long blocks = ((long long)total + kThreads / 32 - 1) / (kThreads / 32), most = (long long)n_sm * kCtas;
    const cudaError_t e = launch_unit<WriteArgs>(unit, write_kernel<uint4>, write_kernel<uint2>, write_kernel<unsigned>, write_kernel<unsigned short>,
                                                 (unsigned)(blocks < most ? blocks : most), st, a);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, "cache write launch");
}

stream_status launch_read(const CacheGeom &c, int elem, const void *k_pages, const void *v_pages, const int32_t *cu, int total, void *k_out, void *v_out, cudaStream_t st) {
    ReadArgs a = {};
    a.c = c; a.k_pages = (const char *)k_pages; a.v_pages = (const char *)v_pages; a.k = (char *)k_out; a.v = (char *)v_out;
    a.cu = cu; a.total = total; a.elem = elem;
    const long long row = (long long)c.d * elem, all = row * c.G;
    const int unit = unit_of({(long long)(uintptr_t)k_pages, (long long)(uintptr_t)v_pages, (long long)(uintptr_t)k_out, (long long)(uintptr_t)v_out,
                              c.s_p * elem, c.s_t * elem, c.s_h * elem, row});
    a.per_token = (int)(all / unit);
    a.run = c.G == 1 || c.s_h == c.d ? a.per_token : (int)(row / unit);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    const long long blocks = ((long long)total + kThreads / 32 - 1) / (kThreads / 32), most = (long long)n_sm * kCtas;
    const cudaError_t e = launch_unit<ReadArgs>(unit, read_kernel<uint4>, read_kernel<uint2>, read_kernel<unsigned>, read_kernel<unsigned short>,
                                                (unsigned)(blocks < most ? blocks : most), st, a);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, "cache read launch");
}

}  // namespace stream
