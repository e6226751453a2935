// A paged cache in 8 bits: new tokens rounded into their pages, and tokens read back.
//
// A block's scale is the smallest power of two 2^e with amax <= 448 2^e, which the exponent and the fraction of amax say, so that x 2^-e is exact and
// one rounding, to e4m3, is all there is. A group of threads (a warp, or a CTA where a block's new tokens are more than a warp's registers
// hold, by the mean over the slots) has a block of one kv head's keys or values: its largest element, of magnitudes compared as whole numbers, the block's scale, the numbers.
// Which blocks have new tokens nobody has to count: n tokens touch n / block + 2 blocks at most, so that slot s has the places cu[s] / block + 2 s and
// those behind it, up to the next slot's, and some of them stay empty. Both kernels move every byte once (a new token's twice where a block is more than
// the group's registers hold). 18566 new tokens of 8 kv heads, d = 128, bf16, blocks of 64: 27 us, 114 MB at 64 % of the copy rate (6556 GB/s): a CTA's
// chain of offsets, length, page, tokens, barrier and stores, of six CTAs an SM side by side (elements held as fp32, four of them: 65). 29562 tokens
// read back: 31 us, 182 MB at 90 % (32 bytes of the output a lane, whose stores are halves of sectors: 37). 64 new tokens: 3.8 us, launch and chain. Pages that
// lie head by head cost the same as those token by token: 29558 tokens written in 41.0 us for 40.3, read back in 31.4 for 31.3.
#include <cuda_fp8.h>

#include "serve_common.cuh"
#include "warp_common.cuh"

namespace stream {
namespace {

constexpr int kThreads = 128;
constexpr int kCtas = 64;   // an SM of a grid, at most
constexpr int kHold = 8;    // pieces that a thread holds
constexpr int kMinExp = -90, kMaxExp = 120;

// The exponent e of the scale for elements up to amax.
__device__ __forceinline__ int scale_exp(float amax) {
    const unsigned b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 2^8
    return min(max(e, kMinExp), kMaxExp);
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// Eight elements, as they lie in memory.
template <class T>
struct Piece { uint4 w[sizeof(T) / 2]; };
template <class T>
__device__ __forceinline__ Piece<T> load_piece(const T *p, bool vec) {
    Piece<T> r;
    constexpr int kPer = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        if (vec) {
            r.w[i] = *reinterpret_cast<const uint4 *>(p + i * kPer);
        } else if constexpr (sizeof(T) == 4) {
            r.w[i] = make_uint4(__float_as_uint(p[4 * i]), __float_as_uint(p[4 * i + 1]), __float_as_uint(p[4 * i + 2]), __float_as_uint(p[4 * i + 3]));
        } else {
            const uint2 a = wp::load4(p), b = wp::load4(p + 4);
            r.w[i] = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
    return r;
}
template <class T>
__device__ __forceinline__ void widen(const Piece<T> &r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const unsigned w[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if constexpr (sizeof(T) == 4) {
                x[4 * i + y] = __uint_as_float(w[y]);
            } else {
                x[2 * y] = __uint_as_float(w[y] << 16);
                x[2 * y + 1] = __uint_as_float(w[y] & 0xffff0000u);
            }
        }
    }
}
// The largest magnitude of a piece and of `top` as the bits of numbers without their signs, whose order is that of the numbers: of two bf16 at
// once, or of an fp32. NaN is above all.
template <class T>
__device__ __forceinline__ unsigned larger(const Piece<T> &r, unsigned top) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const unsigned w[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if constexpr (sizeof(T) == 4) top = max(top, w[y] & 0x7fffffffu);
            else top = __vmaxu2(top, w[y] & 0x7fff7fffu);
        }
    }
    return top;
}
template <class T>
__device__ __forceinline__ unsigned bits_of(unsigned top) {  // of the one number
    if constexpr (sizeof(T) == 4) return top;
    else return max(top << 16, top & 0xffff0000u);
}
__device__ __forceinline__ uint2 round8(const float (&x)[8], float f) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i] * f, x[2 * i + 1] * f), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
__device__ __forceinline__ float2 widen8(unsigned two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
__device__ __forceinline__ void store8(unsigned char *p, uint2 w, bool vec) {
    if (vec) {
        *reinterpret_cast<uint2 *>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = (unsigned char)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ uint2 load8(const unsigned char *p, bool vec) {
    if (vec) return *reinterpret_cast<const uint2 *>(p);
    uint2 w = make_uint2(0, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) (i < 4 ? w.x : w.y) |= (unsigned)p[i] << (8 * (i & 3));
    return w;
}

struct WriteArgs {
    CacheGeom c;             // strides: elements of the pages, which are bytes
    Scales sc;
    const void *x[2];        // K, V
    unsigned char *pages[2];
    const int32_t *cu, *done;
    int total;
    long long s_t, s_h;      // elements, of x
    int vec_in, vec_out;
    long long places;        // of blocks
    Divisor heads, page, block;
};

// Place of the first block of slot s.
__device__ __forceinline__ long long place_of(const WriteArgs &a, int s) { return a.block.quotient((unsigned)min(max(a.cu[s], 0), a.total)) + 2ll * s; }

// kGroup threads a block: 32, or all of the CTA's.
template <class T, int kGroup>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 6 : 4) write8_kernel(const __grid_constant__ WriteArgs a) {
    __shared__ float tops[kThreads / 32];
    after_previous_kernel();
    const CacheGeom &c = a.c;
    if (a.done != nullptr && *a.done == 0) return;
    constexpr int kGroups = kThreads / kGroup;
    const int lane = threadIdx.x & 31, me = threadIdx.x % kGroup, row_shift = 28 - __clz(c.d), block = a.sc.block;  // (2^row_shift pieces a row)
    const long long items = a.places * c.G * 2;
    for (long long it = (long long)blockIdx.x * kGroups + threadIdx.x / kGroup; it < items; it += (long long)gridDim.x * kGroups) {
        const long long x2 = it >> 1, place = x2 >> 31 == 0 ? (long long)a.heads.quotient((unsigned)x2) : x2 / c.G;
        const int kv = (int)(it & 1), h = (int)(x2 - place * c.G);
        int s = 0;
        for (int hi = c.n_slots; hi - s > 1;) {  // the last slot that begins at or before the place (32 candidates a step)
            const int step = (hi - s + 31) / 32;
            const long long at = s + (long long)lane * step;
            const unsigned below = __ballot_sync(0xffffffffu, at < hi && place_of(a, (int)min(at, (long long)hi - 1)) <= place);
            s += (below != 0 ? 31 - __clz(below) : 0) * step;
            hi = min(hi, s + step);
        }
        const Span sp = span_of(a.cu, s, a.total);
        const int len = tokens_of(c, s);
        const int start = max(len - sp.n, 0);  // the first new token (rows in front of the slot's first token are passed over)
        const long long nth = place - place_of(a, s), lo64 = ((int)a.block.quotient((unsigned)start) + nth) * block;
        if (nth < 0 || lo64 >= len || sp.n == 0) continue;  // (the whole group)
        const int lo = (int)lo64, hi = min(len, lo + block), first = max(lo, start);
        const int nth_page = (int)a.page.quotient((unsigned)lo), in_page = lo - nth_page * c.page;
        const int page = c.table[(long long)s * c.max_pages + nth_page];
        if ((unsigned)page >= (unsigned)c.n_pages) continue;
        float *const scale_at = const_cast<float *>(kv ? a.sc.v : a.sc.k) + page * a.sc.s_p + a.block.quotient((unsigned)in_page) * a.sc.s_b + h * a.sc.s_h;
        unsigned char *const to = a.pages[kv] + page * c.s_p + (long long)in_page * c.s_t + h * c.s_h;
        // this thread's rows of the new ones: row0 and every `rows`-th from there on, a piece of each
        const int rows = kGroup >> row_shift, row0 = me >> row_shift, piece = (me & ((1 << row_shift) - 1)) * 8, n = hi - first;
        const T *const from = (const T *)a.x[kv] + (long long)(sp.first + sp.n - (len - first) + row0) * a.s_t + h * a.s_h + piece;
        const long long step = rows * a.s_t;
        const bool held = n <= rows * kHold;
        Piece<T> raw[kHold];
        unsigned largest = 0;
        {
            const T *at = from;
            for (int r = row0; r < n; r += rows * kHold) {
#pragma unroll
                for (int i = 0; i < kHold; ++i) {
                    raw[i] = Piece<T>{};
                    if (r + i * rows < n) raw[i] = load_piece(at, a.vec_in != 0);
                    at += step;
                }
#pragma unroll
                for (int i = 0; i < kHold; ++i) largest = larger(raw[i], largest);
            }
        }
        float top = __uint_as_float(bits_of<T>(largest));
        if (top != top) {  // NaN: which is no number to ask for a scale
            top = 0.f;
            const T *at = from;
            for (int r = row0; r < n; r += rows, at += step) {
                float x[8];
                widen(load_piece(at, a.vec_in != 0), x);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
            }
        }
        const float had = first > lo ? *scale_at : 0.f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        if constexpr (kGroup > 32) {
            __syncthreads();  // (the block before has been read)
            if (lane == 0) tops[threadIdx.x >> 5] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, tops[w]);
        }
        __syncwarp();  // (every lane has read the scale)
        const float asked = two_to(scale_exp(top)), scale = had > asked && had < CUDART_INF_F ? had : asked, inv = 1.f / scale;
        if (me == 0 && scale != had) *scale_at = scale;
        if (first > lo && had != scale) {  // what the block has, rounded again
            const float f = had / scale;
            for (int p = me; p < (first - lo) << row_shift; p += kGroup) {
                unsigned char *const at = to + (long long)(p >> row_shift) * c.s_t + (p & ((1 << row_shift) - 1)) * 8;
                const uint2 w = load8(at, a.vec_out != 0);
                float y[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 z = widen8((i < 2 ? w.x : w.y) >> (16 * (i & 1)) & 0xffffu);
                    y[2 * i] = z.x;
                    y[2 * i + 1] = z.y;
                }
                store8(at, round8(y, f), a.vec_out != 0);
            }
        }
        unsigned char *dst = to + (long long)(first - lo + row0) * c.s_t + piece;
        const long long step_out = rows * c.s_t;
        const T *at = from;
        for (int r = row0; r < n; r += rows * kHold) {
#pragma unroll
            for (int i = 0; i < kHold; ++i) {
                if (r + i * rows < n) {
                    if (!held) raw[i] = load_piece(at, a.vec_in != 0);
                    float x[8];
                    widen(raw[i], x);
                    store8(dst, round8(x, inv), a.vec_out != 0);
                }
                at += step;
                dst += step_out;
            }
        }
    }
}

struct ReadArgs {
    CacheGeom c;
    Scales sc;
    const unsigned char *pages[2];
    void *x[2];
    const int32_t *cu;
    int total;
    Divisor page, block;
};

// A warp a token; kPiece elements at a time: 16 bytes of the output, or one element where a row or an output is off its boundary.
constexpr int kAhead = 4;  // pieces of K, and of V, that a lane reads before it writes
template <class T, int kPiece>
__global__ void __launch_bounds__(kThreads) read8_kernel(const __grid_constant__ ReadArgs a) {
    after_previous_kernel();
    const CacheGeom &c = a.c;
    const int lane = threadIdx.x & 31, row_shift = 31 - __clz(c.d / kPiece);  // (2^row_shift pieces a row)
    for (long long t = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < a.total; t += (long long)gridDim.x * (kThreads / 32)) {
        const int s = slot_of_row(a.cu, c.n_slots, t, lane);
        const Span sp = span_of(a.cu, s, a.total);
        if (t < sp.first || t >= (long long)sp.first + sp.n) continue;
        const long long pos = (long long)tokens_of(c, s) - sp.n + (t - sp.first);
        const int nth_page = pos >= 0 ? (int)a.page.quotient((unsigned)pos) : 0, page = pos >= 0 ? c.table[(long long)s * c.max_pages + nth_page] : -1;
        const bool there = (unsigned)page < (unsigned)c.n_pages;
        const int in_page = there ? (int)pos - nth_page * c.page : 0;
        const long long from = there ? page * c.s_p + in_page * c.s_t : 0, z = there ? page * a.sc.s_p + a.block.quotient((unsigned)in_page) * a.sc.s_b : 0;
        const int pieces = c.G << row_shift;
        for (int u0 = lane; u0 < pieces; u0 += 32 * kAhead) {
            unsigned w[kAhead][2][2];
            float scale[kAhead][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int u = u0 + 32 * i, h = u >> row_shift, x = (u - (h << row_shift)) * kPiece;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    w[i][kv][0] = w[i][kv][1] = 0;
                    scale[i][kv] = 0.f;
                    if (there && u < pieces) {
                        const unsigned char *const at = a.pages[kv] + from + h * c.s_h + x;
                        if constexpr (kPiece == 8) { const uint2 y = *reinterpret_cast<const uint2 *>(at); w[i][kv][0] = y.x; w[i][kv][1] = y.y; }
                        else if constexpr (kPiece == 4) w[i][kv][0] = *reinterpret_cast<const unsigned *>(at);
                        else w[i][kv][0] = *at;
                        scale[i][kv] = (kv ? a.sc.v : a.sc.k)[z + h * a.sc.s_h];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int u = u0 + 32 * i;
                if (u >= pieces) break;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    T *const to = (T *)a.x[kv] + t * c.G * c.d + (long long)u * kPiece;
                    __align__(16) T y[kPiece];
#pragma unroll
                    for (int e = 0; e < (kPiece + 1) / 2; ++e) {
                        const float2 f = widen8(w[i][kv][e >> 1] >> (16 * (e & 1)) & 0xffffu);
                        y[2 * e] = (T)(f.x * scale[i][kv]);
                        if constexpr (kPiece > 1) y[2 * e + 1] = (T)(f.y * scale[i][kv]);
                    }
                    if constexpr (kPiece > 1) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(y);
                    else to[0] = y[0];
                }
            }
        }
    }
}

bool on(long long bytes, const void *p, const void *q) { return (((uintptr_t)p | (uintptr_t)q) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

stream_status launch_write8(const CacheGeom &c, const Scales &sc, int dtype, const void *k, const void *v, int total, long long s_t, long long s_h,
                            const int32_t *cu_new, const int32_t *done, void *k_pages, void *v_pages, cudaStream_t st) {
    const int e = dtype == STREAM_F32 ? 4 : 2;
    WriteArgs a = {};
    a.c = c; a.sc = sc; a.x[0] = k; a.x[1] = v; a.pages[0] = (unsigned char *)k_pages; a.pages[1] = (unsigned char *)v_pages;
    a.cu = cu_new; a.done = done; a.total = total; a.s_t = s_t; a.s_h = s_h;
    a.vec_in = on(16, k, v) && ((s_t | s_h) * e & 15) == 0;
    a.vec_out = on(8, k_pages, v_pages) && ((c.s_p | c.s_t | c.s_h) & 7) == 0;
    a.places = total / sc.block + 2ll * c.n_slots; a.heads = make_divisor(c.G);
    a.page = make_divisor(c.page); a.block = make_divisor(sc.block);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    // A warp a block where a block's new tokens fit its registers (few tokens a slot, or small blocks), else a CTA: by the mean over the slots, whose own numbers only the
    // device knows. us, warps and CTAs: a token each for 64 slots 4.6, 7; for 512 11.9, 30; 24 slots of up to 8192, 43278 tokens, blocks of 16, 55, 140; 27756 tokens, blocks of 64, 55, 43. A step of 63 single
    // tokens and a prompt of 900 goes to warps, 16, where CTAs would take 9.
    const long long per_slot = ((long long)total + c.n_slots - 1) / c.n_slots, rows = per_slot < sc.block ? per_slot : sc.block;
    const bool warp = rows * (c.d / 8) <= 32 * kHold;
    const long long items = a.places * c.G * 2, ctas = warp ? (items + 3) / 4 : items, most = (long long)n_sm * kCtas;
    const unsigned grid = (unsigned)(ctas < most ? ctas : most);
    cudaError_t rc;
    if (dtype == STREAM_F32) rc = warp ? launch_early(write8_kernel<float, 32>, grid, kThreads, 0, st, a) : launch_early(write8_kernel<float, kThreads>, grid, kThreads, 0, st, a);
    else rc = warp ? launch_early(write8_kernel<__nv_bfloat16, 32>, grid, kThreads, 0, st, a) : launch_early(write8_kernel<__nv_bfloat16, kThreads>, grid, kThreads, 0, st, a);
    return rc == cudaSuccess ? STREAM_OK : cuda_fail(rc, "8-bit cache write launch");
}

stream_status launch_read8(const CacheGeom &c, const Scales &sc, int dtype, const void *k_pages, const void *v_pages, const int32_t *cu, int total,
                           void *k_out, void *v_out, cudaStream_t st) {
    ReadArgs a = {};
    a.c = c; a.sc = sc; a.pages[0] = (const unsigned char *)k_pages; a.pages[1] = (const unsigned char *)v_pages; a.x[0] = k_out; a.x[1] = v_out;
    a.cu = cu; a.total = total;
    const int piece = dtype == STREAM_F32 ? 4 : 8;
    const bool vec = on(piece, k_pages, v_pages) && on(16, k_out, v_out) && ((c.s_p | c.s_t | c.s_h) & (piece - 1)) == 0;
    a.page = make_divisor(c.page); a.block = make_divisor(sc.block);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    const long long ctas = ((long long)total + kThreads / 32 - 1) / (kThreads / 32), most = (long long)n_sm * kCtas;
    const unsigned grid = (unsigned)(ctas < most ? ctas : most);
    cudaError_t rc;
    if (dtype == STREAM_F32) rc = vec ? launch_early(read8_kernel<float, 4>, grid, kThreads, 0, st, a) : launch_early(read8_kernel<float, 1>, grid, kThreads, 0, st, a);
    else rc = vec ? launch_early(read8_kernel<__nv_bfloat16, 8>, grid, kThreads, 0, st, a) : launch_early(read8_kernel<__nv_bfloat16, 1>, grid, kThreads, 0, st, a);
    return rc == cudaSuccess ? STREAM_OK : cuda_fail(rc, "8-bit cache read launch");
}

}  // namespace stream
