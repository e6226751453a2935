// Attention of one new token of every slot over a paged cache.
//
// The keys of all slots and kv heads are cut into units of 64 and dealt to the CTAs in one long row, slot by slot, head by
// head, as many to each CTA: whatever the slots' lengths, every SM reads as much of the cache as any other, which is all there is to
// be fast at (a key and its value are read once, 4 d FLOP a query head). A CTA walks its stretch segment by segment, a segment
// being what it has of one slot's head, with the running maximum and sum of a softmax. A segment that holds all of its head's keys
// is written out; of the others m, l and O go to the workspace (a CTA has two at most), and a second
// kernel, launched beside the first one's end, joins the pieces of a head in the order of its keys: no atomics, the
// same bits every time. The FMA kernel here, for what decode_warp.cu does not take: fp32, d = 256, nine slots of 2500, 8 heads 216 us (1.70 TB/s); bf16 off 16 bytes, element by
// element, 16 slots of 2000, 32 / 8 heads, d = 128, 394 us (0.33).
#include "decode.cuh"

namespace stream {
namespace {

using namespace decode;

// ----------------------------------------------------------------------------------------------
// fp32 FMA: every type and head dimension
// ----------------------------------------------------------------------------------------------
template <class T, int D>
struct Form {
    static constexpr int kKeys = D <= 64 ? 64 : 4096 / D;        // of a tile: a unit, or a part of one
    static constexpr int kRow = D * (int)sizeof(T) + 16;         // bytes of a row in shared memory
    static constexpr int kSplit = kThreads / kKeys;              // threads that share a key's query heads
    static constexpr int kGroups = D < kThreads ? kThreads / D : 1, kChan = D > kThreads ? D / kThreads : 1;
};
template <class T, int D>
struct Smem {
    using F = Form<T, D>;
    unsigned char k[2][F::kKeys * F::kRow], v[2][F::kKeys * F::kRow];
    float q[kMaxHeads * D];
    float p[kMaxHeads * F::kKeys];
    float m[kMaxHeads], l[kMaxHeads], f[kMaxHeads];
    int page[3][F::kKeys];   // page of every key of a tile, -1: none
};

template <class T>
__device__ __forceinline__ float4 read4(const unsigned char *p) {
    if constexpr (sizeof(T) == 4) {
        return *reinterpret_cast<const float4 *>(p);
    } else {
        const uint2 x = *reinterpret_cast<const uint2 *>(p);
        const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x.y));
        return make_float4(a.x, a.y, b.x, b.y);
    }
}

template <class T, int D, bool W>
__global__ void __launch_bounds__(kThreads) decode_kernel(Args A, int vec) {
    using F = Form<T, D>;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<T, D> &sm = *reinterpret_cast<Smem<T, D> *>(smem_raw);
    const CacheGeom &c = A.a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    after_previous_kernel();
    T *const out = (T *)A.a.out;
    write_empty_slots<T>(A);
    const Share mine = share_of(A, all_places<W>(A, lane), (int)blockIdx.x);
    unsigned bad = 0;
    Place pl = {0, 0, 0};
    int n_parts = 0;
    Left left = {};
    for (Segment sg = open_segment<W>(A, mine.first, mine.end, lane, pl); sg.next >= 0; sg = open_segment<W>(A, sg.next, mine.end, lane, pl)) {
        const int s = sg.slot, nh = sg.heads, h0 = sg.h0, key0 = sg.key0, key_end = sg.key_end;
        const int n_tiles = (key_end - key0 + F::kKeys - 1) / F::kKeys;
        const int32_t *const row = c.table + (long long)s * c.max_pages;
        const Seen seen = seen_of<W, kUnit64>(A.a, s);
        auto page_of = [&](int tile) -> int {  // of this thread's key
            const int walked = key0 + tile * F::kKeys + tid, key = W ? seen.key(walked) : walked;
            if (walked >= key_end || (W && !seen.sees(key))) return -1;
            const int page = row[key / c.page];
            if ((unsigned)page < (unsigned)c.n_pages) return page;
            bad = (unsigned)s + 1u;
            return -1;
        };
        auto fetch = [&](int tile, int buf) {
            constexpr int kPieces = D * (int)sizeof(T) / 16;
            const int *const pages = sm.page[tile % 3];
            for (int i = tid; i < F::kKeys * kPieces; i += kThreads) {
                const int r = i / kPieces, x = i % kPieces, page = pages[r];
                const long long e = (long long)max(page, 0) * c.s_p + (long long)((W ? seen.key(key0 + tile * F::kKeys + r) : key0 + tile * F::kKeys + r) % c.page) * c.s_t + (long long)sg.kvh * c.s_h + x * (16 / (int)sizeof(T));
                const T *const ks = (const T *)A.a.k + e, *const vs = (const T *)A.a.v + e;
                unsigned char *const kd = sm.k[buf] + r * F::kRow + x * 16, *const vd = sm.v[buf] + r * F::kRow + x * 16;
                if (vec) {
                    wp::cp_async16((unsigned)__cvta_generic_to_shared(kd), ks, page >= 0 ? 16 : 0);
                    wp::cp_async16((unsigned)__cvta_generic_to_shared(vd), vs, page >= 0 ? 16 : 0);
                } else {
#pragma unroll
                    for (int y = 0; y < 16 / (int)sizeof(T); ++y) {
                        reinterpret_cast<T *>(kd)[y] = page >= 0 ? ks[y] : (T)0.f;
                        reinterpret_cast<T *>(vd)[y] = page >= 0 ? vs[y] : (T)0.f;
                    }
                }
            }
            wp::cp_async_commit();
        };
        __syncthreads();  // (the segment before has been read)
        if (tid < F::kKeys) {
            sm.page[0][tid] = page_of(0);
            sm.page[1][tid] = n_tiles > 1 ? page_of(1) : -1;
        }
        for (int i = tid; i < nh * D; i += kThreads)
            sm.q[i] = to_float(((const T *)A.a.q)[(long long)s * A.a.qs_s + (long long)(h0 + i / D) * A.a.qs_h + i % D]) * A.a.scale_log2;
        if (tid < kMaxHeads) { sm.m[tid] = -CUDART_INF_F; sm.l[tid] = 0.f; }
        __syncthreads();
        fetch(0, 0);
        constexpr int kHeads = kMaxHeads / F::kGroups;  // of a thread's O
        const int chan = (tid % (D < kThreads ? D : kThreads)) * F::kChan, group = D < kThreads ? tid / D : 0;
        float o[kHeads][F::kChan];
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
#pragma unroll
            for (int x = 0; x < F::kChan; ++x) o[h][x] = 0.f;
        for (int t = 0; t < n_tiles; ++t) {
            int next_page = -1;
            if (t + 2 < n_tiles && tid < F::kKeys) next_page = page_of(t + 2);
            if (t + 1 < n_tiles) {
                fetch(t + 1, (t + 1) & 1);
                wp::cp_async_wait<1>();
            } else {
                wp::cp_async_wait<0>();
            }
            __syncthreads();
            {  // logits: a key and every kSplit-th query head a thread
                const int key = tid / F::kSplit, part = tid % F::kSplit;
                const unsigned char *const kr = sm.k[t & 1] + key * F::kRow;
                constexpr int kMine = (kMaxHeads + F::kSplit - 1) / F::kSplit;
                float acc[kMine];
#pragma unroll
                for (int i = 0; i < kMine; ++i) acc[i] = 0.f;
#pragma unroll 4
                for (int x = 0; x < D; x += 4) {
                    const float4 b = read4<T>(kr + x * (int)sizeof(T));
#pragma unroll
                    for (int i = 0; i < kMine; ++i)
                        if (i * F::kSplit + part < nh) {
                            const float4 a = *reinterpret_cast<const float4 *>(&sm.q[(i * F::kSplit + part) * D + x]);
                            acc[i] = fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, acc[i]))));
                        }
                }
                const bool there = sm.page[t % 3][key] >= 0;
#pragma unroll
                for (int i = 0; i < kMine; ++i)
                    if (i * F::kSplit + part < nh) sm.p[(i * F::kSplit + part) * F::kKeys + key] = there ? acc[i] : -CUDART_INF_F;
            }
            __syncthreads();
            for (int h = warp; h < nh; h += kThreads / 32) {
                float x[(F::kKeys + 31) / 32], mx = sm.m[h];
                const float was = mx;
#pragma unroll
                for (int i = 0; i < (F::kKeys + 31) / 32; ++i) {
                    x[i] = lane + 32 * i < F::kKeys ? sm.p[h * F::kKeys + lane + 32 * i] : -CUDART_INF_F;
                    mx = fmaxf(mx, x[i]);
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                const float base = mx == -CUDART_INF_F ? 0.f : mx;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < (F::kKeys + 31) / 32; ++i) {
                    const float p = fast_exp2(x[i] - base);
                    sum += p;
                    if (lane + 32 * i < F::kKeys) sm.p[h * F::kKeys + lane + 32 * i] = p;
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane == 0) {
                    const float f = fast_exp2(was - base);
                    sm.m[h] = mx;
                    sm.f[h] = f;
                    sm.l[h] = sm.l[h] * f + sum;
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kHeads; ++i) {
                const int h = i * F::kGroups + group;
                if (h < nh) {
                    const float f = sm.f[h];
#pragma unroll
                    for (int x = 0; x < F::kChan; ++x) o[i][x] *= f;
                }
            }
            for (int j = 0; j < F::kKeys; j += 4) {
                float w[4][F::kChan];
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int x = 0; x < F::kChan; ++x) w[y][x] = to_float(reinterpret_cast<const T *>(sm.v[t & 1] + (j + y) * F::kRow)[chan + x]);
#pragma unroll
                for (int i = 0; i < kHeads; ++i) {
                    const int h = i * F::kGroups + group;
                    if (h < nh) {
                        const float4 p = *reinterpret_cast<const float4 *>(&sm.p[h * F::kKeys + j]);
#pragma unroll
                        for (int x = 0; x < F::kChan; ++x) o[i][x] = fmaf(p.w, w[3][x], fmaf(p.z, w[2][x], fmaf(p.y, w[1][x], fmaf(p.x, w[0][x], o[i][x]))));
                    }
                }
            }
            if (tid < F::kKeys) sm.page[(t + 2) % 3][tid] = next_page;
            __syncthreads();  // (the buffers and the pages of the tile after next)
        }
        float *const part = part_of(A, (int)blockIdx.x, n_parts);
        if (!sg.whole) {
            if (sg.key0 == 0) left = {pieces_of(sg.owner_end, mine), n_parts, sg.heads, 0u, (long long)sg.slot * A.a.H + sg.h0, 0ll};
            ++n_parts;
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            const int h = i * F::kGroups + group;
            if (h < nh) {
                const float l = sm.l[h], inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
                for (int x = 0; x < F::kChan; ++x) {
                    if (sg.whole) out[((long long)s * A.a.H + h0 + h) * D + chan + x] = (T)(o[i][x] * inv);
                    else part[2 * kMaxHeads + h * D + chan + x] = o[i][x];
                }
            }
        }
        if (tid < nh) {
            if (!sg.whole) { part[tid] = sm.m[tid]; part[kMaxHeads + tid] = sm.l[tid]; }
            else if (A.a.lse != nullptr) A.a.lse[(long long)s * A.a.H + h0 + tid] = lse_of(sm.m[tid], sm.l[tid]);
        }
    }
    leave_to_joins(A, left, bad);
}

// ----------------------------------------------------------------------------------------------
// The pieces of an owner joined, a query head a CTA: column c of the grid has what CTA c of the first kernel left. One more column
// writes the header. A thread has four channels of every n-th piece, so that the pieces of a long slot (up to all CTAs' of the first
// kernel: one slot, one head, 32954 keys, 258 pieces) are read 16 to 64 side by side. Its time is that of loads that wait for
// one another (what is left; m, l and the first of O), and of its launch.
// ----------------------------------------------------------------------------------------------
constexpr int kJoinThreads = 256;
template <class T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Args A) {
    const int tid = threadIdx.x, lane = tid & 31, h = blockIdx.y, d = A.a.c.d;
    __shared__ unsigned any;
    __shared__ float f[kMaxGrid];
    __shared__ float wm[kJoinThreads / 32], wl[kJoinThreads / 32];
    __shared__ float4 sums[kJoinThreads];
    if (tid == 0) any = 0;
    after_previous_kernel();
    if ((int)blockIdx.x == A.grid) {
        if (h != 0) return;
        __syncthreads();
        for (int i = tid; i < A.grid; i += kJoinThreads)
            if (A.left[i].bad != 0) atomicMax(&any, A.left[i].bad);
        for (int i = tid; i < (int)sizeof(WorkspaceHeader) / 4; i += kJoinThreads) reinterpret_cast<unsigned *>(A.header)[i] = 0;
        __syncthreads();
        if (tid == 0) {
            A.header->rows = (unsigned long long)A.a.c.n_slots * A.a.H;
            if (any != 0) { A.header->error = 701; A.header->error_info = any - 1; }
        }
        return;
    }
    const Left left = A.left[blockIdx.x];
    if (h >= left.heads || left.n == 0) return;
    const int n = left.n, quads = d / 4, groups = kJoinThreads / quads, group = tid / quads, at = (tid - group * quads) * 4;
    auto piece = [&](int x) { return part_of(A, (int)blockIdx.x + x, x == 0 ? left.which : 0); };
    auto o_of = [&](int x) { return *reinterpret_cast<const float4 *>(piece(x) + 2 * kMaxHeads + h * d + at); };
    constexpr int kFirst = 4;
    float4 first[kFirst];  // of O, before its weights are known
    float ls[2] = {0.f, 0.f}, m = -CUDART_INF_F;
    static_assert(kMaxGrid <= 2 * kJoinThreads, "two pieces' m and l a thread");
#pragma unroll
    for (int i = 0; i < kFirst; ++i) first[i] = group + i * groups < n ? o_of(group + i * groups) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int x = tid + i * kJoinThreads;
        if (x < n) {
            m = fmaxf(m, f[x] = piece(x)[h]);
            ls[i] = piece(x)[kMaxHeads + h];
        }
    }
    m = warp_maximum(m);
    if (lane == 0) wm[tid >> 5] = m;
    __syncthreads();
    m = wm[0];
#pragma unroll
    for (int i = 1; i < kJoinThreads / 32; ++i) m = fmaxf(m, wm[i]);
    const float base = m == -CUDART_INF_F ? 0.f : m;
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int x = tid + i * kJoinThreads;
        if (x < n) {
            f[x] = fast_exp2(f[x] - base);
            l = fmaf(f[x], ls[i], l);
        }
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    if (lane == 0) wl[tid >> 5] = l;
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float w, const float4 &y) { o.x = fmaf(w, y.x, o.x); o.y = fmaf(w, y.y, o.y); o.z = fmaf(w, y.z, o.z); o.w = fmaf(w, y.w, o.w); };
#pragma unroll
    for (int i = 0; i < kFirst; ++i)
        if (group + i * groups < n) add(f[group + i * groups], first[i]);
#pragma unroll 4
    for (int x = group + kFirst * groups; x < n; x += groups) add(f[x], o_of(x));
    sums[tid] = o;
    __syncthreads();
    if (group > 0) return;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinThreads / 32; ++i) l += wl[i];
    for (int i = 1; i < groups && i < n; ++i) add(1.f, sums[i * quads + tid]);
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const long long to = left.to + h;
    T *const out = (T *)A.a.out + to * d + at;
    out[0] = (T)(o.x * inv); out[1] = (T)(o.y * inv); out[2] = (T)(o.z * inv); out[3] = (T)(o.w * inv);
    if (A.a.lse != nullptr && tid == 0) A.a.lse[to] = lse_of(m, l);
}

template <class T, int D, bool W>
cudaError_t launch_fma(const Args &A, int vec, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<T, D>);
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(decode_kernel<T, D, W>, smem, done);
    if (e != cudaSuccess) return e;
    return launch_early(decode_kernel<T, D, W>, (unsigned)A.grid, kThreads, smem, st, A, vec);
}
template <class T, bool W>
cudaError_t launch_fma_d(const Args &A, int vec, cudaStream_t st) {
    switch (A.a.c.d) {
        case 16: return launch_fma<T, 16, W>(A, vec, st);
        case 32: return launch_fma<T, 32, W>(A, vec, st);
        case 64: return launch_fma<T, 64, W>(A, vec, st);
        case 128: return launch_fma<T, 128, W>(A, vec, st);
        default: return launch_fma<T, 256, W>(A, vec, st);
    }
}
template <bool W>
cudaError_t launch_keys(Args &A, int dtype, int n_sm, cudaStream_t st) {
    const int e = dtype == STREAM_F32 ? 4 : 2;
    const DecodeCall &a = A.a;
    const long long any = (long long)(uintptr_t)a.k | (long long)(uintptr_t)a.v | a.c.s_p * e | a.c.s_t * e | a.c.s_h * e;
    const int vec = any % 16 == 0 ? 1 : 0;
    if (warp_supported(a, dtype)) return launch_warp(A, dtype, n_sm, st);
    return dtype == STREAM_F32 ? launch_fma_d<float, W>(A, vec, st) : launch_fma_d<__nv_bfloat16, W>(A, vec, st);
}

constexpr size_t kLeftBytes = (kMaxGrid * sizeof(Left) + 255) & ~(size_t)255;

}  // namespace

namespace decode {

Args args_of(const DecodeCall &a, void *workspace, int n_sm, int unit, int open, int least) {
    Args A;
    A.a = a;
    A.chunks = (a.hpg + kMaxHeads - 1) / kMaxHeads;
    A.per_slot = a.c.G * A.chunks;
    A.header = (WorkspaceHeader *)workspace;
    A.left = (Left *)((char *)workspace + sizeof(WorkspaceHeader));
    A.parts = (float *)((char *)A.left + kLeftBytes);
    long long keys = (long long)a.c.max_pages * a.c.page;  // of a slot, at most
    if (a.window > 0) keys = std::min(keys, (long long)a.window + a.sinks + 2 * (unit - 1));
    const long long most = (long long)a.c.n_slots * A.per_slot * ((keys + unit - 1) / unit + open), ctas = (most + least - 1) / least;
    const int want = 2 * n_sm < kMaxGrid ? 2 * n_sm : kMaxGrid;
    A.grid = (int)(ctas < want ? ctas : want);
    return A;
}

cudaError_t launch_joins(const Args &A, int dtype, cudaStream_t st) {
    const dim3 joins(A.grid + 1, A.a.hpg < kMaxHeads ? A.a.hpg : kMaxHeads);
    return dtype == STREAM_F32 ? launch_early(join_kernel<float>, joins, kJoinThreads, 0, st, A) : launch_early(join_kernel<__nv_bfloat16>, joins, kJoinThreads, 0, st, A);
}

}  // namespace decode

size_t decode_workspace_bytes(const CacheGeom &c) {
    return sizeof(WorkspaceHeader) + kLeftBytes + (size_t)kMaxGrid * 2 * kMaxHeads * (c.d + 2) * sizeof(float);
}

stream_status launch_decode(const DecodeCall &a, int dtype, void *workspace, cudaStream_t st) {
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    Args A = args_of(a, workspace, n_sm);
    cudaError_t rc = a.window > 0 ? launch_keys<true>(A, dtype, n_sm, st) : launch_keys<false>(A, dtype, n_sm, st);
    if (rc != cudaSuccess) return cuda_fail(rc, "decode attention launch");
    rc = launch_joins(A, dtype, st);
    return rc == cudaSuccess ? STREAM_OK : cuda_fail(rc, "decode join launch");
}

}  // namespace stream
