// Attention of one new token of every slot over a paged cache.
//
// The keys of all slots and kv heads are cut into units of 64 and dealt to the CTAs in one long row, slot by slot, head by
// head, as many to each CTA: whatever the slots' lengths, every SM reads as much of the cache as any other, which is all there is to
// be fast at (a key and its value are read once, 4 d FLOP a query head). A CTA walks its stretch segment by segment, a segment
// being what it has of one slot's head, with the running maximum and sum of a softmax. A segment that holds all of its head's keys
// is written out; of the others m, l and O go to the workspace (a CTA has two at most, its first and its last), and a second
// kernel, launched beside the first one's end, joins the pieces of a head in the order of its keys: no atomics, the
// same bits every time.
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

template <class T, int D>
__global__ void __launch_bounds__(kThreads) decode_kernel(Args A, int vec) {
    using F = Form<T, D>;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<T, D> &sm = *reinterpret_cast<Smem<T, D> *>(smem_raw);
    const CacheGeom &c = A.a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    after_previous_kernel();
    T *const out = (T *)A.a.out;
    write_empty_slots<T>(A);
    const Share mine = share_of(A, all_units(c, lane) * A.per_slot, (int)blockIdx.x);
    unsigned bad = 0;
    Place at = {0, 0, 0};
    for (long long u = mine.first; u < mine.end;) {
        at = place_of(c, A.per_slot, u, lane, at);
        const Segment sg = segment_of(A, at, u, mine.end);
        const int s = at.slot, nh = sg.heads, h0 = sg.h0, key0 = sg.key0, key_end = sg.key_end;
        const int n_tiles = (key_end - key0 + F::kKeys - 1) / F::kKeys;
        const int32_t *const row = c.table + (long long)s * c.max_pages;
        auto page_of = [&](int tile) -> int {  // of this thread's key
            const int key = key0 + tile * F::kKeys + tid;
            if (key >= key_end) return -1;
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
                const long long e = (long long)max(page, 0) * c.s_p + (long long)((key0 + tile * F::kKeys + r) % c.page) * c.s_t + (long long)sg.kvh * c.s_h + x * (16 / (int)sizeof(T));
                const T *const ks = (const T *)A.a.k + e, *const vs = (const T *)A.a.v + e;
                unsigned char *const kd = sm.k[buf] + r * F::kRow + x * 16, *const vd = sm.v[buf] + r * F::kRow + x * 16;
                if (vec) {
                    cp_async16((unsigned)__cvta_generic_to_shared(kd), ks, page >= 0);
                    cp_async16((unsigned)__cvta_generic_to_shared(vd), vs, page >= 0);
                } else {
#pragma unroll
                    for (int y = 0; y < 16 / (int)sizeof(T); ++y) {
                        reinterpret_cast<T *>(kd)[y] = page >= 0 ? ks[y] : (T)0.f;
                        reinterpret_cast<T *>(vd)[y] = page >= 0 ? vs[y] : (T)0.f;
                    }
                }
            }
            cp_commit();
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
                cp_wait<1>();
            } else {
                cp_wait<0>();
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
        float *const part = part_of(A, (int)blockIdx.x, u == mine.first ? 0 : 1);
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
            else if (A.a.lse != nullptr) A.a.lse[(long long)s * A.a.H + h0 + tid] = sm.l[tid] > 0.f ? (sm.m[tid] + log2f(sm.l[tid])) * kLn2 : -CUDART_INF_F;
        }
        u += sg.units;
    }
    record_bad(A, bad);
}

// ----------------------------------------------------------------------------------------------
// The pieces of a head joined. CTA c stands for the border between the shares c and c + 1: the first border within an
// owner's units has the join of all of them. One more CTA writes the header.
// ----------------------------------------------------------------------------------------------
template <class T>
__global__ void __launch_bounds__(kThreads) join_kernel(Args A) {
    const CacheGeom &c = A.a.c;
    const int tid = threadIdx.x, lane = tid & 31;
    after_previous_kernel();
    if ((int)blockIdx.x == A.grid - 1) {
        __shared__ unsigned any;
        if (tid == 0) any = 0;
        __syncthreads();
        for (int i = tid; i < A.grid; i += kThreads)
            if (A.bad[i] != 0) atomicMax(&any, A.bad[i]);
        for (int i = tid; i < (int)sizeof(WorkspaceHeader) / 4; i += kThreads) reinterpret_cast<unsigned *>(A.header)[i] = 0;
        __syncthreads();
        if (tid == 0) {
            A.header->rows = (unsigned long long)c.n_slots * A.a.H;
            if (any != 0) { A.header->error = 701; A.header->error_info = any - 1; }
        }
        return;
    }
    const long long all = all_units(c, lane) * A.per_slot;
    const Share left = share_of(A, all, (int)blockIdx.x);
    const long long border = left.end;
    if (border >= all || left.first >= border) return;
    const Place at = place_of(c, A.per_slot, border, lane, {0, 0, 0});
    const int owner = (int)((border - at.first) / at.units);
    const long long first = at.first + (long long)owner * at.units, end = first + at.units;
    if (border == first || left.first > first) return;  // (no owner is cut here, or not for the first time)
    const int cta0 = (int)blockIdx.x, cta1 = (int)((end - 1) / left.per);  // all that have some of it
    const int s = at.slot, kvh = owner / A.chunks, h0 = kvh * A.a.hpg + owner % A.chunks * kMaxHeads;
    const int nh = min(kMaxHeads, A.a.hpg - owner % A.chunks * kMaxHeads), d = c.d;
    auto piece = [&](int x) { return part_of(A, x, x == cta0 && left.first != first ? 1 : 0); };
    T *const out = (T *)A.a.out;
    for (int i = tid; i < nh * d; i += kThreads) {
        const int h = i / d;
        float m = -CUDART_INF_F, l = 0.f, o = 0.f;
        for (int x = cta0; x <= cta1; ++x) m = fmaxf(m, piece(x)[h]);
        const float base = m == -CUDART_INF_F ? 0.f : m;
        for (int x = cta0; x <= cta1; ++x) {
            const float *const p = piece(x);
            const float f = fast_exp2(p[h] - base);
            l = fmaf(f, p[kMaxHeads + h], l);
            o = fmaf(f, p[2 * kMaxHeads + i], o);
        }
        out[((long long)s * A.a.H + h0) * d + i] = (T)(l > 0.f ? o / l : 0.f);
        if (A.a.lse != nullptr && i % d == 0) A.a.lse[(long long)s * A.a.H + h0 + h] = l > 0.f ? (m + log2f(l)) * kLn2 : -CUDART_INF_F;
    }
}

template <class T, int D>
cudaError_t launch_fma(const Args &A, int vec, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<T, D>);
    cudaError_t e = cudaFuncSetAttribute(decode_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_early(decode_kernel<T, D>, (unsigned)A.grid, kThreads, smem, st, A, vec);
}
template <class T>
cudaError_t launch_fma_d(const Args &A, int vec, cudaStream_t st) {
    switch (A.a.c.d) {
        case 16: return launch_fma<T, 16>(A, vec, st);
        case 32: return launch_fma<T, 32>(A, vec, st);
        case 64: return launch_fma<T, 64>(A, vec, st);
        case 128: return launch_fma<T, 128>(A, vec, st);
        default: return launch_fma<T, 256>(A, vec, st);
    }
}

constexpr size_t kFlagBytes = (kMaxGrid * sizeof(unsigned) + 255) & ~(size_t)255;

}  // namespace

size_t decode_workspace_bytes(const CacheGeom &c) {
    return sizeof(WorkspaceHeader) + kFlagBytes + (size_t)kMaxGrid * 2 * kMaxHeads * (c.d + 2) * sizeof(float);
}

stream_status launch_decode(const DecodeCall &a, int dtype, void *workspace, cudaStream_t st) {
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    const int e = dtype == STREAM_F32 ? 4 : 2;
    Args A;
    A.a = a;
    A.chunks = (a.hpg + kMaxHeads - 1) / kMaxHeads;
    A.per_slot = a.c.G * A.chunks;
    A.header = (WorkspaceHeader *)workspace;
    A.bad = (unsigned *)((char *)workspace + sizeof(WorkspaceHeader));
    A.parts = (float *)((char *)A.bad + kFlagBytes);
    const long long most = (long long)a.c.n_slots * A.per_slot * (((long long)a.c.max_pages * a.c.page + kUnit - 1) / kUnit);
    const int want = 2 * n_sm < kMaxGrid ? 2 * n_sm : kMaxGrid;
    A.grid = (int)(most < want ? most : want);
    const long long any = (long long)(uintptr_t)a.k | (long long)(uintptr_t)a.v | a.c.s_p * e | a.c.s_t * e | a.c.s_h * e;
    const int vec = any % 16 == 0 ? 1 : 0;
    cudaError_t rc = mma_supported(a, dtype) ? launch_mma(A, n_sm, st)
                     : dtype == STREAM_F32   ? launch_fma_d<float>(A, vec, st)
                                             : launch_fma_d<__nv_bfloat16>(A, vec, st);
    if (rc != cudaSuccess) return cuda_fail(rc, "decode attention launch");
    rc = dtype == STREAM_F32 ? launch_early(join_kernel<float>, (unsigned)A.grid, kThreads, 0, st, A)
                             : launch_early(join_kernel<__nv_bfloat16>, (unsigned)A.grid, kThreads, 0, st, A);
    return rc == cudaSuccess ? STREAM_OK : cuda_fail(rc, "decode join launch");
}

}  // namespace stream
