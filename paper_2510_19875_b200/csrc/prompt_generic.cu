// Dense attention of packed prompts on fp32 FMA: fp32 with d = 256, and rows of either type that do not lie on 16 bytes.
//
// A CTA has 64 rows (token, query head) of one kv head, so that the query heads of a group share every key tile, and
// walks the keys in tiles of 64 with the running maximum and sum of a softmax:
//     m' = max(m, max_j s_j),   l' = l 2^(m - m') + sum_j 2^(s_j - m'),   O' = O 2^(m - m') + sum_j 2^(s_j - m') v_j,
// logits in units of log2. A thread holds 4 x 4 logits and 4 rows x d / 16 channels of O. Where the row tiles are fewer than
// the SMs, a cluster of up to eight CTAs has the tile: each walks every n-th key tile, and their m, l and O meet
// through shared memory, in a fixed order, every CTA joining its share of the rows. 2048 tokens: fp32, 8 heads, d = 256 498 us (34.5 TFLOP/s); off 16 bytes, 8 heads of fp32,
// d = 64, 253 us (17.0), 32 / 8 heads of bf16, d = 128, 1298 us (26.5).
#include "serve_common.cuh"
#include "warp_common.cuh"

namespace stream {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64, kKeys = 64;

template <int D>
struct Smem {
    static constexpr int kPad = D + 4;        // (16-byte reads of eight rows side by side touch every bank once)
    static constexpr int kBufs = D <= 128 ? 2 : 1;  // key tiles in shared memory
    float q[kRows * kPad];
    float k[kBufs][kKeys * kPad];
    float v[kBufs][kKeys * D];
    float p[kRows * (kKeys + 4)];
    float m[kRows], l[kRows];
};

// Four channels of a row.
template <class T>
__device__ __forceinline__ float4 load4(const T *p, bool vec) {
    if constexpr (sizeof(T) == 4) {
        if (vec) return *reinterpret_cast<const float4 *>(p);
        return make_float4(p[0], p[1], p[2], p[3]);
    } else {
        if (vec) {
            const uint2 x = *reinterpret_cast<const uint2 *>(p);
            const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x.y));
            return make_float4(a.x, a.y, b.x, b.y);
        }
        return make_float4(to_float(p[0]), to_float(p[1]), to_float(p[2]), to_float(p[3]));
    }
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads) prompt_kernel(PromptGeom g, const T *q, const T *k, const T *v, int vec) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<D> &sm = *reinterpret_cast<Smem<D> *>(smem_raw);
    constexpr int kPad = Smem<D>::kPad, kCols = D >= 64 ? 4 : D / 16;  // channels side by side of a thread's O, in D / (16 * kCols) places
    constexpr int kParts = D / (16 * kCols);
    const unsigned ctas = wp::cluster_size(), rank = wp::cluster_rank();
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31;
    if (ctas == 1) after_previous_kernel();
    // which rows: kv head fastest, then the sequences' row tiles one after the other
    const int tile = (int)(blockIdx.x / ctas), kvh = tile % g.G, nth = tile / g.G;
    const RowTile rt = row_tile(g, nth, kRows, lane);
    if (rt.seq < 0) return;  // (the whole cluster)
    const int seq = rt.seq;
    const Span sq = span_of(g.cu_q, seq, g.total_q), sk = span_of(g.cu_k, seq, g.total_k);
    const long long row_base = ((long long)sq.n * g.hpg - 1) / kRows * kRows - (long long)rt.nth * kRows;  // late tokens, with the most keys, first  // (a sequence's rows may be more than 32 bits count)
    const int n_rows = (int)min((long long)sq.n * g.hpg - row_base, (long long)kRows);
    const int shift = sk.n - sq.n;  // query i sees the keys up to i + shift
    auto keys_of = [&](int r) -> int {  // keys that row r of the tile sees
        if (r >= n_rows) return 0;
        if (!g.causal) return sk.n;
        const int tok = (int)((row_base + r) / g.hpg);
        return min(sk.n, max(0, tok + shift + 1));
    };
    const int most = keys_of(n_rows - 1);
    const T *const qs = q + (long long)sq.first * g.qs_t + (long long)kvh * g.hpg * g.qs_h;
    const T *const ks = k + (long long)sk.first * g.ks_t + (long long)kvh * g.ks_h;
    const T *const vs = v + (long long)sk.first * g.ks_t + (long long)kvh * g.ks_h;
    for (int i = tid; i < kRows * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = (i % (D / 4)) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < n_rows) {
            const long long row = row_base + r;
            x = load4(qs + (row / g.hpg) * g.qs_t + (row % g.hpg) * g.qs_h + c, vec);
        }
        *reinterpret_cast<float4 *>(&sm.q[r * kPad + c]) = make_float4(x.x * g.scale_log2, x.y * g.scale_log2, x.z * g.scale_log2, x.w * g.scale_log2);
    }
    float m[4], l[4], o[4][kParts * kCols];
    int see[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -CUDART_INF_F;
        l[i] = 0.f;
        see[i] = keys_of(ty * 4 + i);
#pragma unroll
        for (int c = 0; c < kParts * kCols; ++c) o[i][c] = 0.f;
    }
    constexpr int kBufs = Smem<D>::kBufs;
    const long long step = (long long)ctas * kKeys;
    auto fetch = [&](long long j0, int buf) {
        if (j0 < most) {
            for (int i = tid; i < kKeys * (D / 4); i += kThreads) {
                const int r = i / (D / 4), c = (i % (D / 4)) * 4;
                const long long key = j0 + r;
                const bool there = key < sk.n;
                const T *const kp = ks + (there ? key * g.ks_t : 0) + c, *const vp = vs + (there ? key * g.ks_t : 0) + c;
                float *const kd = &sm.k[buf][r * kPad + c], *const vd = &sm.v[buf][r * D + c];
                if (sizeof(T) == 4 && vec) {
                    wp::cp_async16(wp::smem_addr(kd), kp, there ? 16 : 0);
                    wp::cp_async16(wp::smem_addr(vd), vp, there ? 16 : 0);
                } else {
                    *reinterpret_cast<float4 *>(kd) = there ? load4(kp, vec) : make_float4(0.f, 0.f, 0.f, 0.f);
                    *reinterpret_cast<float4 *>(vd) = there ? load4(vp, vec) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
        }
        wp::cp_async_commit();
    };
    const long long j_first = (long long)rank * kKeys;
    if (kBufs == 2) fetch(j_first, 0);
    int buf = 0;
    for (long long j0 = j_first; j0 < most; j0 += step, buf ^= kBufs - 1) {
        if (kBufs == 2) {
            fetch(j0 + step, buf ^ 1);
            wp::cp_async_wait<1>();
        } else {
            __syncthreads();
            fetch(j0, 0);
            wp::cp_async_wait<0>();
        }
        __syncthreads();
        float s[4][4];  // rows ty * 4 + i, keys tx + 16 * j
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
            float4 a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4 *>(&sm.q[(ty * 4 + i) * kPad + c]);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4 *>(&sm.k[buf][(tx + 16 * j) * kPad + c]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = fmaf(a[i].w, b[j].w, fmaf(a[i].z, b[j].z, fmaf(a[i].y, b[j].y, fmaf(a[i].x, b[j].x, s[i][j]))));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mx = -CUDART_INF_F;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j0 + tx + 16 * j >= see[i]) s[i][j] = -CUDART_INF_F;
                mx = fmaxf(mx, s[i][j]);
            }
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            const float now = fmaxf(m[i], mx), base = now == -CUDART_INF_F ? 0.f : now, f = fast_exp2(m[i] - base);
            m[i] = now;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = fast_exp2(s[i][j] - base);
                sum += p;
                sm.p[(ty * 4 + i) * (kKeys + 4) + tx + 16 * j] = p;
            }
            l[i] = l[i] * f + sum;  // (this thread's keys; the threads of a row have one m, and add up at the end)
#pragma unroll
            for (int c = 0; c < kParts * kCols; ++c) o[i][c] *= f;
        }
        __syncwarp();  // (a row's weights come from 16 lanes of one warp)
#pragma unroll 2
        for (int j = 0; j < kKeys; j += 4) {
            float4 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4 *>(&sm.p[(ty * 4 + i) * (kKeys + 4) + j]);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                float w[kParts * kCols];
#pragma unroll
                for (int part = 0; part < kParts; ++part) {
                    const float *at = &sm.v[buf][(j + x) * D + part * 64 + tx * kCols];
                    if constexpr (kCols == 4) {
                        const float4 y = *reinterpret_cast<const float4 *>(at);
                        w[part * 4] = y.x; w[part * 4 + 1] = y.y; w[part * 4 + 2] = y.z; w[part * 4 + 3] = y.w;
                    } else {
#pragma unroll
                        for (int c = 0; c < kCols; ++c) w[part * kCols + c] = at[c];
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = x == 0 ? p[i].x : x == 1 ? p[i].y : x == 2 ? p[i].z : p[i].w;
#pragma unroll
                    for (int c = 0; c < kParts * kCols; ++c) o[i][c] = fmaf(f, w[c], o[i][c]);
                }
            }
        }
        if (kBufs == 2) __syncthreads();  // (the buffer of the tile after next)
    }
    wp::cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
    if (ctas > 1) {
        // every CTA leaves its m, l and O (over its key tiles, no longer needed); the rows are then dealt out to the CTAs
        __syncthreads();
        float *const acc = sm.k[0];  // [kRows][D]
        if (tx == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { sm.m[ty * 4 + i] = m[i]; sm.l[ty * 4 + i] = l[i]; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int c = 0; c < kCols; ++c) acc[(ty * 4 + i) * D + part * 64 + tx * kCols + c] = o[i][part * kCols + c];
        wp::cluster_arrive();
        wp::cluster_wait();
        for (int r = (int)rank + (int)ctas * ty; r < n_rows; r += (int)ctas * 16) {  // a row per 16 threads and step
            float mx = -CUDART_INF_F;
            for (unsigned x = 0; x < ctas; ++x) mx = fmaxf(mx, wp::load_in_cluster(&sm.m[r], x));
            const float base = mx == -CUDART_INF_F ? 0.f : mx;
            float sum = 0.f, w[kParts * kCols];
#pragma unroll
            for (int c = 0; c < kParts * kCols; ++c) w[c] = 0.f;
            for (unsigned x = 0; x < ctas; ++x) {
                const float f = fast_exp2(wp::load_in_cluster(&sm.m[r], x) - base);
                sum = fmaf(f, wp::load_in_cluster(&sm.l[r], x), sum);
#pragma unroll
                for (int part = 0; part < kParts; ++part)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) w[part * kCols + c] = fmaf(f, wp::load_in_cluster(&acc[r * D + part * 64 + tx * kCols + c], x), w[part * kCols + c]);
            }
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const long long row = row_base + r, tok = sq.first + row / g.hpg;
            const int h = kvh * g.hpg + (int)(row % g.hpg);
            T *const to = (T *)g.out + (tok * g.H + h) * D;
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int c = 0; c < kCols; ++c) to[part * 64 + tx * kCols + c] = (T)(w[part * kCols + c] * inv);
            if (g.lse != nullptr && tx == 0) g.lse[(long long)h * g.total_q + tok] = sum > 0.f ? (mx + log2f(sum)) * kLn2 : -CUDART_INF_F;
        }
        wp::cluster_arrive();
        wp::cluster_wait();  // (nobody leaves while its shared memory is read)
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty * 4 + i;
        if (r >= n_rows) continue;
        const long long row = row_base + r, tok = sq.first + row / g.hpg;
        const int h = kvh * g.hpg + (int)(row % g.hpg);
        const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
        T *const to = (T *)g.out + (tok * g.H + h) * D;
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int c = 0; c < kCols; ++c) to[part * 64 + tx * kCols + c] = (T)(o[i][part * kCols + c] * inv);
        if (g.lse != nullptr && tx == 0) g.lse[(long long)h * g.total_q + tok] = l[i] > 0.f ? (m[i] + log2f(l[i])) * kLn2 : -CUDART_INF_F;
    }
}

template <class T, int D>
stream_status launch(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<D>);
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(prompt_kernel<T, D>, smem, done);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(prompt)");
    const long long tiles = most_row_tiles(g, kRows);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    // several CTAs a tile where one each leaves SMs without, as long as there are keys for all
    unsigned cluster = 1;
    while (cluster < 8 && tiles * cluster <= n_sm && (long long)g.total_k > (long long)cluster * kKeys) cluster *= 2;
    if (tiles * cluster > 0x7fffffffLL) { set_error("too many rows for one launch"); return STREAM_ERR_UNSUPPORTED; }
    const long long any = (long long)(uintptr_t)q | (long long)(uintptr_t)k | (long long)(uintptr_t)v;
    const long long strides = g.qs_t | g.qs_h | g.ks_t | g.ks_h;
    const int vec = any % (4 * (int)sizeof(T)) == 0 && strides % 4 == 0 ? 1 : 0;
    if (cluster == 1) e = launch_early(prompt_kernel<T, D>, (unsigned)tiles, kThreads, smem, st, g, (const T *)q, (const T *)k, (const T *)v, vec);
    else e = launch_clusters(prompt_kernel<T, D>, (unsigned)tiles * cluster, kThreads, smem, st, cluster, g, (const T *)q, (const T *)k, (const T *)v, vec);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, "prompt attention launch");
}

template <class T>
stream_status launch_d(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    switch (g.d) {
        case 16: return launch<T, 16>(g, q, k, v, st);
        case 32: return launch<T, 32>(g, q, k, v, st);
        case 64: return launch<T, 64>(g, q, k, v, st);
        case 128: return launch<T, 128>(g, q, k, v, st);
        default: return launch<T, 256>(g, q, k, v, st);
    }
}

}  // namespace

stream_status launch_prompt_generic(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v, cudaStream_t st) {
    return dtype == STREAM_F32 ? launch_d<float>(g, q, k, v, st) : launch_d<__nv_bfloat16>(g, q, k, v, st);
}

}  // namespace stream
