// Dense attention of packed prompts in fp32 on the tensor cores: every operand as the sum of two tf32 numbers.
//
// x = hi + lo, hi the nearest tf32 (11 significant bits), lo the rest, of which the tensor core takes 11 bits: a b = hi hi + hi lo + lo hi leaves
// out 2^-24 of a product and rounds the parts at 2^-22, no worse than what fp32 sums of some hundred terms lose. The products add
// up in fp32, 16 channels or keys in the tensor core, whose sums are cut instead of rounded, and those parts by ordinary additions (all in
// the tensor core: 1.6e-6 off, relative, at 2048 keys; so: 2.7e-7; fp32 FMA: 3.6e-7). Three mma.sync m16n8k8 instead of 1024 FMA in each of 32 lanes: what bounds it is issue slots, a quarter of the FMA kernel's.
//
// A CTA has 64 rows (token, query head) of one kv head, a warp 16, and walks the keys in tiles that come by cp.async, two of K and
// two of V. Neither contraction cares for the order of its terms nor the product with V for that of its columns, so that fragments are
// 16-byte reads: lane (g, t) of Q K^T reads four consecutive channels of a key for two k steps; a key pair 2 t, 2 t + 1 of P V is where
// the logits' accumulators have it; column p of product j is channel 4 p + j of 32, so that a lane ends up with eight consecutive ones.
// `ref` is moved only when a logit has outgrown it by 2^30. Where the row tiles are fewer than the SMs, a cluster of up to eight
// CTAs has the tile: each walks every n-th key tile, and their m, l and O meet through shared memory, in a fixed order.
// With a window (W) the sinks' tiles are walked, and behind a gap those from the first key on that the tile's first row sees (one head of 2048 tokens, d = 64,
// window 256: 13.7 us, for 26.1 without one).
#include "serve_common.cuh"
#include "warp_common.cuh"

namespace stream {
namespace {

constexpr int kThreads = 128, kRows = 64;
constexpr float kOutgrown = 30.f;  // log2

template <int D>
struct Form {
    // Of a tile: half the code of 64 (the first pass through it, from cold instruction caches, takes 5 us). us with 64 and with 32, d = 64: one head of
    // 2048 tokens 27.0, 26.6; 25 prompts of up to 45, 16 heads, 20.0, 16.4; eight heads of 8192 1314, 1350. d = 128: eight heads of 4096 1062, 744 (with 64 the
    // registers do not do; with 32 eight bytes are spilled). Two CTAs an SM.
    static constexpr int kKeys = D >= 64 ? 32 : 64;
    static constexpr int kRow = D + 16;               // floats of a row of Q and K: eight lanes, two rows of four pieces, touch every bank
    static constexpr int kVRow = D + 4;               // of V: four pairs of rows, two pieces
};
template <int D>
struct Smem {
    using F = Form<D>;
    float q[kRows * F::kRow];                         // in the end O
    float k[2][F::kKeys * F::kRow], v[2][F::kKeys * F::kVRow];
    float m[kRows], l[kRows];
};

__device__ __forceinline__ void mma_tf32(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void split(float x, unsigned &hi, unsigned &lo) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(x));
    lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ void product(float (&c)[4], const unsigned (&ah)[4], const unsigned (&al)[4], unsigned bh0, unsigned bl0, unsigned bh1, unsigned bl1) {
    mma_tf32(c, al, bh0, bh1);  // (the small parts first)
    mma_tf32(c, ah, bl0, bl1);
    mma_tf32(c, ah, bh0, bh1);
}

template <int D, bool W>
__global__ void __launch_bounds__(kThreads, 2) prompt_f32_kernel(const __grid_constant__ PromptGeom g, const float *q, const float *k, const float *v) {
    using F = Form<D>;
    constexpr int kKeys = F::kKeys, kTiles = kKeys / 8, kPieces = D / 4;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<D> &sm = *reinterpret_cast<Smem<D> *>(smem_raw);
    const unsigned ctas = wp::cluster_size(), rank = wp::cluster_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2, t = lane & 3;
    if (ctas == 1) after_previous_kernel();
    const unsigned tile = blockIdx.x / ctas;
    const int kvh = (int)(tile % (unsigned)g.G);
    const RowTile rt = row_tile(g, (int)(tile / (unsigned)g.G), kRows, lane);
    if (rt.seq < 0) return;  // (the whole cluster)
    const Span sq = span_of(g.cu_q, rt.seq, g.total_q), sk = span_of(g.cu_k, rt.seq, g.total_k);
    const long long all_rows = (long long)sq.n * g.hpg, row_base = (all_rows - 1) / kRows * kRows - (long long)rt.nth * kRows;  // late tokens first
    const int n_rows = (int)min(all_rows - row_base, (long long)kRows);
    const int tok_base = (int)(row_base / g.hpg), head_base = (int)(row_base - (long long)tok_base * g.hpg);
    auto token_of = [&](int r) { return tok_base + (head_base + r) / g.hpg; };
    auto head_of = [&](int r) { return kvh * g.hpg + (head_base + r) % g.hpg; };
    auto keys_of = [&](int r) -> int {  // keys that row r of the tile sees (rows behind the last see what it does)
        return g.causal ? min(sk.n, max(0, token_of(min(r, n_rows - 1)) + sk.n - sq.n + 1)) : sk.n;
    };
    Walked wk = {};
    if constexpr (W) wk = walked_keys(g, kKeys, tok_base + (sk.n - sq.n), sk.n);
    const int most = keys_of(n_rows - 1), walked = most - wk.gap, warp_most = keys_of(warp * 16 + 15), warp_least = keys_of(warp * 16);
    const int see[2] = {keys_of(warp * 16 + quad), keys_of(warp * 16 + quad + 8)};
    const float *const ks = k + (long long)sk.first * g.ks_t + (long long)kvh * g.ks_h;
    const float *const vs = v + (long long)sk.first * g.ks_t + (long long)kvh * g.ks_h;
    const unsigned q_s = wp::smem_addr(sm.q), k_s = wp::smem_addr(sm.k[0]), v_s = wp::smem_addr(sm.v[0]);
    auto fetch = [&](int j, int buf) {
        if (j < walked) {
            const int j0 = W ? wk.key(j) : j;
            for (int i = tid; i < kKeys * kPieces; i += kThreads) {
                const int r = i / kPieces, x = i % kPieces, key = j0 + r;
                const bool there = key < sk.n;
                const long long e = (there ? key * g.ks_t : 0) + x * 4;
                wp::cp_async16(k_s + (unsigned)((buf * kKeys + r) * F::kRow + x * 4) * 4u, ks + e, there ? 16 : 0);
                wp::cp_async16(v_s + (unsigned)((buf * kKeys + r) * F::kVRow + x * 4) * 4u, vs + e, there ? 16 : 0);
            }
        }
        wp::cp_async_commit();
    };
    for (int i = tid; i < kRows * kPieces; i += kThreads) {
        const int r = i / kPieces, x = i % kPieces;
        const bool there = r < n_rows;
        const long long e = there ? (long long)(sq.first + token_of(r)) * g.qs_t + (long long)head_of(r) * g.qs_h : 0;
        wp::cp_async16(q_s + (unsigned)(r * F::kRow + x * 4) * 4u, q + e + x * 4, there ? 16 : 0);
    }
    const int first = (int)rank * kKeys, stride = (int)ctas * kKeys;
    fetch(first, 0);  // (Q is in its group)
    float o[D / 8][4];
#pragma unroll
    for (int x = 0; x < D / 8; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
    float ref[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};  // of rows quad and quad + 8, in units of log2
    int low[2] = {0, 0};  // the first keys of their windows
    if constexpr (W) {
#pragma unroll
        for (int r = 0; r < 2; ++r) low[r] = window_begin(g, token_of(min(warp * 16 + quad + 8 * r, n_rows - 1)) + (sk.n - sq.n));
    }
    for (int jw = first, buf = 0; jw < walked; jw += stride, buf ^= 1) {
        const int j = W ? wk.key(jw) : jw;
        fetch(jw + stride, buf ^ 1);
        wp::cp_async_wait<1>();
        __syncthreads();
        if (j < warp_most) {
            const float *const kt = sm.k[buf] + quad * F::kRow + t * 4, *const vt = sm.v[buf] + 2 * t * F::kVRow + quad * 4;
            const float *const qt = sm.q + (warp * 16 + quad) * F::kRow + t * 4;
            float sc[kTiles][4];
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int y = 0; y < 4; ++y) sc[n][y] = 0.f;
#pragma unroll 4
            for (int c = 0; c < D / 16; ++c) {  // 16 channels: two steps of the contraction
                const float4 x0 = *reinterpret_cast<const float4 *>(qt + c * 16), x1 = *reinterpret_cast<const float4 *>(qt + 8 * F::kRow + c * 16);
                unsigned ah[2][4], al[2][4];
                split(x0.x, ah[0][0], al[0][0]); split(x1.x, ah[0][1], al[0][1]); split(x0.y, ah[0][2], al[0][2]); split(x1.y, ah[0][3], al[0][3]);
                split(x0.z, ah[1][0], al[1][0]); split(x1.z, ah[1][1], al[1][1]); split(x0.w, ah[1][2], al[1][2]); split(x1.w, ah[1][3], al[1][3]);
#pragma unroll
                for (int n = 0; n < kTiles; ++n) {
                    const float4 y = *reinterpret_cast<const float4 *>(kt + n * 8 * F::kRow + c * 16);
                    unsigned bh[4], bl[4];
                    split(y.x, bh[0], bl[0]); split(y.y, bh[1], bl[1]); split(y.z, bh[2], bl[2]); split(y.w, bh[3], bl[3]);
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
                    product(part, ah[0], al[0], bh[0], bl[0], bh[1], bl[1]);
                    product(part, ah[1], al[1], bh[2], bl[2], bh[3], bl[3]);
#pragma unroll
                    for (int y2 = 0; y2 < 4; ++y2) sc[n][y2] += part[y2];
                }
            }
            const bool hidden = j + kKeys > warp_least;
            bool outgrown = false;
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    sc[n][y] *= g.scale_log2;
                    const int key = j + n * 8 + t * 2 + (y & 1);
                    if (hidden && key >= see[y >> 1]) sc[n][y] = -CUDART_INF_F;
                    if (W && key < low[y >> 1] && key >= g.sinks) sc[n][y] = -CUDART_INF_F;
                    outgrown = outgrown || sc[n][y] - ref[y >> 1] > kOutgrown;  // (the first: infinity)
                }
            if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float mx = -CUDART_INF_F;
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) mx = fmaxf(mx, fmaxf(sc[n][2 * r], sc[n][2 * r + 1]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const float now = fmaxf(ref[r], mx), f = now == -CUDART_INF_F ? 1.f : fast_exp2(ref[r] - now);
                    ref[r] = now;
                    l[r] *= f;
#pragma unroll
                    for (int x = 0; x < D / 8; ++x) { o[x][2 * r] *= f; o[x][2 * r + 1] *= f; }
                }
            }
            const float base[2] = {ref[0] == -CUDART_INF_F ? 0.f : ref[0], ref[1] == -CUDART_INF_F ? 0.f : ref[1]};
#pragma unroll
            for (int n2 = 0; n2 < kTiles; n2 += 2) {  // 16 keys
                unsigned ph[2][4], pl[2][4];  // k index t: key 2 t, index t + 4: key 2 t + 1
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float(&x)[4] = sc[n2 + i];
                    const float p0 = fast_exp2(x[0] - base[0]), p1 = fast_exp2(x[1] - base[0]), p2 = fast_exp2(x[2] - base[1]), p3 = fast_exp2(x[3] - base[1]);
                    l[0] += p0 + p1;
                    l[1] += p2 + p3;
                    split(p0, ph[i][0], pl[i][0]); split(p2, ph[i][1], pl[i][1]); split(p1, ph[i][2], pl[i][2]); split(p3, ph[i][3], pl[i][3]);
                }
                // columns: kWide products share a lane's reads, column p of the x-th of them being channel kWide p + x
                constexpr int kWide = D >= 32 ? 4 : 2;
                const float *const vn = vt + n2 * 8 * F::kVRow - (4 - kWide) * quad;
#pragma unroll
                for (int c = 0; c < D / (8 * kWide); ++c) {
                    __align__(16) float y[2][2][kWide];  // [8 keys][key of the pair]
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float *const at = vn + (i * 8 + e) * F::kVRow + c * 32;
                            if constexpr (kWide == 4) *reinterpret_cast<float4 *>(y[i][e]) = *reinterpret_cast<const float4 *>(at);
                            else *reinterpret_cast<float2 *>(y[i][e]) = *reinterpret_cast<const float2 *>(at);
                        }
#pragma unroll
                    for (int x = 0; x < kWide; ++x) {
                        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            unsigned bh[2], bl[2];
                            split(y[i][0][x], bh[0], bl[0]); split(y[i][1][x], bh[1], bl[1]);
                            product(part, ph[i], pl[i], bh[0], bl[0], bh[1], bl[1]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[kWide * c + x][e] += part[e];
                    }
                }
            }
        }
        __syncthreads();  // (the buffers of the tile after next)
    }
    wp::cp_async_wait<0>();
    __syncthreads();
    // O over Q: not divided where others have a part of it
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        const int row = warp * 16 + quad + 8 * r;
        const float f = ctas > 1 ? 1.f : l[r] > 0.f ? 1.f / l[r] : 0.f;
        float *const to = sm.q + row * F::kRow;
        if constexpr (D >= 32) {
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    *reinterpret_cast<float4 *>(to + c * 32 + t * 8 + p * 4) =
                        make_float4(o[4 * c][2 * r + p] * f, o[4 * c + 1][2 * r + p] * f, o[4 * c + 2][2 * r + p] * f, o[4 * c + 3][2 * r + p] * f);
        } else {
            *reinterpret_cast<float4 *>(to + t * 4) = make_float4(o[0][2 * r] * f, o[1][2 * r] * f, o[0][2 * r + 1] * f, o[1][2 * r + 1] * f);
        }
        if (t == 0) { sm.m[row] = ref[r]; sm.l[row] = l[r]; }
    }
    float *const out = (float *)g.out;
    if (ctas == 1) {
        __syncwarp();
        for (int i = lane; i < 16 * kPieces; i += 32) {
            const int r = warp * 16 + i / kPieces, x = i % kPieces;
            if (r < n_rows)
                *reinterpret_cast<float4 *>(out + ((long long)(sq.first + token_of(r)) * g.H + head_of(r)) * D + x * 4) = *reinterpret_cast<const float4 *>(sm.q + r * F::kRow + x * 4);
        }
        const int r = warp * 16 + lane;
        if (g.lse != nullptr && lane < 16 && r < n_rows)
            g.lse[(long long)head_of(r) * g.total_q + sq.first + token_of(r)] = sm.l[r] > 0.f ? (sm.m[r] + log2f(sm.l[r])) * kLn2 : -CUDART_INF_F;
        return;
    }
    wp::cluster_arrive();
    wp::cluster_wait();
    // the rows are dealt to the CTAs, four channels of a row to a thread
    for (int i = tid; ; i += kThreads) {
        const int r = (int)rank + (int)ctas * (i / kPieces), x = (i % kPieces) * 4;
        if (r >= n_rows) break;
        float ms[8], mx = -CUDART_INF_F, sum = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            ms[c] = c < (int)ctas ? wp::load_in_cluster(&sm.m[r], (unsigned)c) : -CUDART_INF_F;
            mx = fmaxf(mx, ms[c]);
        }
        const float base = mx == -CUDART_INF_F ? 0.f : mx;
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c < (int)ctas) {
                const float f = fast_exp2(ms[c] - base);
                const float4 y = wp::load4_in_cluster(sm.q + r * F::kRow + x, (unsigned)c);
                sum = fmaf(f, wp::load_in_cluster(&sm.l[r], (unsigned)c), sum);
                w.x = fmaf(f, y.x, w.x); w.y = fmaf(f, y.y, w.y); w.z = fmaf(f, y.z, w.z); w.w = fmaf(f, y.w, w.w);
            }
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        const long long tok = sq.first + token_of(r);
        const int h = head_of(r);
        *reinterpret_cast<float4 *>(out + (tok * g.H + h) * D + x) = make_float4(w.x * inv, w.y * inv, w.z * inv, w.w * inv);
        if (g.lse != nullptr && x == 0) g.lse[(long long)h * g.total_q + tok] = sum > 0.f ? (mx + log2f(sum)) * kLn2 : -CUDART_INF_F;
    }
    wp::cluster_arrive();
    wp::cluster_wait();  // (nobody leaves while its shared memory is read)
}

template <int D, bool W>
stream_status launch_form(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<D>);
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(prompt_f32_kernel<D, W>, smem, done);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(prompt_f32)");
    const long long tiles = most_row_tiles(g, kRows);
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    // several CTAs a tile where one each leaves SMs without, as long as there are keys for all
    unsigned cluster = 1;
    while (cluster < 8 && tiles * cluster <= n_sm && (long long)g.total_k > (long long)cluster * Form<D>::kKeys) cluster *= 2;
    if (tiles * cluster > 0x7fffffffLL) { set_error("too many rows for one launch"); return STREAM_ERR_UNSUPPORTED; }
    if (cluster == 1) e = launch_early(prompt_f32_kernel<D, W>, (unsigned)tiles, kThreads, smem, st, g, (const float *)q, (const float *)k, (const float *)v);
    else e = launch_clusters(prompt_f32_kernel<D, W>, (unsigned)tiles * cluster, kThreads, smem, st, cluster, g, (const float *)q, (const float *)k, (const float *)v);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, "prompt_f32 launch");
}

template <int D>
stream_status launch(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    return g.window > 0 ? launch_form<D, true>(g, q, k, v, st) : launch_form<D, false>(g, q, k, v, st);
}

}  // namespace

bool prompt_f32_supported(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v) {
    if (dtype != STREAM_F32 || g.d > 128 || g.total_k > 0x7fff0000) return false;  // (a tile's end is counted in 32 bits)
    return (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)g.out) & 15) == 0 && ((g.qs_t | g.qs_h | g.ks_t | g.ks_h) & 3) == 0;
}

stream_status launch_prompt_f32(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    switch (g.d) {
        case 16: return launch<16>(g, q, k, v, st);
        case 32: return launch<32>(g, q, k, v, st);
        case 64: return launch<64>(g, q, k, v, st);
        default: return launch<128>(g, q, k, v, st);
    }
}

}  // namespace stream
