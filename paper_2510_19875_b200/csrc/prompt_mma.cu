// Dense attention of packed prompts on mma.sync: bf16 in the head dimensions and head groups that the tcgen05 kernel does not take.
//
// A CTA has 128 rows (token, query head of the group), a warp 16 of them: the heads of a group share every key tile. Tiles of 64 keys
// come by cp.async, two of K and two of V in shared memory (rows padded by 16 bytes: eight of them touch every bank), zeros behind a
// sequence's last key. A warp's logits stay in registers, turn into bf16 weights 2^(scale (s - ref)) there and are the A operand
// of the product with V as they lie. `ref` is a row's maximum at its first tile, moved (O and the sum with it) only when a logit has
// outgrown it by 2^30; the sum is that of the unrounded weights. Late tokens, with the most keys, come first. Bound by the
// latency of dependent steps at eight to sixteen warps an SM: 32 / 8 heads, 4096 tokens, d = 256 920 us (299 TFLOP/s), d = 32 175 us (196); 597 tokens, d = 256, 46.5 us
// (126: 152 CTAs for 148 SMs).
// With a window (W) the sinks' tiles are walked, and behind a gap those from the first key on that the tile's first row sees.
#include "serve_common.cuh"
#include "warp_common.cuh"

namespace stream {
namespace {

constexpr int kThreads = 256, kRows = 128, kKeys = 64;
constexpr float kOutgrown = 30.f;  // log2

template <int D>
struct Form {
    static constexpr int kRow = D * 2 + 16;                     // bytes
    static constexpr bool kQInRegs = D <= 128;
    static constexpr int kCtas = D <= 32 ? 2 : 1;
};
template <int D>
struct Smem {
    unsigned char q[kRows * Form<D>::kRow];
    unsigned char k[2][kKeys * Form<D>::kRow], v[2][kKeys * Form<D>::kRow];
};

template <int D, bool W>
__global__ void __launch_bounds__(kThreads, Form<D>::kCtas) prompt_mma_kernel(const __grid_constant__ PromptGeom g, const __nv_bfloat16 *q,
                                                                             const __nv_bfloat16 *k, const __nv_bfloat16 *v) {
    using F = Form<D>;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<D> &sm = *reinterpret_cast<Smem<D> *>(smem_raw);
    constexpr int kPieces = D / 8;  // of 16 bytes, of a row
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2;
    after_previous_kernel();
    const int kvh = (int)(blockIdx.x % (unsigned)g.G), nth = (int)(blockIdx.x / (unsigned)g.G);
    const RowTile rt = row_tile(g, nth, kRows, lane);
    if (rt.seq < 0) return;
    const Span sq = span_of(g.cu_q, rt.seq, g.total_q), sk = span_of(g.cu_k, rt.seq, g.total_k);
    const long long all_rows = (long long)sq.n * g.hpg, row_base = (all_rows - 1) / kRows * kRows - (long long)rt.nth * kRows;
    const int n_rows = (int)min(all_rows - row_base, (long long)kRows);
    auto keys_of = [&](int r) -> int {  // keys that row r of the tile sees (rows behind the last see what it does)
        if (!g.causal) return sk.n;
        const int tok = (int)((row_base + min(r, n_rows - 1)) / g.hpg);
        return min(sk.n, max(0, tok + sk.n - sq.n + 1));
    };
    Walked wk = {};
    if constexpr (W) wk = walked_keys(g, kKeys, (int)(row_base / g.hpg) + (sk.n - sq.n), sk.n);
    const int most = keys_of(n_rows - 1), walked = most - wk.gap, warp_most = keys_of(warp * 16 + 15);
    const __nv_bfloat16 *const qs = q + (long long)sq.first * g.qs_t + (long long)kvh * g.hpg * g.qs_h;
    const __nv_bfloat16 *const ks = k + (long long)sk.first * g.ks_t + (long long)kvh * g.ks_h;
    const __nv_bfloat16 *const vs = v + (long long)sk.first * g.ks_t + (long long)kvh * g.ks_h;
    const unsigned q_s = wp::smem_addr(sm.q), k_s = wp::smem_addr(sm.k[0]), v_s = wp::smem_addr(sm.v[0]);
    auto fetch = [&](int j, int buf) {
        if (j < walked) {
            const int j0 = W ? wk.key(j) : j;
            for (int i = tid; i < kKeys * kPieces; i += kThreads) {
                const int r = i / kPieces, x = i % kPieces, key = j0 + r;
                const bool there = key < sk.n;
                const long long e = (there ? key * g.ks_t : 0) + x * 8;
                const unsigned to = (unsigned)(buf * kKeys * F::kRow + r * F::kRow + x * 16);
                wp::cp_async16(k_s + to, ks + e, there ? 16 : 0);
                wp::cp_async16(v_s + to, vs + e, there ? 16 : 0);
            }
        }
        wp::cp_async_commit();
    };
    for (int i = tid; i < kRows * kPieces; i += kThreads) {
        const int r = i / kPieces, x = i % kPieces;
        const long long row = row_base + r;
        const bool there = r < n_rows;
        wp::cp_async16(q_s + (unsigned)(r * F::kRow + x * 16), qs + (there ? (row / g.hpg) * g.qs_t + (row % g.hpg) * g.qs_h : 0) + x * 8, there ? 16 : 0);
    }
    fetch(0, 0);  // (Q is in its group)
    const unsigned q_addr = q_s + (unsigned)((warp * 16 + (lane & 15)) * F::kRow + (lane >> 4) * 16);
    const unsigned k_lane = (unsigned)(((lane >> 4) * 8 + (lane & 7)) * F::kRow + ((lane >> 3) & 1) * 16);
    const unsigned v_lane = (unsigned)((((lane >> 3) & 1) * 8 + (lane & 7)) * F::kRow + (lane >> 4) * 16);
    unsigned qa[F::kQInRegs ? D / 16 : 1][4];
    float o[D / 8][4];
#pragma unroll
    for (int x = 0; x < D / 8; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
    float ref[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};  // of rows quad and quad + 8, in units of log2
    const int see[2] = {keys_of(warp * 16 + quad), keys_of(warp * 16 + quad + 8)};
    const int warp_least = keys_of(warp * 16);
    int low[2] = {0, 0};  // the first keys of their windows
    if constexpr (W) {
#pragma unroll
        for (int r = 0; r < 2; ++r) low[r] = window_begin(g, (int)((row_base + min(warp * 16 + quad + 8 * r, n_rows - 1)) / g.hpg) + (sk.n - sq.n));
    }
    for (int jw = 0, buf = 0; jw < walked; jw += kKeys, buf ^= 1) {
        const int j = W ? wk.key(jw) : jw;
        fetch(jw + kKeys, buf ^ 1);
        wp::cp_async_wait<1>();
        __syncthreads();
        if (F::kQInRegs && jw == 0) {
#pragma unroll
            for (int x = 0; x < D / 16; ++x) wp::ldmatrix4(q_addr + x * 32, qa[F::kQInRegs ? x : 0]);
        }
        if (j < warp_most) {
            const unsigned kt = k_s + (unsigned)(buf * kKeys * F::kRow) + k_lane, vt = v_s + (unsigned)(buf * kKeys * F::kRow) + v_lane;
            float sc[8][4];
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int y = 0; y < 4; ++y) sc[n][y] = 0.f;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) {
                unsigned a[4];
                if constexpr (F::kQInRegs) {
#pragma unroll
                    for (int y = 0; y < 4; ++y) a[y] = qa[x][y];
                } else {
                    wp::ldmatrix4(q_addr + x * 32, a);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    unsigned b[4];
                    wp::ldmatrix4(kt + (unsigned)(n * 16 * F::kRow) + x * 32, b);
                    wp::mma_bf16(sc[2 * n], a[0], a[1], a[2], a[3], b[0], b[1]);
                    wp::mma_bf16(sc[2 * n + 1], a[0], a[1], a[2], a[3], b[2], b[3]);
                }
            }
            const bool hidden = j + kKeys > warp_least;
            bool outgrown = false;
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    sc[n][y] *= g.scale_log2;
                    const int key = j + n * 8 + (lane & 3) * 2 + (y & 1);
                    if (hidden && key >= see[y >> 1]) sc[n][y] = -CUDART_INF_F;
                    if (W && key < low[y >> 1] && key >= g.sinks) sc[n][y] = -CUDART_INF_F;
                    outgrown = outgrown || sc[n][y] - ref[y >> 1] > kOutgrown;  // (the first: infinity)
                }
            if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float mx = -CUDART_INF_F;
#pragma unroll
                    for (int n = 0; n < 8; ++n) mx = fmaxf(mx, fmaxf(sc[n][2 * r], sc[n][2 * r + 1]));
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
            for (int n = 0; n < 4; ++n) {
                unsigned pa[4];
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float p0 = fast_exp2(sc[2 * n + half][2 * r] - base[r]), p1 = fast_exp2(sc[2 * n + half][2 * r + 1] - base[r]);
                        l[r] += p0 + p1;
                        const __nv_bfloat162 pk = __floats2bfloat162_rn(p0, p1);
                        pa[2 * half + r] = *reinterpret_cast<const unsigned *>(&pk);
                    }
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    unsigned b[4];
                    wp::ldmatrix4_t(vt + (unsigned)(n * 16 * F::kRow) + x * 32, b);
                    wp::mma_bf16(o[2 * x], pa[0], pa[1], pa[2], pa[3], b[0], b[1]);
                    wp::mma_bf16(o[2 * x + 1], pa[0], pa[1], pa[2], pa[3], b[2], b[3]);
                }
            }
        }
        __syncthreads();  // (the buffers of the tile after next)
    }
    wp::cp_async_wait<0>();
    // The output over the warp's own rows of Q, and from there in pieces of 16 bytes. Those rows came by copies of other warps' threads, which no
    // barrier has waited for where no row of the tile sees a key (the loop did not run).
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        const float inv = l[r] > 0.f ? 1.f / l[r] : 0.f;
#pragma unroll
        for (int x = 0; x < D / 8; ++x) {
            const __nv_bfloat162 pk = __floats2bfloat162_rn(o[x][2 * r] * inv, o[x][2 * r + 1] * inv);
            *reinterpret_cast<__nv_bfloat162 *>(sm.q + (warp * 16 + quad + 8 * r) * F::kRow + x * 16 + (lane & 3) * 4) = pk;
        }
        const int row = warp * 16 + quad + 8 * r;
        if (g.lse != nullptr && (lane & 3) == 0 && row < n_rows) {
            const long long at = row_base + row;
            g.lse[(long long)(kvh * g.hpg + (int)(at % g.hpg)) * g.total_q + sq.first + at / g.hpg] = l[r] > 0.f ? (ref[r] + log2f(l[r])) * kLn2 : -CUDART_INF_F;
        }
    }
    __syncwarp();
    for (int i = lane; i < 16 * kPieces; i += 32) {
        const int r = warp * 16 + i / kPieces, x = i % kPieces;
        if (r < n_rows) {
            const long long at = row_base + r, to = ((sq.first + at / g.hpg) * g.H + kvh * g.hpg + at % g.hpg) * D + x * 8;
            *reinterpret_cast<uint4 *>((__nv_bfloat16 *)g.out + to) = *reinterpret_cast<const uint4 *>(sm.q + r * F::kRow + x * 16);
        }
    }
}

template <int D, bool W>
stream_status launch_form(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<D>);
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(prompt_mma_kernel<D, W>, smem, done);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(prompt_mma)");
    const long long tiles = most_row_tiles(g, kRows);
    if (tiles > 0x7fffffffLL) { set_error("too many rows for one launch"); return STREAM_ERR_UNSUPPORTED; }
    e = launch_early(prompt_mma_kernel<D, W>, (unsigned)tiles, kThreads, smem, st, g, (const __nv_bfloat16 *)q, (const __nv_bfloat16 *)k, (const __nv_bfloat16 *)v);
    return e == cudaSuccess ? STREAM_OK : cuda_fail(e, "prompt_mma launch");
}

template <int D>
stream_status launch(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    return g.window > 0 ? launch_form<D, true>(g, q, k, v, st) : launch_form<D, false>(g, q, k, v, st);
}

}  // namespace

bool prompt_mma_supported(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v) {
    if (dtype != STREAM_BF16) return false;
    return (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)g.out) & 15) == 0 && ((g.qs_t | g.qs_h | g.ks_t | g.ks_h) & 7) == 0;
}

stream_status launch_prompt_mma(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    switch (g.d) {
        case 16: return launch<16>(g, q, k, v, st);
        case 32: return launch<32>(g, q, k, v, st);
        case 64: return launch<64>(g, q, k, v, st);
        case 128: return launch<128>(g, q, k, v, st);
        default: return launch<256>(g, q, k, v, st);
    }
}

}  // namespace stream
