// Decode attention whose warps work alone: rows of 16-byte pieces, up to 512 bytes; bf16 on mma.sync, fp32 on FMA.
//
// The up to 16 query heads of a segment meet a key together, so that it and its value are read from shared memory once for all of
// them. (It is the cache that has to be read: 4 d FLOP a head and 4 d bytes a key in bf16; tcgen05's tiles of 64 or 128
// rows would be empty but for these heads, m16n8k16 has 16 rows.) The four warps of a CTA take 16 keys each in turn and know nothing of one
// another until the segment's end: a warp has its own ring of K and V tiles, filled by cp.async, its own softmax reference and sums
// (ref is moved only when a logit has outgrown it by 2^30: fp32 sums and bf16 weights keep their relative precision), and its own O in
// registers; at the end the four meet in shared memory. Before a segment is written out the next one's first tiles
// are on their way. Keys behind the slot's last one, or without a page, are zeros there.
//   bf16  the heads are the rows of the products; weights are rounded to bf16 (2^-8 of each at most), their sum is not
//   fp32  a logit's channels are halved between two lanes; O is dealt to the lanes by channels, and the weights come from shared memory
// Measured against the copy rate (6567 GB/s), joins and launches included, 32 / 8 heads, d = 128, bf16: 93 % (four slots of up to 131072 tokens, 546 MB in 89 us),
// 97 % (four slots, two of them of some 130000, 1077 MB in 169); the rest is the way to the first tile and the joins.
#include "decode.cuh"

namespace stream {
namespace {

using namespace decode;

constexpr float kOutgrown = 30.f;  // log2
constexpr int kStep = 16;          // keys of a warp's tile

template <class T, int D>
struct Form {
    static constexpr bool kMma = sizeof(T) == 2;
    static constexpr int kRow = D * (int)sizeof(T);            // bytes
    static constexpr int kPieces = kRow / 16;                  // of a row
    static constexpr int kTile = kStep * kRow;
    static constexpr int kStages = kRow <= 128 ? 4 : 3;        // steps in the ring (their keys' flags fit 64 bits)
    static constexpr int kWarp = kStages * 2 * kTile;          // bytes of a warp's ring
    static constexpr bool kQInRegs = kMma && D <= 128;
    static constexpr int kCtas = kRow <= 256 ? 2 : 1;          // of an SM
    static constexpr int kVec = 16 / (int)sizeof(T);           // elements of a piece
    static constexpr int kChan = D >= 32 ? D / 32 : 1;         // fp32: channels of O a lane
    static_assert(kMaxHeads * D * 4 <= 2 * kTile && kStages <= 4, "O in the place of a step");
    static_assert(kPieces <= 32 && kPieces >= 2, "a row is fetched by one pass of a warp at most");
};
template <class T, int D>
struct Smem {
    unsigned char ring[kThreads / 32][Form<T, D>::kWarp];
    unsigned char q[kMaxHeads * Form<T, D>::kRow];
    float p[kThreads / 32][Form<T, D>::kMma ? 1 : kMaxHeads * kStep];  // fp32: the weights of a step
    float m[kThreads / 32][kMaxHeads], l[kThreads / 32][kMaxHeads];
    unsigned o_at[kThreads / 32];  // where in its ring a warp has left its O
};

// Byte of piece x (16 bytes) of row r in a tile: turned, so that eight rows' same piece touch every bank.
template <class T, int D>
__device__ __forceinline__ unsigned piece_at(int r, int x) {
    constexpr int n = Form<T, D>::kPieces;
    const int turn = n >= 8 ? r & 7 : n == 4 ? (r >> 1) & 3 : (r >> 2) & 1;
    return (unsigned)(r * Form<T, D>::kRow + ((x ^ turn) << 4));
}

// What a warp gathers of a segment: bf16.
template <class T, int D>
struct Walk {
    using F = Form<T, D>;
    unsigned q_addr, qa[F::kQInRegs ? D / 16 : 1][4];
    float o[D / 8][4], ref[2], l[2];  // of rows (heads) quad and quad + 8; ref in units of log2

    __device__ __forceinline__ void begin(Smem<T, D> &sm, int lane) {
        q_addr = wp::smem_addr(sm.q);
        if constexpr (F::kQInRegs) {
#pragma unroll
            for (int x = 0; x < D / 16; ++x) wp::ldmatrix4(q_addr + piece_at<T, D>(lane & 15, 2 * x + (lane >> 4)), qa[x]);
        }
#pragma unroll
        for (int x = 0; x < D / 8; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
        ref[0] = ref[1] = -CUDART_INF_F;
        l[0] = l[1] = 0.f;
    }

    // The tiles at shared-memory address kt (V behind K); `keys`: which are there.
    __device__ __forceinline__ void step(Smem<T, D> &, int, unsigned kt, const unsigned char *, unsigned keys, int, float scale_log2, int lane) {
        const unsigned vt = kt + F::kTile;
        // ldmatrix rows of this lane
        const int k_row = (lane >> 4) * 8 + (lane & 7), k_half = (lane >> 3) & 1, v_row = ((lane >> 3) & 1) * 8 + (lane & 7), v_half = lane >> 4;
        float sc[2][4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) sc[x][y] = 0.f;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            unsigned b[4], a[4];
            wp::ldmatrix4(kt + piece_at<T, D>(k_row, 2 * x + k_half), b);
            if constexpr (F::kQInRegs) {
#pragma unroll
                for (int y = 0; y < 4; ++y) a[y] = qa[x][y];
            } else {
                wp::ldmatrix4(q_addr + piece_at<T, D>(lane & 15, 2 * x + (lane >> 4)), a);
            }
            wp::mma_bf16(sc[0], a[0], a[1], a[2], a[3], b[0], b[1]);
            wp::mma_bf16(sc[1], a[0], a[1], a[2], a[3], b[2], b[3]);
        }
        bool outgrown = false;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int key = x * 8 + (lane & 3) * 2 + (y & 1);
                sc[x][y] = (keys >> key) & 1u ? sc[x][y] * scale_log2 : -CUDART_INF_F;
                outgrown = outgrown || sc[x][y] - ref[y >> 1] > kOutgrown;  // (the first: infinity)
            }
        if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float mx = fmaxf(fmaxf(sc[0][2 * r], sc[0][2 * r + 1]), fmaxf(sc[1][2 * r], sc[1][2 * r + 1]));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const float now = fmaxf(ref[r], mx), f = now == -CUDART_INF_F ? 1.f : fast_exp2(ref[r] - now);
                ref[r] = now;
                l[r] *= f;
#pragma unroll
                for (int x = 0; x < D / 8; ++x) { o[x][2 * r] *= f; o[x][2 * r + 1] *= f; }
            }
        }
        unsigned pa[4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float base = ref[r] == -CUDART_INF_F ? 0.f : ref[r];
                const float p0 = fast_exp2(sc[x][2 * r] - base), p1 = fast_exp2(sc[x][2 * r + 1] - base);
                l[r] += p0 + p1;
                const __nv_bfloat162 pk = __floats2bfloat162_rn(p0, p1);
                pa[2 * x + r] = *reinterpret_cast<const unsigned *>(&pk);
            }
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            unsigned b[4];
            wp::ldmatrix4_t(vt + piece_at<T, D>(v_row, 2 * x + v_half), b);
            wp::mma_bf16(o[2 * x], pa[0], pa[1], pa[2], pa[3], b[0], b[1]);
            wp::mma_bf16(o[2 * x + 1], pa[0], pa[1], pa[2], pa[3], b[2], b[3]);
        }
    }

    __device__ __forceinline__ void leave(Smem<T, D> &sm, int warp, float *own, int lane) {
        const int quad = lane >> 2;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
            if ((lane & 3) == 0) { sm.m[warp][quad + 8 * r] = ref[r]; sm.l[warp][quad + 8 * r] = l[r]; }
        }
#pragma unroll
        for (int x = 0; x < D / 8; ++x) {
            *reinterpret_cast<float2 *>(own + quad * D + x * 8 + (lane & 3) * 2) = make_float2(o[x][0], o[x][1]);
            *reinterpret_cast<float2 *>(own + (quad + 8) * D + x * 8 + (lane & 3) * 2) = make_float2(o[x][2], o[x][3]);
        }
    }
};

// The same in fp32. Lanes 2 i and 2 i + 1 have key i of a step, half of its pieces each; lane i has O's channels kChan i ...; a
// head's reference and sum (of every lane's own keys) are in registers, the loop over heads unrolled by four.
template <int D>
struct Walk<float, D> {
    using F = Form<float, D>;
    float o[kMaxHeads][F::kChan], ref[kMaxHeads], l[kMaxHeads];

    __device__ __forceinline__ void begin(Smem<float, D> &, int) {
#pragma unroll
        for (int h = 0; h < kMaxHeads; ++h) {
            ref[h] = -CUDART_INF_F;
            l[h] = 0.f;
#pragma unroll
            for (int x = 0; x < F::kChan; ++x) o[h][x] = 0.f;
        }
    }

    __device__ __forceinline__ void step(Smem<float, D> &sm, int warp, unsigned, const unsigned char *tile, unsigned keys, int heads, float scale_log2, int lane) {
        const int key = lane >> 1, half = lane & 1;
        const bool there = (keys >> key) & 1u;
        float *const p = sm.p[warp];
        const float *const q = reinterpret_cast<const float *>(sm.q);
        const unsigned char *const vt = tile + F::kTile;
        float4 k[F::kPieces / 2];  // every second piece
#pragma unroll
        for (int x = 0; x < F::kPieces / 2; ++x) k[x] = *reinterpret_cast<const float4 *>(tile + piece_at<float, D>(key, 2 * x + half));
#pragma unroll
        for (int h4 = 0; h4 < kMaxHeads; h4 += 4) {
            if (h4 >= heads) break;
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < F::kPieces / 2; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // (heads behind the last are zeros)
                    const float4 a = *reinterpret_cast<const float4 *>(q + (h4 + i) * D + (2 * x + half) * 4);
                    s[i] = fmaf(a.w, k[x].w, fmaf(a.z, k[x].z, fmaf(a.y, k[x].y, fmaf(a.x, k[x].x, s[i]))));
                }
            bool outgrown = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] += __shfl_xor_sync(0xffffffffu, s[i], 1);
                s[i] = there ? s[i] * scale_log2 : -CUDART_INF_F;
                outgrown = outgrown || s[i] - ref[h4 + i] > kOutgrown;  // (the first: infinity)
            }
            if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float now = fmaxf(ref[h4 + i], warp_maximum(s[i])), f = now == -CUDART_INF_F ? 1.f : fast_exp2(ref[h4 + i] - now);
                    ref[h4 + i] = now;
                    l[h4 + i] *= f;
#pragma unroll
                    for (int x = 0; x < F::kChan; ++x) o[h4 + i][x] *= f;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = fast_exp2(s[i] - (ref[h4 + i] == -CUDART_INF_F ? 0.f : ref[h4 + i]));
                if (half == 0) {
                    l[h4 + i] += w;
                    p[(h4 + i) * kStep + key] = w;
                }
            }
        }
        __syncwarp();
        const int at = lane * F::kChan;  // (D = 16: the upper lanes repeat the lower ones)
#pragma unroll
        for (int j = 0; j < kStep; j += 4) {
            float v[4][F::kChan];
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < F::kChan; ++x) {
                    const int c = (at + x) % D;
                    v[y][x] = *reinterpret_cast<const float *>(vt + piece_at<float, D>(j + y, c / 4) + (c % 4) * 4);
                }
#pragma unroll
            for (int h = 0; h < kMaxHeads; ++h) {
                if (h >= heads) break;
                const float4 w = *reinterpret_cast<const float4 *>(p + h * kStep + j);
#pragma unroll
                for (int x = 0; x < F::kChan; ++x) o[h][x] = fmaf(w.w, v[3][x], fmaf(w.z, v[2][x], fmaf(w.y, v[1][x], fmaf(w.x, v[0][x], o[h][x]))));
            }
        }
    }

    __device__ __forceinline__ void leave(Smem<float, D> &sm, int warp, float *own, int lane) {
#pragma unroll
        for (int h = 0; h < kMaxHeads; ++h) {
            float sum = l[h];
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (lane == 0) { sm.m[warp][h] = ref[h]; sm.l[warp][h] = sum; }
#pragma unroll
            for (int x = 0; x < F::kChan; ++x)
                if (lane * F::kChan + x < D) own[h * D + lane * F::kChan + x] = o[h][x];
        }
    }
};

template <class T, int D, bool W>
__global__ void __launch_bounds__(kThreads, Form<T, D>::kCtas) decode_warp_kernel(const __grid_constant__ Args A) {
    using F = Form<T, D>;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Smem<T, D> &sm = *reinterpret_cast<Smem<T, D> *>(smem_raw);
    const CacheGeom &c = A.a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    after_previous_kernel();
    T *const out = (T *)A.a.out;
    write_empty_slots<T>(A);
    const Share mine = share_of(A, all_places<W>(A, lane), (int)blockIdx.x);
    unsigned char *const ring_ptr = sm.ring[warp];
    const unsigned ring = wp::smem_addr(ring_ptr), q_smem = wp::smem_addr(sm.q);
    const bool one_page = c.page % kStep == 0;  // a tile's keys lie side by side
    constexpr int kPieces = F::kPieces, kRowsAtOnce = 32 / kPieces;  // rows that 32 lanes fetch at once
    const int row_l = lane / kPieces, piece_l = lane % kPieces;
    unsigned bad = 0;
    // What this warp fetches: its steps of the segment that is open, step n in the ring's place (at + n) % kStages
    const int32_t *table = nullptr;
    const T *ks = nullptr, *vs = nullptr;
    int slot = 0, key_w = 0, key_end = 0, n_steps = 0;
    unsigned at = 0;
    unsigned long long keys_there = 0;  // 16 flags a place of the ring
    int page = -1;                      // lane i < 16: the page of key i of the next step to be fetched, -1: none
    Seen seen = {};
    auto page_of = [&](int n) -> int {
        const int walked = key_w + 4 * n * kStep + lane, key = W ? seen.key(walked) : walked;
        if (n >= n_steps || lane >= kStep || walked >= key_end) return -1;
        const int x = table[key / c.page];
        if ((unsigned)x < (unsigned)c.n_pages) return x;
        if (!W || seen.sees(key)) bad = (unsigned)slot + 1u;
        return -1;
    };
    auto fetch = [&](int n) {  // step n, and the pages of the one after it are looked up
        const int own_page = page;
        page = page_of(n + 1);
        if (n < n_steps) {
            const int walked = key_w + 4 * n * kStep + lane, key = W ? seen.key(walked) : walked;
            const unsigned place = (at + (unsigned)n) % F::kStages, there = __ballot_sync(0xffffffffu, own_page >= 0 && (!W || seen.sees(key)));
            keys_there = (keys_there & ~(0xffffull << (16 * place))) | (unsigned long long)there << (16 * place);
            const long long own = own_page >= 0 ? (long long)own_page * c.s_p + (long long)(key % c.page) * c.s_t : 0;
            const unsigned dst = ring + place * 2 * F::kTile;
            const long long base = __shfl_sync(0xffffffffu, own, 0) + row_l * c.s_t;
#pragma unroll
            for (int r0 = 0; r0 < kStep; r0 += kRowsAtOnce) {
                const int r = r0 + row_l;
                const bool is = (there >> r) & 1u;
                long long e = base + r0 * c.s_t;
                if (!one_page) e = __shfl_sync(0xffffffffu, own, r);
                e = (is ? e : 0) + piece_l * F::kVec;
                const unsigned to = dst + piece_at<T, D>(r, piece_l);
                wp::cp_async16(to, ks + e, is ? 16 : 0);
                wp::cp_async16(to + F::kTile, vs + e, is ? 16 : 0);
            }
        }
        wp::cp_async_commit();
    };
    constexpr int kQ = (kMaxHeads * kPieces + kThreads - 1) / kThreads;  // pieces of Q a thread
    uint4 qr[kQ];
    // The first steps of a segment are on their way before the one before it is written out, and so is its Q
    auto open = [&](const Segment &sg) {
        at += (unsigned)n_steps;
        slot = sg.slot;
        if constexpr (W) seen = seen_of<W, kUnit64>(A.a, slot);
        table = c.table + (long long)slot * c.max_pages;
        ks = (const T *)A.a.k + (long long)sg.kvh * c.s_h;
        vs = (const T *)A.a.v + (long long)sg.kvh * c.s_h;
        key_w = sg.key0 + warp * kStep;
        key_end = sg.key_end;
        n_steps = key_end > key_w ? (key_end - key_w + 4 * kStep - 1) / (4 * kStep) : 0;
        page = page_of(0);
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
            const int h = (tid + i * kThreads) / kPieces, x = (tid + i * kThreads) % kPieces;
            const T *const src = (const T *)A.a.q + (long long)slot * A.a.qs_s + (long long)(sg.h0 + h) * A.a.qs_h + x * F::kVec;
            qr[i] = make_uint4(0, 0, 0, 0);
            if (h < sg.heads) {
                if (A.q_vec) {
                    qr[i] = *reinterpret_cast<const uint4 *>(src);
                } else if constexpr (F::kMma) {
                    unsigned y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __nv_bfloat162 two = __halves2bfloat162(src[2 * e], src[2 * e + 1]);
                        y[e] = *reinterpret_cast<const unsigned *>(&two);
                    }
                    qr[i] = make_uint4(y[0], y[1], y[2], y[3]);
                } else {
                    qr[i] = make_uint4(__float_as_uint(src[0]), __float_as_uint(src[1]), __float_as_uint(src[2]), __float_as_uint(src[3]));
                }
            }
        }
#pragma unroll
        for (int n = 0; n < F::kStages - 1; ++n) fetch(n);
    };
    Place pl = {0, 0, 0};
    int n_parts = 0;
    Left left = {};
    Segment sg = open_segment<W>(A, mine.first, mine.end, lane, pl);
    if (sg.next >= 0) open(sg);
    while (sg.next >= 0) {
        const int s = sg.slot;
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
            const int h = (tid + i * kThreads) / kPieces, x = (tid + i * kThreads) % kPieces;
            if (h < kMaxHeads) *reinterpret_cast<uint4 *>(sm.q + (F::kMma ? piece_at<T, D>(h, x) : (unsigned)(h * F::kRow + x * 16))) = qr[i];
        }
        __syncthreads();
        Walk<T, D> walk;
        walk.begin(sm, lane);
        for (int n = 0; n < n_steps; ++n) {
            fetch(n + F::kStages - 1);
            wp::cp_async_wait<F::kStages - 1>();
            __syncwarp();
            const unsigned place = (at + (unsigned)n) % F::kStages, keys = (unsigned)(keys_there >> (16 * place)) & 0xffffu;
            const unsigned kt = ring + place * 2 * F::kTile;
            walk.step(sm, warp, kt, ring_ptr + place * 2 * F::kTile, keys, sg.heads, A.a.scale_log2, lane);
            __syncwarp();  // (the tile is read before its place is filled again)
        }
        const Segment next = open_segment<W>(A, sg.next, mine.end, lane, pl);
        if (next.next >= 0) {
            open(next);
        } else {
            at += (unsigned)n_steps;
            wp::cp_async_wait<0>();
        }
        // the place behind the first steps of the next segment is free: for O
        const unsigned o_place = (at + F::kStages - 1) % F::kStages * 2 * F::kTile;
        // the four warps' m, l and O meet
        walk.leave(sm, warp, reinterpret_cast<float *>(ring_ptr + o_place), lane);
        if (lane == 0) sm.o_at[warp] = o_place;
        __syncthreads();
        float *const part = part_of(A, (int)blockIdx.x, n_parts);
        if (!sg.whole) {
            if (sg.key0 == 0) left = {pieces_of(sg.owner_end, mine), n_parts, sg.heads, 0u, (long long)sg.slot * A.a.H + sg.h0, 0ll};
            ++n_parts;
        }
        for (int i = tid; i < sg.heads * (D / 4); i += kThreads) {
            const int h = i / (D / 4), x = (i % (D / 4)) * 4;
            float m = sm.m[0][h];
#pragma unroll
            for (int w = 1; w < kThreads / 32; ++w) m = fmaxf(m, sm.m[w][h]);
            const float base = m == -CUDART_INF_F ? 0.f : m;
            float sum = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) {
                const float f = fast_exp2(sm.m[w][h] - base);
                const float4 z = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(sm.ring[w] + sm.o_at[w]) + h * D + x);
                sum = fmaf(f, sm.l[w][h], sum);
                y.x = fmaf(f, z.x, y.x); y.y = fmaf(f, z.y, y.y); y.z = fmaf(f, z.z, y.z); y.w = fmaf(f, z.w, y.w);
            }
            if (sg.whole) {
                const float inv = sum > 0.f ? 1.f / sum : 0.f;
                T *const to = out + ((long long)s * A.a.H + sg.h0 + h) * D + x;
                to[0] = (T)(y.x * inv); to[1] = (T)(y.y * inv); to[2] = (T)(y.z * inv); to[3] = (T)(y.w * inv);
                if (x == 0 && A.a.lse != nullptr) A.a.lse[(long long)s * A.a.H + sg.h0 + h] = lse_of(m, sum);
            } else {
                *reinterpret_cast<float4 *>(part + 2 * kMaxHeads + h * D + x) = y;
                if (x == 0) { part[h] = m; part[kMaxHeads + h] = sum; }
            }
        }
        __syncthreads();  // (the places of O are filled again)
        sg = next;
    }
    leave_to_joins(A, left, bad);
}

template <class T, int D, bool W>
cudaError_t launch_form(Args &A, int n_sm, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<T, D>);
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(decode_warp_kernel<T, D, W>, smem, done);
    if (e != cudaSuccess) return e;
    const int most = Form<T, D>::kCtas * n_sm;
    if (A.grid > most) A.grid = most;
    return launch_early(decode_warp_kernel<T, D, W>, (unsigned)A.grid, kThreads, smem, st, A);
}
template <class T, int D>
cudaError_t launch(Args &A, int n_sm, cudaStream_t st) {
    return A.a.window > 0 ? launch_form<T, D, true>(A, n_sm, st) : launch_form<T, D, false>(A, n_sm, st);
}

}  // namespace

namespace decode {

bool warp_supported(const DecodeCall &a, int dtype) {
    const int e = dtype == STREAM_F32 ? 4 : 2;
    if (a.c.d * e > 512) return false;
    return (((uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0 && ((a.c.s_p | a.c.s_t | a.c.s_h) * e & 15) == 0;
}

cudaError_t launch_warp(Args &A, int dtype, int n_sm, cudaStream_t st) {
    const int e = dtype == STREAM_F32 ? 4 : 2;
    A.q_vec = ((uintptr_t)A.a.q & 15) == 0 && ((A.a.qs_s | A.a.qs_h) * e & 15) == 0 ? 1 : 0;
    if (dtype == STREAM_F32) {
        switch (A.a.c.d) {
            case 16: return launch<float, 16>(A, n_sm, st);
            case 32: return launch<float, 32>(A, n_sm, st);
            case 64: return launch<float, 64>(A, n_sm, st);
            default: return launch<float, 128>(A, n_sm, st);
        }
    }
    switch (A.a.c.d) {
        case 16: return launch<__nv_bfloat16, 16>(A, n_sm, st);
        case 32: return launch<__nv_bfloat16, 32>(A, n_sm, st);
        case 64: return launch<__nv_bfloat16, 64>(A, n_sm, st);
        case 128: return launch<__nv_bfloat16, 128>(A, n_sm, st);
        default: return launch<__nv_bfloat16, 256>(A, n_sm, st);
    }
}

}  // namespace decode
}  // namespace stream
