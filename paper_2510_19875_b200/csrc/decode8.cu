// Decode attention over a cache in 8 bits: e4m3 numbers with a scale for each block of tokens and kv head.
//
//     x_t = scale log2(e) sk_t (q . k8_t),     out = sum_t 2^(x_t - m) sv_t v8_t / sum_t 2^(x_t - m)
//
// The keys of all slots and heads are dealt to the CTAs as in decode.cu, and a warp walks its tiles of 16 keys alone, as in decode_warp.cu. Half the bytes
// a key leave half the time for it, so that the products turn: the keys are the rows of S^T = K Q^T and V's channels those of O^T = V^T P^T, the
// query heads, of which a kv head has mostly eight or fewer, the eight columns (16 heads: two products from the same K and V). e4m3
// is exact in fp16. A lane's four bytes of K are four channels side by side of one key: Q's channels are taken in that order. Two rows of V
// are turned by ldmatrix two bytes at a time, so that a lane has two channels of two keys, rows g and g + 8 of the product. The weights are turned by movmatrix.
//
// fp16 has eleven bits but a short range, which powers of two see to: a head's q is brought to [2^14, 2^15); a weight for the product is
// 2^(x - r) sv 2^14, r following the largest x + log2(sv) of the warp's keys within a factor of 2, so that what fp16 cuts off, below 2^-24, is 2^-39
// of the largest. The sum has a reference of its own and is that of the unrounded weights. bf16 caches: q (eight bits) is so exact, a weight off by
// 2^-11. fp32 ones: q and the weights as two fp16 numbers each, and parts of 16 terms are added by ordinary additions (the tensor core's own sums are cut).
#include <cuda_fp16.h>

#include "decode.cuh"

namespace stream {
namespace {

using namespace decode;

constexpr int kStep = 16;            // keys of a warp's tile
constexpr float kOutgrown = 30.f;    // log2: of the sum's reference
constexpr float kTop = 14.f;         // log2: a weight for the product at its reference

template <class T, int D, int N>
struct Form {
    static constexpr bool kPair = sizeof(T) == 4;               // two fp16 numbers an operand
    static constexpr int kPieces = D / 16;                      // of 16 bytes of a row, and steps of K Q^T
    static constexpr int kTile = kStep * D;                     // bytes
    static constexpr int kPlace = 2 * kTile + 2 * kStep * 4;    // K, V, the keys' scales
    static constexpr int kStages = D == 128 ? (N == 1 ? 5 : 4) : D == 256 ? 4 : 8;
    static constexpr int kCtas = D == 256 ? 1 : 2;              // of an SM
    static constexpr int kHeads = 8 * N;
    static constexpr bool kQInRegs = D * N * (kPair ? 2 : 1) <= 256;
    static constexpr int kLane = D >= 32 ? D / 32 : 1;          // channels of a head's q a lane
};
template <class T, int D, int N>
struct Smem {
    using F = Form<T, D, N>;
    unsigned char ring[kThreads / 32][F::kStages * F::kPlace];
    float o[kThreads / 32][F::kHeads * D];
    __half q[F::kPair ? 2 : 1][F::kHeads * D];   // the rest of each number behind
    float unit[F::kHeads];                       // what a logit of this q is worth
    float m[kThreads / 32][F::kHeads], l[kThreads / 32][F::kHeads];
};

// Byte of piece x (16 bytes) of row r in a tile: turned, so that eight rows' same piece touch every bank.
template <int D>
__device__ __forceinline__ unsigned piece_at(int r, int x) {
    constexpr int n = D / 16;
    const int turn = n >= 8 ? r & 7 : n == 4 ? (r >> 1) & 3 : n == 2 ? (r >> 2) & 1 : 0;
    return (unsigned)(r * D + ((x ^ turn) << 4));
}

__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two e4m3 numbers (the lower or the upper half of w) to fp16.
__device__ __forceinline__ unsigned widen_low(unsigned w) {
    unsigned r;
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %1; cvt.rn.f16x2.e4m3x2 %0, a;}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ unsigned widen_high(unsigned w) {
    unsigned r;
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %1; cvt.rn.f16x2.e4m3x2 %0, b;}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ unsigned turned(unsigned x) {  // an 8 x 8 matrix of 16-bit elements
    unsigned r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ unsigned pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned *>(&h);
}
__device__ __forceinline__ float log2_of(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void cp_async4_or_zero(unsigned dst, const void *src, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// What a warp gathers of a segment. A lane (g = lane / 4, t = lane % 4) has the heads 8 n + 2 t and 8 n + 2 t + 1, of a tile the keys g and g + 8, and of O
// the channels 16 c + 2 g and 16 c + 2 g + 1.
template <class T, int D, int N>
struct Walk {
    using F = Form<T, D, N>;
    static constexpr int kParts = F::kPair ? 2 : 1;
    unsigned q[kParts][F::kQInRegs ? F::kPieces : 1][N][2];
    float o[F::kPieces][N][4], unit[N][2], ref[N][2], top[N][2], l[N][2];  // ref: of the sum, top: of the weights for the product; units of log2

    __device__ __forceinline__ void load_q(const Smem<T, D, N> &sm, int part, int c, int n, int lane, unsigned (&r)[2]) const {
        const uint2 x = *reinterpret_cast<const uint2 *>(&sm.q[part][(8 * n + (lane >> 2)) * D + 16 * c + 4 * (lane & 3)]);
        r[0] = x.x;
        r[1] = x.y;
    }
    __device__ __forceinline__ void begin(const Smem<T, D, N> &sm, float scale_log2, int lane) {
        if constexpr (F::kQInRegs) {
#pragma unroll
            for (int p = 0; p < kParts; ++p)
#pragma unroll
                for (int c = 0; c < F::kPieces; ++c)
#pragma unroll
                    for (int n = 0; n < N; ++n) load_q(sm, p, c, n, lane, q[p][c][n]);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int c = 0; c < F::kPieces; ++c)
#pragma unroll
                for (int y = 0; y < 4; ++y) o[c][n][y] = 0.f;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                unit[n][y] = sm.unit[8 * n + 2 * (lane & 3) + y] * scale_log2;
                ref[n][y] = top[n][y] = -CUDART_INF_F;
                l[n][y] = 0.f;
            }
        }
    }

    // The tile at shared-memory address kt: K, V behind it, and the keys' scales at z.
    __device__ __forceinline__ void step(const Smem<T, D, N> &sm, unsigned kt, const float *z, int lane) {
        const unsigned vt = kt + F::kTile;
        const int r8 = (lane >> 3 & 1) * 8 + (lane & 7), half = lane >> 4;  // ldmatrix: this lane's row, and which of two pieces
        float s[N][4];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 4; ++y) s[n][y] = 0.f;
#pragma unroll
        for (int c = 0; c < F::kPieces; c += 2) {
            unsigned w[4];
            wp::ldmatrix4(kt + piece_at<D>(r8, F::kPieces > 1 ? c + half : 0), w);
#pragma unroll
            for (int i = 0; i < (F::kPieces > 1 ? 2 : 1); ++i) {
                const unsigned a0 = widen_low(w[2 * i]), a2 = widen_high(w[2 * i]), a1 = widen_low(w[2 * i + 1]), a3 = widen_high(w[2 * i + 1]);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
                    float(&to)[4] = F::kPair ? part : s[n];
#pragma unroll
                    for (int p = kParts - 1; p >= 0; --p) {  // (the small parts first)
                        unsigned b[2];
                        if constexpr (F::kQInRegs) {
                            b[0] = q[p][F::kQInRegs ? c + i : 0][n][0];
                            b[1] = q[p][F::kQInRegs ? c + i : 0][n][1];
                        } else {
                            load_q(sm, p, c + i, n, lane, b);
                        }
                        mma_f16(to, a0, a1, a2, a3, b[0], b[1]);
                    }
                    if constexpr (F::kPair) {
#pragma unroll
                        for (int y = 0; y < 4; ++y) s[n][y] += part[y];
                    }
                }
            }
        }
        const float sk[2] = {z[lane >> 2], z[(lane >> 2) + 8]}, sv[2] = {z[kStep + (lane >> 2)], z[kStep + (lane >> 2) + 8]};
        const float lv[2] = {log2_of(sv[0]), log2_of(sv[1])};
        bool outgrown = false;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 4; ++y) {  // head y & 1, key y >> 1
                s[n][y] = sk[y >> 1] != 0.f ? s[n][y] * (unit[n][y & 1] * sk[y >> 1]) : -CUDART_INF_F;
                outgrown = outgrown || s[n][y] - ref[n][y & 1] > kOutgrown || s[n][y] + lv[y >> 1] - top[n][y & 1] > 1.f;  // (the first: infinity)
            }
        if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float a = fmaxf(s[n][y], s[n][y + 2]), b = fmaxf(s[n][y] + lv[0], s[n][y + 2] + lv[1]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
                        b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, d));
                    }
                    a = fmaxf(a, ref[n][y]);
                    b = fmaxf(b, top[n][y]);
                    l[n][y] *= a == -CUDART_INF_F ? 1.f : fast_exp2(ref[n][y] - a);
                    const float f = b == -CUDART_INF_F ? 1.f : fast_exp2(top[n][y] - b);
                    ref[n][y] = a;
                    top[n][y] = b;
#pragma unroll
                    for (int c = 0; c < F::kPieces; ++c) { o[c][n][y] *= f; o[c][n][y + 2] *= f; }
                }
        }
        unsigned p[kParts][N][2];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int key = 0; key < 2; ++key) {
                float w[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float x = s[n][2 * key + y];
                    l[n][y] += fast_exp2(x - (ref[n][y] == -CUDART_INF_F ? 0.f : ref[n][y]));
                    w[y] = x == -CUDART_INF_F || sv[key] == 0.f ? 0.f : fast_exp2(x - top[n][y] + kTop) * sv[key];
                }
                const unsigned hi = pack(w[0], w[1]);
                p[0][n][key] = turned(hi);
                if constexpr (F::kPair) {
                    const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
                    p[kParts - 1][n][key] = turned(pack(w[0] - h.x, w[1] - h.y));
                }
            }
#pragma unroll
        for (int c = 0; c < F::kPieces; c += 2) {
            unsigned w[4];
            wp::ldmatrix4_t(vt + piece_at<D>(r8, F::kPieces > 1 ? c + half : 0), w);
#pragma unroll
            for (int i = 0; i < (F::kPieces > 1 ? 2 : 1); ++i) {
                // bytes: two channels of one key, two of the next; turned to two keys of one channel, two of the other
                const unsigned u0 = __byte_perm(w[2 * i], 0, 0x3120), u1 = __byte_perm(w[2 * i + 1], 0, 0x3120);
                const unsigned a0 = widen_low(u0), a1 = widen_high(u0), a2 = widen_low(u1), a3 = widen_high(u1);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
                    float(&to)[4] = F::kPair ? part : o[c + i][n];
#pragma unroll
                    for (int y = kParts - 1; y >= 0; --y) mma_f16(to, a0, a1, a2, a3, p[y][n][0], p[y][n][1]);
                    if constexpr (F::kPair) {
#pragma unroll
                        for (int y = 0; y < 4; ++y) o[c + i][n][y] += part[y];
                    }
                }
            }
        }
    }

    // m, l and O = sum_t 2^(x - m) v to shared memory.
    __device__ __forceinline__ void leave(Smem<T, D, N> &sm, int warp, int lane) {
        float *const own = sm.o[warp];
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int h = 8 * n + 2 * t + y;
                float sum = l[n][y];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (g == 0) { sm.m[warp][h] = ref[n][y]; sm.l[warp][h] = sum; }
                const float f = ref[n][y] == -CUDART_INF_F ? 0.f : fast_exp2(top[n][y] - kTop - ref[n][y]);
#pragma unroll
                for (int c = 0; c < F::kPieces; ++c)
                    *reinterpret_cast<float2 *>(own + h * D + 16 * c + 2 * g) = make_float2(o[c][n][y] * f, o[c][n][y + 2] * f);
            }
    }
};

struct Args8 {
    Args A;
    Scales sc;
    int vec;   // rows of the cache are read in pieces of 16 bytes
};

template <class T, int D, int N, bool W>
__global__ void __launch_bounds__(kThreads, Form<T, D, N>::kCtas) decode8_kernel(const __grid_constant__ Args8 B) {
    using F = Form<T, D, N>;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Smem<T, D, N> &sm = *reinterpret_cast<Smem<T, D, N> *>(smem_raw);
    const Args &A = B.A;
    const CacheGeom &c = A.a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    after_previous_kernel();
    T *const out = (T *)A.a.out;
    write_empty_slots<T>(A);
    const Share mine = share_of(A, all_places<W>(A, lane), (int)blockIdx.x);
    unsigned char *const ring_ptr = sm.ring[warp];
    const unsigned ring = wp::smem_addr(ring_ptr);
    const bool one_page = c.page % kStep == 0;  // a tile's keys lie side by side
    constexpr int kPieces = F::kPieces, kRowsAtOnce = 32 / kPieces < kStep ? 32 / kPieces : kStep;  // rows that 32 lanes fetch at once
    const int row_l = lane / kPieces, piece_l = lane % kPieces;
    unsigned bad = 0;
    // What this warp fetches: its steps of the segment that is open, step n in the ring's place (at + n) % kStages
    const int32_t *table = nullptr;
    const unsigned char *ks = nullptr, *vs = nullptr;
    const float *zs = nullptr;          // lanes 0 .. 15: K's scales, the others: V's
    int slot = 0, key_w = 0, key_end = 0, n_steps = 0;
    unsigned at = 0;
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
            const int walked = key_w + 4 * n * kStep + lane, key = W ? seen.key(walked) : walked, in_page = key % c.page;
            const unsigned place = (at + (unsigned)n) % F::kStages, there = __ballot_sync(0xffffffffu, own_page >= 0 && (!W || seen.sees(key)));
            const long long own = own_page >= 0 ? (long long)own_page * c.s_p + (long long)in_page * c.s_t : 0;
            const long long z = own_page >= 0 ? (long long)own_page * B.sc.s_p + (long long)(in_page / B.sc.block) * B.sc.s_b : 0;
            const unsigned dst = ring + place * F::kPlace;
            const long long base = __shfl_sync(0xffffffffu, own, 0) + row_l * c.s_t;
#pragma unroll
            for (int r0 = 0; r0 < kStep; r0 += kRowsAtOnce) {
                const int r = r0 + row_l;
                long long e = base + r0 * c.s_t;
                if (!one_page) e = __shfl_sync(0xffffffffu, own, r & 31);
                if (r - r0 < kRowsAtOnce) {
                    const bool is = (there >> r) & 1u;
                    e = (is ? e : 0) + piece_l * 16;
                    const unsigned to = place * F::kPlace + piece_at<D>(r, piece_l);
                    if (B.vec) {
                        wp::cp_async16(ring + to, ks + e, is ? 16 : 0);
                        wp::cp_async16(ring + to + F::kTile, vs + e, is ? 16 : 0);
                    } else {
#pragma unroll 4
                        for (int i = 0; i < 16; ++i) {
                            ring_ptr[to + i] = is ? ks[e + i] : 0;
                            ring_ptr[to + F::kTile + i] = is ? vs[e + i] : 0;
                        }
                    }
                }
            }
            const long long z_at = __shfl_sync(0xffffffffu, z, lane & 15);
            const bool is = (there >> (lane & 15)) & 1u;
            cp_async4_or_zero(dst + 2 * F::kTile + lane * 4, zs + (is ? z_at : 0), is ? 4 : 0);
        }
        wp::cp_async_commit();
    };
    constexpr int kOwn = F::kHeads / (kThreads / 32);  // heads whose q a warp reads: lane i their channels kLane i ...
    float qr[kOwn][F::kLane];
    // The first steps of a segment are on their way before the one before it is written out, and so is its Q
    auto open = [&](const Segment &sg) {
        at += (unsigned)n_steps;
        slot = sg.slot;
        if constexpr (W) seen = seen_of<W>(A.a, slot);
        table = c.table + (long long)slot * c.max_pages;
        ks = (const unsigned char *)A.a.k + (long long)sg.kvh * c.s_h;
        vs = (const unsigned char *)A.a.v + (long long)sg.kvh * c.s_h;
        zs = (lane < kStep ? B.sc.k : B.sc.v) + (long long)sg.kvh * B.sc.s_h;
        key_w = sg.key0 + warp * kStep;
        key_end = sg.key_end;
        n_steps = key_end > key_w ? (key_end - key_w + 4 * kStep - 1) / (4 * kStep) : 0;
        page = page_of(0);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int h = warp + 4 * i;
            const T *const src = (const T *)A.a.q + (long long)slot * A.a.qs_s + (long long)(sg.h0 + h) * A.a.qs_h + lane * F::kLane;
#pragma unroll
            for (int e = 0; e < F::kLane; ++e) qr[i][e] = h < sg.heads && lane * F::kLane < D ? to_float(src[e]) : 0.f;
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
        for (int i = 0; i < kOwn; ++i) {  // q times a power of two, in [2^14, 2^15) at its largest
            const int h = warp + 4 * i;
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < F::kLane; ++e) most = fmaxf(most, fabsf(qr[i][e]));
            most = warp_maximum(most);
            const int up = min(max(141 - (int)(__float_as_uint(most) >> 23), -114), 126);
            const float f = __uint_as_float((unsigned)(up + 127) << 23);
            if (lane == 0) sm.unit[h] = 1.f / f;
            if (lane * F::kLane < D) {
#pragma unroll
                for (int e = 0; e < F::kLane; ++e) {
                    const float x = qr[i][e] * f;
                    const __half hi = __float2half_rn(x);
                    sm.q[0][h * D + lane * F::kLane + e] = hi;
                    if constexpr (F::kPair) sm.q[F::kPair ? 1 : 0][h * D + lane * F::kLane + e] = __float2half_rn(x - __half2float(hi));
                }
            }
        }
        __syncthreads();
        Walk<T, D, N> walk;
        walk.begin(sm, A.a.scale_log2, lane);
        for (int n = 0; n < n_steps; ++n) {
            fetch(n + F::kStages - 1);
            wp::cp_async_wait<F::kStages - 1>();
            __syncwarp();
            const unsigned place = (at + (unsigned)n) % F::kStages * F::kPlace;
            walk.step(sm, ring + place, reinterpret_cast<const float *>(ring_ptr + place + 2 * F::kTile), lane);
            __syncwarp();  // (the tile is read before its place is filled again)
        }
        const Segment next = open_segment<W>(A, sg.next, mine.end, lane, pl);
        if (next.next >= 0) {
            open(next);
        } else {
            at += (unsigned)n_steps;
            wp::cp_async_wait<0>();
        }
        // the four warps' m, l and O meet
        walk.leave(sm, warp, lane);
        __syncthreads();
        float *const part = part_of(A, (int)blockIdx.x, n_parts);
        if (!sg.whole) {
            if (sg.key0 == 0) left = {pieces_of(sg, mine), n_parts, sg.heads, 0u, (long long)sg.slot * A.a.H + sg.h0, 0ll};
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
                const float4 z = *reinterpret_cast<const float4 *>(sm.o[w] + h * D + x);
                sum = fmaf(f, sm.l[w][h], sum);
                y.x = fmaf(f, z.x, y.x); y.y = fmaf(f, z.y, y.y); y.z = fmaf(f, z.z, y.z); y.w = fmaf(f, z.w, y.w);
            }
            if (sg.whole) {
                const float inv = sum > 0.f ? 1.f / sum : 0.f;
                T *const to = out + ((long long)s * A.a.H + sg.h0 + h) * D + x;
                to[0] = (T)(y.x * inv); to[1] = (T)(y.y * inv); to[2] = (T)(y.z * inv); to[3] = (T)(y.w * inv);
                if (x == 0 && A.a.lse != nullptr) A.a.lse[(long long)s * A.a.H + sg.h0 + h] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -CUDART_INF_F;
            } else {
                *reinterpret_cast<float4 *>(part + 2 * kMaxHeads + h * D + x) = y;
                if (x == 0) { part[h] = m; part[kMaxHeads + h] = sum; }
            }
        }
        __syncthreads();  // (O, m, l and q are written again)
        sg = next;
    }
    leave_to_joins(A, left, bad);
}

template <class T, int D, int N, bool W>
cudaError_t launch(Args8 &B, int n_sm, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<T, D, N>);
    static_assert(Form<T, D, N>::kCtas * (sizeof(Smem<T, D, N>) + 1024) <= 233472, "what an SM has");
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(decode8_kernel<T, D, N, W>, smem, done);
    if (e != cudaSuccess) return e;
    const int most = Form<T, D, N>::kCtas * n_sm;
    if (B.A.grid > most) B.A.grid = most;
    return launch_early(decode8_kernel<T, D, N, W>, (unsigned)B.A.grid, kThreads, smem, st, B);
}
template <class T, int D>
cudaError_t launch_n(Args8 &B, int n_sm, cudaStream_t st) {
    const bool w = B.A.a.window > 0;
    if (B.A.a.hpg <= 8) return w ? launch<T, D, 1, true>(B, n_sm, st) : launch<T, D, 1, false>(B, n_sm, st);
    return w ? launch<T, D, 2, true>(B, n_sm, st) : launch<T, D, 2, false>(B, n_sm, st);
}
template <class T>
cudaError_t launch_d(Args8 &B, int n_sm, cudaStream_t st) {
    switch (B.A.a.c.d) {
        case 16: return launch_n<T, 16>(B, n_sm, st);
        case 32: return launch_n<T, 32>(B, n_sm, st);
        case 64: return launch_n<T, 64>(B, n_sm, st);
        case 128: return launch_n<T, 128>(B, n_sm, st);
        default: return launch_n<T, 256>(B, n_sm, st);
    }
}

}  // namespace

stream_status launch_decode8(const DecodeCall &a, const Scales &sc, int dtype, void *workspace, cudaStream_t st) {
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    Args8 B;
    B.A = args_of(a, workspace, n_sm);
    B.sc = sc;
    B.vec = (((uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0 && ((a.c.s_p | a.c.s_t | a.c.s_h) & 15) == 0 ? 1 : 0;
    cudaError_t rc = dtype == STREAM_F32 ? launch_d<float>(B, n_sm, st) : launch_d<__nv_bfloat16>(B, n_sm, st);
    if (rc != cudaSuccess) return cuda_fail(rc, "8-bit decode attention launch");
    rc = launch_joins(B.A, dtype, st);
    return rc == cudaSuccess ? STREAM_OK : cuda_fail(rc, "decode join launch");
}

}  // namespace stream
