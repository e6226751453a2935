// Decode attention over a cache in 8 bits: e4m3 numbers with a scale for each block of tokens and kv head.
//
//     x_t = scale log2(e) sk_t (q . k8_t),     out = sum_t 2^(x_t - m) sv_t v8_t / sum_t 2^(x_t - m)
//
// Half the bytes a key leave half the time for it, so that the products turn against those of decode_warp.cu: the keys are the rows of S^T = K Q^T and
// V's channels those of O^T = V^T P^T, the query heads, of which a kv head has mostly eight or fewer, the eight columns (up to 16 heads: two products from
// the same K and V). e4m3 is exact in fp16. A lane's four bytes of K are four channels side by side of one key: Q's channels are taken in that order.
// Two rows of V are turned by ldmatrix two bytes at a time, so that a lane has two channels of two keys, rows g and g + 8 of the product. The weights are
// turned by movmatrix.
//
// fp16 has eleven bits but a short range, which powers of two see to: a head's q is brought to [2^14, 2^15); a weight for the product is 2^(x - r) sv 2^14,
// r following the largest x + log2(sv) of the warp's keys within a factor of 2, so that what fp16 cuts off, below 2^-24, is 2^-38 of the largest. The sum
// has a reference of its own and is that of the unrounded weights. bf16 caches: q (eight bits) is so exact, a weight off by 2^-11. fp32 ones: q and
// the weights as two fp16 numbers each, and parts of 16 or 32 terms are added by ordinary additions (the tensor core's own sums are cut).
//
// The keys of all slots and heads lie in one row, as in decode.cu, in units of 32; a CTA's share of it is cut in four once more, a warp's each, and the
// warps walk alone, tile by tile of 32 keys (one a lane where pages are looked up), without a barrier until all are done. (Four warps that shared every segment: 52.9 us
// for 64 slots of up to 8192 tokens, 87.5 for four of up to 131072, the warps waiting for one another at every segment's end; so: 41.6, 68.8.) The
// ring is fed a segment ahead: the next one's first tiles come while this one's last are multiplied (35.9, 61.7), and a tile that is all there takes
// the short way through the addresses (33, 60). Then the warps' pieces of an owner meet, and what is not all of it is left to the joins.
//
// What bounds it: rows of 128 bytes that lie a token apart. Four slots of up to 131072 tokens, 32 / 8 heads, d = 128: 273 MB in 60 us, 69 % of the copy
// rate (6556 GB/s), with head after head within a page 52 us, 80 %; the rest is the way to the first tile (4 us) and the joins. Tried: three CTAs an SM
// with rings of two tiles (64 us), a prefetch of 256 bytes to L2 with each row (73), two kv heads whose rows lie side by side walked by one warp (57, but 36 for the
// 64 slots, for 33, and 12.7 for 10 where one slot of 1219 is all: twice the registers, half the owners). 16 query heads a kv head (32 / 2 heads): 64 slots of up to 8192
// tokens 28.9 us in bf16, d = 128, 62 in bf16, d = 256, 107 in fp32, d = 256, the last two with 0.7 to 1.6 KB of spilled registers a thread.
#include <cuda_fp16.h>

#include "decode.cuh"

namespace stream {
namespace {

using namespace decode;

constexpr int kWarps = kThreads / 32;
constexpr int kStep = 32;            // keys of a warp's tile: one a lane where pages are looked up. And the keys of a unit
// What a segment costs a warp beside its keys, in units. (us with 1, 2, 3, 4, 5, 64 slots of up to 8192 tokens: 37.9, 33.7, 33.0, 32.9, 32.8; four of up to
// 131072: 69.0, 60.3, 60.4, 60.2, 60.4.)
constexpr int kOpen = 3;
constexpr float kOutgrown = 30.f;    // log2: of the sum's reference
constexpr float kTop = 14.f;         // log2: a weight for the product where it is the largest, times its value's scale
constexpr float kNone = -3e38f;      // a reference before the first key, finite so that it has differences
constexpr float kLeastScale = 7.8886090522101181e-31f;  // 2^-100: of a value's scale, for the reference (a smaller one, 0 or NaN counts as this there)

template <class T, int D, int N>
struct Form {
    static constexpr bool kPair = sizeof(T) == 4;               // two fp16 numbers an operand
    static constexpr int kParts = kPair ? 2 : 1;
    static constexpr int kPieces = D / 16;                      // of 16 bytes of a row, and steps of K Q^T
    static constexpr int kTile = kStep * D;                     // bytes
    static constexpr int kPlace = 2 * kTile + 2 * kStep * 4;    // K, V, the keys' scales
    static constexpr int kHeads = 8 * N;
    static constexpr bool kQInRegs = kParts * N * kPieces <= 16;
    static constexpr bool kQEarly = !kPair && N * kPieces <= 8; // the next segment's q is in registers beside the present one
    static constexpr int kStages = D == 256 ? (kQInRegs ? 3 : 2) : D == 128 ? 3 : D == 64 ? 5 : 8;
    static constexpr int kCtas = D == 256 || (D == 128 && !kQInRegs) ? 1 : 2;  // of an SM
    static constexpr int kLeave = (2 * kMaxHeads + kHeads * D) * 4;    // bytes of a piece: m, l, O
    static_assert(kLeave <= kStages * kPlace, "a warp's last piece in its ring");
    // the first pieces of the warps but the first beside the rings, where shared memory is large enough, else in a place of the warp's ring
    static constexpr bool kFirstBeside = kCtas * (kWarps * kStages * kPlace + (kWarps - 1) * kLeave + (kQInRegs ? 0 : kWarps * kParts * kPieces * N * 256) + 2048) <= 233472;
    static_assert(kFirstBeside || (kLeave <= kPlace && kStages > 1), "a warp's first piece in a place of its ring");
};
// A piece of an owner that a warp leaves to its CTA.
struct Piece {
    const float *at;      // m, l, O as in Args::parts
    long long owner_end;
    int slot, h0, heads;  // slot < 0: there is no piece
    int starts, ends;     // with the owner's first key, its last
};
template <class T, int D, int N>
struct Smem {
    using F = Form<T, D, N>;
    unsigned char ring[kWarps][F::kStages * F::kPlace];
    uint2 q[kWarps][F::kQInRegs ? 1 : F::kParts * F::kPieces * N * 32];  // what a lane multiplies with
    float first[F::kFirstBeside ? kWarps - 1 : 1][F::kFirstBeside ? F::kLeave / 4 : 1];
    Piece piece[2 * kWarps];
    unsigned there[kWarps][F::kStages];  // the keys of each place that are there
    int n_parts;   // that the first warp has left to the joins
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

// Four channels of a query head, as they lie in memory.
template <class T>
struct Four { unsigned w[sizeof(T)]; };
template <class T>
__device__ __forceinline__ Four<T> load_four(const T *p, bool vec) {
    Four<T> r;
    if constexpr (sizeof(T) == 4) {
        const uint4 x = vec ? *reinterpret_cast<const uint4 *>(p)
                            : make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
        r.w[0] = x.x; r.w[1] = x.y; r.w[2] = x.z; r.w[3] = x.w;
    } else {
        const uint2 x = vec ? *reinterpret_cast<const uint2 *>(p) : wp::load4(p);
        r.w[0] = x.x; r.w[1] = x.y;
    }
    return r;
}
template <class T>
__device__ __forceinline__ void widen(const Four<T> &f, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(f.w[i]);
        else x[i] = __uint_as_float(i & 1 ? f.w[i >> 1] & 0xffff0000u : f.w[i >> 1] << 16);
    }
}

// What a warp gathers of a segment. A lane (g = lane / 4, t = lane % 4) has the heads 8 n + 2 t and 8 n + 2 t + 1, of a tile the keys g + 8 i, and of O
// the channels 16 c + 2 g and 16 c + 2 g + 1. As a column of K Q^T it has the channels 16 c + 4 t ... of the heads 8 n + g.
template <class T, int D, int N>
struct Walk {
    using F = Form<T, D, N>;
    static constexpr int kParts = F::kParts;
    unsigned q[kParts][F::kQInRegs ? F::kPieces : 1][N][2];
    float o[F::kPieces][N][4], unit[N][2], ref[N][2], top[N][2], l[N][2];  // ref: of the sum, top: of the weights for the product; units of log2

    __device__ __forceinline__ void begin(Smem<T, D, N> &sm, int warp, const Four<T> (&raw)[F::kPieces][N], float scale_log2, int lane) {
#pragma unroll
        for (int n = 0; n < N; ++n) {  // q times a power of two, in [2^14, 2^15) at its largest
            float most = 0.f, x[4];
#pragma unroll
            for (int c = 0; c < F::kPieces; ++c) {
                widen(raw[c][n], x);
                most = fmaxf(most, fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))));
            }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int up = min(max(141 - (int)(__float_as_uint(most) >> 23), -114), 126);
            const float f = __uint_as_float((unsigned)(up + 127) << 23);
#pragma unroll
            for (int c = 0; c < F::kPieces; ++c) {
                widen(raw[c][n], x);
                unsigned r[kParts][2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float a = x[2 * y] * f, b = x[2 * y + 1] * f;
                    r[0][y] = pack(a, b);
                    if constexpr (F::kPair) {
                        const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&r[0][y]));
                        r[kParts - 1][y] = pack(a - h.x, b - h.y);
                    }
                }
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    if constexpr (F::kQInRegs) {
                        q[p][F::kQInRegs ? c : 0][n][0] = r[p][0];
                        q[p][F::kQInRegs ? c : 0][n][1] = r[p][1];
                    } else {
                        sm.q[warp][F::kQInRegs ? 0 : ((p * F::kPieces + c) * N + n) * 32 + lane] = make_uint2(r[p][0], r[p][1]);
                    }
                }
            }
            const float worth = scale_log2 / f;  // a logit of this q
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                unit[n][y] = __shfl_sync(0xffffffffu, worth, 8 * (lane & 3) + 4 * y);
                ref[n][y] = top[n][y] = kNone;
                l[n][y] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < F::kPieces; ++c)
#pragma unroll
                for (int y = 0; y < 4; ++y) o[c][n][y] = 0.f;
        }
    }

    // A tile: K, V behind it, then the keys' scales and the values'; the keys that it has tokens for. Keys g, g + 8, g + 16 and g + 24 of it are this lane's.
    __device__ __forceinline__ void step(const Smem<T, D, N> &sm, int warp, unsigned char *tile, const unsigned *there, int lane) {
        const unsigned kt = wp::smem_addr(tile), vt = kt + F::kTile;
        const float *const z = reinterpret_cast<const float *>(tile + 2 * F::kTile);
        float s[N][2][4];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 8; ++y) s[n][y >> 2][y & 3] = 0.f;
#pragma unroll
        for (int c = 0; c < F::kPieces; ++c) {
            unsigned w[4];
            wp::ldmatrix4(kt + piece_at<D>(lane, c), w);
            unsigned b[kParts][N][2];
#pragma unroll
            for (int p = 0; p < kParts; ++p)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    if constexpr (F::kQInRegs) {
                        b[p][n][0] = q[p][F::kQInRegs ? c : 0][n][0];
                        b[p][n][1] = q[p][F::kQInRegs ? c : 0][n][1];
                    } else {
                        const uint2 x = sm.q[warp][F::kQInRegs ? 0 : ((p * F::kPieces + c) * N + n) * 32 + lane];
                        b[p][n][0] = x.x;
                        b[p][n][1] = x.y;
                    }
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // 16 keys
                const unsigned a0 = widen_low(w[2 * i]), a2 = widen_high(w[2 * i]), a1 = widen_low(w[2 * i + 1]), a3 = widen_high(w[2 * i + 1]);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
                    float(&to)[4] = F::kPair ? part : s[n][i];
#pragma unroll
                    for (int p = kParts - 1; p >= 0; --p) mma_f16(to, a0, a1, a2, a3, b[p][n][0], b[p][n][1]);  // (the small parts first)
                    if constexpr (F::kPair) {
#pragma unroll
                        for (int y = 0; y < 4; ++y) s[n][i][y] += part[y];
                    }
                }
            }
        }
        float sk[4], sv[4], lv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sk[k] = z[(lane >> 2) + 8 * k];
            sv[k] = z[kStep + (lane >> 2) + 8 * k];
            lv[k] = log2_of(fmaxf(sv[k], kLeastScale));
        }
        const bool lacks = sk[0] == 0.f || sk[1] == 0.f || sk[2] == 0.f || sk[3] == 0.f;  // keys that are not there
        bool outgrown = false;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float a = -CUDART_INF_F, b = -CUDART_INF_F;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float &x = s[n][k >> 1][2 * (k & 1) + y];
                    x *= unit[n][y] * sk[k];
                    a = fmaxf(a, x);
                    b = fmaxf(b, x + lv[k]);
                }
                outgrown = outgrown || a > ref[n][y] + kOutgrown || b > top[n][y] + (kTop + 1.f);
            }
        bool moves = __any_sync(0xffffffffu, lacks || outgrown);
        if (moves) {
            moves = __any_sync(0xffffffffu, outgrown);
            // what is not there, whatever its bytes and its value's scale are (NaN times a weight of zero would be NaN)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (sk[k] == 0.f) {
                    sv[k] = 1.f;
                    lv[k] = 0.f;
#pragma unroll
                    for (int n = 0; n < N; ++n) s[n][k >> 1][2 * (k & 1)] = s[n][k >> 1][2 * (k & 1) + 1] = -CUDART_INF_F;
                }
            const unsigned unset = __ballot_sync(0xffffffffu, z[lane] == 0.f) & *there;
            if (unset != 0) {  // (what the tile has no token for is zeros)
#pragma unroll
                for (int i = 0; i < F::kPieces; ++i) {
                    const int at = (i * 32 + lane) * 16;
                    if ((unset >> (at / D)) & 1u) *reinterpret_cast<uint4 *>(tile + F::kTile + at) = make_uint4(0, 0, 0, 0);
                }
                __syncwarp();
            }
        }
        if (moves) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float a = -CUDART_INF_F, b = -CUDART_INF_F;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        a = fmaxf(a, s[n][k >> 1][2 * (k & 1) + y]);
                        b = fmaxf(b, s[n][k >> 1][2 * (k & 1) + y] + lv[k]);
                    }
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
                        b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, d));
                    }
                    a = fmaxf(a, ref[n][y]);
                    b = fmaxf(b - kTop, top[n][y]);
                    l[n][y] *= fast_exp2(ref[n][y] - a);
                    const float f = fast_exp2(top[n][y] - b);
                    ref[n][y] = a;
                    top[n][y] = b;
#pragma unroll
                    for (int c = 0; c < F::kPieces; ++c) { o[c][n][y] *= f; o[c][n][y + 2] *= f; }
                }
        }
        unsigned p[kParts][N][4];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float w[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float x = s[n][k >> 1][2 * (k & 1) + y];
                    l[n][y] += fast_exp2(x - ref[n][y]);
                    w[y] = fast_exp2(x - top[n][y]) * sv[k];
                }
                const unsigned hi = pack(w[0], w[1]);
                p[0][n][k] = turned(hi);
                if constexpr (F::kPair) {
                    const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
                    p[kParts - 1][n][k] = turned(pack(w[0] - h.x, w[1] - h.y));
                }
            }
#pragma unroll
        for (int c = 0; c < F::kPieces; ++c) {
            unsigned w[4];
            wp::ldmatrix4_t(vt + piece_at<D>(lane, c), w);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __byte_perm(w[i], 0, 0x3120);  // two channels of one key, two of the next: two keys of one channel, two of the other
            float part[N][4] = {};
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // 16 keys
                const unsigned a0 = widen_low(w[2 * i]), a1 = widen_high(w[2 * i]), a2 = widen_low(w[2 * i + 1]), a3 = widen_high(w[2 * i + 1]);
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int y = kParts - 1; y >= 0; --y) mma_f16(F::kPair ? part[n] : o[c][n], a0, a1, a2, a3, p[y][n][2 * i], p[y][n][2 * i + 1]);
            }
            if constexpr (F::kPair) {
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int y = 0; y < 4; ++y) o[c][n][y] += part[n][y];
            }
        }
    }

    // m, l and O = sum_t 2^(x - m) v
    __device__ __forceinline__ void leave(float *to, int lane) {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int h = 8 * n + 2 * t + y;
                if (g == 0) { to[h] = ref[n][y] == kNone ? -CUDART_INF_F : ref[n][y]; to[kMaxHeads + h] = l[n][y]; }
#pragma unroll
                for (int c = 0; c < F::kPieces; ++c)
                    *reinterpret_cast<float2 *>(to + 2 * kMaxHeads + h * D + 16 * c + 2 * g) = make_float2(o[c][n][y], o[c][n][y + 2]);
            }
    }
    // l of all keys, and O to l's reference.
    __device__ __forceinline__ void close() {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][y] += __shfl_xor_sync(0xffffffffu, l[n][y], d);
                const float f = fast_exp2(top[n][y] - ref[n][y]);  // (1 where no key was there)
#pragma unroll
                for (int c = 0; c < F::kPieces; ++c) { o[c][n][y] *= f; o[c][n][y + 2] *= f; }
            }
    }
    // The output of a segment with all of its owner's keys; row: of its first head.
    __device__ __forceinline__ void write(const Args &A, long long row, int heads, bool pairs, int lane) {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int h = 8 * n + 2 * t + y;
                if (h >= heads) continue;
                const float inv = l[n][y] > 0.f ? 1.f / l[n][y] : 0.f;
                T *const to = (T *)A.a.out + (row + h) * D + 2 * g;
#pragma unroll
                for (int c = 0; c < F::kPieces; ++c) {
                    const float a = o[c][n][y] * inv, b = o[c][n][y + 2] * inv;
                    if (!pairs) {
                        to[16 * c] = (T)a;
                        to[16 * c + 1] = (T)b;
                    } else if constexpr (F::kPair) {
                        *reinterpret_cast<float2 *>(to + 16 * c) = make_float2(a, b);
                    } else {
                        *reinterpret_cast<__nv_bfloat162 *>(to + 16 * c) = __floats2bfloat162_rn(a, b);
                    }
                }
                if (g == 0 && A.a.lse != nullptr) A.a.lse[row + h] = lse_of(ref[n][y], l[n][y]);
            }
    }
};

__device__ __forceinline__ void cp_async16_whole(unsigned dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Waits until no more than `pending` of the last kMost groups of copies are on their way.
template <int kMost>
__device__ __forceinline__ void wait_for(unsigned pending) {
    if constexpr (kMost == 0) {
        wp::cp_async_wait<0>();
    } else {
        if (pending >= kMost) wp::cp_async_wait<kMost>();
        else wait_for<kMost - 1>(pending);
    }
}

struct Args8 {
    Args A;
    Scales sc;
    Divisor page, block;
    int vec;   // rows of the cache are read in pieces of 16 bytes
    int pairs; // the output is written two elements at a time
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
    // the share of a CTA, and of it a warp's: a quarter of the places
    const long long all = all_places<W, kStep, kOpen>(A, lane);
    const unsigned n_warps = (unsigned)A.grid * kWarps;
    const long long per_warp = all >> 31 == 0 ? ((unsigned)all + n_warps - 1) / n_warps : (all + n_warps - 1) / n_warps;
    const Share mine = {per_warp * kWarps, min(all, per_warp * kWarps * blockIdx.x), min(all, per_warp * kWarps * (blockIdx.x + 1))};
    const long long first = min(all, mine.first + per_warp * warp), end = min(all, mine.first + per_warp * (warp + 1));
    unsigned char *const ring_ptr = sm.ring[warp];
    const unsigned ring = wp::smem_addr(ring_ptr);
    const bool plain = c.page % 16 == 0 && B.vec != 0;  // 16 keys of a tile lie side by side, in pieces of 16 bytes
    constexpr int kPieces = F::kPieces, kRowsAtOnce = 32 / kPieces;  // rows that 32 lanes fetch at once
    const int row_l = lane / kPieces, piece_l = lane % kPieces;
    unsigned bad = 0;

    // What is fetched: one tile after the other of one segment after the other, up to kStages tiles and a segment ahead of the one that is
    // multiplied, so that a segment's first tiles come while the one before it is finished and written out.
    struct Source {
        const int32_t *table;
        int slot, kvh, key0, key_end, n_steps;
        Seen seen;
    } src = {};
    int src_n = 0;                      // the step of it that is fetched next
    int page = -1, row = 0;             // lane i: the page of key i of that step, -1: none; and its row there
    unsigned put = 0, take = 0, ahead = 0;  // the ring's places that are filled next, and multiplied next; how many are filled
    unsigned held = F::kStages;             // the place that has the warp's first piece, if one has
    auto behind = [&](unsigned place) {
        place = place + 1 == F::kStages ? 0 : place + 1;
        if (!F::kFirstBeside && place == held) place = place + 1 == F::kStages ? 0 : place + 1;
        return place;
    };
    auto look_up = [&](const Source &f, int n, int &to, int &to_row) {
        const int walked = f.key0 + n * kStep + lane, key = W ? f.seen.key(walked) : walked;
        to = -1;
        if (walked >= f.key_end) return;
        const unsigned nth = B.page.quotient((unsigned)key);
        to_row = key - (int)(nth * B.page.d);
        to = f.table[nth];
        if ((unsigned)to >= (unsigned)c.n_pages) {
            to = -1;
            if (!W || f.seen.sees(key)) bad = (unsigned)f.slot + 1u;
        }
    };
    auto source_of = [&](const Segment &sg) {
        Source f;
        f.table = c.table + (long long)sg.slot * c.max_pages;
        f.slot = sg.slot;
        f.kvh = sg.kvh;
        f.key0 = sg.key0;
        f.key_end = sg.key_end;
        f.n_steps = (sg.key_end - sg.key0 + kStep - 1) / kStep;
        if constexpr (W) f.seen = seen_of<W, kStep>(A.a, sg.slot);
        return f;
    };
    auto fetch = [&] {  // the next tile of src, and the pages of the one after it are looked up
        const int own_page = page, own_row = row;
        if (src_n + 1 < src.n_steps) look_up(src, src_n + 1, page, row);
        const bool mine = own_page >= 0 && (!W || src.seen.sees(src.seen.key(src.key0 + src_n * kStep + lane)));
        const unsigned there = __ballot_sync(0xffffffffu, mine);
        const long long own = own_page >= 0 ? (long long)own_page * c.s_p + (long long)own_row * c.s_t : 0;
        const long long z = mine ? (long long)own_page * B.sc.s_p + (long long)B.block.quotient((unsigned)own_row) * B.sc.s_b + src.kvh * B.sc.s_h : 0;
        const unsigned to = ring + put * F::kPlace;
        cp_async4_or_zero(to + 2 * F::kTile + lane * 4, B.sc.k + z, mine ? 4 : 0);
        cp_async4_or_zero(to + 2 * F::kTile + kStep * 4 + lane * 4, B.sc.v + z, mine ? 4 : 0);
        if (lane == 0) sm.there[warp][put] = there;
        const long long head = src.kvh * c.s_h + piece_l * 16;
        if (plain && there == 0xffffffffu) {
#pragma unroll
            for (int half = 0; half < (kRowsAtOnce > 16 ? 1 : 2); ++half) {
                const long long base = __shfl_sync(0xffffffffu, own, kRowsAtOnce > 16 ? lane & 16 : half * 16) + head + (row_l & 15) * c.s_t;
                const unsigned char *ks = (const unsigned char *)A.a.k + base, *vs = (const unsigned char *)A.a.v + base;
#pragma unroll
                for (int r0 = half * 16; r0 < (kRowsAtOnce > 16 ? 32 : half * 16 + 16); r0 += kRowsAtOnce) {
                    const unsigned at = to + piece_at<D>(r0 + row_l, piece_l);
                    cp_async16_whole(at, ks);
                    cp_async16_whole(at + F::kTile, vs);
                    ks += kRowsAtOnce * c.s_t;
                    vs += kRowsAtOnce * c.s_t;
                }
            }
        } else {
#pragma unroll 1
            for (int r0 = 0; r0 < kStep; r0 += kRowsAtOnce) {
                const int r = r0 + row_l;
                const long long e0 = __shfl_sync(0xffffffffu, own, r);
                const bool is = (there >> r) & 1u;
                const long long e = is ? e0 + head : 0;
                const unsigned char *const ks = (const unsigned char *)A.a.k + e, *const vs = (const unsigned char *)A.a.v + e;
                const unsigned at = put * F::kPlace + piece_at<D>(r, piece_l);
                if (B.vec) {
                    wp::cp_async16(ring + at, ks, is ? 16 : 0);
                    wp::cp_async16(ring + at + F::kTile, vs, is ? 16 : 0);
                } else {
#pragma unroll 1
                    for (int i = 0; i < 16; ++i) {
                        ring_ptr[at + i] = is ? ks[i] : 0;
                        ring_ptr[at + F::kTile + i] = is ? vs[i] : 0;
                    }
                }
            }
        }
        wp::cp_async_commit();
        put = behind(put);
        ++ahead;
        ++src_n;
    };
    Four<T> raw[F::kPieces][N];
    auto load_q = [&](const Segment &sg) {
        const T *const src = (const T *)A.a.q + (long long)sg.slot * A.a.qs_s + (long long)(sg.h0 + (lane >> 2)) * A.a.qs_h + 4 * (lane & 3);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int c = 0; c < F::kPieces; ++c)
                raw[c][n] = 8 * n + (lane >> 2) < sg.heads ? load_four<T>(src + 8 * n * A.a.qs_h + 16 * c, A.q_vec != 0) : Four<T>{};
    };
    Place pl = {0, 0, 0};
    int n_pieces = 0;
    if (lane < 2) sm.piece[2 * warp + lane].slot = -1;
    if (tid == 0) sm.n_parts = 0;
    __syncwarp();
    // (Every part of the work stands once in the code: its first pass comes from cold instruction caches.)
    Segment sg = {};
    sg.next = first;
    for (bool begun = false; ; begun = true) {
        // the segment behind sg, and the pages of its first tile
        const Segment next = open_segment<W, kStep, kOpen>(A, sg.next, end, lane, pl);
        bool waits = next.next >= 0;  // it is not yet fetched from
        int next_page = -1, next_row = 0;
        Source follows = {};
        if (waits) {
            follows = source_of(next);
            look_up(follows, 0, next_page, next_row);
        }
        auto go_on = [&] {
            waits = false;
            src = follows;
            src_n = 0;
            page = next_page;
            row = next_row;
        };
        if (!begun) {
            if (!waits) break;
            go_on();
            if constexpr (F::kQInRegs) load_q(next);
            sg = next;
            continue;
        }
        if constexpr (!F::kQInRegs) load_q(sg);
        Walk<T, D, N> walk;
        const int n_steps = (sg.key_end - sg.key0 + kStep - 1) / kStep;
        for (int n = 0; n < n_steps; ++n) {
            while (ahead < (F::kFirstBeside || held == F::kStages ? F::kStages : F::kStages - 1)) {
                if (src_n == src.n_steps) {
                    if (!waits) break;
                    go_on();
                }
                fetch();
            }
            if (n == 0) {
                walk.begin(sm, warp, raw, A.a.scale_log2, lane);
                if (F::kQEarly && next.next >= 0) load_q(next);
                __syncwarp();
            }
            wait_for<F::kStages - 1>(ahead - 1);  // copies that may still be on their way: those of later tiles
            __syncwarp();
            walk.step(sm, warp, ring_ptr + take * F::kPlace, &sm.there[warp][take], lane);
            __syncwarp();  // (the tile is read before its place is filled again)
            take = behind(take);
            --ahead;
        }
        if (waits) go_on();
        if (F::kQInRegs && !F::kQEarly && next.next >= 0) load_q(next);
        walk.close();
        const long long to_row = (long long)sg.slot * A.a.H + sg.h0;
        if (sg.whole) {
            walk.write(A, to_row, sg.heads, B.pairs != 0, lane);
        } else {
            // The warp's first segment or its last one, which stays in the ring: that is done with. A first one that others follow ends its owner: the
            // first warp's began in another CTA and is left to the joins as it is. Where another one's has no room beside the rings it takes the
            // place that is filled next, which is empty, and the others go round without it (a warp that has met an owner's end has a tile
            // less ahead: bf16, d = 128 and fp32, d = 256 with more than eight heads).
            const bool last = next.next < 0;
            float *to;
            if (last) {
                to = reinterpret_cast<float *>(ring_ptr + (!F::kFirstBeside && held == 0 ? F::kPlace : 0));
            } else if (warp == 0) {
                to = part_of(A, (int)blockIdx.x, 0);
            } else if constexpr (F::kFirstBeside) {
                to = sm.first[warp - 1];
            } else {
                held = put;
                to = reinterpret_cast<float *>(ring_ptr + held * F::kPlace);
                put = behind(put);
                if (take == held) take = put;
            }
            walk.leave(to, lane);
            if (!last && warp == 0) {
                if (lane == 0) sm.n_parts = 1;
            } else {
                if (lane == 0) sm.piece[2 * warp + n_pieces] = {to, sg.owner_end, sg.slot, sg.h0, sg.heads, sg.key0 == 0, sg.next == sg.owner_end};
                ++n_pieces;
            }
        }
        if (next.next < 0) break;
        sg = next;
    }
    __syncthreads();
    // The warps' pieces side by side: those of one owner are joined, and what is not all of it is left to the joins (two at most)
    int n_parts = sm.n_parts;
    Left left = {};
    for (int k0 = 0, k1; k0 < 2 * kWarps; k0 = k1) {
        const Piece p = sm.piece[k0];
        int ends = p.ends;
        for (k1 = k0 + 1; k1 < 2 * kWarps; ++k1) {
            const Piece &o = sm.piece[k1];
            if (o.slot >= 0 && (o.slot != p.slot || o.h0 != p.h0)) break;
            if (o.slot >= 0) ends = o.ends;
        }
        if (p.slot < 0) { k1 = k0 + 1; continue; }
        const bool whole = p.starts && ends;
        const long long to_row = (long long)p.slot * A.a.H + p.h0;
        float *const part = part_of(A, (int)blockIdx.x, n_parts);
        if (!whole) {
            if (p.starts) left = {pieces_of(p.owner_end, mine), n_parts, p.heads, 0u, to_row, 0ll};
            ++n_parts;
        }
        for (int e = tid; e < p.heads * (D / 4); e += kThreads) {
            const int h = e / (D / 4), x = (e % (D / 4)) * 4;
            float m = -CUDART_INF_F, sum = 0.f;
            for (int k = k0; k < k1; ++k)
                if (sm.piece[k].slot >= 0) m = fmaxf(m, sm.piece[k].at[h]);
            const float base = m == -CUDART_INF_F ? 0.f : m;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = k0; k < k1; ++k)
                if (sm.piece[k].slot >= 0) {
                    const float *const a = sm.piece[k].at;
                    const float f = fast_exp2(a[h] - base);
                    const float4 z = *reinterpret_cast<const float4 *>(a + 2 * kMaxHeads + h * D + x);
                    sum = fmaf(f, a[kMaxHeads + h], sum);
                    y.x = fmaf(f, z.x, y.x); y.y = fmaf(f, z.y, y.y); y.z = fmaf(f, z.z, y.z); y.w = fmaf(f, z.w, y.w);
                }
            if (whole) {
                const float inv = sum > 0.f ? 1.f / sum : 0.f;
                T *const to = out + (to_row + h) * D + x;
                to[0] = (T)(y.x * inv); to[1] = (T)(y.y * inv); to[2] = (T)(y.z * inv); to[3] = (T)(y.w * inv);
                if (x == 0 && A.a.lse != nullptr) A.a.lse[to_row + h] = lse_of(m, sum);
            } else {
                *reinterpret_cast<float4 *>(part + 2 * kMaxHeads + h * D + x) = y;
                if (x == 0) { part[h] = m; part[kMaxHeads + h] = sum; }
            }
        }
    }
    leave_to_joins(A, left, bad);
}

template <class T, int D, int N, bool W>
cudaError_t launch(Args8 &B, int n_sm, cudaStream_t st) {
    const int smem = (int)sizeof(Smem<T, D, N>);
    static_assert(Form<T, D, N>::kCtas * (sizeof(Smem<T, D, N>) + 1024 + 256) <= 233472, "what an SM has");
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
    B.A = args_of(a, workspace, n_sm, kStep, kOpen, kWarps);
    B.sc = sc;
    B.page = make_divisor(a.c.page);
    B.block = make_divisor(sc.block);
    const int e = dtype == STREAM_F32 ? 4 : 2;
    B.A.q_vec = ((uintptr_t)a.q & (4 * e - 1)) == 0 && ((a.qs_s | a.qs_h) & 3) == 0 ? 1 : 0;
    B.pairs = ((uintptr_t)a.out & (2 * e - 1)) == 0 ? 1 : 0;
    B.vec = (((uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0 && ((a.c.s_p | a.c.s_t | a.c.s_h) & 15) == 0 ? 1 : 0;
    cudaError_t rc = dtype == STREAM_F32 ? launch_d<float>(B, n_sm, st) : launch_d<__nv_bfloat16>(B, n_sm, st);
    if (rc != cudaSuccess) return cuda_fail(rc, "8-bit decode attention launch");
    rc = launch_joins(B.A, dtype, st);
    return rc == cudaSuccess ? STREAM_OK : cuda_fail(rc, "decode join launch");
}

}  // namespace stream
