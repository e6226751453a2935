// Dense attention of packed prompts on the 5th-generation tensor cores: bf16, d = 64 or 128.
//
// A row is a token and a query head; the rows of a kv head's queries lie token by token, so that a tile of 128 rows is
// 128 / hpg tokens of all hpg query heads of the group: the heads share every key tile, short sequences fill the rows, and the causal
// border cuts few tokens. One persistent CTA per SM has an item at a time: two such tiles, X = 0 and 1, which walk the
// sequence's keys together in tiles of 128:
//     S_X = Q_X K_j^T  (128 x 128, both from shared memory),     O_X += P_X V_j  (P from TMEM, in the columns of S_X).
// While the tensor core multiplies for one tile, four warps compute P = 2^(scale (s - ref)) of the other, a thread a row. `ref` is
// the row's maximum at the first key tile, moved (with O and the sum, which are multiplied by 2^(scale (old - new))) only when a
// later one has outgrown it by more than 2^30: fp32 sums and bf16 weights keep their relative precision whatever the reference.
// P is rounded to bf16 for the product (2^-8 of a weight at most, as the bf16 output is in the end); the sum l is that of the unrounded
// weights in fp32, and so exact enough for the logarithm that is returned.
//
// Order of the issuing warp, per key tile: P_0 V_j, Q_0 K_(j+1), P_1 V_j, Q_1 K_(j+1). MMAs of one thread run in order, so that S_X
// may overwrite P_X behind its product, and a tile's logits being there says that its last product is, too.
//
// Where there is a window, a pair of tiles walks the sinks and then, behind a gap, the keys from the first row's window on, wherever that begins. Up to 16 sinks
// are the first rows of the first tile (which comes in pieces of 16 rows), more of them have tiles of their own. 12 prompts of up to 4500 tokens, 28 / 4 heads,
// window 1024, 4 sinks: 149 us (with a tile for the sinks 161); 32768 tokens, 32 / 8 heads, window 4096: 1620 us, 1280 TFLOP/s of the pairs that are seen.
// An item of the 12 prompts has nine key tiles (1075 keys) and costs 3 us beside them: the way from the last product over the output to the next item's first weights.
//
// Roles (384 threads): warp 0 loads Q, K and V by TMA (one ring for K and V, in the order of their use); warp 1 issues the MMAs and
// owns TMEM; warp 2 writes zeros over the rows of a V tile behind the sequence's last key (a weight of zero times what lies
// there, which may be anything, has to be zero); warps 4..7 and 8..11 are the softmax of the two tiles and store their output.
// A row's 128 logits stay in registers. Every wait is bounded, or for a role whose waits are.
#include <math_constants.h>

#include "serve_common.cuh"
#include "tc_common.cuh"

namespace stream {

// Status words of this kernel: 0, or the code of the bounded wait that ran out (with the block index beside it).
__device__ unsigned int g_prompt_status[2];

namespace {

using namespace tc;

constexpr int kThreads = 384;
constexpr int kRows = 128, kKeys = 128;  // of a tile
constexpr int kFewSinks = 16;            // rows of a box of the tile that sinks share with others
constexpr int kMaxSeqs = 256;            // of a launch
constexpr int kKnown = 64;               // items of a CTA that are worked out once (each role would take some 2000 cycles for each of them)
constexpr int kMaxLevels = 2048;         // items of a kv head that are put in order
constexpr long long kMaxItems = 0x7fffffffll - (1 << 20);
constexpr float kOutgrown = 30.f;        // log2
// K and V bytes of the kv heads whose items are walked together, of the 126 MB of L2; of this kernel, which reads every key tile (the sparse passes have kL2KvBytes) (32 / 8 heads, TFLOP/s: 131072 tokens, all heads
// 1094 to 1117, one at a time 1202 to 1217; 65536, all 1196 to 1219, two 1193 to 1207, three 1250 to 1268; 16384 in halves 1285 for 1372).
constexpr long long kKvInL2 = 110ll << 20;

template <int D_>
struct Form {
    static constexpr int D = D_, kHalves = D / 64;
    static constexpr int kHalf = 128 * 128;              // 128 rows of 64 channels
    static constexpr int kTile = kHalves * kHalf;        // of Q, K or V
    static constexpr int kStages = D == 128 ? 4 : 8;     // K and V tiles in flight
    static constexpr int kSCol = 0, kOCol = 256;         // TMEM: S_X at 128 X (P_X in its first 64 columns), O_X at 256 + 128 X
    static constexpr unsigned kIdescQK = idesc_bf16(128, 128, false), kIdescPV = idesc_bf16(128, D, true);
};
constexpr unsigned kHi = desc_hi_sw128(1024);

struct Seq { int q_first, q_n, k_first, k_n; };

// What a CTA works on.
struct Item {
    Seq s;
    int kvh, tok0;        // the first tile's first token; the second one's is per_tile later
    int n[2];             // key tiles of each; -1: there is no such tile
    int most;             // of both
    Walked wk;            // (where there is a window)
};

template <class F>
struct Tail {
    unsigned long long full[F::kStages], empty[F::kStages];
    unsigned long long v_raw[F::kStages];                // a V tile that needs zeros is there
    unsigned long long q_full[2], q_free[2];
    unsigned long long s_full[2], p_half[2][2];          // P's first and last 64 keys
    unsigned long long o_done[2], o_free[2];
    unsigned int tmem_base;
    int abort_flag;
    int n_levels, n_items;                               // items of a kv head; of all
    int sorted;                                          // `order` holds the items of a kv head
    unsigned order[kMaxLevels];                          // sequence << 12 | level, the most keys first
    Seq seq[kMaxSeqs];                                   // the longest first
    int level_end[kMaxSeqs];                             // levels (pairs of tiles, items of a kv head) of the sequences up to and with this one
    uint4 stage[8][128];                                 // of each softmax warp: 32 rows x 32 channels of the output
    Item items[kKnown];                                  // of this CTA: the first ones
};

struct Params {
    PromptGeom g;
    int sink_unit; // kFewSinks: the sinks share a tile with the window's first keys; kKeys: they have their own
    int per_tile;  // tokens of a tile: 128 / hpg
    int heads;     // kv heads whose items are walked together
};

// The key that column 0 of key tile j has, or would have if the sinks were not in its place.
template <bool W>
__device__ __forceinline__ int first_key(const Params &P, const Item &it, int j) {
    if constexpr (!W) return j * kKeys;
    return j * kKeys < it.wk.sink_keys && P.sink_unit == kKeys ? j * kKeys : j * kKeys + it.wk.gap;
}

// The first sequence whose levels end behind the nth.
template <class F>
__device__ __forceinline__ int sequence_of(const Tail<F> *tl, int n_seqs, int nth) {
    int lo = 0, hi = n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (tl->level_end[mid] > nth) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// (Not inline: in each role it costs registers that the softmax needs. With it in line, d = 64: 76 bytes of spilled stores for 20, 8192 tokens, 32 / 8
// heads, 368 us for 354, 64 prompts of 500 175 for 163; d = 128 the same with both.)
template <bool W, class F>
__device__ __noinline__ Item item_at(const Params &P, const Tail<F> *tl, int id) {
    const PromptGeom &g = P.g;
    Item it;
    // some kv heads at a time, and of them the sequences' levels (pairs of tiles) in order, head by head
    const unsigned per_phase = (unsigned)(tl->n_levels * P.heads), phase = P.heads == g.G ? 0 : (unsigned)id / per_phase, rem = (unsigned)id - phase * per_phase;
    const unsigned heads = (unsigned)min(P.heads, g.G - (int)phase * P.heads);
    const int nth = (int)(rem / heads);
    it.kvh = (int)(phase * P.heads + rem - nth * heads);
    int lo = 0, level;
    if (tl->sorted) {
        lo = (int)(tl->order[nth] >> 12);
        level = (int)(tl->order[nth] & 4095u);
    } else {
        lo = sequence_of(tl, g.n_seqs, nth);
        level = nth - (lo > 0 ? tl->level_end[lo - 1] : 0);
    }
    it.s = tl->seq[lo];
    const int pairs = ceil_div(it.s.q_n, 2 * P.per_tile);
    it.tok0 = (pairs - 1 - level) * 2 * P.per_tile;  // late tokens, with the most keys, first
    it.most = 0;
    it.wk = W ? walked_keys(g, P.sink_unit, it.tok0 + (it.s.k_n - it.s.q_n), it.s.k_n) : Walked{0, 0};
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int t0 = it.tok0 + x * P.per_tile;
        const int last = min(t0 + P.per_tile, it.s.q_n) - 1;
        const int keys = g.causal ? min(it.s.k_n, max(0, last + 1 + it.s.k_n - it.s.q_n)) : it.s.k_n;
        it.n[x] = t0 < it.s.q_n ? (int)(((long long)max(0, keys - it.wk.gap) + kKeys - 1) / kKeys) : -1;
        it.most = max(it.most, it.n[x]);
    }
    return it;
}

template <bool W, class F>
__device__ __forceinline__ Item nth_of_cta(const Params &P, const Tail<F> *tl, int round, int id) {
    if (round < kKnown) return tl->items[round];
    return item_at<W>(P, tl, id);
}

template <class F>
__device__ __forceinline__ bool wait_w(const void *bar, unsigned parity, Tail<F> *tl, unsigned code, long long limit = kWaitCycles) {
    return mbar_wait_warp(smem_u32(bar), parity, &tl->abort_flag, &g_prompt_status[0], &g_prompt_status[1], code, limit);
}
// For the roles that pass over items and may so wait for one that is far ahead, seconds long where the items in front are many and have
// a million keys: what they wait for comes from roles whose own waits are limited, and ends with their abort.
constexpr long long kWhileOthersWork = 1ll << 62;

// A place in the ring of K and V tiles: use u of it.
template <class F>
struct Use {
    unsigned u = 0;
    __device__ __forceinline__ unsigned stage() const { return u % F::kStages; }
    __device__ __forceinline__ unsigned phase() const { return (u / F::kStages) & 1u; }
};

template <bool W, class F>
__device__ void load_role(const Params &P, const CUtensorMap *tq, const CUtensorMap *tk, const CUtensorMap *tv, const CUtensorMap *few, Tail<F> *tl,
                          unsigned q_smem, unsigned ring) {
    Use<F> use;
    unsigned n_q[2] = {0, 0};
    auto kv = [&](const Item &it, const CUtensorMap *map, int j, bool raw) -> bool {
        if (!wait_w(&tl->empty[use.stage()], use.phase() ^ 1, tl, 1001)) return false;
        if (elect_one()) {
            const unsigned bar = smem_u32(raw ? &tl->v_raw[use.stage()] : &tl->full[use.stage()]), dst = ring + use.stage() * F::kTile;
            mbar_arrive_expect_tx(bar, F::kTile);
            if (W && j == 0 && P.sink_unit == kFewSinks && it.wk.gap > 0 && it.wk.sink_keys > 0) {
#pragma unroll 1
                for (int r = 0; r < kKeys; r += kFewSinks)
#pragma unroll
                    for (int c = 0; c < F::kHalves; ++c)
                        tma_load_4d(dst + c * F::kHalf + r * 128, few + (map == tv ? 1 : 0), bar, c * 64, it.s.k_first + it.wk.key(r), it.kvh, 0);
            } else {
#pragma unroll
                for (int c = 0; c < F::kHalves; ++c) tma_load_4d(dst + c * F::kHalf, map, bar, c * 64, it.s.k_first + first_key<W>(P, it, j), it.kvh, 0);
            }
        }
        __syncwarp();
        ++use.u;
        return true;
    };
    for (int round = 0, id; (id = nth_item(round)) < tl->n_items; ++round) {
        const Item it = nth_of_cta<W>(P, tl, round, id);
        if (it.most == 0) continue;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (it.n[x] <= 0) continue;
            if (!wait_w(&tl->q_free[x], (n_q[x]++ & 1u) ^ 1u, tl, 1002)) return;
            if (elect_one()) {
                const unsigned bar = smem_u32(&tl->q_full[x]);
                mbar_arrive_expect_tx(bar, F::kHalves * 128 * P.g.hpg * P.per_tile);
#pragma unroll
                for (int c = 0; c < F::kHalves; ++c)
                    tma_load_4d(q_smem + x * F::kTile + c * F::kHalf, tq, bar, c * 64, 0, it.s.q_first + it.tok0 + x * P.per_tile, it.kvh);
            }
            __syncwarp();
            if (x == 0 && !kv(it, tk, 0, false)) return;
        }
        if (it.n[0] <= 0 && !kv(it, tk, 0, false)) return;
        for (int j = 0; j < it.most; ++j) {
            if (!kv(it, tv, j, (long long)first_key<W>(P, it, j) + kKeys > it.s.k_n)) return;
            if (j + 1 < it.most && !kv(it, tk, j + 1, false)) return;
        }
    }
}

// Zeros over the rows of a V tile behind the last key.
template <bool W, class F>
__device__ void zero_role(const Params &P, Tail<F> *tl, unsigned char *ring, int lane) {
    Use<F> use;
    unsigned parity = 0;  // of each stage's barrier
    for (int round = 0, id; (id = nth_item(round)) < tl->n_items; ++round) {
        const Item it = nth_of_cta<W>(P, tl, round, id);
        if (it.most == 0) continue;
        use.u += 2 * (unsigned)it.most;
        const int last_key = first_key<W>(P, it, it.most - 1);  // (of the tiles the last alone can reach beyond the last key)
        if ((long long)last_key + kKeys <= it.s.k_n) continue;
        Use<F> last;
        last.u = use.u - 1;
        if (!wait_w(&tl->v_raw[last.stage()], (parity >> last.stage()) & 1u, tl, 1003, kWhileOthersWork)) return;
        parity ^= 1u << last.stage();
        const int there = it.s.k_n - last_key;
        unsigned char *const tile = ring + last.stage() * F::kTile;
#pragma unroll
        for (int c = 0; c < F::kHalves; ++c)
            for (int i = there * 8 + lane; i < kKeys * 8; i += 32) *reinterpret_cast<uint4 *>(tile + c * F::kHalf + i * 16) = make_uint4(0, 0, 0, 0);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&tl->full[last.stage()]));
        __syncwarp();
    }
}

template <bool W, class F>
__device__ void mma_role(const Params &P, Tail<F> *tl, unsigned q_smem, unsigned ring, unsigned tmem) {
    Use<F> use;
    unsigned n_q[2] = {0, 0}, n_p[2] = {0, 0};
    const unsigned q_lo = desc_lo_sw128(q_smem, 16), k_lo = desc_lo_sw128(ring, 16), v_lo = desc_lo_sw128(ring, F::kHalf);
    auto scores = [&](int x, unsigned stage, bool last) {  // S_x = Q_x K^T; last: Q_x has been read
        if (elect_one()) {
#pragma unroll
            for (int c = 0; c < F::kHalves; ++c)
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4)
                    tc_mma_bf16_split(tmem + F::kSCol + x * 128, q_lo + ((x * F::kTile + c * F::kHalf + k4 * 32) >> 4), kHi,
                                      k_lo + stage * (F::kTile >> 4) + ((c * F::kHalf + k4 * 32) >> 4), kHi, F::kIdescQK, (c | k4) != 0);
            tc_commit(smem_u32(&tl->s_full[x]));
            if (last) tc_commit(smem_u32(&tl->q_free[x]));
        }
        __syncwarp();
    };
    auto product = [&](int x, unsigned stage, int half, bool first) {  // O_x (+)= P_x V, 64 keys
        if (elect_one()) {
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4)
                tc_mma_bf16_ta(tmem + F::kOCol + x * 128, tmem + F::kSCol + x * 128 + half * 32 + s4 * 8,
                               v_lo + stage * (F::kTile >> 4) + (((half * 4 + s4) * 2048) >> 4), kHi, F::kIdescPV, !(first && half == 0 && s4 == 0));
        }
        __syncwarp();
    };
    auto release = [&](unsigned stage) {
        if (elect_one()) tc_commit(smem_u32(&tl->empty[stage]));
        __syncwarp();
    };
    for (int round = 0, id; (id = nth_item(round)) < tl->n_items; ++round) {
        const Item it = nth_of_cta<W>(P, tl, round, id);
        if (it.most == 0) continue;
        if (!wait_w(&tl->full[use.stage()], use.phase(), tl, 1011)) return;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (it.n[x] <= 0) continue;
            if (!wait_w(&tl->q_full[x], n_q[x] & 1u, tl, 1012)) return;
            tc_fence_after();
            scores(x, use.stage(), it.n[x] == 1);
        }
        release(use.stage());
        ++use.u;
        for (int j = 0; j < it.most; ++j) {
            const Use<F> v = use;
            Use<F> k = use;
            ++k.u;
            if (!wait_w(&tl->full[v.stage()], v.phase(), tl, 1013)) return;
            bool k_there = false;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (j >= it.n[x]) continue;
                if (!wait_w(&tl->p_half[x][0], n_p[x] & 1u, tl, 1014)) return;
                if (j == 0 && !wait_w(&tl->o_free[x], (n_q[x] & 1u) ^ 1u, tl, 1015)) return;  // the item before has been read
                tc_fence_after();
                product(x, v.stage(), 0, j == 0);
                if (!wait_w(&tl->p_half[x][1], n_p[x]++ & 1u, tl, 1016)) return;
                tc_fence_after();
                product(x, v.stage(), 1, j == 0);
                if (j + 1 < it.n[x]) {
                    if (!k_there && !wait_w(&tl->full[k.stage()], k.phase(), tl, 1017)) return;
                    k_there = true;
                    tc_fence_after();
                    scores(x, k.stage(), j + 2 == it.n[x]);
                } else {
                    if (elect_one()) tc_commit(smem_u32(&tl->o_done[x]));
                    __syncwarp();
                    ++n_q[x];
                }
            }
            release(v.stage());
            ++use.u;
            if (j + 1 < it.most) {
                release(k.stage());
                ++use.u;
            }
        }
    }
    // no arrival is on its way when the CTA leaves
    for (unsigned i = 0; i < F::kStages && use.u > 0; ++i) {
        --use.u;
        if (!wait_w(&tl->empty[use.stage()], use.phase(), tl, 1018)) return;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (n_q[x] > 0 && !wait_w(&tl->q_free[x], (n_q[x] - 1) & 1u, tl, 1019)) return;
}

// Multiplies fp32 columns of this thread's TMEM lane by f (eight at a time: the logits are in registers beside them).
template <int kColumns>
__device__ __forceinline__ void rescale(unsigned taddr, float f) {
#pragma unroll 1
    for (int c = 0; c < kColumns; c += 8) {
        unsigned r[8];
        tmem_ld_32x8_issue(taddr + c, r);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"r"(taddr + c), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                     : "memory");
    }
    tmem_st_wait();
}

template <bool W, class F>
__device__ void softmax_role(const Params &P, Tail<F> *tl, unsigned tmem, int t) {
    const PromptGeom &g = P.g;
    const int x = t >> 7, row = t & 127, lane = t & 31, wq = row >> 5;
    const int tok_r = row / g.hpg, head_r = row - tok_r * g.hpg;  // within the tile
    const unsigned lanes = tmem + ((unsigned)(row & ~31) << 16), s_addr = lanes + F::kSCol + x * 128, o_addr = lanes + F::kOCol + x * 128;
    const unsigned long long scale2 = pack_f32x2(g.scale_log2, g.scale_log2);
    uint4 *const stage = tl->stage[t >> 5];
    int out_tok[4];        // of the four output rows that this lane stores a piece of: the token within the tile, and where
    long long out_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int rr = wq * 32 + i * 8 + (lane >> 2);
        out_tok[i] = rr / g.hpg;
        out_at[i] = ((long long)out_tok[i] * g.H + (rr - out_tok[i] * g.hpg)) * F::D;
    }
    unsigned n_s = 0, n_o = 0;
    __nv_bfloat16 *const out = (__nv_bfloat16 *)g.out;
    for (int round = 0, id; (id = nth_item(round)) < tl->n_items; ++round) {
        const Item it = nth_of_cta<W>(P, tl, round, id);
        const int n_tiles = x == 0 ? it.n[0] : it.n[1];
        if (n_tiles < 0) continue;
        const int tok0 = it.tok0 + x * P.per_tile, tok = tok0 + tok_r;
        // rows that are none see what the last one does, so that they cost nothing
        const int last = min(tok, min(tok0 + P.per_tile, it.s.q_n) - 1);
        const int keys = g.causal ? min(it.s.k_n, max(0, last + 1 + it.s.k_n - it.s.q_n)) : it.s.k_n;
        const int low = W ? window_begin(g, last + (it.s.k_n - it.s.q_n)) : 0;
        const bool mine = tok_r < P.per_tile && tok < it.s.q_n;
        float ref = -CUDART_INF_F, l = 0.f;
        for (int j = 0; j < n_tiles; ++j) {
            if (!wait_w(&tl->s_full[x], n_s++ & 1u, tl, 1021, kWhileOthersWork)) return;
            tc_fence_after();
            unsigned sr[2][64];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32_issue(s_addr + c * 32, sr[c >> 1] + (c & 1) * 32);
            tmem_ld_wait();
            const int base = first_key<W>(P, it, j);
            int n_hi = min(keys - base, kKeys);
            if constexpr (W) {  // keys between the sinks and the window
                const bool gap = it.wk.gap > 0, own_tile = P.sink_unit == kKeys;
                const int to = min(low - base, kKeys);  // columns from there on are the window's
                if (gap && own_tile && j * kKeys < it.wk.sink_keys) {
                    n_hi = min(n_hi, g.sinks - base);
                } else {
                    // columns in front of `from` are sinks: none where the sinks are further back, few where they share the tile
                    const int from = gap ? (j == 0 && !own_tile ? min(g.sinks, kFewSinks) : 0) : max(g.sinks - base, 0);
                    if (__any_sync(0xffffffffu, from < to)) {
                        if (gap) {
#pragma unroll
                            for (int i = 0; i < 64; ++i) {
                                if (i < kFewSinks) sr[0][i] = i < to && i >= from ? 0xff800000u : sr[0][i];
                                else sr[0][i] = i < to ? 0xff800000u : sr[0][i];
                                sr[1][i] = i + 64 < to ? 0xff800000u : sr[1][i];
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 64; ++i) {
                                sr[0][i] = i >= from && i < to ? 0xff800000u : sr[0][i];
                                sr[1][i] = i + 64 >= from && i + 64 < to ? 0xff800000u : sr[1][i];
                            }
                        }
                    }
                }
            }
            if (__any_sync(0xffffffffu, n_hi < kKeys)) {
#pragma unroll
                for (int i = 0; i < 64; ++i) {
                    sr[0][i] = i < n_hi ? sr[0][i] : 0xff800000u;
                    sr[1][i] = i + 64 < n_hi ? sr[1][i] : 0xff800000u;
                }
            }
            const float mx = fmaxf(max_of_64(reinterpret_cast<const float *>(sr[0])), max_of_64(reinterpret_cast<const float *>(sr[1])));
            const bool outgrown = (mx - ref) * g.scale_log2 > kOutgrown;  // (the first of a row that sees anything: infinity)
            if (__any_sync(0xffffffffu, outgrown)) {
                float f = 1.f;
                if (outgrown) {
                    f = fast_exp2((ref - mx) * g.scale_log2);
                    ref = mx;
                    l *= f;
                }
                if (j > 0) rescale<F::D>(o_addr, f);  // (the product before this one is complete: these logits came behind it)
            }
            const float shift = ref == -CUDART_INF_F ? 0.f : -ref * g.scale_log2;
            const unsigned long long shift2 = pack_f32x2(shift, shift);
            unsigned long long sum2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                unsigned packed[16];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    float a, b;
                    unpack_f32x2(fma_f32x2(pack_u32x2(sr[c >> 1][32 * (c & 1) + i], sr[c >> 1][32 * (c & 1) + i + 1]), scale2, shift2), a, b);
                    a = fast_exp2(a);
                    b = fast_exp2(b);
                    sum2[(i >> 1) & 3] = add_f32x2(sum2[(i >> 1) & 3], pack_f32x2(a, b));
                    const __nv_bfloat162 pk = __floats2bfloat162_rn(a, b);
                    packed[i >> 1] = *reinterpret_cast<const unsigned *>(&pk);
                }
                tmem_st_32x16_issue(s_addr + c * 16, packed);
                if (c & 1) {
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    mbar_arrive_if(smem_u32(&tl->p_half[x][c >> 1]), lane == 0);
                }
            }
            float e0, e1;
            unpack_f32x2(add_f32x2(add_f32x2(sum2[0], sum2[1]), add_f32x2(sum2[2], sum2[3])), e0, e1);
            l += e0 + e1;
        }
        const int head = it.kvh * g.hpg + head_r;
        if (mine && g.lse != nullptr)
            g.lse[(long long)head * g.total_q + it.s.q_first + tok] = l > 0.f ? (ref * g.scale_log2 + log2f(l)) * kLn2 : -CUDART_INF_F;
        // 32 channels at a time through shared memory, where a row's 16-byte pieces are turned so that eight rows touch every bank, and
        // from there four lanes a row: whole sectors
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int n_tok = min(P.per_tile, it.s.q_n - tok0);
        __nv_bfloat16 *const to = out + ((long long)(it.s.q_first + tok0) * g.H + it.kvh * g.hpg) * F::D + (lane & 3) * 8;
        if (n_tiles > 0) {
            if (!wait_w(&tl->o_done[x], n_o++ & 1u, tl, 1022)) return;
            tc_fence_after();
        }
        unsigned r[F::D / 32][32];  // (in the place of the logits: the next item's products need not wait for the output)
        if (n_tiles > 0) {
#pragma unroll
            for (int c = 0; c < F::D / 32; ++c) tmem_ld_32x32_issue(o_addr + c * 32, r[c]);
            tmem_ld_wait();
            tc_fence_before();
            mbar_arrive_if(smem_u32(&tl->o_free[x]), lane == 0);
        } else {  // (no key for any row)
#pragma unroll
            for (int c = 0; c < F::D / 32; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i) r[c][i] = 0u;
        }
#pragma unroll
        for (int c = 0; c < F::D / 32; ++c) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                unsigned w[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const __nv_bfloat162 pk = __floats2bfloat162_rn(__uint_as_float(r[c][8 * u + 2 * y]) * inv, __uint_as_float(r[c][8 * u + 2 * y + 1]) * inv);
                    w[y] = *reinterpret_cast<const unsigned *>(&pk);
                }
                stage[lane * 4 + (u ^ ((lane >> 1) & 3))] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = i * 8 + (lane >> 2);
                const uint4 w = stage[rr * 4 + ((lane & 3) ^ ((rr >> 1) & 3))];
                if (out_tok[i] < n_tok) *reinterpret_cast<uint4 *>(to + out_at[i] + c * 32) = w;
            }
            __syncwarp();
        }
    }
}

struct Few { CUtensorMap map[2]; };  // K and V in boxes of kFewSinks rows

template <class F, bool W>
__global__ void __launch_bounds__(kThreads, 1)
prompt_tc_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                 const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ Few few, const __grid_constant__ Params P) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char *const smem = aligned_smem(smem_raw);
    unsigned char *const ring = smem + 2 * F::kTile;
    Tail<F> *const tl = reinterpret_cast<Tail<F> *>(ring + F::kStages * F::kTile);
    const PromptGeom &g = P.g;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < F::kStages; ++i) { mbar_init(smem_u32(&tl->full[i]), 1); mbar_init(smem_u32(&tl->empty[i]), 1); mbar_init(smem_u32(&tl->v_raw[i]), 1); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&tl->q_full[x]), 1);
            mbar_init(smem_u32(&tl->q_free[x]), 1);
            mbar_init(smem_u32(&tl->s_full[x]), 1);
            mbar_init(smem_u32(&tl->p_half[x][0]), 4);
            mbar_init(smem_u32(&tl->p_half[x][1]), 4);
            mbar_init(smem_u32(&tl->o_done[x]), 1);
            mbar_init(smem_u32(&tl->o_free[x]), 4);
        }
        tl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(&tl->tmem_base));  // all columns: one CTA per SM
    after_previous_kernel();
    // The sequences, those with the most keys first (a thread a sequence counts those in front), and their items
    auto span = [&](int s) {
        const Span a = span_of(g.cu_q, s, g.total_q), b = span_of(g.cu_k, s, g.total_k);
        return Seq{a.first, a.n, b.first, b.n};
    };
    if (tid < g.n_seqs) tl->level_end[tid] = span(tid).k_n;
    __syncthreads();
    static_assert(kMaxSeqs <= kThreads, "a thread a sequence");
    int at = 0;
    if (tid < g.n_seqs) {
        const int own = tl->level_end[tid];
        for (int o = 0; o < g.n_seqs; ++o) at += tl->level_end[o] > own || (tl->level_end[o] == own && o < tid) ? 1 : 0;
    }
    __syncthreads();
    if (tid < g.n_seqs) {
        const Seq q = span(tid);
        tl->seq[at] = q;
        tl->level_end[at] = ceil_div(q.q_n, 2 * P.per_tile);
    }
    __syncthreads();
    if (warp == 0) {
        long long sum = 0;
        for (int s0 = 0; s0 < g.n_seqs; s0 += 32) {
            long long v = s0 + lane < g.n_seqs ? tl->level_end[s0 + lane] : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, v, d);
                if (lane >= d) v += y;
            }
            if (s0 + lane < g.n_seqs) tl->level_end[s0 + lane] = (int)(sum + v);
            sum += __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) {
            // (the host has seen that the sequences' items can be counted, unless their offsets fall and sequences overlap: then nothing is done)
            const bool fits = sum * g.G <= kMaxItems;
            tl->n_levels = fits ? (int)sum : 0;
            tl->n_items = fits ? (int)sum * g.G : 0;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = tl->tmem_base;
    // Items in the order of their key tiles, over all sequences (in the sequences' order the last CTA was 9 % behind the mean: 12 prompts of up to 4500
    // tokens; in this one 2 %). An item's place is how many stand in front of it, which each sequence says in closed form. Not where every
    // item has a CTA of its own, nor where there is too much to count (16 terms a thread take 2 us): the items are many and small against
    // a CTA's sum then, and counting costs more than order gives (us as the sequences lie, and put in order all the same, 28 / 4 heads: 64 prompts of 500 tokens
    // 222, 273; of 100 to 900 311, 351; of 50 to 2000 337, 361; 32 / 8 heads 234, 259; 304, 315; 361, 363).
    const int n_levels = tl->n_levels;
    const bool sorted = g.n_seqs > 1 && tl->n_items > (int)gridDim.x && n_levels <= kMaxLevels && n_levels * g.n_seqs <= 16 * kThreads;
    if (tid == 0) tl->sorted = sorted ? 1 : 0;
    for (int i = tid; sorted && i < n_levels; i += kThreads) {
        const int own = sequence_of(tl, g.n_seqs, i), level = i - (own > 0 ? tl->level_end[own - 1] : 0), span2 = 2 * P.per_tile;
        // key tiles of a sequence's item at `level`; its items with more than v of them
        auto tiles = [&](const Seq &q, int lv) {
            const int end = min((ceil_div(q.q_n, span2) - lv) * span2, q.q_n);
            return ceil_div(g.causal ? max(0, end + q.k_n - q.q_n) : q.k_n, kKeys);
        };
        auto above = [&](const Seq &q, int v) {
            const int n = ceil_div(q.q_n, span2);
            if (v < 0) return n;
            if ((long long)q.k_n <= (long long)v * kKeys) return 0;
            if (!g.causal) return n;
            const long long need = (long long)v * kKeys - q.k_n + q.q_n;  // queries up to there see no more
            return need < span2 ? n : n - (int)(need / span2);
        };
        const int v = tiles(tl->seq[own], level);
        int place = level;
        for (int o = 0; o < g.n_seqs; ++o)
            if (o != own) place += above(tl->seq[o], o < own ? v - 1 : v);
        tl->order[place] = (unsigned)own << 12 | (unsigned)level;
    }
    __syncthreads();
    if (tid < kKnown && nth_item(tid) < tl->n_items) tl->items[tid] = item_at<W>(P, tl, nth_item(tid));
    __syncthreads();
    if (warp < 4) {
        if (warp == 0) load_role<W>(P, &tmap_q, &tmap_k, &tmap_v, few.map, tl, smem_u32(smem), smem_u32(ring));
        else if (warp == 1) mma_role<W>(P, tl, smem_u32(smem), smem_u32(ring), tmem);
        else if (warp == 2) zero_role<W>(P, tl, ring, lane);
    } else {
        softmax_role<W>(P, tl, tmem, tid - 128);
    }
    __syncwarp();
    leave(&tl->abort_flag, tmem, warp == 1);
}

// Q as [G][token][head of the group][channel]: a box is 64 channels of all heads of some tokens, rows in the order of a tile.
stream_status make_map_q(CUtensorMap *map, const PromptGeom &g, const void *q, int per_tile) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) { set_error("cuTensorMapEncodeTiled is not available from this driver"); return STREAM_ERR_CUDA; }
    cuuint64_t dims[4] = {(cuuint64_t)g.d, (cuuint64_t)g.hpg, (cuuint64_t)g.total_q, (cuuint64_t)g.G};
    cuuint64_t strides[3] = {(cuuint64_t)g.qs_h * 2, (cuuint64_t)g.qs_t * 2, (cuuint64_t)g.qs_h * g.hpg * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)g.hpg, (cuuint32_t)per_tile, 1}, estr[4] = {1, 1, 1, 1};
    CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_error("cuTensorMapEncodeTiled(q) failed with %d", (int)r); return STREAM_ERR_CUDA; }
    return STREAM_OK;
}

template <class F, bool W>
stream_status launch(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    Params P;
    P.g = g;
    P.per_tile = kRows / g.hpg;
    const long long fit = kKvInL2 / ((long long)g.total_k * F::D * 4);
    // (A window of some thousand keys has a working set that L2 holds whatever the length: all heads side by side, which is faster then: 32768 tokens, window 4096,
    // 32 / 8 heads 1610 us, walked as the dense call does 1660. Windows beyond L2 lose by it: 131072 tokens, window 4096 the same, 16384 27.9 ms for 26.0, 65536 94 for 88, 131072 126 for 120.)
    P.heads = W || fit > g.G ? g.G : (int)(fit < 1 ? 1 : fit);
    CUtensorMap tq, tk, tv;
    stream_status rc = make_map_q(&tq, g, q, P.per_tile);
    if (rc != STREAM_OK) return rc;
    rc = make_map_bf16(&tk, k, g.total_k, g.G, 1, g.ks_t, g.ks_h, 0, "k", kKeys, g.d);
    if (rc != STREAM_OK) return rc;
    rc = make_map_bf16(&tv, v, g.total_k, g.G, 1, g.ks_t, g.ks_h, 0, "v", kKeys, g.d);
    if (rc != STREAM_OK) return rc;
    P.sink_unit = W && g.sinks <= kFewSinks ? kFewSinks : kKeys;
    Few few = {};
    if (W && g.sinks > 0 && g.sinks <= kFewSinks) {
        rc = make_map_bf16(&few.map[0], k, g.total_k, g.G, 1, g.ks_t, g.ks_h, 0, "k", kFewSinks, g.d);
        if (rc == STREAM_OK) rc = make_map_bf16(&few.map[1], v, g.total_k, g.G, 1, g.ks_t, g.ks_h, 0, "v", kFewSinks, g.d);
        if (rc != STREAM_OK) return rc;
    }
    const int smem = (2 + F::kStages) * F::kTile + (int)sizeof(Tail<F>) + 1024;
    static_assert((2 + F::kStages) * F::kTile + (int)sizeof(Tail<F>) + 1024 <= 232448, "what a CTA may have");
    static DeviceFlags done;
    cudaError_t e = allow_smem_once(prompt_tc_kernel<F, W>, smem, done);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(prompt_tc)");
    const int n_sm = current_sm_count();
    if (n_sm <= 0) { set_error("cannot read the SM count of the current device"); return STREAM_ERR_CUDA; }
    for (int s0 = 0; s0 < g.n_seqs; s0 += kMaxSeqs) {
        P.g.n_seqs = g.n_seqs - s0 < kMaxSeqs ? g.n_seqs - s0 : kMaxSeqs;
        P.g.cu_q = g.cu_q + s0;
        P.g.cu_k = g.cu_k + s0;
        const long long items = ((long long)g.total_q / (2 * P.per_tile) + P.g.n_seqs) * g.G;  // at most
        e = launch_early(prompt_tc_kernel<F, W>, (unsigned)(items < n_sm ? items : n_sm), kThreads, smem, st, tq, tk, tv, few, P);
        if (e != cudaSuccess) return cuda_fail(e, "prompt_tc launch");
    }
    return STREAM_OK;
}

}  // namespace

bool prompt_tc_supported(const PromptGeom &g, int dtype, const void *q, const void *k, const void *v) {
    if (dtype != STREAM_BF16 || (g.d != 64 && g.d != 128) || g.hpg > kRows || g.total_k < 1) return false;
    if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)g.out) & 15) != 0 || ((g.qs_t | g.qs_h | g.ks_t | g.ks_h) & 7) != 0) return false;
    return ((long long)g.total_q / (2 * (kRows / g.hpg)) + g.n_seqs) * g.G <= kMaxItems;
}

stream_status launch_prompt_tc(const PromptGeom &g, const void *q, const void *k, const void *v, cudaStream_t st) {
    if (g.window > 0) return g.d == 128 ? launch<Form<128>, true>(g, q, k, v, st) : launch<Form<64>, true>(g, q, k, v, st);
    return g.d == 128 ? launch<Form<128>, false>(g, q, k, v, st) : launch<Form<64>, false>(g, q, k, v, st);
}

stream_status read_prompt_status(unsigned int out[2], cudaStream_t st) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(out, g_prompt_status, 2 * sizeof(unsigned int), 0, cudaMemcpyDeviceToHost, st);
    if (e != cudaSuccess) return cuda_fail(e, "cudaMemcpyFromSymbolAsync(prompt attention status)");
    e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return cuda_fail(e, "cudaStreamSynchronize");
    return STREAM_OK;
}

}  // namespace stream
