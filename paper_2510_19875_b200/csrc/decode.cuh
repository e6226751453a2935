// How the keys of a paged cache are dealt to the CTAs of decode attention, for its kernels.
#pragma once
#include "serve_common.cuh"
#include "warp_common.cuh"

namespace stream {
namespace decode {

constexpr int kThreads = 128;
// The kernels that have the cache's own numbers deal units of 64 keys.
constexpr int kUnit64 = 64;

// A segment costs a CTA kOpen64 units beside its own: the way from one owner's last key to the next one's first, the warps' meeting and
// the output. So an owner takes up as many places more in the row that is dealt out, in front of its units. (Without them a CTA with
// many short slots was the last by far: four slots of up to 131072 tokens, 32 / 8 heads: 80 us most CTAs, 126 the last.) With 1, 2, 3, 4, us: 64 slots of up to
// 8192 tokens 54.2, 46.4, 45.8, 47.3; the four 96.3, 88.5, 88.5, 88.6; nine of up to 5003, fp32, 21.0, 20.0, 20.0, 19.8; slots of some tokens 7 to 10 with any.
constexpr int kOpen64 = 2;
constexpr int kMaxHeads = 16;    // query heads of a segment (a larger group is walked in several segments)
constexpr int kMaxGrid = 320;

// What a CTA leaves to the joins: the owner whose first piece, but not all of it, it has (none: n = 0), and what it has met.
struct Left {
    int n;         // pieces: its own and the first ones of the n - 1 CTAs behind it
    int which;     // its own: its first or its second
    int heads;
    unsigned bad;  // slot + 1 with a page outside the cache, or 0
    long long to;  // row of the output of the owner's first query head
    long long pad;
};

struct Args {
    DecodeCall a;
    int grid;                    // CTAs of the first kernel
    int per_slot;                // owners of a slot's units: (kv head, up to 16 of its query heads)
    int chunks;                  // owners of a kv head
    float *parts;                // [grid][2][kMaxHeads * (d + 2)]: m, l, O
    struct Left *left;           // [grid]
    WorkspaceHeader *header;
    int q_vec;                   // q is read in pieces (decode_warp.cu: of 16 bytes; decode8.cu: of four elements)
};

// The arguments that follow from the call, and the grid at most; the joins' launch.
Args args_of(const DecodeCall &a, void *workspace, int n_sm, int unit = kUnit64, int open = kOpen64, int least = 1);  // least: places of a CTA
cudaError_t launch_joins(const Args &A, int dtype, cudaStream_t st);

// Rows of 16-byte pieces, up to 512 bytes. May lower A.grid.
bool warp_supported(const DecodeCall &a, int dtype);
cudaError_t launch_warp(Args &A, int dtype, int n_sm, cudaStream_t st);

// Which keys of a slot are walked where there is a window (W; 64 slots of up to 8192 tokens, window 1024, 32 / 8 heads, bf16: 30 to 36 us, 106 MB; a
// segment's own cost, which is 3 us, is what bounds it): the units of the sinks, then, behind a gap, those from the window's first key on. A
// segment counts its keys without the gap; units are whole on both sides of it, so that a tile's keys lie as they do without.
struct Seen {
    int n;          // keys that are walked
    int sink_keys;  // of them in front of the gap
    int gap;        // keys
    int sinks, low; // seen are keys < sinks and keys >= low
    __device__ __forceinline__ int key(int walked) const { return walked < sink_keys ? walked : walked + gap; }
    __device__ __forceinline__ bool sees(int key) const { return key < sinks || key >= low; }
};
template <bool W, int kUnit>
__device__ __forceinline__ Seen seen_of(const DecodeCall &a, int s) {
    const int n = tokens_of(a.c, s);
    if constexpr (!W) return {n, n, 0, n, 0};
    const int low = max(0, n - a.window), sink = (min(a.sinks, n) + kUnit - 1) / kUnit, gap = max(0, low / kUnit - sink) * kUnit;
    return {n - gap, sink * kUnit, gap, a.sinks, low};
}

// Sums over the slots, by whole warps (the same in every lane).
template <bool W, int kUnit, int kOpen>
__device__ __forceinline__ int places_of(const DecodeCall &a, int s) {
    const int u = s < a.c.n_slots ? (seen_of<W, kUnit>(a, s).n + kUnit - 1) / kUnit : 0;
    return u > 0 ? u + kOpen : 0;
}
template <bool W, int kUnit = kUnit64, int kOpen = kOpen64>
__device__ __forceinline__ long long all_places(const Args &A, int lane) {
    long long sum = 0;
    for (int s = lane; s < A.a.c.n_slots; s += 32) sum += places_of<W, kUnit, kOpen>(A.a, s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum * A.per_slot;
}
// Whose a place is: the slot, where that slot's places begin, how many it has for one owner. `from`: one at or before it.
struct Place { int slot, n; long long first; };
template <bool W, int kUnit, int kOpen>
__device__ __forceinline__ Place place_of(const Args &A, long long at, int lane, Place from) {
    const CacheGeom &c = A.a.c;
    long long sum = from.first;
    for (int s0 = from.slot; s0 < c.n_slots; s0 += 32) {
        const int n = places_of<W, kUnit, kOpen>(A.a, s0 + lane);
        long long incl = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, at < sum + incl * A.per_slot);
        if (past != 0) {
            const int x = __ffs(past) - 1;
            return {s0 + x, __shfl_sync(0xffffffffu, n, x), sum + __shfl_sync(0xffffffffu, (incl - n) * A.per_slot, x)};
        }
        sum += __shfl_sync(0xffffffffu, incl, 31) * A.per_slot;
    }
    return {c.n_slots, 0, sum};
}

// The places of a CTA. The last place of an owner is always a unit, so that a share with any of its places holds work
// or is followed by one that does.
struct Share { long long per, first, end; };
__device__ __forceinline__ Share share_of(const Args &A, long long all, int cta) {
    const long long per = (all + A.grid - 1) / A.grid;
    return {per, min(all, per * cta), min(all, per * (cta + 1))};
}

// What a CTA has of the owner of place `at`, from there to the end of its share.
struct Segment {
    long long next;      // the place behind it
    long long owner_end; // the place behind all of its owner's
    int slot, kvh, h0, heads;
    int key0, key_end;   // keys of the slot (none where key0 = key_end), as Seen counts them
    bool whole;          // all of them
};
template <bool W, int kUnit, int kOpen>
__device__ __forceinline__ Segment segment_of(const Args &A, const Place &pl, long long at, long long end) {
    Segment sg;
    const long long ahead = at - pl.first;  // (a division of 64 bits is hundreds of cycles)
    const int owner = ahead >> 32 == 0 ? (int)((unsigned)ahead / (unsigned)pl.n) : (int)(ahead / pl.n);
    const int chunk = A.chunks == 1 ? 0 : owner % A.chunks;
    sg.kvh = A.chunks == 1 ? owner : owner / A.chunks;
    const long long first = pl.first + (long long)owner * pl.n;
    sg.owner_end = first + pl.n;
    sg.next = min(sg.owner_end, end);
    sg.slot = pl.slot;
    sg.h0 = sg.kvh * A.a.hpg + chunk * kMaxHeads;
    sg.heads = min(kMaxHeads, A.a.hpg - chunk * kMaxHeads);
    const int unit0 = (int)max(at - first - kOpen, 0ll), unit1 = (int)max(sg.next - first - kOpen, 0ll);
    sg.key0 = unit0 * kUnit;
    sg.key_end = (int)min((long long)seen_of<W, kUnit>(A.a, pl.slot).n, (long long)unit1 * kUnit);
    if (unit0 == unit1) sg.key_end = sg.key0;
    sg.whole = unit0 == 0 && unit1 == pl.n - kOpen;
    return sg;
}
// The first segment with keys at or behind place `at` of a share that ends at `end`; pl: a place at or before it. next = -1: none.
template <bool W, int kUnit = kUnit64, int kOpen = kOpen64>
__device__ __forceinline__ Segment open_segment(const Args &A, long long at, long long end, int lane, Place &pl) {
    while (at < end) {
        if (pl.n == 0 || at >= pl.first + (long long)pl.n * A.per_slot) pl = place_of<W, kUnit, kOpen>(A, at, lane, pl);
        const Segment sg = segment_of<W, kUnit, kOpen>(A, pl, at, end);
        if (sg.key_end > sg.key0) return sg;
        at = sg.next;
    }
    Segment none = {};
    none.next = -1;
    return none;
}

__device__ __forceinline__ float *part_of(const Args &A, int cta, int which) { return A.parts + ((long long)cta * 2 + which) * kMaxHeads * (A.a.c.d + 2); }

// Zeros and -inf for the slots without tokens, which are dealt to the CTAs in turn.
template <class T>
__device__ __forceinline__ void write_empty_slots(const Args &A) {
    for (int s = blockIdx.x; s < A.a.c.n_slots; s += A.grid)
        if (tokens_of(A.a.c, s) == 0) {
            const long long n = (long long)A.a.H * A.a.c.d;
            for (long long i = threadIdx.x; i < n; i += blockDim.x) ((T *)A.a.out)[s * n + i] = (T)0.f;
            if (A.a.lse != nullptr)
                for (int h = threadIdx.x; h < A.a.H; h += blockDim.x) A.a.lse[(long long)s * A.a.H + h] = -CUDART_INF_F;
        }
}

// The n of Left for a segment that begins with its owner's first key and is not all of it.
__device__ __forceinline__ int pieces_of(long long owner_end, const Share &mine) { return (int)((owner_end - 1) / mine.per) - (int)blockIdx.x + 1; }
// `bad`: of every thread. The other fields are thread 0's.
__device__ __forceinline__ void leave_to_joins(const Args &A, Left left, unsigned bad) {
    __shared__ unsigned any;
    bad = __reduce_max_sync(0xffffffffu, bad);
    if (threadIdx.x == 0) any = 0;
    __syncthreads();
    if ((threadIdx.x & 31) == 0 && bad != 0) atomicMax(&any, bad);
    __syncthreads();
    left.bad = any;
    if (threadIdx.x == 0) A.left[blockIdx.x] = left;
}

// The logarithm of a softmax sum l, of weights relative to 2^m; NaN where a logit is.
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2; }

__device__ __forceinline__ float warp_maximum(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}

}  // namespace decode
}  // namespace stream
