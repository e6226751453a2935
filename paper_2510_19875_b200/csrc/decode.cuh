// How the keys of a paged cache are dealt to the CTAs of decode attention, for its kernels.
#pragma once
#include "serve_common.cuh"

namespace stream {
namespace decode {

constexpr int kThreads = 128;
constexpr int kUnit = 64;        // keys
constexpr int kMaxHeads = 16;    // query heads of a segment (a larger group is walked in several segments)
constexpr int kMaxGrid = 320;

struct Args {
    DecodeCall a;
    int grid;                    // CTAs of the first kernel
    int per_slot;                // owners of a slot's units: (kv head, up to 16 of its query heads)
    int chunks;                  // owners of a kv head
    float *parts;                // [grid][2][kMaxHeads * (d + 2)]: m, l, O
    unsigned *bad;               // [grid]: slot + 1 with a page outside the cache, or 0
    WorkspaceHeader *header;
    int q_vec;                   // (mma.sync) q is read in pieces of 16 bytes
};

// bf16 on mma.sync. May lower A.grid.
bool mma_supported(const DecodeCall &a, int dtype);
cudaError_t launch_mma(Args &A, int n_sm, cudaStream_t st);

// Sums over the slots, by whole warps (the same in every lane).
__device__ __forceinline__ int units_of(const CacheGeom &c, int s) { return s < c.n_slots ? (tokens_of(c, s) + kUnit - 1) / kUnit : 0; }
__device__ __forceinline__ long long all_units(const CacheGeom &c, int lane) {
    long long sum = 0;
    for (int s = lane; s < c.n_slots; s += 32) sum += units_of(c, s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum;
}
// Where a unit lies: its slot, that slot's first unit and how many it has for one owner. `from`: a place at or before it.
struct Place { int slot, units; long long first; };
__device__ __forceinline__ Place place_of(const CacheGeom &c, int per_slot, long long unit, int lane, Place from) {
    long long sum = from.first;
    for (int s0 = from.slot; s0 < c.n_slots; s0 += 32) {
        const int u = units_of(c, s0 + lane);
        long long incl = u;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, unit < sum + incl * per_slot);
        if (past != 0) {
            const int at = __ffs(past) - 1;
            return {s0 + at, __shfl_sync(0xffffffffu, u, at), sum + __shfl_sync(0xffffffffu, (incl - u) * per_slot, at)};
        }
        sum += __shfl_sync(0xffffffffu, incl, 31) * per_slot;
    }
    return {c.n_slots, 0, sum};
}

// The units of a CTA.
struct Share { long long per, first, end; };
__device__ __forceinline__ Share share_of(const Args &A, long long all, int cta) {
    const long long per = (all + A.grid - 1) / A.grid;
    return {per, min(all, per * cta), min(all, per * (cta + 1))};
}

// What a CTA whose share ends at `end` has of the owner of unit u.
struct Segment {
    int units, kvh, h0, heads;
    int key0, key_end;   // keys of the slot
    bool whole;          // all of them
};
__device__ __forceinline__ Segment segment_of(const Args &A, const Place &at, long long u, long long end) {
    Segment sg;
    const int owner = (int)((u - at.first) / at.units), unit0 = (int)((u - at.first) % at.units), chunk = owner % A.chunks;
    sg.units = (int)min((long long)(at.units - unit0), end - u);
    sg.kvh = owner / A.chunks;
    sg.h0 = sg.kvh * A.a.hpg + chunk * kMaxHeads;
    sg.heads = min(kMaxHeads, A.a.hpg - chunk * kMaxHeads);
    sg.key0 = unit0 * kUnit;
    sg.key_end = (int)min((long long)tokens_of(A.a.c, at.slot), (long long)(unit0 + sg.units) * kUnit);
    sg.whole = sg.units == at.units;
    return sg;
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

// Every thread's `bad` (slot + 1, or 0) to the CTA's word.
__device__ __forceinline__ void record_bad(const Args &A, unsigned bad) {
    __shared__ unsigned any;
    bad = __reduce_max_sync(0xffffffffu, bad);
    if (threadIdx.x == 0) any = 0;
    __syncthreads();
    if ((threadIdx.x & 31) == 0 && bad != 0) atomicMax(&any, bad);
    __syncthreads();
    if (threadIdx.x == 0) A.bad[blockIdx.x] = any;
}

__device__ __forceinline__ void cp_async16(unsigned dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory"); }

}  // namespace decode
}  // namespace stream
