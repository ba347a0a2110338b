// A stable counting sort of n entries by a number below `buckets`, in three kernels: every wavefront counts the numbers in
// its stretch of entries, the counts are scanned, every wavefront places its stretch's entries.  No atomics on memory and
// the same result whatever runs first.  Used for the slots of experts and for the table's gradient.
#ifndef FS_SLOTS_H
#define FS_SLOTS_H

#include "fs_mixture.h"

namespace fs {

constexpr int kSlotWaves = 4;               // of a workgroup
constexpr int kSlotMostBuckets = 1025;      // experts, and one for choices without a slot
constexpr int kSlotMostStretches = 4096;
constexpr int kSlotScanThreads = 1024;

struct SlotShape {
    int32_t n, buckets, stretch, stretches;
};
inline SlotShape slot_shape(int64_t n, int buckets)
{
    SlotShape s = {(int32_t)n, buckets, 1024, 0};
    const int64_t least = (n + kSlotMostStretches - 1) / kSlotMostStretches;
    if (least > s.stretch)
        s.stretch = (int32_t)((least + 63) / 64 * 64);
    s.stretches = (int32_t)((n + s.stretch - 1) / s.stretch);
    return s;
}
inline size_t slot_count_bytes(const SlotShape &s) { return ((size_t)s.buckets * s.stretches * 4 + 255) / 256 * 256; }

// The lanes whose number is this lane's, among the lanes that are there.
__device__ __forceinline__ uint64_t same_number(int number, int bits, bool there)
{
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const bool set = (number >> b) & 1;
        const uint64_t with = __ballot(set);
        same &= set ? with : ~with;
    }
    return same;
}
__host__ __device__ inline int bits_of(int n)        // of numbers below n
{
    int b = 0;
    while ((1 << b) < n)
        ++b;
    return b;
}

// count[number * stretches + stretch]
template <class Number>
__global__ void __launch_bounds__(kSlotWaves * 64)
slot_count_kernel(Number number, SlotShape s, int32_t *count)
{
    __shared__ int32_t lds[kSlotWaves * kSlotMostBuckets];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mine = (int)blockIdx.x * kSlotWaves + wave;
    int32_t *c = lds + wave * s.buckets;
    for (int b = lane; b < s.buckets; b += 64)
        c[b] = 0;
    __syncthreads();
    if (mine < s.stretches) {
        const int64_t begin = (int64_t)mine * s.stretch, end = min(begin + s.stretch, (int64_t)s.n);
        for (int64_t i = begin + lane; i < end; i += 64)
            atomicAdd(&c[number(i)], 1);
    }
    __syncthreads();
    if (mine < s.stretches)
        for (int b = lane; b < s.buckets; b += 64)
            count[(int64_t)b * s.stretches + mine] = c[b];
}

// Counts to the sums of all counts before them, in place.  One workgroup.
static __global__ void __launch_bounds__(kSlotScanThreads)
slot_scan_kernel(int32_t *count, int32_t n)
{
    __shared__ int32_t sums[kSlotScanThreads];
    const int t = threadIdx.x;
    const int per = (n + kSlotScanThreads - 1) / kSlotScanThreads;
    const int begin = min((int64_t)t * per, (int64_t)n), end = min(begin + per, n);
    int32_t sum = 0;
    for (int i = begin; i < end; ++i)
        sum += count[i];
    sums[t] = sum;
    __syncthreads();
    for (int off = 1; off < kSlotScanThreads; off <<= 1) {
        const int32_t v = t >= off ? sums[t - off] : 0;
        __syncthreads();
        sums[t] += v;
        __syncthreads();
    }
    int32_t at = sums[t] - sum;
    for (int i = begin; i < end; ++i) {
        const int32_t v = count[i];
        count[i] = at;
        at += v;
    }
}

template <class Number, class Put>
__global__ void __launch_bounds__(kSlotWaves * 64)
slot_place_kernel(Number number, Put put, SlotShape s, const int32_t *count)
{
    __shared__ int32_t lds[kSlotWaves * kSlotMostBuckets];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mine = (int)blockIdx.x * kSlotWaves + wave;
    int32_t *next = lds + wave * s.buckets;
    if (mine < s.stretches)
        for (int b = lane; b < s.buckets; b += 64)
            next[b] = count[(int64_t)b * s.stretches + mine];
    __syncthreads();
    if (mine >= s.stretches)
        return;
    const int bits = bits_of(s.buckets);
    const int64_t begin = (int64_t)mine * s.stretch, end = min(begin + s.stretch, (int64_t)s.n);
    for (int64_t i0 = begin; i0 < end; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool there = i < end;
        const int m = there ? number(i) : 0;
        const uint64_t same = same_number(m, bits, there);
        const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
        int slot = 0;
        if (there)
            slot = next[m] + before;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (there && before == 0)
            next[m] = slot + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (there)
            put(i, m, slot);
    }
}

template <class Number, class Put>
void launch_slots(const Number &number, const Put &put, const SlotShape &s, int32_t *count, hipStream_t stream)
{
    const dim3 grid((unsigned)((s.stretches + kSlotWaves - 1) / kSlotWaves)), block(kSlotWaves * 64);
    hipLaunchKernelGGL(slot_count_kernel<Number>, grid, block, 0, stream, number, s, count);
    hipLaunchKernelGGL(slot_scan_kernel, dim3(1), dim3(kSlotScanThreads), 0, stream, count, s.buckets * s.stretches);
    hipLaunchKernelGGL((slot_place_kernel<Number, Put>), grid, block, 0, stream, number, put, s, (const int32_t *)count);
}

}  // namespace fs
#endif
