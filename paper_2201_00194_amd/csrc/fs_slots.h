// A stable counting sort of n entries by a number below `buckets`, in three kernels: every wavefront counts the numbers in
// its stretch of entries; a number's counts are summed along the stretches; every wavefront places its stretch's entries.
// No atomics on memory, and the same result whatever runs first.  Used for the slots of experts and for the table's gradient.
#ifndef FS_SLOTS_H
#define FS_SLOTS_H

#include "fs_mixture.h"

namespace fs {

constexpr int kSlotWaves = 4;               // of a workgroup
constexpr int kSlotMostBuckets = 1025;      // experts, and one for choices without a slot
constexpr int kSlotMostStretches = 4096;
constexpr int kSlotScanThreads = 256;
constexpr int kSlotScanPer = kSlotMostStretches / kSlotScanThreads;

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
// The counts, and behind them every number's total.
inline size_t slot_count_bytes(const SlotShape &s) { return s.n == 0 ? 0 : ((size_t)s.buckets * (s.stretches + 1) * 4 + 255) / 256 * 256; }

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
    lds_sync();
    if (mine >= s.stretches)
        return;
    const int64_t begin = (int64_t)mine * s.stretch, end = min(begin + s.stretch, (int64_t)s.n);
    for (int64_t i = begin + lane; i < end; i += 64)
        atomicAdd(&c[number(i)], 1);
    lds_sync();
    for (int b = lane; b < s.buckets; b += 64)
        count[(int64_t)b * s.stretches + mine] = c[b];
}

__device__ __forceinline__ int32_t wave_inclusive_sum(int32_t v, int lane)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int32_t t = __shfl_up(v, off);
        if (lane >= off)
            v += t;
    }
    return v;
}

// A workgroup a number: its counts become the sums of those before them, and their total goes behind all counts.
static __global__ void __launch_bounds__(kSlotScanThreads)
slot_scan_kernel(int32_t *count, SlotShape s)
{
    __shared__ int32_t wave_total[kSlotScanThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t *const row = count + (int64_t)blockIdx.x * s.stretches;
    const int per = (s.stretches + kSlotScanThreads - 1) / kSlotScanThreads, first = threadIdx.x * per;
    int32_t v[kSlotScanPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kSlotScanPer; ++i) {
        v[i] = i < per && first + i < s.stretches ? row[first + i] : 0;
        sum += v[i];
    }
    const int32_t upto = wave_inclusive_sum(sum, lane);
    if (lane == 63)
        wave_total[wave] = upto;
    __syncthreads();
    int32_t at = upto - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kSlotScanThreads / 64; ++w) {
        at += w < wave ? wave_total[w] : 0;
        total += wave_total[w];
    }
#pragma unroll
    for (int i = 0; i < kSlotScanPer; ++i) {
        if (i < per && first + i < s.stretches)
            row[first + i] = at;
        at += v[i];
    }
    if (threadIdx.x == 0)
        count[(int64_t)s.buckets * s.stretches + blockIdx.x] = total;
}

// put(i, number, slot) for every entry; put.start(number, slot of its first), once for every number.
template <class Number, class Put>
__global__ void __launch_bounds__(kSlotWaves * 64)
slot_place_kernel(Number number, Put put, SlotShape s, const int32_t *count)
{
    constexpr int kThreads = kSlotWaves * 64, kPer = (kSlotMostBuckets + kThreads - 1) / kThreads;
    __shared__ int32_t lds[kSlotWaves * kSlotMostBuckets], base[kSlotMostBuckets], wave_total[kSlotWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mine = (int)blockIdx.x * kSlotWaves + wave;
    const int32_t *const total = count + (int64_t)s.buckets * s.stretches;
    const int first = threadIdx.x * kPer;
    int32_t v[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        v[i] = first + i < s.buckets ? total[first + i] : 0;
        sum += v[i];
    }
    const int32_t upto = wave_inclusive_sum(sum, lane);
    if (lane == 63)
        wave_total[wave] = upto;
    __syncthreads();
    int32_t at = upto - sum;
#pragma unroll
    for (int w = 0; w < kSlotWaves; ++w)
        at += w < wave ? wave_total[w] : 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (first + i < s.buckets) {
            base[first + i] = at;
            if (blockIdx.x == 0)
                put.start(first + i, at);
        }
        at += v[i];
    }
    __syncthreads();
    if (mine >= s.stretches)
        return;
    int32_t *next = lds + wave * s.buckets;
    for (int b = lane; b < s.buckets; b += 64)
        next[b] = base[b] + count[(int64_t)b * s.stretches + mine];
    lds_sync();
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
        lds_sync();
        if (there && before == 0)
            next[m] = slot + __popcll(same);
        lds_sync();
        if (there)
            put(i, m, slot);
    }
}

template <class Number, class Put>
void launch_slots(const Number &number, const Put &put, const SlotShape &s, int32_t *count, hipStream_t stream)
{
    const dim3 grid((unsigned)((s.stretches + kSlotWaves - 1) / kSlotWaves)), block(kSlotWaves * 64);
    hipLaunchKernelGGL(slot_count_kernel<Number>, grid, block, 0, stream, number, s, count);
    hipLaunchKernelGGL(slot_scan_kernel, dim3((unsigned)s.buckets), dim3(kSlotScanThreads), 0, stream, count, s);
    hipLaunchKernelGGL((slot_place_kernel<Number, Put>), grid, block, 0, stream, number, put, s, (const int32_t *)count);
}

}  // namespace fs
#endif
