// A stable counting sort of n entries by a number below `buckets`.  Long lists take three kernels: every wavefront counts the
// numbers in its stretch of entries; a number's counts are summed along the stretches; every wavefront places its stretch's
// entries.  Up to kSlotFew entries are one workgroup's, in one kernel.  No atomics on memory, and the same result
// whatever runs first.  Used for the slots of experts and for the table's gradient.
//
// A Source says what the entries are: load(items, i) takes entries i, i + 64, ... (the last one, where that is past it), int
// number(item), put(item, i, number, slot), and start(number, slot of its first), called once for every number.
#ifndef FS_SLOTS_H
#define FS_SLOTS_H

#include "fs_mixture.h"

namespace fs {

constexpr int kSlotWaves = 4;               // of a workgroup
constexpr int kSlotMostBuckets = 1025;      // experts, and one for choices without a slot
constexpr int kSlotMostBits = 11;
constexpr int kSlotMostStretches = 4096;
constexpr int kSlotScanThreads = 256;
constexpr int kSlotScanPer = kSlotMostStretches / kSlotScanThreads;
constexpr int kSlotAhead = 8;               // loads of a lane on their way at once
constexpr int kSlotFew = 16384;
constexpr int kSlotFewWaves = 16;
constexpr int kSlotFewPer = kSlotFew / (kSlotFewWaves * 64);

struct SlotShape {
    int32_t n, buckets, stretch, stretches;
};
// Stretches as short as 128 entries, for as many wavefronts, but not shorter than the numbers are many: the counts then
// are no more than the entries.
inline SlotShape slot_shape(int64_t n, int buckets)
{
    SlotShape s = {(int32_t)n, buckets, 0, 0};
    int64_t stretch = (n + kSlotMostStretches - 1) / kSlotMostStretches;
    stretch = stretch < buckets ? buckets : stretch;
    stretch = stretch < 128 ? 128 : stretch;
    s.stretch = (int32_t)((stretch + 63) / 64 * 64);
    s.stretches = (int32_t)((n + s.stretch - 1) / s.stretch);
    return s;
}
// The counts, and behind them every number's total.
inline size_t slot_count_bytes(const SlotShape &s)
{
    return s.n <= kSlotFew ? 0 : ((size_t)s.buckets * (s.stretches + 1) * 4 + 255) / 256 * 256;
}

// The lanes whose number is this lane's, among the lanes that are there.
// Four instructions a bit: its sign, a compare, two three-way bit operations.
__device__ __forceinline__ uint64_t same_number(int number, int bits, bool there)
{
    const uint64_t all = __ballot(there);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
    for (int b = 0; b < kSlotMostBits; ++b) {
        if (b < bits) {
            const int mine = (int)((uint32_t)number << (31 - b)) >> 31;
            const uint64_t with = __ballot(mine != 0);
            lo &= ~((uint32_t)with ^ (uint32_t)mine);
            hi &= ~((uint32_t)(with >> 32) ^ (uint32_t)mine);
        }
    }
    return (uint64_t)hi << 32 | lo;
}
__host__ __device__ inline int bits_of(int n)        // of numbers below n
{
    int b = 0;
    while ((1 << b) < n)
        ++b;
    return b;
}
__device__ __forceinline__ int lanes_before(uint64_t lanes)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
}
// The slot of this lane's number: next[number] and up, in the order of the lanes; next moves on.
__device__ __forceinline__ int take_slot(int32_t *next, int number, int bits, bool there)
{
    const uint64_t same = same_number(number, bits, there);
    const int before = lanes_before(same);
    int slot = 0;
    if (there)
        slot = next[number] + before;
    lds_sync();
    if (there && before == 0)
        next[number] = slot + __popcll(same);
    lds_sync();
    return slot;
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

// count[number * stretches + stretch]
template <class Source>
__global__ void __launch_bounds__(kSlotWaves * 64)
slot_count_kernel(Source source, SlotShape s, int32_t *count)
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
    for (int64_t i0 = begin; i0 < end; i0 += kSlotAhead * 64) {
        typename Source::Item item[kSlotAhead];
        source.load(item, i0 + lane, end);
#pragma unroll
        for (int u = 0; u < kSlotAhead; ++u)
            if (i0 + u * 64 + lane < end)
                atomicAdd(&c[source.number(item[u])], 1);
    }
    lds_sync();
    for (int b = lane; b < s.buckets; b += 64)
        count[(int64_t)b * s.stretches + mine] = c[b];
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

template <class Source>
__global__ void __launch_bounds__(kSlotWaves * 64)
slot_place_kernel(Source source, SlotShape s, const int32_t *count)
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
                source.start(first + i, at);
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
    for (int64_t i0 = begin; i0 < end; i0 += kSlotAhead * 64) {
        typename Source::Item item[kSlotAhead];
        source.load(item, i0 + lane, end);
#pragma unroll
        for (int u = 0; u < kSlotAhead; ++u) {
            const int64_t i = i0 + u * 64 + lane;
            if (i0 + u * 64 < end) {
                const int number = source.number(item[u]);
                const int slot = take_slot(next, number, bits, i < end);
                if (i < end)
                    source.put(item[u], i, number, slot);
            }
        }
    }
}

// ---- few entries: one workgroup ----------------------------------------------------------------------------------------

// Sixteen wavefronts' counts (c[wave * buckets + number]) become every wavefront's first slot of a number; start(number, slot).
// All threads of the workgroup call it, after a barrier; it ends with one.
template <class F>
__device__ __forceinline__ void first_slots(int32_t *c, int buckets, int32_t *wave_total, F start)
{
    constexpr int kThreads = kSlotFewWaves * 64, kPer = (kSlotMostBuckets + kThreads - 1) / kThreads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (buckets + kThreads - 1) / kThreads, first = threadIdx.x * per;      // 1 or 2 numbers a thread
    int32_t sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < per && first + i < buckets)
            for (int w = 0; w < kSlotFewWaves; ++w)
                sum += c[w * buckets + first + i];
    const int32_t upto = wave_inclusive_sum(sum, lane);
    if (lane == 63)
        wave_total[wave] = upto;
    __syncthreads();
    int32_t at = upto - sum;
    for (int w = 0; w < wave; ++w)
        at += wave_total[w];
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < per && first + i < buckets) {
            start(first + i, at);
            for (int w = 0; w < kSlotFewWaves; ++w) {
                const int32_t n = c[w * buckets + first + i];
                c[w * buckets + first + i] = at;
                at += n;
            }
        }
    __syncthreads();
}

template <class Source>
__global__ void __launch_bounds__(kSlotFewWaves * 64)
slot_few_kernel(Source source, int32_t n, int32_t buckets)
{
    __shared__ int32_t c[kSlotFewWaves * kSlotMostBuckets], wave_total[kSlotFewWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int steps = (n + kSlotFewWaves * 64 - 1) / (kSlotFewWaves * 64);       // of a wavefront, at most kSlotFewPer
    const int begin = wave * steps * 64 + lane;
    typename Source::Item item[kSlotFewPer];
    source.load(item, begin, n);
    for (int b = threadIdx.x; b < kSlotFewWaves * buckets; b += kSlotFewWaves * 64)
        c[b] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSlotFewPer; ++u)
        if (u < steps && begin + u * 64 < n)
            atomicAdd(&c[wave * buckets + source.number(item[u])], 1);
    __syncthreads();
    first_slots(c, buckets, wave_total, [&](int number, int slot) { source.start(number, slot); });
    const int bits = bits_of(buckets);
#pragma unroll
    for (int u = 0; u < kSlotFewPer; ++u)
        if (u < steps) {
            const bool there = begin + u * 64 < n;
            const int number = source.number(item[u]);
            const int slot = take_slot(c + wave * buckets, number, bits, there);
            if (there)
                source.put(item[u], begin + u * 64, number, slot);
        }
}

template <class Source>
void launch_few_slots(const Source &source, const SlotShape &s, hipStream_t stream)
{
    hipLaunchKernelGGL(slot_few_kernel<Source>, dim3(1), dim3(kSlotFewWaves * 64), 0, stream, source, s.n, s.buckets);
}
template <class Source>
void launch_slots(const Source &source, const SlotShape &s, int32_t *count, hipStream_t stream)
{
    const dim3 grid((unsigned)((s.stretches + kSlotWaves - 1) / kSlotWaves)), block(kSlotWaves * 64);
    hipLaunchKernelGGL(slot_count_kernel<Source>, grid, block, 0, stream, source, s, count);
    hipLaunchKernelGGL(slot_scan_kernel, dim3((unsigned)s.buckets), dim3(kSlotScanThreads), 0, stream, count, s);
    hipLaunchKernelGGL(slot_place_kernel<Source>, grid, block, 0, stream, source, s, (const int32_t *)count);
}

}  // namespace fs
#endif
