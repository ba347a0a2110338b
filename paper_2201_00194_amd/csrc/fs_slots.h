// A stable counting sort of n entries by a number below `buckets`.  Long lists take three kernels: every workgroup counts the
// numbers in its stretch of entries; a number's counts are summed along the stretches; every workgroup places its stretch's
// entries, a tile after the other, which it puts in order in LDS so that they leave in runs.  Up to kSlotFew entries are
// one workgroup's, in one kernel.  No atomics on memory, and the same result whatever runs first.  Used for the slots of
// experts and for the table's gradient.
//
// A Source says what the entries are: load(items, i) takes entries i, i + 64, ... (the last one, where that is past it), int
// number(item), place(i, number, slot) tells where entry i goes, put(what(item, i), number, slot) puts it there, and start(number, slot
// of its first) is called once for every number.  The launches that count and that place have more workgroups, for what can
// be done beside them: more_counting() that call beside_count(which, of how many), and the same for placing.
#ifndef FS_SLOTS_H
#define FS_SLOTS_H

#include "fs_mixture.h"

namespace fs {

constexpr int kSlotWaves = 8;               // of a workgroup
constexpr int kSlotThreads = kSlotWaves * 64;
constexpr int kSlotMostBuckets = 1025;      // experts, and one for choices without a slot
constexpr int kSlotMostBits = 11;
constexpr int kSlotMostPer = 8;             // entries of a lane in a tile
constexpr int kSlotManyGroups = 512;
constexpr int kSlotMostGroups = 2048;
constexpr int kSlotScanThreads = 256;
constexpr int kSlotScanPer = kSlotMostGroups / kSlotScanThreads;
constexpr int kSlotFew = 16384;
constexpr int kSlotFewWaves = 16;
constexpr int kSlotFewPer = kSlotFew / (kSlotFewWaves * 64);

struct SlotShape {
    int32_t n, buckets, per, tiles, groups;      // groups of `tiles` tiles of per * kSlotThreads entries
};
constexpr size_t slot_place_bytes(int per, int buckets, int what_bytes)
{
    return (size_t)per * kSlotThreads * (what_bytes + 2) + ((size_t)(kSlotWaves + 2) * buckets + kSlotWaves) * 4;
}
// Tiles short enough for kSlotManyGroups workgroups, but not shorter than the numbers are many: the counts then are no more
// than the entries.  A tile and its counts stay within 64 KB of LDS.  what_bytes: of what a tile puts in order.
inline SlotShape slot_shape(int64_t n, int buckets, int what_bytes)
{
    SlotShape s = {(int32_t)n, buckets, 0, 0, 0};
    int64_t per = (n + kSlotThreads * kSlotManyGroups - 1) / (kSlotThreads * kSlotManyGroups);
    const int64_t least = (buckets + kSlotThreads - 1) / kSlotThreads;
    per = per < least ? least : per;
    s.per = (int32_t)(per < 1 ? 1 : per > kSlotMostPer ? kSlotMostPer : per);
    while (s.per > 1 && slot_place_bytes(s.per, buckets, what_bytes) > 65536)
        --s.per;
    const int64_t tiles = (n + s.per * kSlotThreads - 1) / (s.per * kSlotThreads);
    s.tiles = (int32_t)((tiles + kSlotMostGroups - 1) / kSlotMostGroups);
    s.groups = s.tiles ? (int32_t)((tiles + s.tiles - 1) / s.tiles) : 0;
    return s;
}
// The counts, and behind them every number's total.
inline size_t slot_count_bytes(const SlotShape &s, int few)       // up to `few` entries need none
{
    return s.n <= few ? 0 : ((size_t)s.buckets * (s.groups + 1) * 4 + 255) / 256 * 256;
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
    while (b < 31 && (1 << b) < n)
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

// count[number * groups + group]
template <class Source>
__global__ void __launch_bounds__(kSlotThreads)
slot_count_kernel(Source source, SlotShape s, int32_t *count)
{
    extern __shared__ int32_t slot_lds[];
    if ((int)blockIdx.x >= s.groups) {
        source.beside_count(blockIdx.x - s.groups, gridDim.x - s.groups);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = threadIdx.x; b < kSlotWaves * s.buckets; b += kSlotThreads)
        slot_lds[b] = 0;
    __syncthreads();
    int32_t *const c = slot_lds + wave * s.buckets;
    const int64_t begin = (int64_t)blockIdx.x * s.tiles * s.per * kSlotThreads;
    const int64_t end = min(begin + (int64_t)s.tiles * s.per * kSlotThreads, (int64_t)s.n);
    for (int64_t i0 = begin + wave * kSlotMostPer * 64; i0 < end; i0 += kSlotMostPer * kSlotThreads) {
        typename Source::Item item[kSlotMostPer];
        source.load(item, i0 + lane, end);
#pragma unroll
        for (int u = 0; u < kSlotMostPer; ++u)
            if (i0 + u * 64 + lane < end)
                atomicAdd(&c[source.number(item[u])], 1);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < s.buckets; b += kSlotThreads) {
        int32_t sum = 0;
#pragma unroll
        for (int w = 0; w < kSlotWaves; ++w)
            sum += slot_lds[w * s.buckets + b];
        count[(int64_t)b * s.groups + blockIdx.x] = sum;
    }
}

// A workgroup a number: its counts become the sums of those before them, and their total goes behind all counts.
static __global__ void __launch_bounds__(kSlotScanThreads)
slot_scan_kernel(int32_t *count, SlotShape s)
{
    __shared__ int32_t wave_total[kSlotScanThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t *const row = count + (int64_t)blockIdx.x * s.groups;
    const int per = (s.groups + kSlotScanThreads - 1) / kSlotScanThreads, first = threadIdx.x * per;
    int32_t v[kSlotScanPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kSlotScanPer; ++i) {
        v[i] = i < per && first + i < s.groups ? row[first + i] : 0;
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
        if (i < per && first + i < s.groups)
            row[first + i] = at;
        at += v[i];
    }
    if (threadIdx.x == 0)
        count[(int64_t)s.buckets * s.groups + blockIdx.x] = total;
}

// Where all counts are few, every workgroup that places entries sums them itself: a kernel less.  131 072 choices of 30 experts (7936
// counts) 11.4 us so, 14.4 with the scan; past the border it depends on how many numbers there are: 80 000 choices of 64 (10 205 counts)
// 12.8 and 14.2, 20 000 of 255 (10 240) 16.3 and 13.9.
constexpr int kSlotFewCounts = 8192;
__host__ __device__ inline bool slots_scan_alone(const SlotShape &s) { return s.buckets * s.groups <= kSlotFewCounts; }
// Every number's total, and its count in the workgroups before this one; a barrier at the end.
__device__ __forceinline__ void sum_counts(const int32_t *count, const SlotShape &s, int32_t *total, int32_t *before)
{
    constexpr int kAtOnce = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b0 = wave * kAtOnce; b0 < s.buckets; b0 += kSlotWaves * kAtOnce) {
        int32_t all[kAtOnce] = {}, mine[kAtOnce] = {};
#pragma unroll 4
        for (int g = lane; g < s.groups; g += 64)
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int32_t v = count[min(b0 + u, s.buckets - 1) * s.groups + g];
                all[u] += v;
                mine[u] += g < (int)blockIdx.x ? v : 0;
            }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int32_t a = row_sum(all[u], 6), m = row_sum(mine[u], 6);
            if (lane == 0 && b0 + u < s.buckets) {
                total[b0 + u] = a;
                before[b0 + u] = m;
            }
        }
    }
    __syncthreads();
}

// f(number, sum of value(numbers before it)) by all threads of a workgroup of kSlotThreads; a barrier at the end.
template <class V, class F>
__device__ __forceinline__ void over_numbers(int buckets, int32_t *wave_total, V value, F f)
{
    constexpr int kPer = (kSlotMostBuckets + kSlotThreads - 1) / kSlotThreads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (buckets + kSlotThreads - 1) / kSlotThreads, first = threadIdx.x * per;
    int32_t v[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        v[i] = i < per && first + i < buckets ? value(first + i) : 0;
        sum += v[i];
    }
    const int32_t upto = wave_inclusive_sum(sum, lane);
    if (lane == 63)
        wave_total[wave] = upto;
    __syncthreads();
    int32_t at = upto - sum;
    for (int w = 0; w < wave; ++w)
        at += wave_total[w];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (i < per && first + i < buckets)
            f(first + i, at);
        at += v[i];
    }
    __syncthreads();
}

template <class Source>
__global__ void __launch_bounds__(kSlotThreads)
slot_place_kernel(Source source, SlotShape s, const int32_t *count)
{
    extern __shared__ int32_t slot_lds[];
    if ((int)blockIdx.x >= s.groups) {
        source.beside_place(blockIdx.x - s.groups, gridDim.x - s.groups);
        return;
    }
    typename Source::What *const staged = (typename Source::What *)slot_lds;         // the tile in order
    const int tile = s.per * kSlotThreads;
    int32_t *const c = (int32_t *)(staged + tile);          // of every wavefront: how often it met a number, then where in the tile
    int32_t *const to = c + kSlotWaves * s.buckets;         // a number's next slot, less its place in the tile
    int32_t *const met_all = to + s.buckets;                // how often the tile met it
    int32_t *const wave_total = met_all + s.buckets;
    uint16_t *const staged_number = (uint16_t *)(wave_total + kSlotWaves);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bits = bits_of(s.buckets);
    const int32_t *const total = count + (int64_t)s.buckets * s.groups;
    const bool scanned = !slots_scan_alone(s);
    if (!scanned)
        sum_counts(count, s, met_all, to);
    over_numbers(s.buckets, wave_total, [&](int b) { return scanned ? total[b] : met_all[b]; }, [&](int b, int32_t at) {
        to[b] = at + (scanned ? count[(int64_t)b * s.groups + blockIdx.x] : to[b]);
        met_all[b] = 0;
        if (blockIdx.x == 0)
            source.start(b, at);
    });
    const int64_t begin = (int64_t)blockIdx.x * s.tiles * tile;
    const int64_t end = min(begin + (int64_t)s.tiles * tile, (int64_t)s.n);
    for (int64_t t0 = begin; t0 < end; t0 += tile) {
        const int64_t i0 = t0 + wave * s.per * 64 + lane;
        typename Source::Item item[kSlotMostPer];
        source.load(item, i0, end);
        for (int b = threadIdx.x; b < kSlotWaves * s.buckets; b += kSlotThreads)
            c[b] = 0;
        __syncthreads();
        int rank[kSlotMostPer];
#pragma unroll
        for (int u = 0; u < kSlotMostPer; ++u)
            if (u < s.per)
                rank[u] = take_slot(c + wave * s.buckets, source.number(item[u]), bits, i0 + u * 64 < end);
        __syncthreads();
        const auto met_in = [&](int b) {
            int32_t sum = 0;
#pragma unroll
            for (int w = 0; w < kSlotWaves; ++w)
                sum += c[w * s.buckets + b];
            return sum;
        };
        over_numbers(s.buckets, wave_total, met_in, [&](int b, int32_t at) {
            to[b] += met_all[b] - at;                        // on past the tile before, less the place in this one
            int32_t sum = 0;
#pragma unroll
            for (int w = 0; w < kSlotWaves; ++w) {
                const int32_t n = c[w * s.buckets + b];
                c[w * s.buckets + b] = at + sum;
                sum += n;
            }
            met_all[b] = at + sum;
        });
#pragma unroll
        for (int u = 0; u < kSlotMostPer; ++u)
            if (u < s.per && i0 + u * 64 < end) {
                const int number = source.number(item[u]), at = c[wave * s.buckets + number] + rank[u];
                staged[at] = source.what(item[u], i0 + u * 64);
                staged_number[at] = (uint16_t)number;
                source.place(i0 + u * 64, number, to[number] + at);
            }
        __syncthreads();
        const int n = (int)min((int64_t)tile, end - t0);
        for (int at = threadIdx.x; at < n; at += kSlotThreads) {
            const int number = staged_number[at];
            source.put(staged[at], number, to[number] + at);
        }
        __syncthreads();
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
            if (there) {
                source.place(begin + u * 64, number, slot);
                source.put(source.what(item[u], begin + u * 64), number, slot);
            }
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
    hipLaunchKernelGGL(slot_count_kernel<Source>, dim3((unsigned)(s.groups + source.more_counting())), dim3(kSlotThreads),
                       (size_t)kSlotWaves * s.buckets * 4, stream, source, s, count);
    if (!slots_scan_alone(s))
        hipLaunchKernelGGL(slot_scan_kernel, dim3((unsigned)s.buckets), dim3(kSlotScanThreads), 0, stream, count, s);
    hipLaunchKernelGGL(slot_place_kernel<Source>, dim3((unsigned)(s.groups + source.more_placing())), dim3(kSlotThreads),
                       slot_place_bytes(s.per, s.buckets, sizeof(typename Source::What)), stream, source, s, (const int32_t *)count);
}

}  // namespace fs
#endif
