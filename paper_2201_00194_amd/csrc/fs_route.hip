// Routing: logits to the k chosen experts of a token and their weights, and the logits' gradient.
//
// A row of E logits lies in 1 << ll neighbouring lanes, 16 a lane, so that a wavefront works on 64 >> ll rows and one
// step of a reduction takes one move between lanes.  The choice goes by 42 bits: a key's 32, made to compare like whole
// numbers, and the expert's number, turned round so that of equal keys the lower expert wins.  They stand in the mantissa of a double
// between 1 and 2, because a compare and exchange of doubles is two instructions at full rate, of 64-bit integers
// six.  Every lane sorts its keys in lists of KP >= k with Batcher's network, and two lists become the best KP of both by
// KP maxima (the one against the other turned round) and a bitonic merge, in the lane first, between lanes then.
//
// Keys with a bias (score + bias) and the sums of groups have to compare as in 64 bits.  They are computed in 32, with a bound
// on their error; a row where two keys that matter are nearer than the bounds say, and not equal by their inputs, or where a
// group at the cut may have as much as one beyond it, is taken again by the whole wavefront in 64 bits.  What that costs depends
// on the values.  Equal sums are taken again too: without a bias and with group_best 1, equal bf16 logits make them (262 144 rows
// of 64 experts in 8 groups 83 us, with group_best 2 41).  And a softmax score's bound does not shrink with the score, so that small
// scores next to each other are in doubt where the bias says nothing: a bias of zeros, 64 experts, k = 8, logits of standard
// deviation 1.5 42 us, 5 114, 8 279 (without the bias 19).
//
// What bounds it: 2 000 000 rows of 64 bf16 experts in 8 groups with a bias, k = 8, take 219 us (1.7 TB/s) at 1022 vector
// instructions a wavefront of 16 rows, with the vector units busy all the time.  Without bias and groups, 262 144 rows of 30 fp32
// experts, k = 4: 12 to 13 us (3.1 TB/s), the vector units half busy: loads, then one chain through the lists.
#include "fs_mixture.h"

#include <math.h>

namespace fs {

constexpr int kRouteWaves = 4;           // of a workgroup
constexpr int kRoutePer = 16;            // experts of a lane
constexpr int kRouteMostGroups = 32;     // more groups than a word has bits: every row in 64 bits

struct RouteArgs {
    fs_route_params p;
    int64_t n_tokens, stride, d_stride;
    const void *logits;
    const float *bias;
    int32_t *expert;
    float *weight;
    const int32_t *chosen;
    const float *d_weight;
    void *d_logits;
    int32_t ll, group_size;
    uint32_t group_magic;                // e / group_size = e * group_magic >> 22 for e < 1024
    int32_t exact;                       // 1: every row in 64 bits
    int32_t wave_lds;                    // bytes
    int64_t block0;                      // of this launch
};

// The value between -infinity and `most`; -infinity for a quiet NaN, as the median of three is defined on this hardware.  The
// compiler, where it sees the -infinity, takes the minimum of the other two instead, which is not.
__device__ __forceinline__ float bounded(float v, float most)
{
    float least = -__builtin_inff();
    asm("" : "+v"(least));
    return __builtin_amdgcn_fmed3f(v, least, most);
}
// NaN masks an expert as -infinity does; +infinity counts as the largest float.
__device__ __forceinline__ float route_logit(float l) { return bounded(__builtin_canonicalizef(l), 3.402823466e38f); }

// The logarithm of a score, but for a term that is the same for all of a row: it falls out of weights that are renormalised.
__device__ __forceinline__ float chosen_log(const RouteArgs &a, float x)
{
    return a.p.score == FS_SCORE_SOFTMAX ? x : fminf(x, 0.0f) - __logf(1.0f + exp_of(-fabsf(x)));
}

// ---- a row in 64 bits ---------------------------------------------------------------------------------------------------

__device__ __forceinline__ double wave_sum(double v) { return row_sum(v, 6); }
// The largest of n values in LDS, the first of equal ones; -1 if all are -infinity.
__device__ __forceinline__ int wave_argmax(const double *v, int n, int lane)
{
    double best = -__builtin_inf();
    int at = 1 << 30;
    for (int i = lane; i < n; i += 64)
        if (v[i] > best)
            best = v[i], at = i;
    for (int o = 32; o; o >>= 1) {
        const double b = __shfl_xor(best, o);
        const int a = __shfl_xor(at, o);
        if (b > best || (b == best && a < at))
            best = b, at = a;
    }
    return at == 1 << 30 ? -1 : at;
}
// The choice by 64-bit keys, in LDS; its weights as everywhere.
template <class T>
__device__ void route_exact(const RouteArgs &a, int64_t row, double *key, int lane)
{
    const int n = a.p.n_experts, k = a.p.k;
    const double none = -__builtin_inf();
    const T *logits = (const T *)a.logits + row * a.stride;
    double *group = key + n;
    const bool softmax = a.p.score == FS_SCORE_SOFTMAX;
    float top = -__builtin_inff();
#pragma nounroll
    for (int e = lane; e < n; e += 64)
        top = fmaxf(top, route_logit((float)logits[e]));
    top = row_max(top, 6);
    top = top == -__builtin_inff() ? 0.0f : top;
    double sum = 0.0;
    lds_sync();
#pragma nounroll
    for (int e = lane; e < n; e += 64) {
        const double x = route_logit((float)logits[e]), v = exp(softmax ? x - (double)top : -x);
        key[e] = softmax ? v : 1.0 / (1.0 + v);
        sum += v;
    }
    sum = wave_sum(sum);
#pragma nounroll
    for (int e = lane; e < n; e += 64) {
        const double s = softmax ? key[e] / sum : key[e], v = a.bias ? s + (double)a.bias[e] : s;
        key[e] = route_logit((float)logits[e]) > -__builtin_inff() && v > none ? v : none;
    }
    lds_sync();
    if (a.p.n_groups > 1) {
        const int per = a.group_size;
#pragma nounroll
        for (int g = lane; g < a.p.n_groups; g += 64) {
            double first = none, second = none;
#pragma nounroll
            for (int e = g * per; e < (g + 1) * per; ++e) {
                const double v = key[e];
                if (v > first)
                    second = first, first = v;
                else if (v > second)
                    second = v;
            }
            group[g] = a.p.group_best == 2 && second > none ? first + second : first;
        }
        lds_sync();
#pragma nounroll
        for (int r = 0; r < a.p.top_groups; ++r) {
            const int g = wave_argmax(group, a.p.n_groups, lane);
            lds_sync();
            if (g >= 0 && lane == 0)
                group[g] = __builtin_nan("");                 // taken
            lds_sync();
        }
#pragma nounroll
        for (int e = lane; e < n; e += 64) {
            const double t = group[e / per];
            if (t == t)
                key[e] = none;
            else if (!a.bias && key[e] > none)
                key[e] = route_logit((float)logits[e]);
        }
        lds_sync();
    }
    int mine = -1;
#pragma nounroll
    for (int j = 0; j < k; ++j) {
        const int e = wave_argmax(key, n, lane);
        lds_sync();
        if (e >= 0 && lane == 0)
            key[e] = none;
        if (lane == j)
            mine = e;
        lds_sync();
    }
    const float x = mine < 0 ? 0.0f : route_logit((float)logits[mine]);
    float w;
    if (a.p.renormalise) {
        const float s = mine < 0 ? -__builtin_inff() : chosen_log(a, x), high = row_max(s, 6);
        w = mine < 0 ? 0.0f : exp_of(s - high);
        const float all = row_sum(w, 6);
        w = all > 0.0f ? w * inverse(all) : 0.0f;
    } else {
        w = mine < 0 ? 0.0f : softmax ? exp_of(x - top) * inverse((float)sum) : inverse(1.0f + exp_of(-x));
    }
    if (lane < k) {
        a.expert[row * k + lane] = mine;
        a.weight[row * k + lane] = w * a.p.scale;
    }
}

// ---- keys and lists -------------------------------------------------------------------------------------------------------

// The key (not -0) and the expert as a double in [1, 2).
__device__ __forceinline__ double packed(float key, int e)
{
    const int bits = __float_as_int(key);
    const uint32_t order = (uint32_t)bits ^ ((uint32_t)(bits >> 31) | 0x80000000u);
    return __hiloint2double((int)__builtin_amdgcn_alignbit(0x3ffu, order, 12), (int)((order << 20) | (uint32_t)(1023 - e)));
}
// Nobody: an expert whose key is -infinity.
__device__ __forceinline__ bool somebody(double v) { return __double2hiint(v) > 0x3ff007ff; }
__device__ __forceinline__ int expert_of(double v) { return 1023 - (__double2loint(v) & 1023); }
__device__ __forceinline__ float key_of(double v)
{
    const uint32_t order = __builtin_amdgcn_alignbit((uint32_t)__double2hiint(v), (uint32_t)__double2loint(v), 20);
    return __uint_as_float(order ^ (~(uint32_t)((int)order >> 31) | 0x80000000u));
}

// 1 where a > b, else 0, from b * -kFar: one instruction, where a compare leaves a mask that the next may only read two cycles
// later.  The difference of two floats of common size times kFar is at least 1, or 0 or less; where sizes are not common, or
// infinite, it may be 0.
constexpr float kFar = 1.2676506e30f;     // 2^100
__device__ __forceinline__ float one_if_more(float a, float minus_b_far) { return __builtin_amdgcn_fmed3f(fmaf(a, kFar, minus_b_far), 0.0f, 1.0f); }
// Two of the largest so far, and another value.
__device__ __forceinline__ void best_two(float &first, float &second, float v)
{
    second = __builtin_amdgcn_fmed3f(first, second, v);
    first = fmaxf(first, v);
}
// __builtin_fmax would first make signalling NaNs quiet; there are none.  The compiler does not know of the wait that a value
// made so needs before another lane takes it: settled() is that wait.
__device__ __forceinline__ double larger(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double smaller(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ void in_order(double &a, double &b)
{
    const double hi = larger(a, b), lo = smaller(a, b);
    a = hi, b = lo;
}
// Largest first: Batcher's odd-even merge sort of N = 2^i values from `at` on.
template <int N>
struct SortNetwork {
    int n = 0, first[N * 4] = {}, second[N * 4] = {};
    constexpr SortNetwork()
    {
        for (int p = 1; p < N; p *= 2)
            for (int q = p; q >= 1; q /= 2)
                for (int j = q % p; j + q < N; j += 2 * q)
                    for (int i = 0; i < q && i + j + q < N; ++i)
                        if ((i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                            first[n] = i + j;
                            second[n++] = i + j + q;
                        }
    }
};
template <int N, int M>
__device__ __forceinline__ void sort_list(double (&v)[M], int at)
{
    constexpr SortNetwork<N> kNetwork;
#pragma unroll
    for (int i = 0; i < kNetwork.n; ++i)
        in_order(v[at + kNetwork.first[i]], v[at + kNetwork.second[i]]);
}
// list becomes the best KP of itself and other, both sorted.
template <int KP>
__device__ __forceinline__ void merge_list(double (&list)[KP], const double (&other)[KP])
{
#pragma unroll
    for (int i = 0; i < KP; ++i)
        list[i] = larger(list[i], other[KP - 1 - i]);
#pragma unroll
    for (int q = KP / 2; q >= 1; q /= 2)
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if ((i & q) == 0)
                in_order(list[i], list[i + q]);
}
template <int KP>
__device__ __forceinline__ void settled(double (&list)[KP])
{
    if constexpr (KP == 2) {
        asm volatile("s_nop 1" : "+v"(list[0]), "+v"(list[1]));
    } else if constexpr (KP == 4) {
        asm volatile("s_nop 1" : "+v"(list[0]), "+v"(list[1]), "+v"(list[2]), "+v"(list[3]));
    } else {
#pragma unroll
        for (int i = 0; i < KP; i += 8)
            asm volatile("s_nop 1"
                         : "+v"(list[i]), "+v"(list[i + 1]), "+v"(list[i + 2]), "+v"(list[i + 3]), "+v"(list[i + 4]), "+v"(list[i + 5]),
                           "+v"(list[i + 6]), "+v"(list[i + 7]));
    }
}
template <int STEP, int KP>
__device__ __forceinline__ void merge_met(double (&list)[KP])
{
    settled<KP>(list);
    double other[KP];
#pragma unroll
    for (int i = 0; i < KP; ++i)
        other[i] = met<STEP>(list[i]);
    merge_list<KP>(list, other);
}

// x[u]: expert expert_at(u) of the row, -infinity past the last.
template <class T>
__device__ __forceinline__ int expert_at(int u, int ll, int h) { return (((u / kChunk<T>) << ll) + h) * kChunk<T> + u % kChunk<T>; }

template <int KP>
__device__ __forceinline__ double entry_at(const double (&list)[KP], int j)
{
    int lo = __double2loint(list[0]), hi = __double2hiint(list[0]);
#pragma unroll
    for (int i = 1; i < KP; ++i) {
        lo = j == i ? __double2loint(list[i]) : lo;
        hi = j == i ? __double2hiint(list[i]) : hi;
    }
    return __hiloint2double(hi, lo);
}
template <int KP>
__device__ __forceinline__ float key_at(const double (&list)[KP], int j) { return key_of(entry_at<KP>(list, j)); }

// Whether two keys of this lane's row that matter are too near to be told apart by what they are in fp32 (each off by at most
// `off`, the sum's rounding on top), unless the same logit and bias made both: that is one key then, and the lower expert goes
// first.
template <class T, int KP>
__device__ __forceinline__ bool in_doubt(const RouteArgs &a, const T *logits, const double (&list)[KP], const float (&key)[kRoutePer], float off,
                                         int ll, int h)
{
    constexpr float kStep = 5.9604645e-8f;
    float size = 0.0f;
    bool again = false;
#pragma unroll
    for (int j = 0; j < KP; ++j)
        if (j < a.p.k && somebody(list[j]))
            size = fmaxf(size, fabsf(key_of(list[j])));
    if (!(size < __builtin_inff()))
        return true;
    const float near = 2.0f * off + 4.0f * kStep * size;
#pragma unroll
    for (int j = 0; j + 1 < KP; ++j)
        if (j + 1 < a.p.k && somebody(list[j + 1]) && !(key_of(list[j]) - key_of(list[j + 1]) > near)) {
            const int e = expert_of(list[j]), o = expert_of(list[j + 1]);
            again |= !(route_logit((float)logits[e]) == route_logit((float)logits[o]) && a.bias[e] == a.bias[o]);
        }
    const double end = entry_at<KP>(list, a.p.k - 1);
    if (somebody(end)) {
        const float last = key_of(end), border = last - 1.0001f * near;
        const int last_e = expert_of(end);
        const float last_x = route_logit((float)logits[last_e]), last_b = a.bias[last_e];
#pragma unroll
        for (int u = 0; u < kRoutePer; ++u) {
            const int e = expert_at<T>(u, ll, h);
            if (key[u] >= border && (key[u] < last || (key[u] == last && e > last_e)))
                again |= !(last_x == route_logit((float)logits[e]) && last_b == a.bias[e]);
        }
    }
    return again;
}

// ---- the kernel -----------------------------------------------------------------------------------------------------------

template <class T>
__device__ __forceinline__ void load_row(const T *logits, int n, int ll, int h, float (&x)[kRoutePer])
{
#pragma unroll
    for (int c = 0; c < kRoutePer / kChunk<T>; ++c) {
        const int e = expert_at<T>(c * kChunk<T>, ll, h);
        float v[kChunk<T>];
        load_chunk<kChunk<T>>(logits + e, n - e, v, -__builtin_inff());
#pragma unroll
        for (int i = 0; i < kChunk<T>; ++i)
            x[c * kChunk<T> + i] = route_logit(v[i]);
    }
}

// Choices i * (1 << LL) + h of the row's list are this lane's: their experts and weights go out.
template <class T, int KP, int LL>
__device__ __forceinline__ void finish(const RouteArgs &a, int64_t row, const T *logits, const double (&list)[KP], int h, float top, float sum,
                                       bool write)
{
    constexpr int kLanes = (1 << LL) < KP ? 1 << LL : KP, kMine = KP / kLanes;
    const float none = -__builtin_inff();
    float s[kMine];
    int expert[kMine];
    float high = none;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        double from[kLanes];
#pragma unroll
        for (int l = 0; l < kLanes; ++l)
            from[l] = list[i * kLanes + l];
#pragma unroll
        for (int half = kLanes / 2; half >= 1; half /= 2)
#pragma unroll
            for (int l = 0; l < half; ++l) {
                const double low = from[l], high_l = from[l + half];
                from[l] = (h & half) ? high_l : low;
            }
        const int j = i * kLanes + h;
        const bool there = h < kLanes && j < a.p.k && somebody(from[0]);
        expert[i] = there ? expert_of(from[0]) : -1;
        s[i] = none;
        if (there) {
            const float x = route_logit((float)logits[expert[i]]);
            s[i] = a.p.renormalise ? chosen_log(a, x) : x;
        }
        high = fmaxf(high, s[i]);
    }
    if (a.p.renormalise) {
        high = row_max(high, a.ll);
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            s[i] = expert[i] < 0 ? 0.0f : exp_of(s[i] - high);
            all += s[i];
        }
        all = row_sum(all, a.ll);
        const float factor = all > 0.0f ? a.p.scale * inverse(all) : 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            s[i] *= factor;
    } else {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (expert[i] < 0)
                s[i] = 0.0f;
            else if (a.p.score == FS_SCORE_SOFTMAX)
                s[i] = exp_of(s[i] - top) * inverse(sum) * a.p.scale;
            else
                s[i] = a.p.scale * inverse(1.0f + exp_of(-s[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int j = i * kLanes + h;
        if (write && h < kLanes && j < a.p.k) {
            a.expert[row * a.p.k + j] = expert[i];
            a.weight[row * a.p.k + j] = s[i];
        }
    }
}

template <int TYPE, int KP, bool EXACT>
__global__ void __launch_bounds__(kRouteWaves * 64, KP > 8 ? 4 : EXACT ? 5 : 8)
route_kernel(RouteArgs a)
{
    typedef typename Element<TYPE>::type T;
    extern __shared__ double lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ll = a.ll, h = lane & ((1 << ll) - 1);
    const int n = a.p.n_experts;
    const float none = -__builtin_inff();
    const int64_t row0 = ((a.block0 + blockIdx.x) * kRouteWaves + wave) << (6 - ll);
    if (row0 >= a.n_tokens)
        return;
    const bool there = row0 + (lane >> ll) < a.n_tokens;
    const int64_t row = there ? row0 + (lane >> ll) : a.n_tokens - 1;
    double *const own = lds + wave * (a.wave_lds / 8);
    bool again = EXACT && a.exact;                                  // this lane's row goes through 64 bits
    if (!(EXACT && a.exact)) {
        const T *logits = (const T *)a.logits + row * a.stride;
        float x[kRoutePer];
        load_row<T>(logits, n, ll, h, x);
        float top = 0.0f, sum = 1.0f;
        if (a.p.score == FS_SCORE_SOFTMAX && (EXACT || !a.p.renormalise)) {
            top = none;
#pragma unroll
            for (int u = 0; u < kRoutePer; ++u)
                top = fmaxf(top, x[u]);
            top = row_max(top, ll);
            top = top == none ? 0.0f : top;
            sum = 0.0f;
#pragma unroll
            for (int u = 0; u < kRoutePer; ++u)
                sum += exp_of(x[u] - top);
            sum = row_sum(sum, ll);
        }
        // Keys.  Bounds on the error of a score in fp32: with d = top - x, an exponential is off by (2 d + 4) 2^-24 of itself and
        // d exp(-d) < 0.37, a quotient and a sum of up to 1024 as a tree add 40: 48 * 2^-24 / sum; a sigmoid, by the same way
        // (s (1 - s) d < 0.23), 8 * 2^-24.  The sum with the bias rounds once more.
        constexpr float kStep = 5.9604645e-8f;                      // 2^-24
        float key[kRoutePer], off = 0.0f;
        if constexpr (EXACT) {
            if (a.p.score == FS_SCORE_SOFTMAX) {
                const float over = inverse(sum);
                off = 48.0f * kStep * over;
#pragma unroll
                for (int u = 0; u < kRoutePer; ++u)
                    key[u] = exp_of(x[u] - top) * over;
            } else {
                off = 8.0f * kStep;
#pragma unroll
                for (int u = 0; u < kRoutePer; ++u)
                    key[u] = inverse(1.0f + exp_of(-x[u]));
            }
            if (a.bias) {
#pragma unroll
                for (int c = 0; c < kRoutePer / kChunk<T>; ++c) {
                    const int e = expert_at<T>(c * kChunk<T>, ll, h);
                    float b[kChunk<T>];
                    load_chunk<kChunk<T>>(a.bias + e, n - e, b);
#pragma unroll
                    for (int i = 0; i < kChunk<T>; ++i)
                        key[c * kChunk<T> + i] += b[i];
                }
            }
#pragma unroll
            for (int u = 0; u < kRoutePer; ++u) {    // a NaN becomes -infinity
                const float v = bounded(key[u], __builtin_inff());
                key[u] = x[u] > none ? v : none;
            }
            if (a.p.n_groups > 1) {
                // A lane ranks groups h, h + (1 << ll), ... of its row by the sums of all, in LDS.  Of groups of one chunk these are
                // its own chunks; else what they are made of meets in LDS too: of groups of whole chunks every chunk's best two
                // keys, else all keys.  A group is taken if fewer than top_groups have more; where more are taken so, or fewer though
                // others are there (sums of 2^28 and more are not compared), or one that is not may have as much as one that is, nothing
                // is decided here.  A sum is off by what its own keys are: `off` and a rounding of each, which is large beside the
                // sum where the keys have opposite signs, and by the rounding of the sum itself; the least and the most that it may be
                // round once more.
                constexpr int kChunks = kRoutePer / kChunk<T>;
                const int padded = (a.p.n_groups + 3) & ~3;         // sums of nobody's groups behind
                float *const sums = (float *)own + ((((n + 3) & ~3) << (6 - ll)) + (lane >> ll) * padded);
                const bool one = a.group_size == kChunk<T>, whole = a.group_size % kChunk<T> == 0;
                float best[kChunks][2];
                if (whole) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) {
                        best[c][0] = key[c * kChunk<T>];
                        best[c][1] = none;
#pragma unroll
                        for (int i = 1; i < kChunk<T>; ++i)
                            best_two(best[c][0], best[c][1], key[c * kChunk<T> + i]);
                    }
                }
                // Two keys of finite size have a sum, whatever fp32 makes of it.
                const float most = 3.402823466e38f, of_best = (float)a.p.group_best;
                const auto sum_of = [&](float first, float second, float &wide) {
                    const bool both = a.p.group_best == 2 && second > none;
                    wide = of_best * fmaf(4.0f * kStep, both ? fmaxf(fabsf(first), fabsf(second)) : fabsf(first), off);
                    return both ? __builtin_amdgcn_fmed3f(first + second, -most, most) : first;
                };
                const auto more_than = [&](float mine) {
                    const float minus = -kFar * mine;
                    float n = 0.0f;
                    for (int o = 0; o < padded; o += 4) {
                        const float4 v = *(const float4 *)(sums + o);
                        n += one_if_more(v.x, minus) + one_if_more(v.y, minus) + (one_if_more(v.z, minus) + one_if_more(v.w, minus));
                    }
                    return n;
                };
                const float top_groups = (float)a.p.top_groups;
                // The least that a taken group may have, the most that another may.  A sum that is infinite is so in 64 bits too: its
                // bounds are NaN and count for nothing.
                float lowest = __builtin_inff(), highest = none, count = 0.0f;
                if (one) {
                    float sum[kChunks], wide[kChunks];
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) {
                        sum[c] = sum_of(best[c][0], best[c][1], wide[c]);
                        if ((c << ll) + h < padded)
                            sums[(c << ll) + h] = sum[c];
                    }
                    if constexpr (kChunks < 4)                                        // 2 groups of 8: nobody's, behind the last chunk
                        for (int g = (kChunks << ll) + h; g < padded; g += 1 << ll)
                            sums[g] = none;
                    lds_sync();
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) {
                        const bool in = sum[c] > none && more_than(sum[c]) < top_groups;
                        lowest = in ? fminf(lowest, sum[c] - wide[c]) : lowest;
                        highest = in ? highest : fmaxf(highest, sum[c] + wide[c]);
                        count += in ? 1.0f : 0.0f;
#pragma unroll
                        for (int i = 0; i < kChunk<T>; ++i)
                            key[c * kChunk<T> + i] = in ? key[c * kChunk<T> + i] : none;
                    }
                    count = row_sum(count, ll);
                } else {
                    const int width = whole ? n / kChunk<T> * 2 : n, per = width / a.p.n_groups;      // per: of a group
                    float *const keys = (float *)own + (lane >> ll) * width;
                    if (whole) {
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) {
                            const int e = expert_at<T>(c * kChunk<T>, ll, h);
                            if (e < n)
                                *(float2 *)(keys + e / kChunk<T> * 2) = make_float2(best[c][0], best[c][1]);
                        }
                    } else {
#pragma unroll
                        for (int u = 0; u < kRoutePer; ++u) {
                            const int e = expert_at<T>(u, ll, h);
                            if (e < n)
                                keys[e] = key[u];
                        }
                    }
                    lds_sync();
                    for (int g = h; g < padded; g += 1 << ll) {
                        float first = none, second = none;
                        if (g < a.p.n_groups)
                            for (int i = 0; i < per; ++i)
                                best_two(first, second, keys[g * per + i]);
                        float wide;
                        sums[g] = sum_of(first, second, wide);
                        if (g < a.p.n_groups)
                            keys[g * per] = wide;                   // this lane's, as its keys were
                    }
                    lds_sync();
                    int taken = 0;
                    for (int g = h; g < a.p.n_groups; g += 1 << ll) {
                        const float mine = sums[g], wide = keys[g * per];
                        const bool in = mine > none && more_than(mine) < top_groups;
                        lowest = in ? fminf(lowest, mine - wide) : lowest;
                        highest = in ? highest : fmaxf(highest, mine + wide);
                        taken |= in ? 1 << g : 0;
                    }
                    taken = row_or(taken, ll);
                    count = (float)__popc(taken);
#pragma unroll
                    for (int u = 0; u < kRoutePer; ++u) {
                        const int e = whole ? expert_at<T>(u / kChunk<T> * kChunk<T>, ll, h) : expert_at<T>(u, ll, h);
                        const bool in = taken >> ((uint32_t)e * a.group_magic >> 22 & 31) & 1;
                        key[u] = in ? key[u] : none;
                    }
                }
                lowest = -row_max(-lowest, ll);
                highest = row_max(highest, ll);
                again |= (highest > none ? count != top_groups : count > top_groups) || !(lowest > highest);
            }
            if (!a.bias)
#pragma unroll
                for (int u = 0; u < kRoutePer; ++u)
                    key[u] = key[u] > none ? x[u] + 0.0f : none;
        } else {
#pragma unroll
            for (int u = 0; u < kRoutePer; ++u)
                key[u] = x[u] + 0.0f;
        }
        double v[kRoutePer], list[KP];
#pragma unroll
        for (int u = 0; u < kRoutePer; ++u)
            v[u] = packed(key[u], expert_at<T>(u, ll, h));
#pragma unroll
        for (int u = 0; u < kRoutePer; u += KP)
            sort_list<KP>(v, u);
#pragma unroll
        for (int i = 0; i < KP; ++i)
            list[i] = v[i];
#pragma unroll
        for (int u = KP; u < kRoutePer; u += KP) {
            double other[KP];
#pragma unroll
            for (int i = 0; i < KP; ++i)
                other[i] = v[u + i];
            merge_list<KP>(list, other);
        }
        if (ll > 0) merge_met<0, KP>(list);
        if (ll > 1) merge_met<1, KP>(list);
        if (ll > 2) merge_met<2, KP>(list);
        if (ll > 3) merge_met<3, KP>(list);
        if (ll > 4) merge_met<4, KP>(list);
        if (ll > 5) merge_met<5, KP>(list);
        if constexpr (EXACT) {
            if (a.bias) {
                // Two of the list's keys nearer than `near` may be in the wrong order, and one that stayed outside may belong in
                // the place of the last: then more keys reach the border than the list has, over all rows of the wavefront.
                const float best = somebody(list[0]) ? key_of(list[0]) : 0.0f, last = key_at<KP>(list, a.p.k - 1);
                const bool full = last > none;
                const float near = 2.0f * off + 4.0f * kStep * fmaxf(fabsf(best), full ? fabsf(last) : 0.0f);
                const float border = full ? last - 1.0001f * near : __builtin_inff();
                float gap = __builtin_inff();
#pragma unroll
                for (int j = 0; j + 1 < KP; ++j)
                    if (j + 1 < a.p.k)
                        gap = fminf(gap, key_of(list[j]) - key_of(list[j + 1]));
                const bool doubt = !full || !(near < __builtin_inff()) || !(gap > near);
                int above = 0;
#pragma unroll
                for (int u = 0; u < kRoutePer; ++u)
                    above += __popcll(__ballot(key[u] >= border));
                if (__ballot(doubt) || above != __popcll(__ballot(full && h == 0)) * a.p.k)
                    again |= in_doubt<T, KP>(a, logits, list, key, off, ll, h);
            }
            again = row_or(again, ll);
        }
        const bool write = there && !again;
        if (ll == 0)
            finish<T, KP, 0>(a, row, logits, list, h, top, sum, write);
        else if (ll == 1)
            finish<T, KP, 1>(a, row, logits, list, h, top, sum, write);
        else if (ll == 2)
            finish<T, KP, 2>(a, row, logits, list, h, top, sum, write);
        else if (ll == 3)
            finish<T, KP, 3>(a, row, logits, list, h, top, sum, write);
        else
            finish<T, KP, 4>(a, row, logits, list, h, top, sum, write);
    }
    if constexpr (EXACT) {
        uint64_t rows = __ballot(again && there && h == 0);
        while (rows) {
            const int l = __builtin_ctzll(rows);
            rows &= rows - 1;
            route_exact<T>(a, row0 + (l >> ll), own, lane);
        }
    }
}

// ---- the gradient ---------------------------------------------------------------------------------------------------------

// The choices' gradients go to the row's logits through LDS; a row's experts lie in its lanes as above, its choices j in lane
// j mod (1 << LL).  262 144 rows of 30 fp32 experts, a dense gradient: 20 us (3.6 TB/s), the chain of loads, LDS and moves between
// lanes (vector units 38 % busy).
template <int TYPE, int LL>
__global__ void __launch_bounds__(kRouteWaves * 64)
route_backward_kernel(RouteArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int kMine = LL < 4 ? 16 >> LL : 1;
    __shared__ float lds[kRouteWaves * 64 * kRoutePer];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane & ((1 << LL) - 1);
    const int n = a.p.n_experts, k = a.p.k;
    const float none = -__builtin_inff();
    const int64_t row0 = ((a.block0 + blockIdx.x) * kRouteWaves + wave) << (6 - LL);
    if (row0 >= a.n_tokens)
        return;
    const bool there = row0 + (lane >> LL) < a.n_tokens;
    const int64_t row = there ? row0 + (lane >> LL) : a.n_tokens - 1;
    const T *logits = (const T *)a.logits + row * a.stride;
    float *const grad = lds + wave * 64 * kRoutePer + ((lane >> LL) << LL) * kRoutePer;      // of this row
    int expert[kMine];
    float g[kMine], l[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int j = (i << LL) + h;
        expert[i] = -1;
        g[i] = 0.0f;
        if (j < k) {
            expert[i] = a.chosen[row * k + j];
            g[i] = a.d_weight[row * k + j];
        }
    }
    float x[kRoutePer];
    load_row<T>(logits, n, LL, h, x);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const bool fits = expert[i] >= 0 && expert[i] < n;
        expert[i] = fits ? expert[i] : -1;
        g[i] = fits ? g[i] : 0.0f;
        l[i] = fits ? route_logit((float)logits[expert[i]]) : none;
    }
#pragma unroll
    for (int u = 0; u < kRoutePer; ++u)
        grad[expert_at<T>(u, LL, h)] = 0.0f;
    if (a.p.renormalise) {        // weight_j = exp(s_j) / sum exp(s_i), s the logit or the logarithm of its sigmoid
        float q[kMine], high = none, all = 0.0f, mean = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            q[i] = l[i] > none ? chosen_log(a, l[i]) : none;
            high = fmaxf(high, q[i]);
        }
        high = row_max(high, LL);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            q[i] = q[i] > none ? exp_of(q[i] - high) : 0.0f;
            all += q[i];
            mean += q[i] > 0.0f ? q[i] * g[i] : 0.0f;
        }
        all = row_sum(all, LL);
        all = all > 0.0f ? inverse(all) : 0.0f;
        mean = row_sum(mean, LL) * all;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            g[i] = q[i] > 0.0f ? q[i] * all * (g[i] - mean) : 0.0f;
            if (a.p.score == FS_SCORE_SIGMOID)
                g[i] *= inverse(1.0f + exp_of(l[i]));
        }
    }
    // An expert that a row names once (fs_route names no other way) gets its number, then its gradient.  Where numbers are
    // lost, the choices are added one after the other.
    lds_sync();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (expert[i] >= 0)
            grad[expert[i]] = (float)((i << LL) + h + 1);
    lds_sync();
    bool twice = false;
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        twice |= expert[i] >= 0 && grad[max(expert[i], 0)] != (float)((i << LL) + h + 1);
    lds_sync();
    if (__ballot(twice)) {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (expert[i] >= 0)
                grad[expert[i]] = 0.0f;
        lds_sync();
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            for (int o = 0; o < 1 << LL; ++o) {
                if (h == o && expert[i] >= 0)
                    grad[expert[i]] += g[i];
                lds_sync();
            }
    } else {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (expert[i] >= 0)
                grad[expert[i]] = g[i];
        lds_sync();
    }
    float d[kRoutePer];
#pragma unroll
    for (int u = 0; u < kRoutePer; ++u)
        d[u] = grad[expert_at<T>(u, LL, h)];
    if (!a.p.renormalise && a.p.score == FS_SCORE_SOFTMAX) {
        float top = none, sum = 0.0f, dot = 0.0f, p[kRoutePer];
#pragma unroll
        for (int u = 0; u < kRoutePer; ++u)
            top = fmaxf(top, x[u]);
        top = row_max(top, LL);
        top = top == none ? 0.0f : top;
#pragma unroll
        for (int u = 0; u < kRoutePer; ++u) {
            p[u] = exp_of(x[u] - top);
            sum += p[u];
            dot += p[u] > 0.0f ? p[u] * d[u] : 0.0f;
        }
        const float factor = inverse(row_sum(sum, LL));
        dot = row_sum(dot, LL) * factor;
#pragma unroll
        for (int u = 0; u < kRoutePer; ++u)
            d[u] = p[u] * factor * (d[u] - dot);
    } else if (!a.p.renormalise) {
#pragma unroll
        for (int u = 0; u < kRoutePer; ++u) {    // s (1 - s) = 1 / (1 + exp(|x|)) * 1 / (1 + exp(-|x|))
            const float small = exp_of(-fabsf(x[u])), over = inverse(1.0f + small);
            d[u] *= small * over * over;
        }
    }
    if (!there)
        return;
    T *out = (T *)a.d_logits + row * a.d_stride;
#pragma unroll
    for (int c = 0; c < kRoutePer / kChunk<T>; ++c) {
        const int e = expert_at<T>(c * kChunk<T>, LL, h);
        float v[kChunk<T>];
#pragma unroll
        for (int i = 0; i < kChunk<T>; ++i) {
            const int u = c * kChunk<T> + i;
            v[i] = x[u] > none ? d[u] * a.p.scale : 0.0f;
        }
        store_chunk<kChunk<T>>(out + e, n - e, v);
    }
}

static int lanes_log(int n_experts)
{
    int ll = 0;
    while ((kRoutePer << ll) < n_experts)
        ++ll;
    return ll;
}

static int check_route(const char *who, const fs_route_params *p, int64_t n_tokens, const void *logits, int32_t type, int64_t stride)
{
    if (!p)
        return fail(FS_EINVAL, "%s: params is NULL", who);
    if (p->n_experts < 1 || p->n_experts > FS_MAX_EXPERTS)
        return fail(p->n_experts < 1 ? FS_EINVAL : FS_EUNSUPPORTED, "%s: n_experts %d outside [1, %d]", who, p->n_experts, FS_MAX_EXPERTS);
    if (p->k < 1 || p->k > p->n_experts)
        return fail(FS_EINVAL, "%s: k %d outside [1, %d experts]", who, p->k, p->n_experts);
    if (p->k > FS_MAX_CHOICES)
        return fail(FS_EUNSUPPORTED, "%s: k %d over %d", who, p->k, FS_MAX_CHOICES);
    if (p->score != FS_SCORE_SOFTMAX && p->score != FS_SCORE_SIGMOID)
        return fail(FS_EINVAL, "%s: unknown score %d", who, p->score);
    if (p->renormalise != 0 && p->renormalise != 1)
        return fail(FS_EINVAL, "%s: renormalise is %d", who, p->renormalise);
    if (p->n_groups < 1 || p->n_groups > p->n_experts || p->n_experts % p->n_groups != 0)
        return fail(FS_EINVAL, "%s: %d experts in %d groups", who, p->n_experts, p->n_groups);
    if (p->top_groups < 1 || p->top_groups > p->n_groups)
        return fail(FS_EINVAL, "%s: top_groups %d outside [1, %d groups]", who, p->top_groups, p->n_groups);
    if (p->group_best != 1 && p->group_best != 2)
        return fail(FS_EINVAL, "%s: group_best %d is neither 1 nor 2", who, p->group_best);
    if (!isfinite(p->scale))
        return fail(FS_EINVAL, "%s: scale is not finite", who);
    FS_TRY(check_tokens(who, n_tokens, p->k));
    return check_matrix(who, "logits", logits, n_tokens, p->n_experts, type, stride);
}

}  // namespace fs

using namespace fs;

extern "C" int fs_route(const fs_route_params *params, int64_t n_tokens, const void *logits, int32_t logit_type, int64_t logit_stride,
                        const float *bias, int32_t *expert, float *weight, void *stream_)
{
    static const char who[] = "fs_route";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_route(who, params, n_tokens, logits, logit_type, logit_stride));
    FS_TRY(check_array(who, "bias", bias, 0, 4));
    FS_TRY(check_array(who, "expert", expert, n_tokens, 4));
    FS_TRY(check_array(who, "weight", weight, n_tokens, 4));
    if (n_tokens == 0)
        return FS_OK;
    const int n = params->n_experts, groups = params->n_groups, ll = lanes_log(n);
    const bool exact = bias || groups > 1;
    size_t wave_lds = 0;
    if (exact) {
        const size_t wide = (size_t)(n + (groups > 1 ? groups : 0)) * 8, rows = groups > 1 ? ((size_t)((n + 3) / 4 + (groups + 3) / 4) << (6 - ll)) * 16 : 0;
        wave_lds = ((wide > rows && wide > 0 ? wide : rows) + 15) / 16 * 16;
    }
    RouteArgs a = {*params, n_tokens, logit_stride, 0, logits, bias, expert, weight, nullptr, nullptr, nullptr, ll, n / groups,
                   (uint32_t)((1 << 22) / (n / groups) + 1),
                   exact && groups > kRouteMostGroups, (int32_t)wave_lds, 0};
    const int64_t rows = (int64_t)kRouteWaves << (6 - ll);
    prof_start(kKernTopk, stream);
    with_type(logit_type, [&](auto t) {
        constexpr int type = decltype(t)::value;
        const auto go = [&](auto kernel) {
            in_pieces((n_tokens + rows - 1) / rows, [&](int64_t at, unsigned blocks) {
                a.block0 = at;
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kRouteWaves * 64), kRouteWaves * wave_lds, stream, a);
            });
        };
        if (params->k <= 2)
            exact ? go(route_kernel<type, 2, true>) : go(route_kernel<type, 2, false>);
        else if (params->k <= 4)
            exact ? go(route_kernel<type, 4, true>) : go(route_kernel<type, 4, false>);
        else if (params->k <= 8)
            exact ? go(route_kernel<type, 8, true>) : go(route_kernel<type, 8, false>);
        else
            exact ? go(route_kernel<type, 16, true>) : go(route_kernel<type, 16, false>);
    });
    prof_stop(stream);
    return launched("route kernel launch");
}

extern "C" int fs_route_backward(const fs_route_params *params, int64_t n_tokens, const void *logits, int32_t logit_type, int64_t logit_stride,
                                 const int32_t *expert, const float *d_weight, void *d_logits, int64_t d_logit_stride, void *stream_)
{
    static const char who[] = "fs_route_backward";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_route(who, params, n_tokens, logits, logit_type, logit_stride));
    FS_TRY(check_array(who, "expert", expert, n_tokens, 4));
    FS_TRY(check_array(who, "d_weight", d_weight, n_tokens, 4));
    FS_TRY(check_matrix(who, "d_logits", d_logits, n_tokens, params->n_experts, logit_type, d_logit_stride));
    if (n_tokens == 0)
        return FS_OK;
    RouteArgs a = {*params, n_tokens, logit_stride, d_logit_stride, logits, nullptr, nullptr, nullptr, expert, d_weight, d_logits,
                   lanes_log(params->n_experts), 0, 0, 0, 0, 0};
    const int64_t rows = (int64_t)kRouteWaves << (6 - a.ll);
    prof_start(kKernTrainOther, stream);
    with_type(logit_type, [&](auto t) {
        constexpr int type = decltype(t)::value;
        const auto go = [&](auto kernel) {
            in_pieces((n_tokens + rows - 1) / rows, [&](int64_t at, unsigned blocks) {
                a.block0 = at;
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kRouteWaves * 64), 0, stream, a);
            });
        };
        switch (a.ll) {
        case 0: go(route_backward_kernel<type, 0>); break;
        case 1: go(route_backward_kernel<type, 1>); break;
        case 2: go(route_backward_kernel<type, 2>); break;
        case 3: go(route_backward_kernel<type, 3>); break;
        case 4: go(route_backward_kernel<type, 4>); break;
        case 5: go(route_backward_kernel<type, 5>); break;
        default: go(route_backward_kernel<type, 6>); break;
        }
    });
    prof_stop(stream);
    return launched("route gradient kernel launch");
}
