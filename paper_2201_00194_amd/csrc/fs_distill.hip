// Distillation from a teacher's largest logits, and its gradient.
//
// With m the largest logit of the row and s the sum of exp((x - m) / T), log p_c = (x_c - m) / T - log s.  The gradient is d_c =
// coefficient * (Q p_c - the entries' q of c) with Q the sum of all q: one factor on exp((x_c - m) / T) for all classes without an entry, whose few
// others are written afterwards.  With a rest, its share of p meets its q in a difference that may be small, so m and s go over the
// classes without an entry alone (a bit a class says which have one), entries are added in 64 bits, and p_rest = 1 / (1 + entries / rest)
// is as exact as they are.
#include "fs_mixture.h"
#include "familyseer_experts.h"

namespace fs {

struct DistillArgs {
    const void *logits, *ids, *teacher;
    const float *total, *d_loss;
    float *loss;
    void *d_logits;
    int64_t n_tokens, logit_stride, d_logit_stride;
    int32_t n_classes, k, id_type, teacher_type;
    int32_t n_bits, ll;         // classes that have a bit; lanes of a row
    float rate, twice_rate;     // log2(e) / T
    double inverse_t, inverse_rate, scale;
};

// -infinity for NaN, the largest float for infinity.  NaN that signals is made quiet first: of it and a number the larger is NaN, of
// quiet NaN and a number it is the number.
__device__ __forceinline__ float clean(float v) { return fminf(fmaxf(__builtin_canonicalizef(v), -__builtin_inff()), 3.402823466e38f); }

__device__ __forceinline__ int64_t id_at(const void *ids, int type, int64_t i) { return type == FS_ID_I64 ? ((const int64_t *)ids)[i] : ((const int32_t *)ids)[i]; }
__device__ __forceinline__ float element_at(const void *p, int type, int64_t i)
{
    return type == FS_F32 ? ((const float *)p)[i] : type == FS_BF16 ? (float)((const __bf16 *)p)[i] : (float)((const _Float16 *)p)[i];
}

// ---- exponential and logarithm in 64 bits --------------------------------------------------------
// From their series, to 1e-12 and better.  They run beside rows that fill the registers: their coefficients are brought where they are
// used and not kept from one call to the next, which the library's functions' are.
__device__ __forceinline__ double brought(double c)
{
    asm volatile("" : "+s"(c));
    return c;
}
// v = n log 2 + f, |f| <= log(2) / 2; the series of exp(f) to f^11 / 11!.  n log 2 is taken off as log 2 rounded to 64 bits, in one rounding of
// what is left, and what that leaves of it.
__device__ __forceinline__ double exp_of_double(double v)
{
    const double n = __builtin_rint(fmax(v, -740.0) * brought(1.4426950408889634)), f = fma(n, brought(-2.3190468138462996e-17), fma(n, brought(-0.69314718055994531), v));
    double e = brought(1.0 / 39916800);
    e = fma(e, f, brought(1.0 / 3628800));
    e = fma(e, f, brought(1.0 / 362880));
    e = fma(e, f, brought(1.0 / 40320));
    e = fma(e, f, brought(1.0 / 5040));
    e = fma(e, f, brought(1.0 / 720));
    e = fma(e, f, brought(1.0 / 120));
    e = fma(e, f, brought(1.0 / 24));
    e = fma(e, f, brought(1.0 / 6));
    e = fma(e, f, 0.5);
    e = fma(e, f, 1.0);
    e = fma(e, f, 1.0);
    return v < -740.0 ? 0.0 : __builtin_ldexp(e, (int)n);
}
// log((1 + t) / (1 - t)) = 2 (t + t^3 / 3 + t^5 / 5 + ...), |t| < 0.172.
__device__ __forceinline__ double log_of_ratio(double t)
{
    const double u = t * t;
    double s = brought(1.0 / 15);
    s = fma(s, u, brought(1.0 / 13));
    s = fma(s, u, brought(1.0 / 11));
    s = fma(s, u, brought(1.0 / 9));
    s = fma(s, u, brought(1.0 / 7));
    s = fma(s, u, brought(1.0 / 5));
    s = fma(s, u, brought(1.0 / 3));
    return 2.0 * fma(s * u, t, t);
}
__device__ __forceinline__ double log_of_double(double v)
{
    int n = __builtin_amdgcn_frexp_exp(v);
    double m = __builtin_amdgcn_frexp_mant(v);            // 1/2 to 1
    if (m < 0.70710678118654752) {
        m += m;
        --n;
    }
    return v > 0 ? fma((double)n, brought(0.69314718055994531), log_of_ratio((m - 1.0) / (m + 1.0))) : -__builtin_inf();
}
__device__ __forceinline__ double log_of_1_and(double v) { return v < 0.4 ? log_of_ratio(v / (2.0 + v)) : log_of_double(1.0 + v); }

// ---- the threads of a row ------------------------------------------------------------------------
// WAVES > 0: a workgroup of so many wavefronts.  0: 1 << ll lanes of a wavefront, of which a workgroup has four.
template <int WAVES>
struct Team {
    static constexpr int threads = WAVES ? WAVES * 64 : 256;
    double *joined;               // LDS: a number a wavefront
    int ll, lanes, h;             // 1 << ll lanes of a wavefront belong together; `lanes` threads in all, of which this is the h-th
    __device__ __forceinline__ Team(double *lds, int lanes_log) : joined(lds)
    {
        ll = WAVES ? 6 : lanes_log;
        lanes = WAVES ? WAVES * 64 : 1 << lanes_log;
        h = WAVES ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
    }
    __device__ __forceinline__ void sync() const
    {
        if constexpr (WAVES > 1)
            __syncthreads();
        else
            lds_sync();
    }
    // Of all threads' values, in an order that the sizes alone decide; all get the result.
    template <class T, class F>
    __device__ __forceinline__ T join(T v, F f) const
    {
        v = row_reduce(v, ll, f);
        if constexpr (WAVES > 1) {
            T *const one = (T *)joined;
            __syncthreads();            // what was here before has been read
            if ((threadIdx.x & 63) == 0)
                one[threadIdx.x >> 6] = v;
            __syncthreads();
            v = one[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
                v = f(v, one[w]);
        }
        return v;
    }
    // The first wavefront's part of the work on entries.
    __device__ __forceinline__ bool leads() const { return !WAVES || threadIdx.x < 64; }
    __device__ __forceinline__ int part() const { return WAVES ? 64 : lanes; }      // lanes that share it
};

// What the entries of a row make of it.
struct Verdict {
    float factor, from;         // d = exp((x - from) / T) * factor
};
// An entry, in LDS.
struct Entry {
    int id;                     // its class; -1: it does not count
    float x, t;                 // student's and teacher's logit; x: afterwards the gradient
    float q;
};
// LDS of a row: the bits of its classes, its entries, the verdict and whether a class is named twice.
struct RowLds {
    unsigned *bits;
    Entry *entry;
    Verdict *verdict;
    int *twice;
};
inline __host__ __device__ size_t row_lds_words(int n_bits, int k) { return (size_t)(n_bits + 31) / 32 + (size_t)k * 4 + 4; }

// M and S: the largest logit, or a number beside it, and the sum of exp((x - M) / T), of classes without an entry where `apart`; M is
// -infinity where there are none.  By the lanes of a wavefront that
// belong together; reductions are theirs.
template <bool GRADIENT>
__device__ __forceinline__ void judge(const DistillArgs &a, const RowLds &row, int64_t r, bool there, bool apart, bool search, double total, float from, double M, double S,
                                      int ll, int h)
{
    const int lanes = 1 << ll;
    float top = -__builtin_inff(), high = -__builtin_inff();
    for (int j = h; j < a.k; j += lanes) {
        const Entry e = row.entry[j];
        if (e.id >= 0) {
            top = fmaxf(top, e.t);
            high = fmaxf(high, e.x);
        }
    }
    top = row_max(top, ll);
    high = row_max(high, ll);
    const bool taught = top > -__builtin_inff(), none = !(M > -__builtin_inf()), rest = apart && !none;
    const double all_high = apart ? fmax((double)high, M) : M;
    const auto owns = [&](int j, int id) {
        bool first = true;
        if (search)
            for (int i = 0; i < j; ++i)
                first &= row.entry[i].id != id;
        return first;
    };
    double beside = 0, q_top = 0;
    for (int j = h; j < a.k; j += lanes) {
        const Entry e = row.entry[j];
        if (e.id < 0)
            continue;
        if (apart && owns(j, e.id))
            beside += exp_of_double(((double)e.x - all_high) * a.inverse_t);
        if (!rest)
            q_top += exp_of_double(((double)e.t - top) * a.inverse_t);
    }
    beside = row_sum(beside, ll);
    q_top = row_sum(q_top, ll);
    const double down = none ? 0.0 : exp_of_double((M - all_high) * a.inverse_t), Z = S * down + beside, log_z = log_of_double(Z);
    // log q = (t - base) / T - log_base
    const double base = rest ? 0.0 : top, log_base = rest ? total : log_of_double(q_top);
    double q_all = 0, loss = 0;
    for (int j = h; j < a.k; j += lanes) {
        const Entry e = row.entry[j];
        float q = 0.0f;
        if (e.id >= 0) {
            const double log_q = fmin(0.0, ((double)e.t - base) * a.inverse_t - log_base), share = exp_of_double(log_q);
            q_all += share;
            loss += share > 0 ? share * (log_q - (((double)e.x - all_high) * a.inverse_t - log_z)) : 0.0;
            q = (float)share;
        }
        row.entry[j].q = q;
    }
    q_all = row_sum(q_all, ll);
    loss = row_sum(loss, ll);
    double q_rest = 0, p_rest = 0;
    if (rest && taught) {
        q_rest = fmax(0.0, 1.0 - q_all);
        const double ratio = beside / (S * down);
        const double log_p = ratio < 1e300 ? -log_of_1_and(ratio) : (M - all_high) * a.inverse_t + log_of_double(S) - log_z;
        p_rest = exp_of_double(log_p);
        if (q_rest > 0)
            loss += q_rest * (log_of_double(q_rest) - log_p);
    }
    if (a.loss && there && h == 0)
        a.loss[r] = taught ? (float)(loss * a.scale) : 0.0f;
    if constexpr (GRADIENT) {
        lds_sync();      // all q are there
        const double coefficient = taught ? (double)a.d_loss[r] * a.scale * a.inverse_t : 0.0, q_sum = q_all + q_rest;
        for (int j = h; j < a.k; j += lanes) {
            const Entry e = row.entry[j];
            if (e.id < 0)
                continue;
            if (!owns(j, e.id)) {
                row.entry[j].t = __builtin_nanf("");      // another entry's
                continue;
            }
            double own = e.q;
            if (search)
                for (int i = j + 1; i < a.k; ++i)
                    own += row.entry[i].id == e.id ? row.entry[i].q : 0.0f;
            row.entry[j].x = (float)(coefficient * (q_sum * exp_of_double(((double)e.x - all_high) * a.inverse_t - log_z) - own));
        }
        if (h == 0) {
            row.verdict->factor = taught && !none ? (float)(coefficient * (rest ? (q_sum * p_rest - q_rest) / S : q_sum * down / Z)) : 0.0f;
            row.verdict->from = from;
        }
    }
}

// A row's entries and, for classes that are looked at apart, its bits, which are 0.
template <class T, int WAVES>
__device__ __forceinline__ void collect(const DistillArgs &a, const RowLds &row, const Team<WAVES> &team, int64_t r, bool bits)
{
    const T *const logits = (const T *)a.logits + r * a.logit_stride;
    for (int j = team.h; j < a.k; j += team.lanes) {
        const int64_t c = id_at(a.ids, a.id_type, r * a.k + j);
        Entry e = {-1, -__builtin_inff(), clean(element_at(a.teacher, a.teacher_type, r * a.k + j)), 0.0f};
        if (c >= 0 && c < a.n_classes)
            e.x = clean((float)logits[c]);
        if (e.x > -__builtin_inff() && e.t > -__builtin_inff())
            e.id = (int)c;
        row.entry[j] = e;
        if (bits && e.id >= 0 && (atomicOr(&row.bits[e.id >> 5], 1u << (e.id & 31)) >> (e.id & 31) & 1))
            *row.twice = 1;
    }
}
template <class T, int WAVES>
__device__ __forceinline__ void store_entries(const DistillArgs &a, const RowLds &row, const Team<WAVES> &team, int64_t r)
{
    T *const d_logits = (T *)a.d_logits + r * a.d_logit_stride;
    for (int j = team.h; j < a.k; j += team.lanes) {
        const Entry e = row.entry[j];
        if (e.id >= 0 && e.t == e.t)
            d_logits[e.id] = (T)e.x;
    }
}
// exp((v - from) / T) of a logit whatever it holds: NaN counts as -infinity, infinity as the largest float, which is `from` then.  The
// difference is of halves, as that of two floats may be no float, and times twice the rate, which is 2^127 * 1.45 at most.
__device__ __forceinline__ float share_of(float v, float from, float twice_rate)
{
    return __builtin_amdgcn_exp2f(fminf(fmaxf(fmaf(v, 0.5f, -0.5f * from), -__builtin_inff()), 0.0f) * twice_rate);
}

// Exponents of 2 are counted from a largest one that is rounded: below this, it is off by less than 1.
constexpr float kPlain = 16777216.0f;

// The same chunk, of which nothing is known: what was made of its elements before is not kept beside it.
template <class T>
__device__ __forceinline__ T anew(T v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// Rows of which a thread keeps C chunks of 16 bytes in registers, so that they are read once.  As a chunk has done its work, the next row's is
// asked for.  4096 rows of 131 072 bf16 and their gradient: 522 us, 4.1 TB/s of reads and writes (a copy reaches 4.7), 1000 rows of 32 001
// fp16 with a rest 36 us, 3.5 TB/s; 5120 rows of 64 fp32, losses alone, 5.9 us, the chain of one verdict.
template <int TYPE, bool GRADIENT, int WAVES, int C>
__global__ void __launch_bounds__(Team<WAVES>::threads, WAVES == 16 ? 4 : C < 16 ? 1 : WAVES ? 4 : 3)
distill_row_kernel(DistillArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int N = kChunk<T>, threads = Team<WAVES>::threads;
    typedef typename ChunkOf<T, N>::type Chunk;
    constexpr int kStash = GRADIENT && WAVES && C == 16 ? 12 : 0;
    __shared__ double joined[16];
    __shared__ Chunk stash[kStash ? kStash * 64 : 1];
    extern __shared__ unsigned lds[];
    const Team<WAVES> team(joined, a.ll);
    const int teams = WAVES ? 1 : threads / team.lanes, mine = WAVES ? 0 : (int)threadIdx.x / team.lanes;
    const bool bits = a.n_bits > 0;
    unsigned *const own = lds + mine * row_lds_words(a.n_bits, a.k);
    const RowLds row = {own, (Entry *)(own + (a.n_bits + 31) / 32), (Verdict *)(own + (a.n_bits + 31) / 32 + a.k * 4), (int *)(own + (a.n_bits + 31) / 32 + a.k * 4 + 2)};
    const int64_t by = (int64_t)gridDim.x * teams;
    const T nothing = (T)-__builtin_inff();
    Chunk x[C];
    const auto load = [&](int c, int64_t r) {
        const T *const p = (const T *)a.logits + r * a.logit_stride;
        const int first = (c * team.lanes + anew(team.h)) * N, n = a.n_classes - first;
        if ((c + 1) * team.lanes * N <= a.n_classes) {
            x[c] = *(const Chunk *)(p + first);
        } else if (c * team.lanes * N < a.n_classes) {
            if (n >= N) {
                x[c] = *(const Chunk *)(p + first);
            } else {
                Chunk v;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    v[i] = i < n ? p[first + i] : nothing;
                x[c] = v;
            }
        }
    };
    const auto has = [&](int c) { return c * team.lanes * N < a.n_classes; };
    int64_t r = (int64_t)blockIdx.x * teams + mine;
#pragma unroll
    for (int c = 0; c < C; ++c)
        load(c, min(r, a.n_tokens - 1));
    // All teams of a wavefront go round together; one whose rows are done does another's without storing anything.
    for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < a.n_tokens; r0 += by, r += by) {
        const bool there = r < a.n_tokens;
        const int64_t now = there ? r : a.n_tokens - 1, next = min(r + by, a.n_tokens - 1);
        const float total = a.total ? a.total[now] : __builtin_inff();
        const bool apart = __builtin_isfinite(total);
        if (bits) {
            for (int i = team.h; i < (a.n_bits + 31) / 32; i += team.lanes)
                row.bits[i] = 0;
            if (team.h == 0)
                *row.twice = 0;
            team.sync();
        }
        collect<T>(a, row, team, now, bits);
        team.sync();
        float m = -__builtin_inff();
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (!has(c))
                continue;
            if (bits && apart) {
                const int first = (c * team.lanes + anew(team.h)) * N;
                const unsigned out = first < a.n_classes ? row.bits[first >> 5] >> (first & 31) & ((1u << N) - 1) : 0;
                if (out) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        x[c][i] = out >> i & 1 ? nothing : x[c][i];
                }
            }
            const Chunk v = anew(x[c]);
#pragma unroll
            for (int i = 0; i < N; ++i)
                m = fmaxf(m, (float)v[i]);
        }
        const auto larger = [](float p, float q) { return fmaxf(p, q); };
        float M = clean(team.join(m, larger));
        const auto zero_if_none = [](float most) { return most > -__builtin_inff() ? most : 0.0f; };
        // Exponents of 2 as one product and sum, from `base`, where it is near enough to the largest logit's and nothing is NaN or infinity: of
        // either, the sum would tell.  (Temperatures far above 1 bring the largest float near enough too.)
        const float base = zero_if_none(M) * a.rate;
        float s = 0.0f;
        bool plain = fabsf(base) < kPlain;
        if (plain) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!has(c))
                    continue;
                const Chunk v = anew(x[c]);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    s += __builtin_amdgcn_exp2f(fmaf((float)v[i], a.rate, -base));
            }
        }
        double S = team.join((double)s, [](double p, double q) { return p + q; });
        plain = plain && S < __builtin_inf();
        if (WAVES ? !plain : __any(!plain)) {
            plain = false;
            m = -__builtin_inff();      // once more: NaN that signals hid what was larger before it
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!has(c))
                    continue;
                const Chunk v = anew(x[c]);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    m = fmaxf(m, __builtin_canonicalizef((float)v[i]));
            }
            M = clean(team.join(m, larger));
            s = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!has(c))
                    continue;
                const Chunk v = anew(x[c]);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    s += share_of((float)v[i], zero_if_none(M), a.twice_rate);
            }
            S = team.join((double)s, [](double p, double q) { return p + q; });
        }
        const float from = zero_if_none(M);
        // What the sum is one of exp((x - .) / T) from.
        const double origin = !(M > -__builtin_inff()) ? -__builtin_inf() : plain ? base * a.inverse_rate : M;
        if (team.leads()) {
            // The registers do not hold all chunks and what the verdict takes: some wait in LDS.
#pragma unroll
            for (int c = C - kStash; c < C; ++c)
                stash[(c - C + kStash) * 64 + threadIdx.x] = x[c];
            asm volatile("" ::: "memory");
            judge<GRADIENT>(a, row, now, there, apart, bits ? *row.twice != 0 : GRADIENT || apart, total, from, origin, S, team.ll, WAVES ? (int)threadIdx.x : team.h);
            asm volatile("" ::: "memory");
#pragma unroll
            for (int c = C - kStash; c < C; ++c)
                x[c] = stash[(c - C + kStash) * 64 + threadIdx.x];
        }
        if constexpr (!GRADIENT) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                load(c, next);
        } else {
            team.sync();
            const Verdict v = *row.verdict;
            T *const d_logits = (T *)a.d_logits + now * a.d_logit_stride;
            plain = plain && fabsf(v.factor) < 1e38f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!has(c))
                    continue;
                const int first = (c * team.lanes + anew(team.h)) * N;
                const Chunk logit = anew(x[c]);
                float d[N];
                if (plain) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        d[i] = __builtin_amdgcn_exp2f(fmaf((float)logit[i], a.rate, -base)) * v.factor;
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float e = share_of((float)logit[i], from, a.twice_rate);
                        d[i] = e > 0.0f ? e * v.factor : 0.0f;
                    }
                }
                store_chunk<N>(d_logits + first, there ? a.n_classes - first : 0, d);
                load(c, next);
            }
            team.sync();            // the entries' classes are written again
            if (there)
                store_entries<T>(a, row, team, now);
        }
        team.sync();                // the entries have been read
    }
}

// Rows of any length: read for their sums, AHEAD chunks of a thread on their way at once, and once more for the gradient.  Losses of many rows: 4096
// of 131 072 bf16 191 us, 5.6 TB/s, 8192 of 32 001 145 us, 3.6 TB/s, as nothing of the next row is on its way during a verdict.  One row stays in one
// workgroup: of 131 072 bf16 12.9 us, what a compute unit takes to issue its exponentials.
template <int TYPE, bool GRADIENT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, WAVES == 16 ? 4 : 1)
distill_long_kernel(DistillArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int N = kChunk<T>, threads = WAVES * 64, AHEAD = 4;
    typedef typename ChunkOf<T, N>::type Chunk;
    __shared__ double joined[16];
    extern __shared__ unsigned lds[];
    const Team<WAVES> team(joined, 6);
    const bool bits = a.n_bits > 0;
    unsigned *const rest_of_lds = lds + (a.n_bits + 31) / 32;
    const RowLds row = {lds, (Entry *)rest_of_lds, (Verdict *)(rest_of_lds + a.k * 4), (int *)(rest_of_lds + a.k * 4 + 2)};
    for (int64_t r = blockIdx.x; r < a.n_tokens; r += gridDim.x) {
        const T *const logits = (const T *)a.logits + r * a.logit_stride;
        const float total = a.total ? a.total[r] : __builtin_inff();
        const bool apart = __builtin_isfinite(total);
        if (bits) {
            for (int i = team.h; i < (a.n_bits + 31) / 32; i += team.lanes)
                row.bits[i] = 0;
            if (team.h == 0)
                *row.twice = 0;
            team.sync();
        }
        collect<T>(a, row, team, r, bits);
        team.sync();
        // Batches of whole chunks, exponents of 2 as one product and sum, from `base`.
        const int batches = a.n_classes / (AHEAD * threads * N);
        float m = -__builtin_inff(), base = 0.0f, s = 0.0f;
        Chunk x[AHEAD];
        const auto load = [&](int batch) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                x[u] = *(const Chunk *)(logits + ((batch * AHEAD + u) * threads + team.h) * N);
        };
        const auto one = [&](int c) {            // a chunk, whatever it holds
            float v[N], most = -__builtin_inff();
            load_chunk(logits + c, a.n_classes - c, v, -__builtin_inff());
            const unsigned out = bits && apart ? row.bits[c >> 5] >> (c & 31) : 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = out >> i & 1 ? -__builtin_inff() : clean(v[i]);
                most = fmaxf(most, v[i]);
            }
            if (most > m) {
                s *= share_of(m, most, a.twice_rate);
                m = most;
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                s += m > -__builtin_inff() ? share_of(v[i], m, a.twice_rate) : 0.0f;
        };
        if (batches > 0)
            load(0);
        bool plain = true;
        for (int batch = 0; batch < batches; ++batch) {
            Chunk now[AHEAD];
            float most = -__builtin_inff();
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                now[u] = x[u];
            if (batch + 1 < batches)
                load(batch + 1);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (bits && apart) {
                    const int first = ((batch * AHEAD + u) * threads + team.h) * N;
                    const unsigned out = row.bits[first >> 5] >> (first & 31) & ((1u << N) - 1);
                    if (out) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            now[u][i] = out >> i & 1 ? (T)-__builtin_inff() : now[u][i];
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
                    most = fmaxf(most, (float)now[u][i]);
            }
            plain = plain && most == most;          // NaN that signals has hidden what was larger before it
            if (most > m) {
                const float before = base;
                base = most * a.rate;
                s = m > -__builtin_inff() ? s * __builtin_amdgcn_exp2f(before - base) : 0.0f;
                m = most;
                plain = plain && fabsf(base) < kPlain;
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    s += __builtin_amdgcn_exp2f(fmaf((float)now[u][i], a.rate, -base));
        }
        if (m > -__builtin_inff())               // from m itself
            s *= __builtin_amdgcn_exp2f(fmaf(-m, a.rate, base));
        if (!(plain && s == s)) {                // infinities and NaN, or logits far above the temperature
            m = -__builtin_inff();
            s = 0.0f;
            for (int c = team.h * N; c < batches * AHEAD * threads * N; c += threads * N)
                one(c);
        }
        for (int c = batches * AHEAD * threads * N + team.h * N; c < a.n_classes; c += threads * N)
            one(c);
        const float M = team.join(m, [](float p, float q) { return fmaxf(p, q); }), from = M > -__builtin_inff() ? M : 0.0f;
        const double S = team.join((double)s * share_of(m, from, a.twice_rate), [](double p, double q) { return p + q; });
        if (team.leads())
            judge<GRADIENT>(a, row, r, true, apart, bits ? *row.twice != 0 : GRADIENT || apart, total, from, M, S, 6, (int)threadIdx.x);
        if constexpr (GRADIENT) {
            team.sync();
            const Verdict verdict = *row.verdict;
            T *const d_logits = (T *)a.d_logits + r * a.d_logit_stride;
            for (int c = team.h * N; c < a.n_classes; c += threads * N) {
                float v[N];
                load_chunk(logits + c, a.n_classes - c, v, -__builtin_inff());
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float e = share_of(v[i], verdict.from, a.twice_rate);
                    v[i] = e > 0.0f ? e * verdict.factor : 0.0f;
                }
                store_chunk<N>(d_logits + c, a.n_classes - c, v);
            }
            team.sync();            // the entries' classes are written again
            store_entries<T>(a, row, team, r);
        }
        team.sync();                // the entries have been read
    }
}

constexpr int kUnits = 256;      // compute units of the card
template <class K>
static int launch_distill(K kernel, DistillArgs a, int threads, int teams, hipStream_t stream)
{
    const size_t lds = row_lds_words(a.n_bits, a.k) * 4 * teams;
    if (lds > 32768) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return fail_hip(e, "distillation kernel's LDS");
    }
    // As many workgroups as run at once, if rows are so many: a thread that goes on to another row has asked for it before.
    const int64_t most = (a.n_tokens + teams - 1) / teams, resident = threads >= 512 ? kUnits : 8 * kUnits;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(most < resident ? most : resident)), dim3(threads), lds, stream, a);
    return FS_OK;
}
template <int TYPE, bool GRADIENT>
static int launch_rows(DistillArgs a, hipStream_t stream)
{
    const int64_t chunks = (a.n_classes * (int64_t)type_bytes(TYPE) + 15) / 16;
    if (chunks <= 16 * 64 && a.k <= 256) {
        // Up to 16 KB: lanes of a wavefront.  The verdict costs a wavefront about the same for one row as for several, so that many rows
        // have few lanes each, if one line's at least; few rows have many.
        const int each = a.n_tokens >= 8192 || chunks > 256 ? 16 : chunks > 64 ? 4 : 1;
        const int64_t least = (chunks + each - 1) / each, line = chunks < 8 ? chunks : 8;
        a.ll = 0;
        while (a.ll < 6 && ((1 << a.ll) < least || (1 << a.ll) < line || (4 << a.ll) < a.k))
            ++a.ll;
        const int teams = 256 >> a.ll;
        return each == 1   ? launch_distill(distill_row_kernel<TYPE, GRADIENT, 0, 1>, a, 256, teams, stream)
               : each == 4 ? launch_distill(distill_row_kernel<TYPE, GRADIENT, 0, 4>, a, 256, teams, stream)
                           : launch_distill(distill_row_kernel<TYPE, GRADIENT, 0, 16>, a, 256, teams, stream);
    }
    if constexpr (GRADIENT) {
        if (chunks <= 16 * 256)
            return launch_distill(distill_row_kernel<TYPE, true, 4, 16>, a, 256, 1, stream);
        if (chunks <= 8 * 1024)
            return launch_distill(distill_row_kernel<TYPE, true, 16, 8>, a, 1024, 1, stream);
        if (chunks <= 16 * 1024)
            return launch_distill(distill_row_kernel<TYPE, true, 16, 16>, a, 1024, 1, stream);
        return launch_distill(distill_long_kernel<TYPE, true, 16>, a, 1024, 1, stream);
    } else {
        return a.n_tokens < kUnits || a.n_bits > 65536 * 8 ? launch_distill(distill_long_kernel<TYPE, false, 16>, a, 1024, 1, stream)
                                                           : launch_distill(distill_long_kernel<TYPE, false, 4>, a, 256, 1, stream);
    }
}

static int check_distill(const char *who, const fs_distill_params *p, int64_t n_tokens)
{
    if (!p)
        return fail(FS_EINVAL, "%s: params is NULL", who);
    if (p->n_classes < 1 || p->n_classes > FS_MAX_CLASSES)
        return fail(p->n_classes < 1 ? FS_EINVAL : FS_EUNSUPPORTED, "%s: n_classes %d outside [1, %d]", who, p->n_classes, FS_MAX_CLASSES);
    if (p->k < 1 || p->k > FS_MAX_LISTED)
        return fail(p->k < 1 ? FS_EINVAL : FS_EUNSUPPORTED, "%s: k %d outside [1, %d]", who, p->k, FS_MAX_LISTED);
    if (!(p->temperature >= 1.17549435e-38f) || p->temperature > 3.402823466e38f)      // below, log2(e) / T would be no fp32
        return fail(FS_EINVAL, "%s: temperature %g is not of at least 2^-126 and finite", who, (double)p->temperature);
    if (!(fabsf(p->scale) <= 3.402823466e38f))
        return fail(FS_EINVAL, "%s: scale %g is not finite", who, (double)p->scale);
    if (n_tokens < 0 || n_tokens >= ((int64_t)1 << 31))
        return fail(FS_EINVAL, "%s: %lld tokens: 0 to 2^31 - 1 are taken", who, (long long)n_tokens);
    return FS_OK;
}

static int distill(const char *who, bool gradient, const fs_distill_params *p, DistillArgs a, int32_t type, const void *work, size_t work_bytes, hipStream_t stream)
{
    FS_TRY(check_distill(who, p, a.n_tokens));
    FS_TRY(check_matrix(who, "logits", a.logits, a.n_tokens, p->n_classes, type, a.logit_stride));
    if (a.id_type != FS_ID_I32 && a.id_type != FS_ID_I64)
        return fail(FS_EINVAL, "%s: type %d of ids is neither FS_ID_I32 nor FS_ID_I64", who, a.id_type);
    FS_TRY(check_array(who, "ids", a.ids, a.n_tokens, a.id_type == FS_ID_I64 ? 8 : 4));
    if (!type_ok(a.teacher_type))
        return fail(FS_EINVAL, "%s: unknown element type %d of teacher", who, a.teacher_type);
    FS_TRY(check_array(who, "teacher", a.teacher, a.n_tokens, type_bytes(a.teacher_type)));
    FS_TRY(check_array(who, "total", a.total, 0, 4));
    FS_TRY(check_array(who, "loss", a.loss, gradient ? 0 : a.n_tokens, 4));
    if (gradient) {
        FS_TRY(check_array(who, "d_loss", a.d_loss, a.n_tokens, 4));
        FS_TRY(check_matrix(who, "d_logits", a.d_logits, a.n_tokens, p->n_classes, type, a.d_logit_stride));
    }
    const size_t need = fs_distill_workspace_bytes(p, a.n_tokens, type);
    FS_TRY(check_array(who, "work", work, (int64_t)need, 256));
    if (work_bytes < need)
        return fail(FS_EINVAL, "%s: %zu bytes of working memory, %zu are needed", who, work_bytes, need);
    if (a.n_tokens == 0)
        return FS_OK;
    a.n_classes = p->n_classes;
    a.k = p->k;
    a.rate = (float)(1.44269504088896340736 / p->temperature);
    a.twice_rate = 2.0f * a.rate;
    a.inverse_rate = 1.0 / a.rate;
    a.inverse_t = 1.0 / p->temperature;
    a.scale = p->scale;
    // Bits of the classes: for a rest, and to see whether two entries name one class (comparing 64 entries with each other instead made
    // a gradient of 4096 rows of 131 072 classes 630 us instead of 560).
    a.n_bits = a.total || gradient ? a.n_classes : 0;
    prof_start(kKernTrainOther, stream);
    int rc = FS_OK;
    with_type(type, [&](auto t) { rc = gradient ? launch_rows<decltype(t)::value, true>(a, stream) : launch_rows<decltype(t)::value, false>(a, stream); });
    prof_stop(stream);
    FS_TRY(rc);
    return launched("distillation kernel launch");
}

}  // namespace fs

using namespace fs;

extern "C" size_t fs_distill_workspace_bytes(const fs_distill_params *params, int64_t n_tokens, int32_t logit_type)
{
    static const char who[] = "fs_distill_workspace_bytes";
    if (check_distill(who, params, n_tokens) != FS_OK)
        return 0;
    if (!type_ok(logit_type))
        fail(FS_EINVAL, "%s: unknown element type %d", who, logit_type);
    return 0;
}

extern "C" int fs_distill(const fs_distill_params *params, int64_t n_tokens, const void *logits, int32_t logit_type, int64_t logit_stride,
                          const void *ids, int32_t id_type, const void *teacher, int32_t teacher_type, const float *total, float *loss,
                          void *work, size_t work_bytes, void *stream)
{
    const DistillArgs a = {logits, ids, teacher, total, nullptr, loss, nullptr, n_tokens, logit_stride, 0, 0, 0, id_type, teacher_type, 0, 0, 0, 0, 0, 0, 0};
    return distill("fs_distill", false, params, a, logit_type, work, work_bytes, (hipStream_t)stream);
}

extern "C" int fs_distill_backward(const fs_distill_params *params, int64_t n_tokens, const void *logits, int32_t logit_type, int64_t logit_stride,
                                   const void *ids, int32_t id_type, const void *teacher, int32_t teacher_type, const float *total,
                                   const float *d_loss, float *loss, void *d_logits, int64_t d_logit_stride, void *work, size_t work_bytes,
                                   void *stream)
{
    const DistillArgs a = {logits, ids, teacher, total, d_loss, loss, d_logits, n_tokens, logit_stride, d_logit_stride, 0, 0, id_type, teacher_type, 0, 0, 0, 0, 0, 0, 0};
    return distill("fs_distill_backward", true, params, a, logit_type, work, work_bytes, (hipStream_t)stream);
}
