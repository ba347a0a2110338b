// Shared by the kernels of mixtures of family models (not installed).
#ifndef FS_MIXTURE_H
#define FS_MIXTURE_H

#include "fs_internal.h"
#include "familyseer_mixture.h"

namespace fs {

// Elements of a matrix: read as fp32, written with one rounding to nearest.
template <int TYPE> struct Element;
template <> struct Element<FS_F32> { typedef float type; };
template <> struct Element<FS_BF16> { typedef __bf16 type; };
template <> struct Element<FS_F16> { typedef _Float16 type; };

inline bool type_ok(int32_t type) { return type == FS_F32 || type == FS_BF16 || type == FS_F16; }
inline size_t type_bytes(int32_t type) { return type == FS_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// f is called with a value whose type says the element type.
template <int TYPE> struct TypeTag { static constexpr int value = TYPE; };
template <class F>
void with_type(int32_t type, F f)
{
    if (type == FS_F32)
        f(TypeTag<FS_F32>());
    else if (type == FS_BF16)
        f(TypeTag<FS_BF16>());
    else
        f(TypeTag<FS_F16>());
}

// A matrix argument: `rows` rows of `width` elements.
inline int check_matrix(const char *who, const char *what, const void *p, int64_t rows, int64_t width, int32_t type, int64_t stride)
{
    if (!type_ok(type))
        return fail(FS_EINVAL, "%s: unknown element type %d of %s", who, type, what);
    if (stride < width)
        return fail(FS_EINVAL, "%s: row stride %lld of %s is less than its width %lld", who, (long long)stride, what, (long long)width);
    if (stride > ((int64_t)1 << 40))
        return fail(FS_EINVAL, "%s: row stride %lld of %s is over 2^40", who, (long long)stride, what);
    if (rows > 0 && !p)
        return fail(FS_EINVAL, "%s: %s is NULL", who, what);
    if (!aligned_to(p, type_bytes(type)))
        return fail(FS_EINVAL, "%s: %s is not aligned to its elements", who, what);
    return FS_OK;
}
// A matrix of 8-bit integers.
inline int check_bytes(const char *who, const char *what, const void *p, int64_t rows, int64_t width, int64_t stride)
{
    if (stride < width || stride > ((int64_t)1 << 40))
        return fail(FS_EINVAL, "%s: row stride %lld of %s, whose width is %lld: 2^40 at most", who, (long long)stride, what, (long long)width);
    if (rows > 0 && !p)
        return fail(FS_EINVAL, "%s: %s is NULL", who, what);
    return FS_OK;
}
inline int check_width(const char *who, int32_t width)
{
    if (width < 1 || width > FS_MAX_WIDTH)
        return fail(width < 1 ? FS_EINVAL : FS_EUNSUPPORTED, "%s: width %d outside [1, %d]", who, width, FS_MAX_WIDTH);
    return FS_OK;
}
inline int check_array(const char *who, const char *what, const void *p, int64_t n, size_t bytes)
{
    if (n > 0 && !p)
        return fail(FS_EINVAL, "%s: %s is NULL", who, what);
    if (!aligned_to(p, bytes))
        return fail(FS_EINVAL, "%s: %s is not aligned to its elements", who, what);
    return FS_OK;
}
inline int check_tokens(const char *who, int64_t n_tokens, int32_t k)
{
    if (k < 1 || k > FS_MAX_CHOICES)
        return fail(FS_EINVAL, "%s: k %d outside [1, %d]", who, k, FS_MAX_CHOICES);
    if (n_tokens < 0 || n_tokens * k >= ((int64_t)1 << 31) || n_tokens >= ((int64_t)1 << 31))
        return fail(FS_EINVAL, "%s: %lld tokens with %d choices: 0 to 2^31 - 1 choices are taken", who, (long long)n_tokens, k);
    return FS_OK;
}
inline int check_experts(const char *who, int32_t n_experts)
{
    if (n_experts < 1 || n_experts > FS_MAX_EXPERTS)
        return fail(n_experts < 1 ? FS_EINVAL : FS_EUNSUPPORTED, "%s: n_experts %d outside [1, %d]", who, n_experts, FS_MAX_EXPERTS);
    return FS_OK;
}
inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FS_OK : fail_hip(e, what);
}

// ---- lanes --------------------------------------------------------------------------------------
// What this wavefront has done in LDS is done.
__device__ __forceinline__ void lds_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 1 << ll neighbouring lanes work on one row.  Step s < ll of a reduction over them meets a lane whose 1 << s neighbours
// this lane's have not met yet: within sixteen lanes by data-parallel moves (pairs, quads swapped, then mirrored halves and
// rows, as all lanes of a quad and of a half hold the same by then).
template <int STEP>
__device__ __forceinline__ int met_int(int v)
{
    if constexpr (STEP == 0)
        return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);     // quad_perm 1 0 3 2
    else if constexpr (STEP == 1)
        return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);     // quad_perm 2 3 0 1
    else if constexpr (STEP == 2)
        return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true);    // row_half_mirror
    else if constexpr (STEP == 3)
        return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, true);    // row_mirror
    else
        return __shfl_xor(v, STEP == 4 ? 16 : 32);
}
template <int STEP> __device__ __forceinline__ float met(float v) { return __int_as_float(met_int<STEP>(__float_as_int(v))); }
template <int STEP> __device__ __forceinline__ int met(int v) { return met_int<STEP>(v); }
template <int STEP> __device__ __forceinline__ double met(double v)
{
    return __hiloint2double(met_int<STEP>(__double2hiint(v)), met_int<STEP>(__double2loint(v)));
}
// f(this lane's, the met lane's) over the 1 << ll lanes of a row, ll the same in the whole wavefront; f is symmetric, so all lanes
// of a row get the same.
template <class T, class F>
__device__ __forceinline__ T row_reduce(T v, int ll, F f)
{
    if (ll > 0) v = f(v, met<0>(v));
    if (ll > 1) v = f(v, met<1>(v));
    if (ll > 2) v = f(v, met<2>(v));
    if (ll > 3) v = f(v, met<3>(v));
    if (ll > 4) v = f(v, met<4>(v));
    if (ll > 5) v = f(v, met<5>(v));
    return v;
}
template <class T> __device__ __forceinline__ T row_sum(T v, int ll) { return row_reduce(v, ll, [](T a, T b) { return a + b; }); }
__device__ __forceinline__ float row_max(float v, int ll) { return row_reduce(v, ll, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ int row_or(int v, int ll) { return row_reduce(v, ll, [](int a, int b) { return a | b; }); }

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896340736f); }

// ---- rows of a matrix ---------------------------------------------------------------------------
// A row's elements lie in 1 << ll neighbouring lanes, 16 bytes of them a lane; wider rows take several column blocks of a
// wavefront's 1 KB.  Rows need not be aligned to more than their elements: unaligned loads are loads all the same.
template <class T> constexpr int kChunk = 16 / (int)sizeof(T);
inline int row_lanes_log(int width, int chunk)
{
    int ll = 0;
    while (ll < 6 && (chunk << ll) < width)
        ++ll;
    return ll;
}
inline int column_blocks(int width, int chunk) { return (width + chunk * 64 - 1) / (chunk * 64); }

template <class T, int N>
struct ChunkOf {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
// N elements, n of them there: the others are `rest`, and nothing behind the n-th is read.
template <int N, class T>
__device__ __forceinline__ void load_chunk(const T *p, int n, float (&v)[N], float rest = 0.0f)
{
    if (n >= N) {
        const typename ChunkOf<T, N>::type c = *(const typename ChunkOf<T, N>::type *)p;
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = (float)c[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = rest;
        if (n > 0) {
            T c[N];
#pragma unroll
            for (int i = 0; i < N; ++i)
                c[i] = p[i < n ? i : n - 1];
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = i < n ? (float)c[i] : rest;
        }
    }
}
// PAST: the stores ask the caches not to keep what they bring; see past_caches.
template <int N, bool PAST = false, class T>
__device__ __forceinline__ void store_chunk(T *p, int n, const float (&v)[N])
{
    if (n >= N) {
        typename ChunkOf<T, N>::type c;
#pragma unroll
        for (int i = 0; i < N; ++i)
            c[i] = (T)v[i];
        if constexpr (PAST)
            __builtin_nontemporal_store(c, (typename ChunkOf<T, N>::type *)p);
        else
            *(typename ChunkOf<T, N>::type *)p = c;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n)
                p[i] = (T)v[i];
    }
}

// Elements c .. c + N - 1 of a row, n of them there.  The last chunk of a row moves back until it is whole, where the row has so many
// elements: its first `skip` are its neighbour's too, and both write the same.  (Element by element it costs twice as many
// loads as all other chunks together.)  `whole` false: it stays where it is, for sums onto what is there.
struct Span {
    int c, n, skip;
};
template <int N>
__device__ __forceinline__ Span span_of(int c, int width, bool whole = true)
{
    const int n = width - c, skip = whole && n > 0 && n < N && width >= N ? N - n : 0;
    return Span{c - skip, n + skip, skip};
}

// The same elements as they are: a quarter or half of the registers of load_chunk's, for what is on its way for long.
template <class T>
struct RawChunk {
    static constexpr int N = kChunk<T>;
    typedef typename ChunkOf<T, N>::type Chunk;
    Chunk c;
    template <bool PAST = false>
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= N) {
            if constexpr (PAST)
                c = __builtin_nontemporal_load((const Chunk *)p);
            else
                c = *(const Chunk *)p;
        } else {
            clear();
            if (n > 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const T v = p[i < n ? i : n - 1];
                    c[i] = i < n ? v : (T)0.0f;
                }
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            c[i] = (T)0.0f;
    }
    __device__ __forceinline__ float operator[](int i) const { return (float)c[i]; }
    template <bool PAST = false>
    __device__ __forceinline__ void store(T *p, int n) const
    {
        if (n >= N) {
            if constexpr (PAST)
                __builtin_nontemporal_store(c, (Chunk *)p);
            else
                *(Chunk *)p = c;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < n)
                    p[i] = c[i];
        }
    }
};

// Looked-up and gathered rows of this many bytes leave past the caches: whoever reads them next would find few of them there, and
// the table's rows stay.  268 MB of looked-up rows 85 us and 58 so, with a pass that reads them next 173 and 168; of gathered
// ones 63 and 51, 153 and 151; 134 MB 36 and 35, 78 and 80.  Gradients of results stay ordinary stores (268 MB 118 and 109, with
// their reader 207 and 217).
constexpr int64_t kPastCaches = 200 << 20;
inline bool past_caches(int64_t rows, int32_t width, int32_t type) { return rows * width * (int64_t)type_bytes(type) >= kPastCaches; }

// The hardware's reciprocal, one step off at most.
__device__ __forceinline__ float inverse(float v) { return __builtin_amdgcn_rcpf(v); }

// A launch has at most 2^32 - 1 threads: f(first block, blocks) for pieces of 2^22 workgroups.
template <class F>
void in_pieces(int64_t blocks, F f)
{
    constexpr int64_t kMost = (int64_t)1 << 22;
    for (int64_t at = 0; at < blocks; at += kMost)
        f(at, (unsigned)(blocks - at < kMost ? blocks - at : kMost));
}

#define FS_TRY(call)               \
    do {                           \
        const int fs_rc_ = (call); \
        if (fs_rc_ != FS_OK)       \
            return fs_rc_;         \
    } while (0)

}  // namespace fs
#endif
