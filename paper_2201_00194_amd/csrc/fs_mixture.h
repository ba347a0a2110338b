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
inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FS_OK : fail_hip(e, what);
}
#define FS_TRY(call)               \
    do {                           \
        const int fs_rc_ = (call); \
        if (fs_rc_ != FS_OK)       \
            return fs_rc_;         \
    } while (0)

}  // namespace fs
#endif
