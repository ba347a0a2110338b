// The exchange between tokens and experts: the plan of slots, rows into the slots, results back.
#include "fs_slots.h"

namespace fs {

struct ChoiceNumber {
    const int32_t *expert;
    int32_t n_experts;
    __device__ __forceinline__ int operator()(int64_t i) const
    {
        const int e = expert[i];
        return e >= 0 && e < n_experts ? e : n_experts;
    }
};
struct ChoicePut {
    int32_t *first, *order, *place;
    int32_t n_experts;
    __device__ __forceinline__ void start(int e, int slot) const { first[e] = slot; }
    __device__ __forceinline__ void operator()(int64_t i, int e, int slot) const
    {
        order[slot] = e < n_experts ? (int32_t)i : -1;
        place[i] = e < n_experts ? slot : -1;
    }
};

// No choices: no slots.
__global__ void __launch_bounds__(256)
expert_none_kernel(int32_t n_experts, int32_t *first)
{
    for (int e = threadIdx.x; e <= n_experts; e += 256)
        first[e] = 0;
}

struct ExchangeArgs {
    int64_t n_tokens, in_stride, y_stride, out_stride;
    int32_t k, n_experts, width;
    const void *in;                  // x, or the gradient of the tokens' results
    const void *y;
    const int32_t *first, *place;
    const float *weight;
    void *out;
    float *d_weight;
};

// The slots behind the last expert's: n_tokens wavefronts share them.
template <class T>
__device__ __forceinline__ void clear_slots_behind(const ExchangeArgs &a, int64_t token, int lane)
{
    const int64_t slots = a.n_tokens * a.k;
    for (int64_t s = max(a.first[a.n_experts], 0) + token; s < slots; s += a.n_tokens)
        for (int c = lane; c < a.width; c += 64)
            ((T *)a.out)[s * a.out_stride + c] = (T)0.0f;
}

template <int TYPE>
__global__ void __launch_bounds__(64)
expert_gather_kernel(ExchangeArgs a)
{
    typedef typename Element<TYPE>::type T;
    const int64_t t = blockIdx.x, slots = a.n_tokens * a.k;
    const T *in = (const T *)a.in + t * a.in_stride;
    for (int j = 0; j < a.k; ++j) {
        const int p = a.place[t * a.k + j];
        if (p >= 0 && p < slots)
            for (int c = threadIdx.x; c < a.width; c += 64)
                ((T *)a.out)[(int64_t)p * a.out_stride + c] = in[c];
    }
    clear_slots_behind<T>(a, t, threadIdx.x);
}

template <int TYPE>
__global__ void __launch_bounds__(64)
expert_combine_kernel(ExchangeArgs a)
{
    typedef typename Element<TYPE>::type T;
    const int64_t t = blockIdx.x, slots = a.n_tokens * a.k;
    for (int c = threadIdx.x; c < a.width; c += 64) {
        float sum = 0.0f;
        for (int j = 0; j < a.k; ++j) {
            const int p = a.place[t * a.k + j];
            if (p >= 0 && p < slots)
                sum = fmaf(a.weight ? a.weight[t * a.k + j] : 1.0f, (float)((const T *)a.y)[(int64_t)p * a.y_stride + c], sum);
        }
        ((T *)a.out)[t * a.out_stride + c] = (T)sum;
    }
}

template <int TYPE>
__global__ void __launch_bounds__(64)
expert_combine_backward_kernel(ExchangeArgs a)
{
    typedef typename Element<TYPE>::type T;
    const int64_t t = blockIdx.x, slots = a.n_tokens * a.k;
    const T *in = (const T *)a.in + t * a.in_stride;
    for (int j = 0; j < a.k; ++j) {
        const int p = a.place[t * a.k + j];
        float dot = 0.0f;
        if (p >= 0 && p < slots) {
            const float w = a.weight[t * a.k + j];
            for (int c = threadIdx.x; c < a.width; c += 64) {
                const float g = (float)in[c];
                dot = fmaf(g, (float)((const T *)a.y)[(int64_t)p * a.y_stride + c], dot);
                ((T *)a.out)[(int64_t)p * a.out_stride + c] = (T)(w * g);
            }
            for (int o = 32; o; o >>= 1)
                dot += __shfl_xor(dot, o);
        }
        if (threadIdx.x == 0)
            a.d_weight[t * a.k + j] = dot;
    }
    clear_slots_behind<T>(a, t, threadIdx.x);
}

static int check_experts(const char *who, int32_t n_experts)
{
    if (n_experts < 1 || n_experts > FS_MAX_EXPERTS)
        return fail(n_experts < 1 ? FS_EINVAL : FS_EUNSUPPORTED, "%s: n_experts %d outside [1, %d]", who, n_experts, FS_MAX_EXPERTS);
    return FS_OK;
}

}  // namespace fs

using namespace fs;

extern "C" size_t fs_expert_plan_workspace_bytes(int64_t n_tokens, int32_t k, int32_t n_experts)
{
    static const char who[] = "fs_expert_plan_workspace_bytes";
    if (check_tokens(who, n_tokens, k) != FS_OK || check_experts(who, n_experts) != FS_OK)
        return 0;
    return slot_count_bytes(slot_shape(n_tokens * k, n_experts + 1));
}

extern "C" int fs_expert_plan(int64_t n_tokens, int32_t k, int32_t n_experts, const int32_t *expert, int32_t *first, int32_t *order,
                              int32_t *place, void *work, size_t work_bytes, void *stream_)
{
    static const char who[] = "fs_expert_plan";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_tokens(who, n_tokens, k));
    FS_TRY(check_experts(who, n_experts));
    FS_TRY(check_array(who, "expert", expert, n_tokens, 4));
    FS_TRY(check_array(who, "first", first, 1, 4));
    FS_TRY(check_array(who, "order", order, n_tokens, 4));
    FS_TRY(check_array(who, "place", place, n_tokens, 4));
    const SlotShape s = slot_shape(n_tokens * k, n_experts + 1);
    const size_t need = slot_count_bytes(s);
    FS_TRY(check_array(who, "work", work, (int64_t)need, 256));
    if (work_bytes < need)
        return fail(FS_EINVAL, "%s: %zu bytes of working memory, %zu are needed", who, work_bytes, need);
    int32_t *count = (int32_t *)work;
    prof_start(kKernPack, stream);
    if (s.n > 0)
        launch_slots(ChoiceNumber{expert, n_experts}, ChoicePut{first, order, place, n_experts}, s, count, stream);
    else
        hipLaunchKernelGGL(expert_none_kernel, dim3(1), dim3(256), 0, stream, n_experts, first);
    prof_stop(stream);
    return launched("expert plan kernels launch");
}

extern "C" int fs_expert_gather(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t width, const void *x, int32_t type, int64_t x_stride,
                                const int32_t *first, const int32_t *place, void *xs, int64_t xs_stride, void *stream_)
{
    static const char who[] = "fs_expert_gather";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_tokens(who, n_tokens, k));
    FS_TRY(check_experts(who, n_experts));
    FS_TRY(check_width(who, width));
    FS_TRY(check_matrix(who, "x", x, n_tokens, width, type, x_stride));
    FS_TRY(check_matrix(who, "xs", xs, n_tokens, width, type, xs_stride));
    FS_TRY(check_array(who, "first", first, n_tokens, 4));
    FS_TRY(check_array(who, "place", place, n_tokens, 4));
    if (n_tokens == 0)
        return FS_OK;
    ExchangeArgs a = {n_tokens, x_stride, 0, xs_stride, k, n_experts, width, x, nullptr, first, place, nullptr, xs, nullptr};
    prof_start(kKernPack, stream);
    with_type(type, [&](auto t) {
        hipLaunchKernelGGL(expert_gather_kernel<decltype(t)::value>, dim3((unsigned)n_tokens), dim3(64), 0, stream, a);
    });
    prof_stop(stream);
    return launched("expert gather kernel launch");
}

extern "C" int fs_expert_combine(int64_t n_tokens, int32_t k, int32_t width, const void *y, int32_t type, int64_t y_stride,
                                 const int32_t *place, const float *weight, void *out, int64_t out_stride, void *stream_)
{
    static const char who[] = "fs_expert_combine";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_tokens(who, n_tokens, k));
    FS_TRY(check_width(who, width));
    FS_TRY(check_matrix(who, "y", y, n_tokens, width, type, y_stride));
    FS_TRY(check_matrix(who, "out", out, n_tokens, width, type, out_stride));
    FS_TRY(check_array(who, "place", place, n_tokens, 4));
    FS_TRY(check_array(who, "weight", weight, 0, 4));
    if (n_tokens == 0)
        return FS_OK;
    ExchangeArgs a = {n_tokens, 0, y_stride, out_stride, k, 0, width, nullptr, y, nullptr, place, weight, out, nullptr};
    prof_start(kKernPack, stream);
    with_type(type, [&](auto t) {
        hipLaunchKernelGGL(expert_combine_kernel<decltype(t)::value>, dim3((unsigned)n_tokens), dim3(64), 0, stream, a);
    });
    prof_stop(stream);
    return launched("expert combine kernel launch");
}

extern "C" int fs_expert_combine_backward(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t width, const void *d_out, int32_t type,
                                          int64_t d_out_stride, const void *y, int64_t y_stride, const int32_t *first, const int32_t *place,
                                          const float *weight, void *d_y, int64_t d_y_stride, float *d_weight, void *stream_)
{
    static const char who[] = "fs_expert_combine_backward";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_tokens(who, n_tokens, k));
    FS_TRY(check_experts(who, n_experts));
    FS_TRY(check_width(who, width));
    FS_TRY(check_matrix(who, "d_out", d_out, n_tokens, width, type, d_out_stride));
    FS_TRY(check_matrix(who, "y", y, n_tokens, width, type, y_stride));
    FS_TRY(check_matrix(who, "d_y", d_y, n_tokens, width, type, d_y_stride));
    FS_TRY(check_array(who, "first", first, n_tokens, 4));
    FS_TRY(check_array(who, "place", place, n_tokens, 4));
    FS_TRY(check_array(who, "weight", weight, n_tokens, 4));
    FS_TRY(check_array(who, "d_weight", d_weight, n_tokens, 4));
    if (n_tokens == 0)
        return FS_OK;
    ExchangeArgs a = {n_tokens, d_out_stride, y_stride, d_y_stride, k, n_experts, width, d_out, y, first, place, weight, d_y, d_weight};
    prof_start(kKernTrainOther, stream);
    with_type(type, [&](auto t) {
        hipLaunchKernelGGL(expert_combine_backward_kernel<decltype(t)::value>, dim3((unsigned)n_tokens), dim3(64), 0, stream, a);
    });
    prof_stop(stream);
    return launched("expert combine gradient kernel launch");
}
