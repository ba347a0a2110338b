// Routing: logits to the k chosen experts of a token and their weights, and the logits' gradient.
#include "fs_mixture.h"

#include <math.h>

namespace fs {

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
};

// NaN masks an expert as -infinity does; +infinity counts as the largest float.
__device__ __forceinline__ float route_logit(float l)
{
    return l != l ? -__builtin_inff() : fminf(l, 3.402823466e38f);
}

__device__ __forceinline__ double wave_max(double v)
{
    for (int o = 32; o; o >>= 1)
        v = fmax(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ double wave_sum(double v)
{
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o);
    return v;
}
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
__device__ __forceinline__ double log_score(double x, double top, double log_sum, int score)
{
    return score == FS_SCORE_SOFTMAX ? x - top - log_sum : fmin(x, 0.0) - log1p(exp(-fabs(x)));
}

// One wavefront a token, everything in 64 bits.
template <int TYPE>
__global__ void __launch_bounds__(64)
route_kernel(RouteArgs a)
{
    typedef typename Element<TYPE>::type T;
    __shared__ double key[FS_MAX_EXPERTS], group[FS_MAX_EXPERTS];
    const int lane = threadIdx.x, n = a.p.n_experts, k = a.p.k;
    const double none = -__builtin_inf();
    const T *logits = (const T *)a.logits + (int64_t)blockIdx.x * a.stride;
    double top = none, sum = 0.0;
    for (int e = lane; e < n; e += 64)
        top = fmax(top, (double)route_logit((float)logits[e]));
    top = wave_max(top);
    if (top == none)
        top = 0.0;
    for (int e = lane; e < n; e += 64)
        sum += exp((double)route_logit((float)logits[e]) - top);
    const double log_sum = log(wave_sum(sum));
    const int per = n / a.p.n_groups;
    for (int e = lane; e < n; e += 64) {
        const double x = route_logit((float)logits[e]);
        double v = x;
        if (x > none && (a.bias || a.p.n_groups > 1)) {
            v = exp(log_score(x, top, log_sum, a.p.score));
            if (a.bias)
                v += (double)a.bias[e];
        }
        key[e] = v > none ? v : none;
    }
    __syncthreads();
    if (a.p.n_groups > 1) {
        for (int g = lane; g < a.p.n_groups; g += 64) {
            double first = none, second = none;
            for (int e = g * per; e < (g + 1) * per; ++e) {
                const double v = key[e];
                if (v > first)
                    second = first, first = v;
                else if (v > second)
                    second = v;
            }
            group[g] = a.p.group_best == 2 && second > none ? first + second : first;
        }
        __syncthreads();
        for (int r = 0; r < a.p.top_groups; ++r) {
            const int g = wave_argmax(group, a.p.n_groups, lane);
            __syncthreads();
            if (g >= 0 && lane == 0)
                group[g] = __builtin_nan("");                 // taken
            __syncthreads();
        }
        for (int e = lane; e < n; e += 64) {
            const double t = group[e / per];
            if (t == t)
                key[e] = none;
            else if (!a.bias && key[e] > none)
                key[e] = route_logit((float)logits[e]);
        }
        __syncthreads();
    }
    int mine = -1;
    for (int j = 0; j < k; ++j) {
        const int e = wave_argmax(key, n, lane);
        __syncthreads();
        if (e >= 0 && lane == 0)
            key[e] = none;
        if (lane == j)
            mine = e;
        __syncthreads();
    }
    double s = none, w;
    if (mine >= 0) {
        const double x = route_logit((float)logits[mine]);
        s = a.p.renormalise && a.p.score == FS_SCORE_SOFTMAX ? x : log_score(x, top, log_sum, a.p.score);
    }
    if (a.p.renormalise) {                 // the softmax over the chosen: a common term of their logarithms falls out
        const double high = wave_max(s);
        w = mine < 0 ? 0.0 : exp(s - high);
        const double all = wave_sum(w);
        w = all > 0.0 ? w / all : 0.0;
    } else {
        w = mine < 0 ? 0.0 : exp(s);
    }
    if (lane < k) {
        a.expert[(int64_t)blockIdx.x * k + lane] = mine;
        a.weight[(int64_t)blockIdx.x * k + lane] = (float)(w * (double)a.p.scale);
    }
}

template <int TYPE>
__global__ void __launch_bounds__(64)
route_backward_kernel(RouteArgs a)
{
    typedef typename Element<TYPE>::type T;
    __shared__ double grad[FS_MAX_EXPERTS];
    const int lane = threadIdx.x, n = a.p.n_experts, k = a.p.k;
    const double none = -__builtin_inf();
    const T *logits = (const T *)a.logits + (int64_t)blockIdx.x * a.stride;
    T *out = (T *)a.d_logits + (int64_t)blockIdx.x * a.d_stride;
    for (int e = lane; e < n; e += 64)
        grad[e] = 0.0;
    __syncthreads();
    int mine = lane < k ? a.chosen[(int64_t)blockIdx.x * k + lane] : -1;
    if (mine < 0 || mine >= n)
        mine = -1;
    const double dw = mine < 0 ? 0.0 : (double)a.d_weight[(int64_t)blockIdx.x * k + lane];
    double g = dw;
    if (a.p.renormalise) {
        const double x = mine < 0 ? none : (double)route_logit((float)logits[mine]);
        const double s = mine < 0 ? none : a.p.score == FS_SCORE_SOFTMAX ? x : fmin(x, 0.0) - log1p(exp(-fabs(x)));
        const double high = wave_max(s);
        double q = s > none ? exp(s - high) : 0.0;
        const double all = wave_sum(q);
        q = all > 0.0 ? q / all : 0.0;
        const double mean = wave_sum(q > 0.0 ? q * dw : 0.0);
        g = q > 0.0 ? q * (dw - mean) : 0.0;
        if (a.p.score == FS_SCORE_SIGMOID)
            g *= 1.0 / (1.0 + exp(x));
    }
    for (int j = 0; j < k; ++j) {
        if (lane == j && mine >= 0)
            grad[mine] += g;
        __syncthreads();
    }
    double top = none, sum = 0.0, dot = 0.0;
    if (!a.p.renormalise && a.p.score == FS_SCORE_SOFTMAX) {
        for (int e = lane; e < n; e += 64)
            top = fmax(top, (double)route_logit((float)logits[e]));
        top = wave_max(top);
        if (top == none)
            top = 0.0;
        for (int e = lane; e < n; e += 64) {
            const double v = exp((double)route_logit((float)logits[e]) - top);
            sum += v;
            dot += v * grad[e];
        }
        sum = wave_sum(sum);
        dot = wave_sum(dot) / sum;
    }
    for (int e = lane; e < n; e += 64) {
        const double x = route_logit((float)logits[e]);
        double d = grad[e];
        if (!(x > none))
            d = 0.0;
        else if (!a.p.renormalise)
            d = a.p.score == FS_SCORE_SOFTMAX ? exp(x - top) / sum * (d - dot) : d / ((1.0 + exp(x)) * (1.0 + exp(-x)));
        out[e] = (T)(float)(d * (double)a.p.scale);
    }
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
    RouteArgs a = {*params, n_tokens, logit_stride, 0, logits, bias, expert, weight, nullptr, nullptr, nullptr};
    prof_start(kKernTopk, stream);
    with_type(logit_type, [&](auto t) {
        hipLaunchKernelGGL(route_kernel<decltype(t)::value>, dim3((unsigned)n_tokens), dim3(64), 0, stream, a);
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
    RouteArgs a = {*params, n_tokens, logit_stride, d_logit_stride, logits, nullptr, nullptr, nullptr, expert, d_weight, d_logits};
    prof_start(kKernTrainOther, stream);
    with_type(logit_type, [&](auto t) {
        hipLaunchKernelGGL(route_backward_kernel<decltype(t)::value>, dim3((unsigned)n_tokens), dim3(64), 0, stream, a);
    });
    prof_stop(stream);
    return launched("route gradient kernel launch");
}
