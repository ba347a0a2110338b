// Distillation from a teacher's largest logits, and its gradient.
//
// With m the largest x = logit / T of the row and s the sum of exp(x - m), log p_c = x_c - m - log s.  A row is read once for m and s;
// its gradient needs it once more, as d_c = coefficient * (Q p_c - the entries' q of c) with Q the sum of all q: one factor for all classes
// without an entry.  With a rest, its share of p meets its q in a difference that may be small, so m and s go over the classes without an entry
// alone (a bit a class says which have one), entries are added in 64 bits, and p_rest = 1 / (1 + entries / rest) is as exact as they are.
#include "fs_mixture.h"
#include "familyseer_experts.h"

namespace fs {

struct DistillArgs {
    const void *logits, *ids, *teacher;
    const float *total, *d_loss;
    float *loss;
    void *d_logits;
    int64_t n_tokens, logit_stride, d_logit_stride, row0;
    int32_t n_classes, k, id_type, teacher_type;
    float rate;                 // log2(e) / T
    double inverse_t, scale;
};

// -infinity for NaN, the largest float for infinity.
__device__ __forceinline__ float clean(float v) { return fminf(fmaxf(v, -__builtin_inff()), 3.402823466e38f); }

// 256 threads' values joined, the same way every time; all get the result.
template <class T, class F>
__device__ __forceinline__ T join_all(T v, T *lds, F f)
{
    v = row_reduce(v, 6, f);
    __syncthreads();            // what was here before has been read
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return f(f(lds[0], lds[1]), f(lds[2], lds[3]));
}
__device__ __forceinline__ double sum_all(double v, double *lds) { return join_all(v, lds, [](double a, double b) { return a + b; }); }
__device__ __forceinline__ float max_all(float v, float *lds) { return join_all(v, lds, [](float a, float b) { return fmaxf(a, b); }); }

__device__ __forceinline__ int64_t id_at(const void *ids, int type, int64_t i) { return type == FS_ID_I64 ? ((const int64_t *)ids)[i] : ((const int32_t *)ids)[i]; }
__device__ __forceinline__ float element_at(const void *p, int type, int64_t i)
{
    return type == FS_F32 ? ((const float *)p)[i] : type == FS_BF16 ? (float)((const __bf16 *)p)[i] : (float)((const _Float16 *)p)[i];
}

constexpr int kEntriesEach = FS_MAX_LISTED / 256;      // of a thread

// A workgroup to a row.
template <int TYPE, bool GRADIENT>
__global__ void __launch_bounds__(256)
distill_kernel(DistillArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int N = kChunk<T>;
    __shared__ double joined[4];
    __shared__ int listed[FS_MAX_LISTED];          // classes, -1: no entry
    __shared__ float share[FS_MAX_LISTED];         // q
    __shared__ int twice;
    extern __shared__ unsigned has_entry[];        // a bit a class
    const int64_t row = a.row0 + blockIdx.x;
    const T *const logits = (const T *)a.logits + row * a.logit_stride;
    const int tid = threadIdx.x;

    const float total = a.total ? a.total[row] : __builtin_inff();
    bool rest = __builtin_isfinite(total);
    if (rest)
        for (int i = tid; i < (a.n_classes + 31) / 32; i += 256)
            has_entry[i] = 0;
    if (tid == 0)
        twice = 0;
    __syncthreads();
    float x[kEntriesEach], t[kEntriesEach], top = -__builtin_inff(), high = top;
    int id[kEntriesEach];
#pragma unroll
    for (int u = 0; u < kEntriesEach; ++u) {
        const int j = tid + u * 256;
        id[u] = -1;
        x[u] = t[u] = -__builtin_inff();
        if (j < a.k) {
            const int64_t c = id_at(a.ids, a.id_type, row * a.k + j);
            t[u] = clean(element_at(a.teacher, a.teacher_type, row * a.k + j));
            if (c >= 0 && c < a.n_classes)
                x[u] = clean((float)logits[c]);
            if (x[u] > -__builtin_inff() && t[u] > -__builtin_inff()) {
                id[u] = (int)c;
                top = fmaxf(top, t[u]);
                high = fmaxf(high, x[u]);
            }
            listed[j] = id[u];
        }
        if (id[u] >= 0 && rest && (atomicOr(&has_entry[id[u] >> 5], 1u << (id[u] & 31)) >> (id[u] & 31) & 1))
            twice = 1;
    }
    top = max_all(top, (float *)joined);
    high = max_all(high, (float *)joined);
    const bool taught = top > -__builtin_inff();

    // the row's largest and sum, without entries where there is a rest
    float m = -__builtin_inff(), s = 0.0f;
    for (int c = tid * N; c < a.n_classes; c += 256 * N) {
        float v[N];
        load_chunk(logits + c, a.n_classes - c, v, -__builtin_inff());
        const unsigned out = rest ? has_entry[c >> 5] >> (c & 31) : 0;
        float most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = out >> i & 1 ? -__builtin_inff() : clean(v[i]);
            most = fmaxf(most, v[i]);
        }
        if (most > m) {
            s *= __builtin_amdgcn_exp2f((m - most) * a.rate);
            m = most;
        }
        if (m > -__builtin_inff()) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                s += __builtin_amdgcn_exp2f((v[i] - m) * a.rate);
        }
    }
    const float M = max_all(m, (float *)joined);
    const double S = sum_all(m > -__builtin_inff() ? (double)s * __builtin_amdgcn_exp2f((m - M) * a.rate) : 0.0, joined);
    const bool none = !(M > -__builtin_inff());      // no class without an entry is to be had
    if (rest && none)
        rest = false;
    const bool apart = a.total && __builtin_isfinite(total);      // entries are not in S

    // which of several entries of a class counts it
    bool owns[kEntriesEach];
    const bool search = apart ? twice != 0 : true;
#pragma unroll
    for (int u = 0; u < kEntriesEach; ++u) {
        owns[u] = id[u] >= 0;
        if (owns[u] && search)
            for (int j = 0; j < tid + u * 256; ++j)
                owns[u] &= listed[j] != id[u];
    }
    const float all_high = fmaxf(apart ? high : M, M);
    double beside = 0, q_top = 0;
#pragma unroll
    for (int u = 0; u < kEntriesEach; ++u) {
        if (owns[u] && apart)
            beside += exp(((double)x[u] - all_high) * a.inverse_t);
        if (id[u] >= 0)
            q_top += exp(((double)t[u] - top) * a.inverse_t);
    }
    beside = sum_all(beside, joined);
    q_top = sum_all(q_top, joined);
    const double down = none ? 0.0 : exp(((double)M - all_high) * a.inverse_t), Z = S * down + beside, log_z = log(Z);
    // log q = (t - base) / T - log_base
    const double base = rest ? 0.0 : top, log_base = rest ? (double)total : log(q_top);
    double q_all = 0, loss = 0;
    float q[kEntriesEach];
#pragma unroll
    for (int u = 0; u < kEntriesEach; ++u) {
        q[u] = 0.0f;
        if (id[u] >= 0) {
            const double log_q = fmin(0.0, ((double)t[u] - base) * a.inverse_t - log_base), e = exp(log_q);
            q_all += e;
            loss += e > 0 ? e * (log_q - (((double)x[u] - all_high) * a.inverse_t - log_z)) : 0.0;
            q[u] = (float)e;
        }
        if (tid + u * 256 < a.k)
            share[tid + u * 256] = q[u];
    }
    q_all = sum_all(q_all, joined);
    loss = sum_all(loss, joined);
    double q_rest = 0, p_rest = 0;
    if (rest && taught) {
        q_rest = fmax(0.0, 1.0 - q_all);
        const double ratio = beside / (S * down);
        const double log_p = ratio < 1e300 ? -log1p(ratio) : ((double)M - all_high) * a.inverse_t + log(S) - log_z;
        p_rest = exp(log_p);
        if (q_rest > 0)
            loss += q_rest * (log(q_rest) - log_p);
    }
    if (a.loss && tid == 0)
        a.loss[row] = taught ? (float)(loss * a.scale) : 0.0f;
    if constexpr (!GRADIENT)
        return;

    const double coefficient = taught ? (double)a.d_loss[row] * a.scale * a.inverse_t : 0.0, q_sum = q_all + q_rest;
    const float factor = taught && !none ? (float)(coefficient * (rest ? (q_sum * p_rest - q_rest) / S : q_sum * down / Z)) : 0.0f;
    const float from = none ? 0.0f : M;
    T *const d_logits = (T *)a.d_logits + row * a.d_logit_stride;
    for (int c = tid * N; c < a.n_classes; c += 256 * N) {
        float v[N];
        load_chunk(logits + c, a.n_classes - c, v, -__builtin_inff());
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = __builtin_amdgcn_exp2f((clean(v[i]) - from) * a.rate);
            v[i] = e > 0.0f ? e * factor : 0.0f;
        }
        store_chunk<N>(d_logits + c, a.n_classes - c, v);
    }
    __syncthreads();            // the entries' classes are written again
#pragma unroll
    for (int u = 0; u < kEntriesEach; ++u) {
        if (!owns[u])
            continue;
        double own = q[u];
        if (search)
            for (int j = tid + u * 256 + 1; j < a.k; ++j)
                own += listed[j] == id[u] ? share[j] : 0.0f;
        const double p = exp(((double)x[u] - all_high) * a.inverse_t - log_z);
        d_logits[id[u]] = (T)(float)(coefficient * (q_sum * p - own));
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
    if (!(p->temperature > 0.0f) || p->temperature > 3.402823466e38f)
        return fail(FS_EINVAL, "%s: temperature %g is not positive and finite", who, (double)p->temperature);
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
    a.inverse_t = 1.0 / p->temperature;
    a.rate = (float)(1.44269504088896340736 / p->temperature);
    a.scale = p->scale;
    const size_t lds = a.total ? (size_t)(a.n_classes + 31) / 32 * 4 : 0;
    prof_start(kKernTrainOther, stream);
    int rc = FS_OK;
    with_type(type, [&](auto t) {
        const auto kernel = gradient ? distill_kernel<decltype(t)::value, true> : distill_kernel<decltype(t)::value, false>;
        if (lds > 32768) {
            const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) {
                rc = fail_hip(e, "distillation kernel's LDS");
                return;
            }
        }
        in_pieces(a.n_tokens, [&](int64_t at, unsigned blocks) {
            a.row0 = at;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), lds, stream, a);
        });
    });
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
    const DistillArgs a = {logits, ids, teacher, total, nullptr, loss, nullptr, n_tokens, logit_stride, 0, 0, 0, 0, id_type, teacher_type, 0, 0, 0};
    return distill("fs_distill", false, params, a, logit_type, work, work_bytes, (hipStream_t)stream);
}

extern "C" int fs_distill_backward(const fs_distill_params *params, int64_t n_tokens, const void *logits, int32_t logit_type, int64_t logit_stride,
                                   const void *ids, int32_t id_type, const void *teacher, int32_t teacher_type, const float *total,
                                   const float *d_loss, float *loss, void *d_logits, int64_t d_logit_stride, void *work, size_t work_bytes,
                                   void *stream)
{
    const DistillArgs a = {logits, ids, teacher, total, d_loss, loss, d_logits, n_tokens, logit_stride, d_logit_stride, 0, 0, 0, id_type, teacher_type, 0, 0, 0};
    return distill("fs_distill_backward", true, params, a, logit_type, work, work_bytes, (hipStream_t)stream);
}
