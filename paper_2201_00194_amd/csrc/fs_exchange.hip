// The exchange between tokens and experts: the plan of slots, rows into the slots, results back.
#include "fs_slots.h"

namespace fs {

struct Choices {
    typedef int32_t Item, What;
    const int32_t *expert;
    int32_t *first, *order, *places;
    int32_t n_experts;
    template <int N>
    __device__ __forceinline__ void load(int32_t (&item)[N], int64_t i, int64_t end) const
    {
#pragma unroll
        for (int u = 0; u < N; ++u)
            item[u] = expert[min(i + u * 64, end - 1)];
    }
    int more_counting() const { return 0; }
    int more_placing() const { return 0; }
    __device__ __forceinline__ void beside_count(int, int) const {}
    __device__ __forceinline__ void beside_place(int, int) const {}
    __device__ __forceinline__ int number(int32_t e) const { return e >= 0 && e < n_experts ? e : n_experts; }
    __device__ __forceinline__ void start(int e, int slot) const { first[e] = slot; }
    __device__ __forceinline__ int32_t what(int32_t, int64_t i) const { return (int32_t)i; }
    __device__ __forceinline__ void place(int64_t i, int e, int slot) const { places[i] = e < n_experts ? slot : -1; }
    __device__ __forceinline__ void put(int32_t i, int e, int slot) const { order[slot] = e < n_experts ? i : -1; }
};

// No choices: no slots.
__global__ void __launch_bounds__(256)
expert_none_kernel(int32_t n_experts, int32_t *first)
{
    for (int e = threadIdx.x; e <= n_experts; e += 256)
        first[e] = 0;
}

constexpr int kExchangeWaves = 4;      // of a workgroup
// From so many bytes of results on, which is more wavefronts than run at once, a lane works on two tokens of up to four choices.
constexpr int64_t kTwoTokens = 16 << 20;

struct ExchangeArgs {
    int64_t n_tokens, in_stride, y_stride, out_stride;
    int32_t k, n_experts, width, ll, columns;
    const void *in;                  // x, or the gradient of the tokens' results
    const void *y;
    const int32_t *first, *place;
    const float *weight;
    void *out;
    float *d_weight;
    int64_t block0;                  // of this launch
};
// Lanes (1 << ll) to a token; of a wide row, `columns` neighbouring wavefronts, so that they read a row at one time.  A lane
// works on tokens token, token + step, ...: `tokens` of them.
struct TokenLanes {
    int h, column, step;
    int64_t token;
    __device__ __forceinline__ explicit TokenLanes(const ExchangeArgs &a, int tokens = 1)
    {
        const int lane = threadIdx.x & 63;
        h = lane & ((1 << a.ll) - 1);
        const int64_t wave = (a.block0 + blockIdx.x) * kExchangeWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        column = a.columns == 1 ? 0 : (int)(wave % a.columns);
        token = a.columns == 1 ? ((wave * tokens) << (6 - a.ll)) + (lane >> a.ll) : wave / a.columns * tokens;
        step = 1 << (6 - a.ll);
    }
};

// The slots behind the last expert's: the tokens' lanes share them.
template <class T, bool PAST = false>
__device__ __forceinline__ void clear_slots_behind(const ExchangeArgs &a, int64_t token, int c, int n)
{
    RawChunk<T> zero;
    zero.clear();
    const int64_t slots = a.n_tokens * a.k;
    for (int64_t s = max(a.first[a.n_experts], 0) + token; s < slots; s += a.n_tokens)
        zero.template store<PAST>((T *)a.out + s * a.out_stride + c, n);
}

// A row is read once and written k times.  65 536 rows of 1024 bf16, k = 4: 143 us, 4.7 TB/s, what memory takes (a large copy 5.0).
template <int TYPE, bool PAST>
__global__ void __launch_bounds__(kExchangeWaves * 64)
expert_gather_kernel(ExchangeArgs a)
{
    typedef typename Element<TYPE>::type T;
    const TokenLanes l(a);
    if (l.token >= a.n_tokens)
        return;
    const Span at = span_of<kChunk<T>>((l.column * 64 + l.h) * kChunk<T>, a.width);
    const int c = at.c, n = at.n;
    const int64_t slots = a.n_tokens * a.k;
    RawChunk<T> x;
    x.load((const T *)a.in + l.token * a.in_stride + c, n);
    const int32_t *const place = a.place + l.token * a.k;
    for (int j = 0; j < a.k; ++j) {
        const int p = place[j];
        if (p >= 0 && p < slots)
            x.template store<PAST>((T *)a.out + (int64_t)p * a.out_stride + c, n);
    }
    clear_slots_behind<T, PAST>(a, l.token, c, n);
}

// Results are read once and not kept in the caches: 32768 rows of 164 features, slots, gather and this in turn, 66 us with them
// kept and 60 so.  Two tokens of a lane are on their way together where tokens are many: 26 us and 22.6 so.  65 536 tokens of 1024
// bf16, k = 4: 121 us, 5.5 TB/s.
template <int TYPE, int AHEAD, int TOKENS>
__global__ void __launch_bounds__(kExchangeWaves * 64)
expert_combine_kernel(ExchangeArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int N = kChunk<T>;
    const TokenLanes l(a, TOKENS);
    if (l.token >= a.n_tokens)
        return;
    const Span at = span_of<N>((l.column * 64 + l.h) * N, a.width);
    const int c = at.c, n = at.n;
    const int64_t slots = a.n_tokens * a.k;
    const T *const y = (const T *)a.y + c;
    float sum[TOKENS][N];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[t][i] = 0.0f;
    for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
        int p[TOKENS][AHEAD];
        float w[TOKENS][AHEAD];
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t at = min(l.token + t * l.step, a.n_tokens - 1) * a.k + min(j0 + u, a.k - 1);
                p[t][u] = a.place[at];
                w[t][u] = a.weight ? a.weight[at] : 1.0f;
            }
        RawChunk<T> x[TOKENS][AHEAD];
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const bool there = j0 + u < a.k && p[t][u] >= 0 && p[t][u] < slots && l.token + t * l.step < a.n_tokens;
                w[t][u] = there ? w[t][u] : 0.0f;
                x[t][u].template load<true>(y + (int64_t)(there ? p[t][u] : 0) * a.y_stride, there ? n : 0);
            }
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sum[t][i] = fmaf(w[t][u], x[t][u][i], sum[t][i]);
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        const int64_t token = l.token + t * l.step;
        store_chunk<N>((T *)a.out + token * a.out_stride + c, token < a.n_tokens ? n : 0, sum[t]);
    }
}

// The products need a token's whole width, so that its lanes go over the column blocks themselves.  At most kMostProducts of a lane
// are added one after the other; a wide row has many such sums, whose sum is another, so that 2^20 columns are 256 and 64
// additions long.  65 536 tokens of 1024 bf16, k = 4: 217 us, 5.6 TB/s.
constexpr int kMostProducts = 256;
template <int TYPE, int AHEAD>
__global__ void __launch_bounds__(kExchangeWaves * 64)
expert_combine_backward_kernel(ExchangeArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int N = kChunk<T>;
    const TokenLanes l(a);
    const bool there = l.token < a.n_tokens;
    const int64_t slots = a.n_tokens * a.k, token = there ? l.token : a.n_tokens - 1;
    if (__ballot(there) == 0)
        return;
    for (int j0 = 0; j0 < a.k; j0 += AHEAD) {
        int p[AHEAD];
        float w[AHEAD], dot[AHEAD], dots[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = min(j0 + u, a.k - 1);
            p[u] = a.place[token * a.k + j];
            if (!there || j0 + u >= a.k || p[u] < 0 || p[u] >= slots)
                p[u] = -1;
            w[u] = a.weight[token * a.k + j];
            dot[u] = dots[u] = 0.0f;
        }
        int products = 0;
        for (int c0 = l.h * N; c0 < a.width; c0 += 64 * N) {
            const Span at = span_of<N>(c0, a.width);
            const int c = at.c, n = at.n;
            RawChunk<T> g, y[AHEAD];
            g.load((const T *)a.in + token * a.in_stride + c, n);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                y[u].template load<true>((const T *)a.y + (int64_t)max(p[u], 0) * a.y_stride + c, p[u] >= 0 ? n : 0);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (p[u] < 0)
                    continue;
                float d[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dot[u] = i < at.skip ? dot[u] : fmaf(g[i], y[u][i], dot[u]);
                    d[i] = w[u] * g[i];
                }
                store_chunk<N>((T *)a.out + (int64_t)p[u] * a.out_stride + c, n, d);
            }
            products += N;
            if (products == kMostProducts) {
                products = 0;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    dots[u] += dot[u];
                    dot[u] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const float all = row_sum(dots[u] + dot[u], a.ll);
            if (there && l.h == 0 && j0 + u < a.k)
                a.d_weight[token * a.k + j0 + u] = all;
        }
    }
    if (there)
        for (int c0 = l.h * N; c0 < a.width; c0 += 64 * N) {
            const Span at = span_of<N>(c0, a.width);
            const int c = at.c, n = at.n;
            clear_slots_behind<T>(a, token, c, n);
        }
}

// f(workgroups) launches what one launch holds; a's numbers of lanes, columns and workgroups are set.
template <class F>
void over_tokens(ExchangeArgs &a, int32_t type, bool whole_rows, int tokens, F f)
{
    const int chunk = 16 / (int)type_bytes(type);
    a.ll = row_lanes_log(a.width, chunk);
    a.columns = whole_rows ? 1 : column_blocks(a.width, chunk);
    const int64_t each = (int64_t)tokens << (6 - a.ll), waves = (a.n_tokens + each - 1) / each * a.columns;
    in_pieces((waves + kExchangeWaves - 1) / kExchangeWaves, [&](int64_t at, unsigned blocks) {
        a.block0 = at;
        f(blocks);
    });
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
    return slot_count_bytes(slot_shape(n_tokens * k, n_experts + 1, sizeof(Choices::What)), kSlotFew);
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
    const SlotShape s = slot_shape(n_tokens * k, n_experts + 1, sizeof(Choices::What));
    const size_t need = slot_count_bytes(s, kSlotFew);
    FS_TRY(check_array(who, "work", work, (int64_t)need, 256));
    if (work_bytes < need)
        return fail(FS_EINVAL, "%s: %zu bytes of working memory, %zu are needed", who, work_bytes, need);
    int32_t *count = (int32_t *)work;
    prof_start(kKernPack, stream);
    const Choices choices = {expert, first, order, place, n_experts};
    if (s.n > kSlotFew)
        launch_slots(choices, s, count, stream);
    else if (s.n > 0)
        launch_few_slots(choices, s, stream);
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
    ExchangeArgs a = {n_tokens, x_stride, 0, xs_stride, k, n_experts, width, 0, 1, x, nullptr, first, place, nullptr, xs, nullptr, 0};
    prof_start(kKernPack, stream);
    with_type(type, [&](auto t) {
        over_tokens(a, type, false, 1, [&](unsigned blocks) {
            const auto kernel = past_caches(n_tokens * k, width, type) ? expert_gather_kernel<decltype(t)::value, true>
                                                                       : expert_gather_kernel<decltype(t)::value, false>;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kExchangeWaves * 64), 0, stream, a);
        });
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
    ExchangeArgs a = {n_tokens, 0, y_stride, out_stride, k, 0, width, 0, 1, nullptr, y, nullptr, place, weight, out, nullptr, 0};
    prof_start(kKernPack, stream);
    with_type(type, [&](auto t) {
        constexpr int element = decltype(t)::value;
        const bool two = k <= 4 && n_tokens * width * (int64_t)type_bytes(type) >= kTwoTokens;
        over_tokens(a, type, false, two ? 2 : 1, [&](unsigned blocks) {
            const auto kernel = two      ? expert_combine_kernel<element, 4, 2>
                                : k <= 4 ? expert_combine_kernel<element, 4, 1>
                                         : expert_combine_kernel<element, 8, 1>;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kExchangeWaves * 64), 0, stream, a);
        });
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
    ExchangeArgs a = {n_tokens, d_out_stride, y_stride, d_y_stride, k, n_experts, width, 0, 1, d_out, y, first, place, weight, d_y, d_weight, 0};
    prof_start(kKernTrainOther, stream);
    with_type(type, [&](auto t) {
        over_tokens(a, type, true, 1, [&](unsigned blocks) {
            const auto kernel = k <= 4 ? expert_combine_backward_kernel<decltype(t)::value, 4> : expert_combine_backward_kernel<decltype(t)::value, 8>;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kExchangeWaves * 64), 0, stream, a);
        });
    });
    prof_stop(stream);
    return launched("expert combine gradient kernel launch");
}
