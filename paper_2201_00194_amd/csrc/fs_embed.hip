// Embedding: tokens, or bags of tokens, to scaled sums of a table's rows, and the table's gradient by sorted tokens.
#include "fs_slots.h"

#include <math.h>

namespace fs {

struct EmbedIds {
    const void *ids;
    const int32_t *col_base;
    int32_t id_type, n_cols, n_vocab;
    // The table's row of entry i, or -1.
    __device__ __forceinline__ int64_t row(int64_t i) const
    {
        int64_t v = id_type == FS_ID_I32 ? (int64_t)((const int32_t *)ids)[i]
                    : id_type == FS_ID_I64 ? ((const int64_t *)ids)[i]
                                           : (int64_t)((const uint16_t *)ids)[i];
        if (v < -2147483648ll || v > 2147483647ll)
            return -1;
        if (col_base)
            v += col_base[i % n_cols];
        return v >= 0 && v < n_vocab ? v : -1;
    }
};

struct EmbedArgs {
    EmbedIds ids;
    const void *in;            // the table, or the gradient of the sums
    int64_t in_stride, out_stride, n_rows;
    int32_t width, accumulate;
    float scale;
    void *out;
    const int32_t *token, *entry;   // sorted
};

template <int IN, int OUT>
__global__ void __launch_bounds__(64)
embed_kernel(EmbedArgs a)
{
    typedef typename Element<IN>::type In;
    typedef typename Element<OUT>::type Out;
    const int64_t r = blockIdx.x;
    for (int c = threadIdx.x; c < a.width; c += 64) {
        float sum = 0.0f;
        for (int j = 0; j < a.ids.n_cols; ++j) {
            const int64_t v = a.ids.row(r * a.ids.n_cols + j);
            if (v >= 0)
                sum += (float)((const In *)a.in)[v * a.in_stride + c];
        }
        ((Out *)a.out)[r * a.out_stride + c] = (Out)(sum * a.scale);
    }
}

// Sorting the entries by token, a digit at a time: the first pass takes ids, the others what the pass before left.
struct DigitOfId {
    EmbedIds ids;
    int32_t mask;
    __device__ __forceinline__ int token(int64_t i) const
    {
        const int64_t v = ids.row(i);
        return v < 0 ? ids.n_vocab : (int)v;
    }
    __device__ __forceinline__ int operator()(int64_t i) const { return token(i) & mask; }
};
struct DigitOfToken {
    const int32_t *from;
    int32_t shift, mask;
    __device__ __forceinline__ int operator()(int64_t i) const { return (from[i] >> shift) & mask; }
};
struct PutId {
    DigitOfId of;
    int32_t *token, *entry;
    __device__ __forceinline__ void operator()(int64_t i, int, int slot) const
    {
        token[slot] = of.token(i);
        entry[slot] = (int32_t)i;
    }
};
struct PutToken {
    const int32_t *from_token, *from_entry;
    int32_t *token, *entry;
    __device__ __forceinline__ void operator()(int64_t i, int, int slot) const
    {
        token[slot] = from_token[i];
        entry[slot] = from_entry[i];
    }
};

__device__ __forceinline__ int64_t first_not_below(const int32_t *token, int64_t n, int v)
{
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (token[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

template <int IN, int OUT>
__global__ void __launch_bounds__(64)
embed_backward_kernel(EmbedArgs a, int64_t n)
{
    typedef typename Element<IN>::type In;
    typedef typename Element<OUT>::type Out;
    const int v = blockIdx.x;
    const int64_t begin = first_not_below(a.token, n, v), end = first_not_below(a.token, n, v + 1);
    for (int c = threadIdx.x; c < a.width; c += 64) {
        double sum = 0.0;
        for (int64_t i = begin; i < end; ++i)
            sum += (double)(float)((const In *)a.in)[(int64_t)(a.entry[i] / a.ids.n_cols) * a.in_stride + c];
        Out &out = ((Out *)a.out)[(int64_t)v * a.out_stride + c];
        const double add = sum * (double)a.scale;
        out = (Out)(float)(a.accumulate ? (double)(float)out + add : add);
    }
}

struct SortPlan {
    int passes, bits;
    SlotShape shape;
    size_t list_bytes, bytes;
};
static SortPlan sort_plan(int32_t n_vocab, int64_t n)
{
    SortPlan p;
    int bits = 1;                                  // of 0 .. n_vocab
    while (((int64_t)1 << bits) <= n_vocab)
        ++bits;
    p.passes = (bits + 9) / 10;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.shape = slot_shape(n, 1 << p.bits);
    p.list_bytes = ((size_t)n * 4 + 255) / 256 * 256;
    p.bytes = 4 * p.list_bytes + slot_count_bytes(p.shape);
    return p;
}

static int check_embed(const char *who, int32_t n_vocab, int32_t width, int64_t n_rows, int32_t n_cols)
{
    if (n_vocab < 1 || n_vocab == 2147483647)
        return fail(FS_EINVAL, "%s: n_vocab %d outside [1, 2^31 - 2]", who, n_vocab);
    if (width < 1)
        return fail(FS_EINVAL, "%s: width %d", who, width);
    if (n_cols < 1)
        return fail(FS_EINVAL, "%s: n_cols %d", who, n_cols);
    if (n_rows < 0 || n_rows >= ((int64_t)1 << 31) || n_rows * n_cols >= ((int64_t)1 << 31))
        return fail(FS_EINVAL, "%s: %lld rows of %d ids: 0 to 2^31 - 1 ids are taken", who, (long long)n_rows, n_cols);
    return FS_OK;
}
static int check_ids(const char *who, int64_t n_rows, const void *ids, int32_t id_type, const int32_t *col_base, float scale)
{
    if (id_type != FS_ID_I32 && id_type != FS_ID_I64 && id_type != FS_ID_U16)
        return fail(FS_EINVAL, "%s: unknown type %d of ids", who, id_type);
    FS_TRY(check_array(who, "ids", ids, n_rows, id_type == FS_ID_I32 ? 4 : id_type == FS_ID_I64 ? 8 : 2));
    FS_TRY(check_array(who, "col_base", col_base, 0, 4));
    return isfinite(scale) ? FS_OK : fail(FS_EINVAL, "%s: scale is not finite", who);
}
static int check_out_type(const char *who, const char *what, int32_t in_type, int32_t out_type)
{
    if (out_type != FS_F32 && out_type != in_type)
        return fail(FS_EINVAL, "%s: %s is of another type than the input and not fp32", who, what);
    return FS_OK;
}

// f(input's type, output's type)
template <class F>
void with_types(int32_t in, int32_t out, F f)
{
    with_type(in, [&](auto i) {
        if (out == FS_F32)
            f(i, TypeTag<FS_F32>());
        else
            f(i, i);
    });
}

}  // namespace fs

using namespace fs;

extern "C" int fs_embed(int32_t n_vocab, int32_t width, const void *table, int32_t table_type, int64_t table_stride, int64_t n_rows,
                        int32_t n_cols, const void *ids, int32_t id_type, const int32_t *col_base, float scale, void *out, int32_t out_type,
                        int64_t out_stride, void *stream_)
{
    static const char who[] = "fs_embed";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_embed(who, n_vocab, width, n_rows, n_cols));
    FS_TRY(check_matrix(who, "table", table, n_vocab, width, table_type, table_stride));
    FS_TRY(check_ids(who, n_rows, ids, id_type, col_base, scale));
    FS_TRY(check_matrix(who, "out", out, n_rows, width, out_type, out_stride));
    FS_TRY(check_out_type(who, "out", table_type, out_type));
    if (n_rows == 0)
        return FS_OK;
    EmbedArgs a = {{ids, col_base, id_type, n_cols, n_vocab}, table, table_stride, out_stride, n_rows, width, 0, scale, out, nullptr, nullptr};
    prof_start(kKernPack, stream);
    with_types(table_type, out_type, [&](auto i, auto o) {
        hipLaunchKernelGGL((embed_kernel<decltype(i)::value, decltype(o)::value>), dim3((unsigned)n_rows), dim3(64), 0, stream, a);
    });
    prof_stop(stream);
    return launched("embedding kernel launch");
}

extern "C" size_t fs_embed_backward_workspace_bytes(int32_t n_vocab, int32_t width, int64_t n_rows, int32_t n_cols)
{
    if (check_embed("fs_embed_backward_workspace_bytes", n_vocab, width, n_rows, n_cols) != FS_OK)
        return 0;
    return sort_plan(n_vocab, n_rows * n_cols).bytes;
}

extern "C" int fs_embed_backward(int32_t n_vocab, int32_t width, const void *d_out, int32_t d_out_type, int64_t d_out_stride, int64_t n_rows,
                                 int32_t n_cols, const void *ids, int32_t id_type, const int32_t *col_base, float scale, int32_t accumulate,
                                 void *d_table, int32_t d_table_type, int64_t d_table_stride, void *work, size_t work_bytes, void *stream_)
{
    static const char who[] = "fs_embed_backward";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_embed(who, n_vocab, width, n_rows, n_cols));
    FS_TRY(check_matrix(who, "d_out", d_out, n_rows, width, d_out_type, d_out_stride));
    FS_TRY(check_ids(who, n_rows, ids, id_type, col_base, scale));
    FS_TRY(check_matrix(who, "d_table", d_table, n_vocab, width, d_table_type, d_table_stride));
    FS_TRY(check_out_type(who, "d_table", d_out_type, d_table_type));
    if (accumulate != 0 && accumulate != 1)
        return fail(FS_EINVAL, "%s: accumulate is %d", who, accumulate);
    const int64_t n = n_rows * n_cols;
    const SortPlan p = sort_plan(n_vocab, n);
    FS_TRY(check_array(who, "work", work, (int64_t)p.bytes, 256));
    if (work_bytes < p.bytes)
        return fail(FS_EINVAL, "%s: %zu bytes of working memory, %zu are needed", who, work_bytes, p.bytes);
    int32_t *token[2], *entry[2];
    for (int i = 0; i < 2; ++i) {
        token[i] = (int32_t *)((char *)work + (2 * i) * p.list_bytes);
        entry[i] = (int32_t *)((char *)work + (2 * i + 1) * p.list_bytes);
    }
    int32_t *count = (int32_t *)((char *)work + 4 * p.list_bytes);
    prof_start(kKernTrainOther, stream);
    const EmbedIds e = {ids, col_base, id_type, n_cols, n_vocab};
    const int mask = (1 << p.bits) - 1;
    int at = 0;
    if (n > 0) {
        const DigitOfId of = {e, mask};
        launch_slots(of, PutId{of, token[0], entry[0]}, p.shape, count, stream);
        for (int pass = 1; pass < p.passes; ++pass, at ^= 1)
            launch_slots(DigitOfToken{token[at], pass * p.bits, mask}, PutToken{token[at], entry[at], token[at ^ 1], entry[at ^ 1]},
                         p.shape, count, stream);
    }
    EmbedArgs a = {e, d_out, d_out_stride, d_table_stride, n_rows, width, accumulate, scale, d_table, token[at], entry[at]};
    with_types(d_out_type, d_table_type, [&](auto i, auto o) {
        hipLaunchKernelGGL((embed_backward_kernel<decltype(i)::value, decltype(o)::value>), dim3((unsigned)n_vocab), dim3(64), 0, stream, a, n);
    });
    prof_stop(stream);
    return launched("embedding gradient kernels launch");
}
