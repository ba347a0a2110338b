// Rows in 8-bit integers with a scale each, where they are or in their experts' slots.
#include "fs_mixture.h"
#include "familyseer_experts.h"

namespace fs {

struct QuantizeArgs {
    int64_t n_rows, x_stride, q_stride;
    int32_t width, ll, k, n_experts;
    const void *x;
    const int32_t *first, *place;      // place NULL: row r's integers are row r
    int8_t *q;
    float *scale;
    int64_t row0;
};

// x / scale to the nearest integer, exactly: the product with the reciprocal names it or a neighbour; what is left of x is exact
// in fp32 (at most about half a step of scale, on a grid that x and scale have in common), and so is its double beside scale.
__device__ __forceinline__ int quotient(float x, float scale, float inverse_scale)
{
    const float n = __builtin_rintf(x * inverse_scale), left = fmaf(-n, scale, x), twice = 2.0f * fabsf(left);
    const bool odd = (int)n & 1;
    return (int)n + (twice > scale || (twice == scale && odd) ? (left > 0.0f ? 1 : -1) : 0);
}

template <int N>
__device__ __forceinline__ void store_bytes(int8_t *p, int n, const int (&v)[N])
{
    typedef int8_t Loose __attribute__((ext_vector_type(N), aligned(1)));
    if (n >= N) {
        Loose c;
#pragma unroll
        for (int i = 0; i < N; ++i)
            c[i] = (int8_t)v[i];
        *(Loose *)p = c;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n)
                p[i] = (int8_t)v[i];
    }
}

// 1 << ll lanes to a row.  C > 0: a lane keeps so many chunks of it; else it is read once for its largest and once more for its integers.
// Bound by memory where rows are many: 32 768 of 1024 fp16 to four slots each 40 us, 5.0 TB/s (quotients that are exact cost nothing
// beside it); eight rows take 7 us, most of it their loads' latency.
template <int TYPE, int C>
__global__ void __launch_bounds__(256)
quantize_kernel(QuantizeArgs a)
{
    typedef typename Element<TYPE>::type T;
    constexpr int N = kChunk<T>;
    const int lane = threadIdx.x & 63, h = lane & ((1 << a.ll) - 1), each = 64 >> a.ll;
    const int64_t wave = (a.row0 + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = wave * each + (lane >> a.ll);
    if (wave * each >= a.n_rows)
        return;
    const bool there = row < a.n_rows;
    const int64_t from = there ? row : a.n_rows - 1;
    const T *const x = (const T *)a.x + from * a.x_stride;
    unsigned most = 0;      // of the values without their signs, as their bits: infinities and NaN are above all others
    RawChunk<T> kept[C ? C : 1];
    if constexpr (C > 0) {
#pragma unroll
        for (int u = 0; u < C; ++u) {
            const int c = (u << a.ll | h) * N;
            kept[u].load(x + c, a.width - c);
        }
#pragma unroll
        for (int u = 0; u < C; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i)
                most = max(most, __float_as_uint(kept[u][i]) & 0x7fffffffu);
    } else {
        for (int c = h * N; c < a.width; c += N << a.ll) {
            float v[N];
            load_chunk(x + c, a.width - c, v);
#pragma unroll
            for (int i = 0; i < N; ++i)
                most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
        }
    }
    most = row_reduce((int)most, a.ll, [](int p, int q) { return max(p, q); });
    const bool good = most < 0x7f800000u;
    const float scale = good ? fmaxf(__uint_as_float(most) / 127.0f, 1.17549435e-38f) : __uint_as_float(0x7fc00000u);
    const float inverse_scale = 1.0f / scale;
    const int64_t slots = a.n_rows * a.k;
    // f(row of q) for each row that this one goes to.
    const auto each_place = [&](auto f) {
        if (!there)
            return;
        if (!a.place) {
            f(row);
            return;
        }
        for (int j = 0; j < a.k; ++j) {
            const int p = a.place[row * a.k + j];
            if (p >= 0 && p < slots)
                f((int64_t)p);
        }
    };
    if (h == 0)
        each_place([&](int64_t p) { a.scale[p] = scale; });
    const auto put = [&](int c, const auto &v) {
        int q[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            q[i] = good ? quotient(v[i], scale, inverse_scale) : 0;
        each_place([&](int64_t p) { store_bytes<N>(a.q + p * a.q_stride + c, a.width - c, q); });
    };
    if constexpr (C > 0) {
#pragma unroll
        for (int u = 0; u < C; ++u) {
            const int c = (u << a.ll | h) * N;
            if (c < a.width)
                put(c, kept[u]);
        }
    } else {
        for (int c = h * N; c < a.width; c += N << a.ll) {
            float v[N];
            load_chunk(x + c, a.width - c, v);
            put(c, v);
        }
    }
    if (a.place && there) {
        const int zero[N] = {};
        for (int64_t s = max(a.first[a.n_experts], 0) + row; s < slots; s += a.n_rows) {
            if (h == 0)
                a.scale[s] = 0.0f;
            for (int c = h * N; c < a.width; c += N << a.ll)
                store_bytes<N>(a.q + s * a.q_stride + c, a.width - c, zero);
        }
    }
}

static void launch_quantize(QuantizeArgs a, int32_t type, hipStream_t stream)
{
    const int chunk = 16 / (int)type_bytes(type), blocks_of_row = column_blocks(a.width, chunk);
    a.ll = row_lanes_log(a.width, chunk);
    const int64_t each = (int64_t)4 << (6 - a.ll);
    with_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        const auto kernel = blocks_of_row <= 1   ? quantize_kernel<T, 1>
                            : blocks_of_row <= 2 ? quantize_kernel<T, 2>
                            : blocks_of_row <= 4 ? quantize_kernel<T, 4>
                            : blocks_of_row <= 8 ? quantize_kernel<T, 8>
                                                 : quantize_kernel<T, 0>;
        in_pieces((a.n_rows + each - 1) / each, [&](int64_t at, unsigned blocks) {
            a.row0 = at;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, a);
        });
    });
}

}  // namespace fs

using namespace fs;

extern "C" int fs_quantize_rows(int64_t n_rows, int32_t width, const void *x, int32_t type, int64_t x_stride, int8_t *q, int64_t q_stride,
                                float *scale, void *stream_)
{
    static const char who[] = "fs_quantize_rows";
    hipStream_t stream = (hipStream_t)stream_;
    if (n_rows < 0 || n_rows >= ((int64_t)1 << 31))
        return fail(FS_EINVAL, "%s: %lld rows: 0 to 2^31 - 1 are taken", who, (long long)n_rows);
    FS_TRY(check_width(who, width));
    FS_TRY(check_matrix(who, "x", x, n_rows, width, type, x_stride));
    FS_TRY(check_bytes(who, "q", q, n_rows, width, q_stride));
    FS_TRY(check_array(who, "scale", scale, n_rows, 4));
    if (n_rows == 0)
        return FS_OK;
    prof_start(kKernPack, stream);
    launch_quantize(QuantizeArgs{n_rows, x_stride, q_stride, width, 0, 1, 0, x, nullptr, nullptr, q, scale, 0}, type, stream);
    prof_stop(stream);
    return launched("row quantizing kernel launch");
}

extern "C" int fs_expert_gather_i8(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t width, const void *x, int32_t type, int64_t x_stride,
                                   const int32_t *first, const int32_t *place, int8_t *q, int64_t q_stride, float *scale, void *stream_)
{
    static const char who[] = "fs_expert_gather_i8";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_tokens(who, n_tokens, k));
    FS_TRY(check_experts(who, n_experts));
    FS_TRY(check_width(who, width));
    FS_TRY(check_matrix(who, "x", x, n_tokens, width, type, x_stride));
    FS_TRY(check_array(who, "first", first, n_tokens, 4));
    FS_TRY(check_array(who, "place", place, n_tokens, 4));
    FS_TRY(check_bytes(who, "q", q, n_tokens, width, q_stride));
    FS_TRY(check_array(who, "scale", scale, n_tokens, 4));
    if (n_tokens == 0)
        return FS_OK;
    prof_start(kKernPack, stream);
    launch_quantize(QuantizeArgs{n_tokens, x_stride, q_stride, width, 0, k, n_experts, x, first, place, q, scale, 0}, type, stream);
    prof_stop(stream);
    return launched("row quantizing kernel launch");
}
