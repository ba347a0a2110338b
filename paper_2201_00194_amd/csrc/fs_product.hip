// Products of rows in slots with their expert's weights, in 32, 16 and 8 bits, and the weights' gradient.
//
// A workgroup takes tiles of one expert's slots and columns one after the other; which, it finds from the experts' bounds by itself, so that no
// launch waits for the host to read them.
#include "fs_product.h"

namespace fs {

struct ProductArgs {
    Bounds bounds;
    const char *x, *w;
    int64_t x_stride, w_stride, w_step;      // bytes
    void *y;
    int64_t y_stride;                        // elements
    int32_t y_type, in_width, out_width, across;      // tiles across a row of results
    const float *scale, *w_scale;            // of 8-bit operands
};

typedef Shape<256, 256, 2, 4, 128, 2> Wide;           // of rows
typedef Shape<256, 256, 2, 4, 64, 4> WideAcross;      // of weights' gradients
typedef Shape<128, 128, 2, 2, 128, 2> Middle;
typedef Shape<128, 64, 4, 1, 64, 2> Small;            // of rows
typedef Shape<64, 64, 2, 1, 128, 2> Little;           // of rows
typedef Shape<128, 64, 2, 1, 64, 2> SmallAcross;

// Results of a tile whose piece and first column are given.
template <int TYPE, class S, class T>
__device__ __forceinline__ void store_product(const ProductArgs &a, const T &t, char *rows, const Piece &piece, int n0)
{
    constexpr int N = 16 / sizeof(S);
    const int thread = thread_here();
    S *const y = (S *)a.y + (int64_t)piece.first * a.y_stride + n0;
    const auto put = [&](int row, int column, const auto &part) {
        if (row < piece.count)
            store_part<S, N>(y + row * a.y_stride + column, a.out_width - n0 - column, part);
    };
    if constexpr (TYPE == kI8) {      // all scales are there before the first store
        struct Scales {
            float v[16];
        };
        float scale[T::MF];
#pragma unroll
        for (int i = 0; i < T::MF; ++i)
            scale[i] = a.scale[piece.first + min(T::row_of(thread, thread & 15, i), piece.count - 1)];
        t.template results<S>(
            rows, thread,
            [&](int column) {
                Scales s;
                const float *const from = a.w_scale + (int64_t)piece.expert * a.out_width;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s.v[i] = from[min(n0 + column + i, a.out_width - 1)];
                return s;
            },
            [&](int i, const auto &v, const Scales &s, float (&out)[16]) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    out[e] = (float)v[e] * scale[i] * s.v[e];
            },
            put);
    } else {
        t.template results<S>(
            rows, thread, [](int) { return 0; },
            [](int, const auto &v, int, float (&out)[16]) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    out[e] = v[e];
            },
            put);
    }
}
template <int TYPE, int RESULT, class T>
__device__ __forceinline__ void store_product_as(const ProductArgs &a, const T &t, char *rows, const Piece &piece, int n0)
{
    if (RESULT != FS_F32 && a.y_type == FS_F32)
        store_product<TYPE, float>(a, t, rows, piece, n0);
    else
        store_product<TYPE, typename Element<RESULT>::type>(a, t, rows, piece, n0);
}

// Nobody's slots, by all workgroups of a launch.
template <class S, int THREADS>
__device__ __forceinline__ void clear_nobodys_as(const ProductArgs &a)
{
    constexpr int N = 16 / sizeof(S), rows = THREADS / 64;
    const S __attribute__((ext_vector_type(N))) zero = {};
    const int from = min(max(a.bounds.first[a.bounds.n_experts], 0), a.bounds.n_slots);
    for (int64_t s = from + (int64_t)blockIdx.x * rows + threadIdx.x / 64; s < a.bounds.n_slots; s += (int64_t)gridDim.x * rows)
        for (int c = (threadIdx.x & 63) * N; c < a.out_width; c += 64 * N)
            store_part<S, N>((S *)a.y + s * a.y_stride + c, a.out_width - c, zero);
}
template <int RESULT, int THREADS>
__device__ __forceinline__ void clear_nobodys(const ProductArgs &a)
{
    if (RESULT != FS_F32 && a.y_type == FS_F32)
        clear_nobodys_as<float, THREADS>(a);
    else
        clear_nobodys_as<typename Element<RESULT>::type, THREADS>(a);
}

// The tiles that a workgroup makes, of `tiles`: an XCD, whose L2 cache is its own, takes neighbouring ones.  Results that fit the card's
// memory have fewer than 2^31 tiles.
struct Share {
    int id, last, by;
    __device__ __forceinline__ explicit Share(int tiles)
    {
        const int each = (tiles + 7) >> 3, xcd = (int)(blockIdx.x & 7);
        last = min((xcd + 1) * each, tiles);
        id = xcd * each + (int)(blockIdx.x >> 3);
        by = (int)(gridDim.x >> 3);
    }
};

// A workgroup makes BM slots of one expert times BN columns, and then others.  This form takes any alignment and is bound by the
// instructions that bring operands through registers: 32 768 slots of 16 experts, 1001 columns to 1001, bf16 108 us, where 1000 to 1000 take 67
// in the next one.
template <int TYPE, int RESULT, class SHAPE, bool TURNED>
__global__ void __launch_bounds__(SHAPE::threads)
product_kernel(ProductArgs a)
{
    typedef Tile<TYPE, SHAPE, false, TURNED> T;
    constexpr int BN = T::BN;
    __shared__ __attribute__((aligned(1024))) char lds[T::lds_bytes];
    __shared__ __attribute__((aligned(1024))) char rows[T::rows_bytes * (T::threads / 64)];
    __shared__ PieceTable<false> table;
    clear_nobodys<RESULT, T::threads>(a);
    for (Share s(table.template fill<T::threads>(a.bounds) * a.across); s.id < s.last; s.id += s.by) {
        const Piece piece = table.find(a.bounds, s.id / a.across);
        const int n0 = s.id % a.across * BN;
        T t;
        t.clear();
        const Operand x = {a.x + (int64_t)piece.first * a.x_stride, a.x_stride, piece.count};
        const char *const w = a.w + (int64_t)piece.expert * a.w_step;
        const Operand b = {TURNED ? w + (int64_t)n0 * T::U::size : w + (int64_t)n0 * a.w_stride, a.w_stride, a.out_width - n0};
        t.run(lds, x, b, a.in_width, a.in_width, TURNED ? a.out_width : a.in_width);
        store_product_as<TYPE, RESULT>(a, t, rows, piece, n0);
        __syncthreads();      // the last step has been read
    }
}

// The same with operands straight to LDS, one tile after the other: the first step of the next tile is on its way while the last
// step of one is multiplied and its results are stored.  131 072 slots of 64 experts, 1024 columns to 2048, bf16: 540 us, 1017 TFLOP/s,
// matrix units half busy; what holds it up is how long a row's first bytes take from memory, for of a quarter of the slots, which stay in the
// last cache, the same launch makes 1370 TFLOP/s.  Tiles in the order of the pieces, bypassing stores, longer and shorter steps, sums
// begun at other places, and loads asked for earlier changed nothing or cost time.
template <int TYPE, int RESULT, class SHAPE, bool TURNED>
__global__ void __launch_bounds__(SHAPE::threads)
product_stream_kernel(ProductArgs a)
{
    typedef Tile<TYPE, SHAPE, false, TURNED> T;
    constexpr int BM = T::BM, BN = T::BN;
    __shared__ __attribute__((aligned(1024))) char lds[T::lds_bytes];
    __shared__ __attribute__((aligned(1024))) char rows[T::rows_bytes * (T::threads / 64)];
    __shared__ PieceTable<false> table;
    clear_nobodys<RESULT, T::threads>(a);
    Share s(table.template fill<T::threads>(a.bounds) * a.across);
    if (s.id >= s.last)
        return;
    constexpr int stores = T::MF * T::NF / 4 * (RESULT == FS_F32 ? 4 : 2);     // of a wavefront and a whole tile, at least
    typename T::template Stream<stores> stream;
    stream.lds = lds;
    int to_load = s.id - s.by;
    const auto next = [&] {
        to_load += s.by;
        if (to_load >= s.last)
            return false;
        const Piece piece = table.find(a.bounds, to_load / a.across);
        const int n0 = to_load % a.across * BN;
        stream.sa = {Operand{a.x + (int64_t)piece.first * a.x_stride, a.x_stride, piece.count}};
        const char *const w = a.w + (int64_t)piece.expert * a.w_step;
        stream.sb = {Operand{TURNED ? w + (int64_t)n0 * T::U::size : w + (int64_t)n0 * a.w_stride, a.w_stride, a.out_width - n0}};
        stream.left = a.in_width;
        return true;
    };
    stream.begin(next);
    for (; s.id < s.last; s.id += s.by) {
        const Piece piece = table.find(a.bounds, s.id / a.across);
        const int n0 = s.id % a.across * BN;
        T t;
        t.clear();
        stream.sum(t, a.in_width, next);
        store_product_as<TYPE, RESULT>(a, t, rows, piece, n0);
        stream.stored(piece.count == BM && n0 + BN <= a.out_width);
    }
    stream.end();
}

// Few rows an expert: what counts is how fast the weights arrive.  A workgroup makes sixteen columns of one expert's results; its
// wavefronts share the sum out, 64 bytes of it each in turn, straight from memory to registers, and meet in LDS.  One row of 30
// experts, 1024 x 1024 bf16: 5 us; 16 slots of 30 of 2048 x 2048 int8, 46 MB of weights: 12.9 us, 3.6 TB/s.
constexpr int kFewWaves = 4;
template <int TYPE, int RESULT, int MF>
__global__ void __launch_bounds__(kFewWaves * 64)
product_few_kernel(ProductArgs a)
{
    typedef Unit16<TYPE> U;
    typedef typename Element<RESULT>::type E;
    constexpr int AHEAD = 4, per = MF * 16;
    __shared__ typename U::Acc others[kFewWaves - 1][MF][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int expert = blockIdx.y, n0 = blockIdx.x * 16, n_slots = a.bounds.n_slots;
    const bool owned = expert < a.bounds.n_experts;
    const int begin = min(max(a.bounds.first[expert], 0), n_slots), end = owned ? max(min(a.bounds.first[expert + 1], n_slots), begin) : n_slots;
    const bool wide = RESULT == FS_F32 || a.y_type == FS_F32;
    const int bytes = a.in_width * U::size, whole = bytes / kUnitBytes;
    const char *const w = a.w + (owned ? expert : 0) * a.w_step + min(n0 + r, a.out_width - 1) * a.w_stride + g * 16;
    for (int64_t s = begin + (int64_t)blockIdx.z * per; s < end; s += (int64_t)gridDim.z * per) {
        typename U::Acc acc[MF];
        const char *x[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            acc[f] = typename U::Acc{0, 0, 0, 0};
            x[f] = a.x + min((int)s + f * 16 + r, end - 1) * a.x_stride + g * 16;
        }
        if (owned) {
            int u = wave;
            for (; u + (AHEAD - 1) * kFewWaves < whole; u += AHEAD * kFewWaves) {
                I4 wv[AHEAD], xv[AHEAD][MF];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int64_t at = (int64_t)(u + i * kFewWaves) * kUnitBytes;
                    wv[i] = *(const typename Bytes16<U::size>::type *)(w + at);
#pragma unroll
                    for (int f = 0; f < MF; ++f)
                        xv[i][f] = *(const typename Bytes16<U::size>::type *)(x[f] + at);
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                    for (int f = 0; f < MF; ++f)
                        acc[f] = U::step(wv[i], xv[i][f], acc[f]);
            }
            for (; u * kUnitBytes < bytes; u += kFewWaves) {
                const int64_t at = (int64_t)u * kUnitBytes;
                const int n = (bytes - u * kUnitBytes - g * 16) / U::size;
                const I4 wv = some_bytes<U::size>(w + at, n);
#pragma unroll
                for (int f = 0; f < MF; ++f)
                    acc[f] = U::step(wv, some_bytes<U::size>(x[f] + at, n), acc[f]);
            }
            __syncthreads();      // the last piece's sums have been read
            if (wave > 0) {
#pragma unroll
                for (int f = 0; f < MF; ++f)
                    others[wave - 1][f][lane] = acc[f];
            }
            __syncthreads();
        }
        if (wave > 0)
            continue;
        const int column = n0 + g * 4, n = a.out_width - column;
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            const int row = (int)s + f * 16 + r;
            if (owned) {
#pragma unroll
                for (int i = 0; i < kFewWaves - 1; ++i)
                    acc[f] += others[i][f][lane];
            }
            if (row >= end || n <= 0)
                continue;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = (float)acc[f][i];
                if constexpr (TYPE == kI8)
                    y[i] = owned ? y[i] * a.scale[row] * a.w_scale[(int64_t)expert * a.out_width + min(column + i, a.out_width - 1)] : 0.0f;
            }
            const int64_t at = row * a.y_stride + column;
            if (wide)
                store_chunk<4>((float *)a.y + at, n, y);
            else
                store_chunk<4>((E *)a.y + at, n, y);
        }
    }
}

struct WeightsArgs {
    Bounds bounds;
    const char *g, *x;
    int64_t g_stride, x_stride;              // bytes
    void *d_w;
    int64_t d_w_stride, d_w_step;            // elements
    int32_t d_w_type, in_width, out_width, across, tiles, accumulate;      // tiles across and of a matrix
    float *work;
};

// Where the partial sum of a piece lies, of an expert that has several: such experts have more than bounds.per slots, so that of each
// bounds.per slots at most two such pieces begin there, a first one and another expert's last.
__device__ __forceinline__ float *partial_sum(const WeightsArgs &a, int first, int number)
{
    return a.work + ((int64_t)(first / a.bounds.per) * 2 + (number > 0 ? 1 : 0)) * a.out_width * a.in_width;
}

template <int TYPE, class T>
__device__ __forceinline__ void store_weights(const WeightsArgs &a, const T &t, char *rows, const Piece &piece, int m0, int n0)
{
    const int thread = thread_here();
    const auto as_they_are = [](int, const auto &v, int, float (&out)[16]) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            out[e] = v[e];
    };
    if (piece.of > 1) {
        float *const to = partial_sum(a, piece.first, piece.number);
        t.template results<float>(rows, thread, [](int) { return 0; }, as_they_are, [&](int row, int column, const auto &part) {
            if (m0 + row < a.out_width)
                store_part<float, 4>(to + (m0 + row) * (int64_t)a.in_width + n0 + column, a.in_width - n0 - column, part);
        });
        return;
    }
    t.template results<float>(rows, thread, [](int) { return 0; }, as_they_are, [&](int row, int column, auto part) {
        if (m0 + row >= a.out_width)
            return;
        const int64_t at = piece.expert * a.d_w_step + (m0 + row) * a.d_w_stride + n0 + column;
        const int n = a.in_width - n0 - column;
        typedef typename Element<TYPE>::type E;
        if (TYPE == FS_F32 || a.d_w_type == FS_F32) {
            float *const to = (float *)a.d_w + at;
            if (a.accumulate) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    part[i] += i < n ? to[i] : 0.0f;
            }
            store_part<float, 4>(to, n, part);
        } else {
            E *const to = (E *)a.d_w + at;
            E __attribute__((ext_vector_type(4))) half;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                half[i] = (E)(part[i] + (a.accumulate && i < n ? (float)to[i] : 0.0f));
            store_part<E, 4>(to, n, half);
        }
    });
}

// A workgroup makes BM x BN of an expert's gradient over one piece of its slots, and then others: the gradient itself where the
// piece is all of them, else a partial sum.  Pieces differ in length.  The longest come first, and each round of tiles goes to the XCDs the
// other way round than the one before, so that all have about the same to do; an XCD's tiles of a round are neighbours.
// 131 072 slots of 64 experts, 1024 x 1024 bf16, a tenth nobody's: 343 us, 725 TFLOP/s, matrix units half busy: rows of both operands come
// from memory as those of products do.  65 536 slots of 30, 164 x 256 fp32: 78 us, 71 TFLOP/s, 64 % busy.
template <int TYPE, class SHAPE, bool DIRECT>
__global__ void __launch_bounds__(SHAPE::threads)
weights_kernel(WeightsArgs a)
{
    typedef Tile<TYPE, SHAPE, true, true> T;
    constexpr int BM = T::BM, BN = T::BN;
    __shared__ __attribute__((aligned(1024))) char lds[T::lds_bytes];
    __shared__ __attribute__((aligned(1024))) char rows[T::rows_bytes * (T::threads / 64)];
    __shared__ PieceTable<true> table;
    const int tiles = table.template fill<T::threads>(a.bounds) * a.tiles, per_xcd = (int)(gridDim.x >> 3), xcd = (int)(blockIdx.x & 7);
    const auto tile_of_round = [&](int round) {
        return (round * 8 + (round & 1 ? 7 - xcd : xcd)) * per_xcd + (int)(blockIdx.x >> 3);
    };
    const int rounds = (tiles + (int)gridDim.x - 1) / (int)gridDim.x;
    struct Place2 {
        Piece piece;
        int m0, n0;
    };
    const auto place_of = [&](int id) {
        const int tile = id % a.tiles;
        return Place2{table.find(a.bounds, id / a.tiles), tile / a.across * BM, tile % a.across * BN};
    };
    const auto operand_g = [&](const Place2 &p) {
        return Operand{a.g + (int64_t)p.piece.first * a.g_stride + (int64_t)p.m0 * T::U::size, a.g_stride, a.out_width - p.m0};
    };
    const auto operand_x = [&](const Place2 &p) {
        return Operand{a.x + (int64_t)p.piece.first * a.x_stride + (int64_t)p.n0 * T::U::size, a.x_stride, a.in_width - p.n0};
    };
    if constexpr (DIRECT) {
        typename T::template Stream<T::MF * T::NF / 4 * 4> stream;
        stream.lds = lds;
        int to_load = -1;
        const auto next = [&] {
            while (++to_load < rounds) {
                const int id = tile_of_round(to_load);
                if (id >= tiles)
                    continue;
                const Place2 p = place_of(id);
                if (p.piece.count <= 0)
                    continue;
                stream.sa = {operand_g(p)};
                stream.sb = {operand_x(p)};
                stream.left = p.piece.count;
                return true;
            }
            return false;
        };
        stream.begin(next);
        for (int round = 0; round < rounds; ++round) {
            const int id = tile_of_round(round);
            if (id >= tiles)
                continue;
            const Place2 p = place_of(id);
            T t;
            t.clear();
            stream.sum(t, p.piece.count, next);
            store_weights<TYPE>(a, t, rows, p.piece, p.m0, p.n0);
            stream.stored(!a.accumulate && a.d_w_type == FS_F32 && p.m0 + BM <= a.out_width && p.n0 + BN <= a.in_width);
        }
        stream.end();
    } else {
        for (int round = 0; round < rounds; ++round) {
            const int id = tile_of_round(round);
            if (id >= tiles)
                continue;
            const Place2 p = place_of(id);
            T t;
            t.clear();
            t.run(lds, operand_g(p), operand_x(p), p.piece.count, a.out_width, a.in_width);
            store_weights<TYPE>(a, t, rows, p.piece, p.m0, p.n0);
            __syncthreads();      // the last step has been read
        }
    }
}

// The partial sums of an expert's pieces, in their order, in 64 bits: a wavefront to a row of the gradient.  8 us for 164 x 256 of 30
// experts of which each has two or three; 16 us for 64 of 1024 x 1024, most of it the start of workgroups that have nothing to join.
template <int TYPE>
__global__ void __launch_bounds__(256)
weights_join_kernel(WeightsArgs a)
{
    typedef typename Element<TYPE>::type E;
    const int expert = (int)(blockIdx.x / a.tiles);
    int begin, end;
    const int pieces = a.bounds.pieces(expert, begin, end);
    if (pieces <= 1)
        return;
    const bool wide = TYPE == FS_F32 || a.d_w_type == FS_F32;
    for (int row = (int)(blockIdx.x % a.tiles) * 4 + (int)(threadIdx.x >> 6); row < a.out_width; row += a.tiles * 4)
        for (int c = (threadIdx.x & 63) * 4; c < a.in_width; c += 256) {
            const int64_t at = expert * a.d_w_step + row * a.d_w_stride + c;
            const int n = a.in_width - c;
            double sum[4] = {};
            if (a.accumulate) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < n)
                        sum[i] = wide ? ((const float *)a.d_w)[at + i] : (float)((const E *)a.d_w)[at + i];
            }
            for (int p = 0; p < pieces; ++p) {
                float v[4];
                load_chunk(partial_sum(a, begin + p * a.bounds.per, p) + (int64_t)row * a.in_width + c, n, v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sum[i] += v[i];
            }
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = (float)sum[i];
            if (wide)
                store_chunk<4>((float *)a.d_w + at, n, v);
            else
                store_chunk<4>((E *)a.d_w + at, n, v);
        }
}

// Workgroups of a launch for at most `pieces` pieces of `tiles` tiles, of which a compute unit holds as many as its LDS does.
constexpr int kUnits = 256;      // compute units of the card
template <class T, class Table>
static unsigned workgroups(int64_t n_slots, int32_t n_experts, int64_t per, int64_t tiles)
{
    constexpr int resident = kUnits * (int)(163840 / (T::lds_bytes + T::rows_bytes * (T::threads / 64) + sizeof(Table)));
    const int64_t most = ((n_slots / per + n_experts) * tiles + 7) / 8 * 8;
    return (unsigned)(most < resident ? most : resident);
}

template <int TYPE, int RESULT, bool TURNED, class SHAPE, bool DIRECT>
static void launch_tiles(ProductArgs a, hipStream_t stream)
{
    a.bounds.per = SHAPE::BM;
    a.across = (a.out_width + SHAPE::BN - 1) / SHAPE::BN;
    const unsigned blocks = workgroups<Tile<TYPE, SHAPE, false, TURNED>, PieceTable<false>>(a.bounds.n_slots, a.bounds.n_experts, SHAPE::BM, a.across);
    if constexpr (DIRECT)
        hipLaunchKernelGGL((product_stream_kernel<TYPE, RESULT, SHAPE, TURNED>), dim3(blocks), dim3(SHAPE::threads), 0, stream, a);
    else
        hipLaunchKernelGGL((product_kernel<TYPE, RESULT, SHAPE, TURNED>), dim3(blocks), dim3(SHAPE::threads), 0, stream, a);
}

template <int TYPE, int RESULT, int MF>
static void launch_few(const ProductArgs &a, hipStream_t stream)
{
    // Pieces of an expert that has more rows than most: four workgroups share them.
    const int64_t pieces = (a.bounds.n_slots + MF * 16 - 1) / (MF * 16);
    const dim3 grid((a.out_width + 15) / 16, a.bounds.n_experts + 1, (unsigned)(pieces < 4 ? pieces : 4));
    hipLaunchKernelGGL((product_few_kernel<TYPE, RESULT, MF>), grid, dim3(kFewWaves * 64), 0, stream, a);
}

// Whether rows can be loaded straight into LDS: 16-byte chunks that are aligned and whole, and a tile's rows within 2^31 bytes.
static bool streams(const void *p, int64_t stride, int64_t step, int64_t width)
{
    return aligned_to(p, 16) && stride % 16 == 0 && step % 16 == 0 && width % 16 == 0 && stride < ((int64_t)1 << 23);
}

template <int TYPE, int RESULT, bool TURNED>
static void launch_product(ProductArgs a, hipStream_t stream)
{
    constexpr int size = Unit16<TYPE>::size;
    const bool direct = streams(a.x, a.x_stride, 0, (int64_t)a.in_width * size) &&
                        streams(a.w, a.w_stride, a.w_step, (int64_t)(TURNED ? a.out_width : a.in_width) * size);
    // Few rows: sixteen columns a workgroup get all compute units to work, and their sums are short, but each reads its expert's rows.
    // us, tiles and this: 30 of 164 x 256 fp32, 64 rows an expert 19.0 and 7.7, 192 19.6 and 15.1; one of 1024 x 1024 bf16,
    // 1 row 15.1 and 7.7, 192 27.9 and 12.1; eight of 4096 x 4096, 1 row each 47 and 30, 8 rows 62 and 54, 16 rows 63 and 69; 64 of
    // 2048 x 1024, 1 row each 28.7 and 29.2, 4 rows 42 and 59.  Of 16 and 8 bits only where sums are long, for a tile takes as long as its sum and this
    // as there are parts: 64 of 1024 to 64, 32 rows each, 256 parts bf16 14.7 and 7.4; 64 of 64 to 1024, 64 rows each, 4096 parts 8.0 and
    // 15.9, int8 8.5 and 21.
    const int64_t met = a.bounds.n_slots < a.bounds.n_experts ? a.bounds.n_slots : a.bounds.n_experts;      // experts, at most
    const int64_t pieces = a.bounds.n_slots / 64 > met ? a.bounds.n_slots / 64 : met;                       // of 64 slots, about
    if constexpr (!TURNED) {
        const int64_t mean = (a.bounds.n_slots + a.bounds.n_experts - 1) / a.bounds.n_experts, row = (int64_t)a.in_width * size;
        const int64_t wide = (a.out_width + 127) / 128, again = (int64_t)a.bounds.n_slots * ((a.out_width + 15) / 16) * row;      // bytes of rows
        const int64_t parts = pieces * ((a.out_width + 15) / 16);
        const bool little = met * a.out_width * row <= (32 << 20) && mean <= 192 && again <= (TYPE == kI8 ? 32 << 20 : 64 << 20);
        const bool alone = (a.bounds.n_slots / 128 + met) * wide <= 64 && mean <= 256 && again <= (128 << 20);
        if ((TYPE == FS_F32 || parts <= row) && (little || alone || (mean <= 8 && met * wide <= kUnits)))
            return mean <= 16 ? launch_few<TYPE, RESULT, 1>(a, stream) : mean <= 32 ? launch_few<TYPE, RESULT, 2>(a, stream) : launch_few<TYPE, RESULT, 4>(a, stream);
    }
    // fp32 is bound by the matrix units whatever the tile, and small ones leave less idle at the edges and the end.
    const bool small = TYPE == FS_F32 || a.out_width <= 64;
    if constexpr (TYPE != FS_F32) {
        // Tiles of 128 x 128 where the card makes all of them at once, two a compute unit: us, of 128 and of 256, in 4096 to out columns
        // bf16: 2048 slots of 8 experts to 1024 48 and 84, to 4096 94 and 125; 4096 slots of 4 to 2048 64 and 88, to 4096 131 and 103.
        const bool at_once = (int64_t)(a.bounds.n_slots / 128) * ((a.out_width + 127) / 128) <= 2 * kUnits;
        if (direct && a.out_width > 128 && a.bounds.n_slots / a.bounds.n_experts >= 192 && !at_once)
            return launch_tiles<TYPE, RESULT, TURNED, Wide, true>(a, stream);
        // Tiles of 64 x 64 in the same case: alone on a compute unit a tile takes the time that its operands take to get there.  us, of 128
        // and of 64, 1024 columns to out bf16: 1000 slots of one expert to 1024 16.4 and 11.7, to 2048 17.1 and 14.7; 2048 slots of 8 to 2048,
        // 1024 tiles, 17.8 and 24.2.
        if (direct && pieces * ((a.out_width + 63) / 64) <= 2 * kUnits)
            return launch_tiles<TYPE, RESULT, TURNED, Little, true>(a, stream);
        if (!small)
            return direct ? launch_tiles<TYPE, RESULT, TURNED, Middle, true>(a, stream) : launch_tiles<TYPE, RESULT, TURNED, Middle, false>(a, stream);
    }
    direct ? launch_tiles<TYPE, RESULT, TURNED, Small, true>(a, stream) : launch_tiles<TYPE, RESULT, TURNED, Small, false>(a, stream);
}

// The shapes of weights' gradients, and how many slots a workgroup adds up: no more than a workgroup's share of all of them, so that the
// longest experts end no later than the others; and 32 768 at most, as a piece is one sum in fp32, whatever the share is, and pieces meet in 64 bits.
enum { kSmall, kMiddle, kWide };
static int shape_of_weights(int32_t type, int64_t n_experts, int64_t in_width, int64_t out_width)
{
    if (type == FS_F32 || in_width <= 64 || out_width <= 64)
        return kSmall;
    return in_width > 128 && out_width > 128 && in_width * out_width * n_experts >= ((int64_t)1 << 24) ? kWide : kMiddle;
}
template <class SHAPE>
static int64_t tiles_of_weights(int64_t in_width, int64_t out_width)
{
    return (in_width + SHAPE::BN - 1) / SHAPE::BN * ((out_width + SHAPE::BM - 1) / SHAPE::BM);
}
static int piece_of_weights(int64_t n_slots, int32_t type, int32_t n_experts, int64_t in_width, int64_t out_width)
{
    const int shape = shape_of_weights(type, n_experts, in_width, out_width);
    const int64_t work = n_slots * (shape == kWide     ? tiles_of_weights<Wide>(in_width, out_width)
                                    : shape == kMiddle ? tiles_of_weights<Middle>(in_width, out_width)
                                                       : tiles_of_weights<SmallAcross>(in_width, out_width));
    const int64_t per = work / (shape == kWide ? kUnits : shape == kMiddle ? 2 * kUnits : 4 * kUnits);
    return (int)(((per < 512 ? 512 : per > 32768 ? 32768 : per) + 255) / 256 * 256);
}

template <int TYPE, class SHAPE, bool DIRECT>
static void launch_weights(WeightsArgs a, hipStream_t stream)
{
    a.across = (a.in_width + SHAPE::BN - 1) / SHAPE::BN;
    a.tiles = (int32_t)tiles_of_weights<SHAPE>(a.in_width, a.out_width);
    const unsigned blocks = workgroups<Tile<TYPE, SHAPE, true, true>, PieceTable<true>>(a.bounds.n_slots, a.bounds.n_experts, a.bounds.per, a.tiles);
    hipLaunchKernelGGL((weights_kernel<TYPE, SHAPE, DIRECT>), dim3(blocks), dim3(SHAPE::threads), 0, stream, a);
}

static int check_shape(const char *who, int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width)
{
    if (n_slots < 0 || n_slots >= ((int64_t)1 << 31))
        return fail(FS_EINVAL, "%s: %lld slots: 0 to 2^31 - 1 are taken", who, (long long)n_slots);
    FS_TRY(check_experts(who, n_experts));
    FS_TRY(check_width(who, in_width));
    FS_TRY(check_width(who, out_width));
    // Tiles are counted in 32 bits: more of them, of 128 x 64 results, would be more than the card holds.
    const int64_t in_tiles = ((int64_t)in_width + 63) / 64, out_tiles = ((int64_t)out_width + 63) / 64;
    const int64_t rows = n_slots / 128 + n_experts, wide = in_tiles > out_tiles ? in_tiles : out_tiles;
    if (rows > INT32_MAX / wide || (n_slots / 512 + n_experts) > INT32_MAX / ((in_tiles * out_tiles + 1) / 2))
        return fail(FS_EUNSUPPORTED, "%s: %lld slots of %d experts, %d to %d columns", who, (long long)n_slots, n_experts, in_width, out_width);
    return FS_OK;
}
// n_experts matrices, `step` apart.
static int check_matrices(const char *who, const char *what, const void *p, int64_t rows, int64_t width, int32_t type, int64_t stride, int64_t step,
                          int64_t least_step)
{
    FS_TRY(check_matrix(who, what, p, rows, width, type, stride));
    if (step < least_step || step > ((int64_t)1 << 50))
        return fail(FS_EINVAL, "%s: %lld elements from matrix to matrix of %s, %lld at least and 2^50 at most are taken", who, (long long)step, what,
                    (long long)least_step);
    return FS_OK;
}
static int check_result(const char *who, const char *what, int32_t result, int32_t type)
{
    if (result != type && result != FS_F32)
        return fail(FS_EINVAL, "%s: %s is of another type (%d) than the operands (%d) or fp32", who, what, result, type);
    return FS_OK;
}

}  // namespace fs

using namespace fs;

extern "C" int fs_expert_matmul(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, const void *x, int32_t type,
                                int64_t x_stride, const int32_t *first, const void *w, int64_t w_stride, int64_t w_step, int32_t turned,
                                void *y, int32_t y_type, int64_t y_stride, void *stream_)
{
    static const char who[] = "fs_expert_matmul";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_shape(who, n_slots, n_experts, in_width, out_width));
    FS_TRY(check_matrix(who, "x", x, n_slots, in_width, type, x_stride));
    FS_TRY(check_array(who, "first", first, n_slots, 4));
    if (turned != 0 && turned != 1)
        return fail(FS_EINVAL, "%s: turned %d is neither 0 nor 1", who, turned);
    FS_TRY(check_matrices(who, "w", w, n_slots, turned ? out_width : in_width, type, w_stride, w_step, 0));
    FS_TRY(check_matrix(who, "y", y, n_slots, out_width, y_type, y_stride));
    FS_TRY(check_result(who, "y", y_type, type));
    if (n_slots == 0)
        return FS_OK;
    const int64_t b = (int64_t)type_bytes(type);
    ProductArgs a = {{first, n_experts, (int)n_slots, 0}, (const char *)x, (const char *)w, x_stride * b, w_stride * b, w_step * b, y, y_stride, y_type,
                     in_width, out_width, 0, nullptr, nullptr};
    prof_start(kKernPack, stream);
    with_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (turned)
            launch_product<T, T, true>(a, stream);
        else
            launch_product<T, T, false>(a, stream);
    });
    prof_stop(stream);
    return launched("expert product kernel launch");
}

extern "C" int fs_expert_matmul_i8(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, const int8_t *q, int64_t q_stride,
                                   const float *scale, const int32_t *first, const int8_t *w, int64_t w_stride, int64_t w_step,
                                   const float *w_scale, void *y, int32_t y_type, int64_t y_stride, void *stream_)
{
    static const char who[] = "fs_expert_matmul_i8";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_shape(who, n_slots, n_experts, in_width, out_width));
    if (in_width > FS_MAX_I8_WIDTH)
        return fail(FS_EUNSUPPORTED, "%s: width %d of a sum in 32 bits, %d at most", who, in_width, FS_MAX_I8_WIDTH);
    FS_TRY(check_bytes(who, "q", q, n_slots, in_width, q_stride));
    FS_TRY(check_array(who, "scale", scale, n_slots, 4));
    FS_TRY(check_array(who, "first", first, n_slots, 4));
    FS_TRY(check_bytes(who, "w", w, n_slots, in_width, w_stride));
    if (w_step < 0 || w_step > ((int64_t)1 << 50))
        return fail(FS_EINVAL, "%s: %lld bytes from matrix to matrix of w", who, (long long)w_step);
    FS_TRY(check_array(who, "w_scale", w_scale, n_slots, 4));
    FS_TRY(check_matrix(who, "y", y, n_slots, out_width, y_type, y_stride));
    if (n_slots == 0)
        return FS_OK;
    ProductArgs a = {{first, n_experts, (int)n_slots, 0}, (const char *)q, (const char *)w, q_stride, w_stride, w_step, y, y_stride, y_type,
                     in_width, out_width, 0, scale, w_scale};
    prof_start(kKernPack, stream);
    with_type(y_type, [&](auto t) { launch_product<kI8, decltype(t)::value, false>(a, stream); });
    prof_stop(stream);
    return launched("expert product kernel launch");
}

extern "C" size_t fs_expert_matmul_backward_workspace_bytes(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, int32_t type)
{
    static const char who[] = "fs_expert_matmul_backward_workspace_bytes";
    if (check_shape(who, n_slots, n_experts, in_width, out_width) != FS_OK)
        return 0;
    if (!type_ok(type)) {
        fail(FS_EINVAL, "%s: unknown element type %d", who, type);
        return 0;
    }
    const int64_t per = piece_of_weights(n_slots, type, n_experts, in_width, out_width);
    if (n_slots <= per)
        return 0;
    // An expert of n > per slots has at most n / per + 1 < 2 n / per pieces.
    return (size_t)(2 * (n_slots / per + 1)) * in_width * out_width * 4;
}

extern "C" int fs_expert_matmul_backward(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, const void *d_y, int32_t type,
                                         int64_t d_y_stride, const void *x, int64_t x_stride, const int32_t *first, int32_t accumulate,
                                         void *d_w, int32_t d_w_type, int64_t d_w_stride, int64_t d_w_step, void *work, size_t work_bytes,
                                         void *stream_)
{
    static const char who[] = "fs_expert_matmul_backward";
    hipStream_t stream = (hipStream_t)stream_;
    FS_TRY(check_shape(who, n_slots, n_experts, in_width, out_width));
    FS_TRY(check_matrix(who, "d_y", d_y, n_slots, out_width, type, d_y_stride));
    FS_TRY(check_matrix(who, "x", x, n_slots, in_width, type, x_stride));
    FS_TRY(check_array(who, "first", first, 1, 4));
    if (accumulate != 0 && accumulate != 1)
        return fail(FS_EINVAL, "%s: accumulate %d is neither 0 nor 1", who, accumulate);
    FS_TRY(check_matrices(who, "d_w", d_w, 1, in_width, d_w_type, d_w_stride, d_w_step, n_experts > 1 ? d_w_stride * out_width : 0));
    FS_TRY(check_result(who, "d_w", d_w_type, type));
    const size_t need = fs_expert_matmul_backward_workspace_bytes(n_slots, n_experts, in_width, out_width, type);
    FS_TRY(check_array(who, "work", work, (int64_t)need, 256));
    if (work_bytes < need)
        return fail(FS_EINVAL, "%s: %zu bytes of working memory, %zu are needed", who, work_bytes, need);
    const int64_t b = (int64_t)type_bytes(type);
    WeightsArgs a = {{first, n_experts, (int)n_slots, piece_of_weights(n_slots, type, n_experts, in_width, out_width)}, (const char *)d_y, (const char *)x,
                     d_y_stride * b, x_stride * b, d_w, d_w_stride, d_w_step, d_w_type, in_width, out_width, 0, 0, accumulate, (float *)work};
    const bool direct = streams(d_y, a.g_stride, 0, out_width * b) && streams(x, a.x_stride, 0, in_width * b);
    prof_start(kKernTrainOther, stream);
    with_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        const int shape = shape_of_weights(type, n_experts, in_width, out_width);
        if constexpr (T != FS_F32) {
            if (shape == kWide && direct)
                launch_weights<T, WideAcross, true>(a, stream);
            else if (shape != kSmall)
                direct ? launch_weights<T, Middle, true>(a, stream) : launch_weights<T, Middle, false>(a, stream);
        }
        if (shape == kSmall)
            direct ? launch_weights<T, SmallAcross, true>(a, stream) : launch_weights<T, SmallAcross, false>(a, stream);
        if (need) {
            const int64_t wanted = ((int64_t)out_width + 3) / 4, most = 8192 / n_experts + 1;
            a.tiles = (int32_t)(wanted < most ? wanted : most);
            hipLaunchKernelGGL(weights_join_kernel<T>, dim3((unsigned)(a.tiles * n_experts)), dim3(256), 0, stream, a);
        }
    });
    prof_stop(stream);
    return launched("expert weights' gradient kernel launch");
}
