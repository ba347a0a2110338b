// Embedding: tokens, or bags of tokens, to scaled sums of a table's rows, and the table's gradient by sorted tokens.
//
// The gradient of a table's row is the sum over the places that named it.  The (token, row) pairs are sorted by token,
// stably, a digit at a time; then the sorted list is cut in chunks, and the lanes that hold a row add a chunk's rows run by run.
// A run inside a chunk is a finished row of the table; what a workgroup's chunks have of a run that goes on beyond them is a
// partial sum, two a workgroup at most, and a last kernel joins them.  The order of additions depends on the ids alone.
#include "fs_slots.h"

#include <math.h>
#include <type_traits>

namespace fs {

constexpr int kEmbedWaves = 4;            // of a workgroup
constexpr int kEmbedAhead = 8;            // rows on their way at once
constexpr int kEmbedFewWaves = 2048;
constexpr int kEmbedMostFp32 = 256;       // rows of a bag that are added in fp32 one after the other
constexpr int kLookupRows = 4;            // rows of a lane
constexpr int kSumMostWaves = 4096;
constexpr int kSumMostChunk = 256, kSumLeastChunk = 8;    // pairs a chunk
constexpr int kSumWaves = 8;              // of a workgroup
constexpr int kJoinAhead = 16;            // partial sums on their way at once
// Ids that need no sorting.  79 of a 3891 x 11 table: 16.2 us sorted, 11.1 so (8.5 of which any call takes).  Past this
// number, one token in all places would cost its one wavefront more than sorting does.
constexpr int kDirectIds = 256;
constexpr int kDirectWaves = 4, kDirectRows = 8192;       // rows of the table that a workgroup clears, at most
constexpr int kBlockSlots = 16;           // a wavefront's sums, where one row takes all its lanes

template <int ID> struct IdOf;
template <> struct IdOf<FS_ID_I32> { typedef int32_t type; };
template <> struct IdOf<FS_ID_I64> { typedef int64_t type; };
template <> struct IdOf<FS_ID_U16> { typedef uint16_t type; };
template <class F>
void with_id_type(int32_t type, F f)
{
    if (type == FS_ID_I32)
        f(TypeTag<FS_ID_I32>());
    else if (type == FS_ID_I64)
        f(TypeTag<FS_ID_I64>());
    else
        f(TypeTag<FS_ID_U16>());
}

struct EmbedIds {
    const void *ids;
    const int32_t *col_base;
    int32_t n_cols, n_vocab;
    uint32_t magic, shift;       // i / n_cols = (i * magic >> 32) >> shift for i < 2^31, n_cols > 1
    // The table's rows that N entries name, or -1.  All ids are on their way before the first is looked at.
    template <int ID, int N, class Entry, class Column>
    __device__ __forceinline__ void rows(int (&row)[N], Entry entry, Column column) const
    {
        typename IdOf<ID>::type id[N];
        int32_t base[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            id[u] = ((const typename IdOf<ID>::type *)ids)[entry(u)];
            base[u] = 0;
        }
        if (col_base)
#pragma unroll
            for (int u = 0; u < N; ++u)
                base[u] = col_base[column(u)];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if constexpr (ID == FS_ID_I64) {       // id + base in [0, n_vocab), without a sum that 64 bits might not hold
                const int64_t v = id[u], least = -(int64_t)base[u];
                row[u] = v >= least && v < least + n_vocab ? (int)(v - least) : -1;
            } else {
                const int64_t v = (int64_t)(int32_t)id[u] + base[u];
                row[u] = v >= 0 && v < n_vocab ? (int)v : -1;
            }
        }
    }
    __device__ __forceinline__ uint32_t row_of(uint32_t i) const { return n_cols == 1 ? i : __umulhi(i, magic) >> shift; }
};
// n_cols = d > 1, s the bits of d - 1: magic = floor(2^(31 + s) / d) + 1 is i / d times 2^(31 + s) with an error that stays below
// 1 / d for i < 2^31.
static EmbedIds embed_ids(const void *ids, const int32_t *col_base, int32_t n_cols, int32_t n_vocab)
{
    EmbedIds e = {ids, col_base, n_cols, n_vocab, 0, 0};
    if (n_cols > 1) {
        const int s = bits_of(n_cols);
        e.magic = (uint32_t)((((uint64_t)1 << (31 + s)) / (uint32_t)n_cols) + 1);
        e.shift = (uint32_t)(s - 1);
    }
    return e;
}

struct EmbedArgs {
    EmbedIds ids;
    const void *in;            // the table
    int64_t in_stride, out_stride, n_rows;
    int32_t width, ll, split;  // a row of the result in 1 << (ll + split) lanes, the bag in 1 << split parts;
    int32_t columns;           // of a wide row, `columns` neighbouring wavefronts
    float scale;
    void *out;
    int64_t block0;            // of this launch
};

// The entries of a bag that a part of it takes: of the 1 << split parts, entries begin .. end - 1, `per` of them in all but the last.
// A bag has up to 2^31 - 1 entries, so that steps beyond its end need the 32nd bit; short ones are counted in int, which is quicker
// (320 bags of 100 rows 8.8 us, 8.9 unsigned).
template <class Count>
struct BagPart {
    Count per, begin, end;
};
template <class Count>
__host__ __device__ constexpr BagPart<Count> bag_part(Count cols, int split, Count part)
{
    const Count per = (cols + (Count)(1 << split) - 1) >> split;
    const Count begin = part * per < cols ? part * per : cols, end = begin + per < cols ? begin + per : cols;
    return BagPart<Count>{per, begin, end};
}
constexpr uint32_t kMostBag = 2147483647u;
static_assert(bag_part<uint32_t>(kMostBag, 0, 0).per == kMostBag && bag_part<uint32_t>(kMostBag, 0, 0).end == kMostBag && kMostBag + kEmbedAhead > kMostBag,
              "one part: all entries, and the step behind them is no smaller");
static_assert(bag_part<uint32_t>(kMostBag, 6, 63).end == kMostBag && bag_part<uint32_t>(kMostBag, 6, 63).begin == bag_part<uint32_t>(kMostBag, 6, 62).end &&
                  bag_part<uint32_t>(kMostBag - 62, 6, 63).end == kMostBag - 62 && bag_part<uint32_t>(65, 6, 63).begin == 65,
              "64 parts: they meet, and the last ends with the bag");

// Bags.  A row of the result in neighbouring lanes, eight rows of the table on their way at once; bags of few rows are split over
// lanes.  320 bags of 100 rows of 64 fp32: 9 us, three rounds of dependent loads and the launch.  LONG: a lane has more than
// kEmbedMostFp32 of a bag's rows; sums of so many are added in 64 bits, so that what is lost does not grow with the bag.
template <int IN, int OUT, int ID, bool LONG>
__global__ void __launch_bounds__(kEmbedWaves * 64)
embed_kernel(EmbedArgs a)
{
    typedef typename Element<IN>::type In;
    typedef typename Element<OUT>::type Out;
    constexpr int N = kChunk<In>;
    const int lane = threadIdx.x & 63, ll = a.ll, h = lane & ((1 << ll) - 1), part = (lane >> ll) & ((1 << a.split) - 1);
    const int64_t wave = (a.block0 + blockIdx.x) * kEmbedWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = a.columns == 1 ? wave << (6 - ll - a.split) : wave / a.columns;
    if (row0 >= a.n_rows)
        return;
    const bool there = row0 + (lane >> (ll + a.split)) < a.n_rows;
    const int64_t row = there ? row0 + (lane >> (ll + a.split)) : a.n_rows - 1;
    const Span at = span_of<N>(((a.columns == 1 ? 0 : (int)(wave % a.columns)) * 64 + h) * N, a.width);
    const int c = at.c, n = at.n;
    typedef typename std::conditional<LONG, uint32_t, int>::type Count;
    const Count cols = (Count)a.ids.n_cols;
    const BagPart<Count> of = bag_part<Count>(cols, a.split, (Count)part);
    const Count per = of.per, begin = of.begin, end = of.end;
    const In *const in = (const In *)a.in + c;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        sum[i] = 0.0f;
    double all[N] = {};
    for (Count j0 = 0; j0 < per; j0 += kEmbedAhead) {     // the same number of times in all lanes
        int v[kEmbedAhead];
        if (ll >= 3) {                                       // eight lanes fetch an id each
            int id[1];
            const Count j = min(begin + j0 + (Count)(h & 7), cols - 1);
            a.ids.template rows<ID>(id, [&](int) { return row * cols + j; }, [&](int) { return j; });
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u)
                v[u] = __shfl(id[0], (lane & ~7) + u);
        } else {
            const auto j = [&](int u) { return min(begin + j0 + (Count)u, cols - 1); };
            a.ids.template rows<ID>(v, [&](int u) { return row * cols + j(u); }, j);
        }
#pragma unroll
        for (int u = 0; u < kEmbedAhead; ++u)
            v[u] = begin + j0 + (Count)u < end ? v[u] : -1;
        RawChunk<In> x[kEmbedAhead];
#pragma unroll
        for (int u = 0; u < kEmbedAhead; ++u)
            x[u].load(in + (int64_t)max(v[u], 0) * a.in_stride, v[u] >= 0 ? n : 0);
#pragma unroll
        for (int u = 0; u < kEmbedAhead; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i)
                sum[i] += x[u][i];
        if (LONG && (j0 + kEmbedAhead) % kEmbedMostFp32 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                all[i] += (double)sum[i];
                sum[i] = 0.0f;
            }
    }
    if (LONG)
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[i] = (float)(all[i] + (double)sum[i]);
    for (int s = 0; s < a.split; ++s)
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[i] += __shfl_xor(sum[i], 1 << (ll + s));
    if (!there || part != 0)
        return;
#pragma unroll
    for (int i = 0; i < N; ++i)
        sum[i] *= a.scale;
    store_chunk<N>((Out *)a.out + row * a.out_stride + c, n, sum);
}

// One id a row: kLookupRows of them a lane.  131 072 rows of 1024 bf16 from a table of 65 536: 57 us, 268 MB written and 119 read,
// 6.8 TB/s, what filling memory reaches.
template <int IN, int OUT, int ID, bool PAST>
__global__ void __launch_bounds__(kEmbedWaves * 64)
embed_lookup_kernel(EmbedArgs a)
{
    typedef typename Element<IN>::type In;
    typedef typename Element<OUT>::type Out;
    constexpr int N = kChunk<In>;
    const int lane = threadIdx.x & 63, ll = a.ll, h = lane & ((1 << ll) - 1);
    const int64_t wave = (a.block0 + blockIdx.x) * kEmbedWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = ((a.columns == 1 ? wave : wave / a.columns) * kLookupRows) << (6 - ll);
    if (row0 >= a.n_rows)
        return;
    const Span at = span_of<N>(((a.columns == 1 ? 0 : (int)(wave % a.columns)) * 64 + h) * N, a.width);
    const int c = at.c, n = at.n;
    const In *const in = (const In *)a.in + c;
    const auto row = [&](int u) { return row0 + (u << (6 - ll)) + (lane >> ll); };
    int v[kLookupRows];
    a.ids.template rows<ID>(v, [&](int u) { return min(row(u), a.n_rows - 1); }, [](int) { return 0; });
    RawChunk<In> x[kLookupRows];
#pragma unroll
    for (int u = 0; u < kLookupRows; ++u)
        x[u].load(in + (int64_t)max(v[u], 0) * a.in_stride, v[u] >= 0 ? n : 0);
#pragma unroll
    for (int u = 0; u < kLookupRows; ++u) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            y[i] = x[u][i] * a.scale;
        store_chunk<N, PAST>((Out *)a.out + row(u) * a.out_stride + c, row(u) < a.n_rows ? n : 0, y);
    }
}

// ---- sorting by token, the lowest digit first: the first pass takes ids, the others what the pass before left ------------

// A token and the row that named it, in 32 bits where both fit, which halves what sorting moves.
struct Pair {
    int32_t token, row;
};
struct Packing {
    int32_t row_bits;              // of a packed pair's
    int32_t token_bits;            // of a token's: those above are the band's
    uint32_t band_magic;           // a row's band: the high word of row * band_magic
};
template <class P> __device__ __forceinline__ P make_pair(const Packing &k, int token, uint32_t row);
template <> __device__ __forceinline__ Pair make_pair<Pair>(const Packing &, int token, uint32_t row) { return Pair{token, (int32_t)row}; }
template <> __device__ __forceinline__ uint32_t make_pair<uint32_t>(const Packing &k, int token, uint32_t row) { return (uint32_t)token << k.row_bits | row; }
__device__ __forceinline__ int token_of(const Packing &, const Pair &p) { return p.token; }
__device__ __forceinline__ int token_of(const Packing &k, uint32_t p) { return (int)(p >> k.row_bits); }
__device__ __forceinline__ uint32_t row_of(const Packing &, const Pair &p) { return (uint32_t)p.row; }
__device__ __forceinline__ uint32_t row_of(const Packing &k, uint32_t p) { return p & ((1u << k.row_bits) - 1u); }

// Bands: see bands_for.  From here on a token is the token in its row's band.
__device__ __forceinline__ int banded(const Packing &k, int token, uint32_t row) { return token | (int)(__umulhi(row, k.band_magic) << k.token_bits); }
__device__ __forceinline__ int plain_token(const Packing &k, int token) { return token & (int)((1u << k.token_bits) - 1u); }

struct ClearArgs {
    void *table;
    int64_t n_rows, stride;
    int32_t type, width, ll;
};
template <class T>
__device__ __forceinline__ void clear_row(const ClearArgs &a, int64_t row, int h)
{
    constexpr int N = kChunk<T>;
    RawChunk<T> zero;
    zero.clear();
    for (int c0 = h * N; c0 < a.width; c0 += 64 * N) {
        const Span at = span_of<N>(c0, a.width);
        zero.store((T *)a.table + row * a.stride + at.c, at.n);
    }
}
// Rows that nobody names are 0: what block b of `blocks` clears.
template <class T>
__device__ __forceinline__ void clear_rows(const ClearArgs &a, int64_t b, int64_t blocks)
{
    const int lane = threadIdx.x & 63, h = lane & ((1 << a.ll) - 1), waves = blockDim.x >> 6;
    for (int64_t r = ((b * waves + (threadIdx.x >> 6)) << (6 - a.ll)) + (lane >> a.ll); r < a.n_rows; r += (blocks * waves) << (6 - a.ll))
        clear_row<T>(a, r, h);
}
__device__ __forceinline__ void clear_table(const ClearArgs &a, int64_t b, int64_t blocks)
{
    if (a.type == FS_F32)
        clear_rows<float>(a, b, blocks);
    else                           // the zeros of bf16 and fp16 are the same
        clear_rows<_Float16>(a, b, blocks);
}
// A pass of the sort clears two parts of the table.
struct ClearBeside {
    ClearArgs counting, placing;
    int32_t count_blocks, place_blocks;
    int more_counting() const { return count_blocks; }
    int more_placing() const { return place_blocks; }
    __device__ __forceinline__ void beside_count(int block, int blocks) const { clear_table(counting, block, blocks); }
    __device__ __forceinline__ void beside_place(int block, int blocks) const { clear_table(placing, block, blocks); }
};

template <int ID, class P>
struct IdDigit : ClearBeside {
    typedef P Item, What;
    EmbedIds ids;
    P *to;
    int32_t mask;
    Packing packing;
    template <int N>
    __device__ __forceinline__ void load(P (&item)[N], int64_t i, int64_t end) const
    {
        int token[N];
        const auto entry = [&](int u) { return (uint32_t)min(i + u * 64, end - 1); };
        ids.template rows<ID>(token, entry, [&](int u) { return entry(u) - ids.row_of(entry(u)) * (uint32_t)ids.n_cols; });
#pragma unroll
        for (int u = 0; u < N; ++u)
            item[u] = make_pair<P>(packing, banded(packing, token[u] < 0 ? ids.n_vocab : token[u], ids.row_of(entry(u))), ids.row_of(entry(u)));
    }
    __device__ __forceinline__ int number(const P &p) const { return token_of(packing, p) & mask; }
    __device__ __forceinline__ void start(int, int) const {}
    __device__ __forceinline__ void place(int64_t, int, int) const {}
    __device__ __forceinline__ P what(const P &p, int64_t) const { return p; }
    __device__ __forceinline__ void put(const P &p, int, int slot) const { to[slot] = p; }
};
template <class P>
struct PairDigit : ClearBeside {
    typedef P Item, What;
    const P *from;
    P *to;
    int32_t shift, mask;
    Packing packing;
    template <int N>
    __device__ __forceinline__ void load(P (&item)[N], int64_t i, int64_t end) const
    {
#pragma unroll
        for (int u = 0; u < N; ++u)
            item[u] = from[min(i + u * 64, end - 1)];
    }
    __device__ __forceinline__ int number(const P &p) const { return (token_of(packing, p) >> shift) & mask; }
    __device__ __forceinline__ void start(int, int) const {}
    __device__ __forceinline__ void place(int64_t, int, int) const {}
    __device__ __forceinline__ P what(const P &p, int64_t) const { return p; }
    __device__ __forceinline__ void put(const P &p, int, int slot) const { to[slot] = p; }
};

static __global__ void __launch_bounds__(kSlotThreads)
embed_clear_kernel(ClearArgs a) { clear_table(a, blockIdx.x, gridDim.x); }
constexpr int kClearBlocks = 2047;

// All digits of up to PER * 1024 entries in one workgroup.  LDS holds the tokens where the entries are and the entries' numbers
// in the order so far, which a pass takes to registers and puts back.  The launch's other workgroups clear the table meanwhile.
constexpr int kFewDigitBits = 9;
// 8192 entries 21 us, 16384 37, and 29 by the six kernels of a long list; but where there is much to clear, it is better cleared beside
// one kernel than in four parts beside the others.  Whole gradients of 1024 bf16, one kernel and six, us: 9000 ids and 16 MB of
// table 35 and 38, 64 MB 41 and 51, 130 MB 42 and 65, 400 MB 92 and 101; 16384 ids and 16 MB 44 and 39, 64 MB 51 and 54, 130 MB 54
// and 68, 400 MB 93 and 105.
constexpr int kEmbedFew = 8192;
constexpr int64_t kClearLong = 64000000;
static bool sort_in_one(int64_t n, int64_t clear_bytes) { return n <= kEmbedFew || (n <= 2 * kEmbedFew && clear_bytes >= kClearLong); }
template <int ID, class P, int PER>
__global__ void __launch_bounds__(kSlotFewWaves * 64)
embed_sort_few_kernel(IdDigit<ID, P> source, int32_t n, int32_t bits)
{
    if (blockIdx.x > 0) {
        source.beside_count(blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    __shared__ int32_t token[PER * 1024], c[kSlotFewWaves << kFewDigitBits], wave_total[kSlotFewWaves];
    __shared__ uint16_t order[PER * 1024];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int steps = (n + kSlotFewWaves * 64 - 1) / (kSlotFewWaves * 64);
    const int begin = wave * steps * 64 + lane;
    P item[PER];
    source.load(item, begin, n);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = begin + u * 64;
        if (u < steps && i < n) {
            token[i] = token_of(source.packing, item[u]);
            order[i] = (uint16_t)i;
        }
    }
    const int passes = (bits + kFewDigitBits - 1) / kFewDigitBits, digit = (bits + passes - 1) / passes, buckets = 1 << digit;
    for (int shift = 0; shift < bits; shift += digit) {
        for (int b = threadIdx.x; b < kSlotFewWaves * buckets; b += kSlotFewWaves * 64)
            c[b] = 0;
        __syncthreads();
        uint16_t mine[PER];
        int number[PER];
#pragma unroll
        for (int u = 0; u < PER; ++u)
            if (u < steps && begin + u * 64 < n) {
                mine[u] = order[begin + u * 64];
                number[u] = (token[mine[u]] >> shift) & (buckets - 1);
                atomicAdd(&c[wave * buckets + number[u]], 1);
            }
        __syncthreads();
        first_slots(c, buckets, wave_total, [](int, int) {});
#pragma unroll
        for (int u = 0; u < PER; ++u)
            if (u < steps) {
                const bool there = begin + u * 64 < n;
                const int slot = take_slot(c + wave * buckets, there ? number[u] : 0, digit, there);
                if (there)
                    order[slot] = mine[u];
            }
        __syncthreads();
    }
    for (int s = threadIdx.x; s < n; s += kSlotFewWaves * 64) {
        const int i = order[s];
        source.to[s] = make_pair<P>(source.packing, token[i], source.ids.row_of((uint32_t)i));       // the token in its band, as it came
    }
}

// ---- sums of the runs -----------------------------------------------------------------------------------------------------

struct SumArgs {
    const void *list;              // pairs
    Packing packing;
    const void *in;
    int64_t in_stride, out_stride, n;
    int32_t width, ll, chunk, n_vocab, accumulate;
    float scale;
    void *out;
    uint32_t *part_token;          // partial sums, two a workgroup: token * 2, + 1 where there is nothing to add
    float *part;
    int64_t part_stride;
    int32_t groups, bands;         // workgroups' stretches of the list
};
constexpr uint32_t kNoToken = 0xffffffffu;
constexpr int kXcds = 8;           // workgroups go round them
// The row of the result for a token: with bands, of a table for each.
__device__ __forceinline__ int64_t row_for(const SumArgs &a, int token)
{
    return (int64_t)(token >> a.packing.token_bits) * a.n_vocab + plain_token(a.packing, token);
}

// A whole row of the table.
template <class Out, int N>
__device__ __forceinline__ void put_row(const SumArgs &a, int token, int c, int n, const float (&sum)[N])
{
    Out *const out = (Out *)a.out + row_for(a, token) * a.out_stride + c;
    float had[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        had[i] = 0.0f;
    if (a.accumulate)
        load_chunk<N>(out, n, had);
#pragma unroll
    for (int i = 0; i < N; ++i)
        had[i] += sum[i] * a.scale;
    store_chunk<N>(out, n, had);
}

// A chunk of the list is added by the lanes of one row, in fp32.  What a workgroup's chunks have of runs that go on beyond
// them, two sums a chunk at most, meets in LDS, where the lanes of a run's first sum add them up, in 64 bits (blocks of sixteen
// are rounded between); what the workgroup has of runs that go on beyond it goes to memory.
//
// 32 768 rows of 256 bytes, each named by 100 tokens: 52 us, 839 MB of rows at 16 TB/s, nearly all from the L2 caches, with 14 vector
// instructions beside every four rows (vector units 52 % busy); the sort in front of it 67 us, of which the chains of 3.3 M
// entries' ballots and LDS steps are 42 (51 and 57 % busy while placing).
template <int IN, int OUT, class P, bool NEAR>
__global__ void __launch_bounds__(kSumWaves * 64)
embed_sum_kernel(SumArgs a)
{
    typedef typename Element<IN>::type In;
    typedef typename Element<OUT>::type Out;
    constexpr int N = kChunk<In>;
    __shared__ uint32_t slot_token[2 * kSumWaves * 64];
    __shared__ float slot_sum[2 * kSumWaves * 64 * N];
    __shared__ uint32_t whole[2 * kSumWaves * 64 / kBlockSlots];
    const int lane = threadIdx.x & 63, ll = a.ll, h = lane & ((1 << ll) - 1);
    const int units = kSumWaves << (6 - ll), unit = ((threadIdx.x >> 6) << (6 - ll)) + (lane >> ll), slots = 2 * units;
    // With bands, an XCD takes stretches of one of them.
    int64_t group = blockIdx.x;
    if (a.bands > 1) {
        const int xcd = blockIdx.x % kXcds, per = kXcds / a.bands, each = (a.groups + a.bands - 1) / a.bands;
        const int in_band = blockIdx.x / kXcds * per + xcd / a.bands;
        group = (int64_t)(xcd % a.bands) * each + in_band;
        if (in_band >= each || group >= a.groups)
            return;
    }
    const int64_t group_begin = group * units * a.chunk, group_end = min(group_begin + (int64_t)units * a.chunk, a.n);
    const int64_t begin = group_begin + (int64_t)unit * a.chunk, end = min(begin + a.chunk, a.n);
    const Span at = span_of<N>(((int)blockIdx.y * 64 + h) * N, a.width, !a.accumulate);
    const int c = at.c, n = at.n;
    const In *const in = (const In *)a.in + c;
    const P *const list = (const P *)a.list;
    // The tokens before and behind the group and the chunk, on their way together.
    const auto token_at = [&](int64_t i) { return token_of(a.packing, list[min(max(i, (int64_t)0), a.n - 1)]); };
    const int group_left = token_at(group_begin - 1), group_right = token_at(group_end);
    const int chunk_left = token_at(begin - 1), chunk_right = token_at(end), chunk_first = token_at(begin);
    const int group_before = group_begin > 0 ? group_left : -1, group_behind = group_end < a.n ? group_right : -1;
    if (begin < a.n) {
        const int before = begin > 0 ? chunk_left : -1, behind = end < a.n ? chunk_right : -1;
        float sum[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[i] = 0.0f;
        int now = chunk_first;
        bool first = true;
        const auto mark = [&](int which, bool partial) {
            if (h == 0)
                slot_token[2 * unit + which] = (uint32_t)now * 2u + (partial ? 0u : 1u);
            if (partial)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    slot_sum[(((2 * unit + which) << ll) + h) * N + i] = sum[i];
        };
        const auto done = [&](bool last) {                       // the run of `now` ends here, or the chunk does
            const bool left = first && before == now, right = last && behind == now, some = plain_token(a.packing, now) < a.n_vocab;
            if (!left && !right && some)
                put_row<Out>(a, now, c, n, sum);
            if (first)
                mark(0, (left || right) && some);
            if (last)
                mark(1, !first && right && some);
        };
        // NEAR: offsets from the rows' start fit in 32 bits, one multiplication instead of four.
        const auto row_at = [&](const P &p) {
            if constexpr (NEAR)
                return (const In *)((const char *)a.in + (row_of(a.packing, p) * (uint32_t)(a.in_stride * (int64_t)sizeof(In)) + (uint32_t)c * (uint32_t)sizeof(In)));
            else
                return in + (int64_t)row_of(a.packing, p) * a.in_stride;
        };
        const auto add = [&](const P (&pair)[kEmbedAhead], const RawChunk<In> (&x)[kEmbedAhead]) {
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u) {
                const int token = token_of(a.packing, pair[u]);
                if (token != now) {
                    done(false);
                    first = false;
                    now = token;
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        sum[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sum[i] += x[u][i];
            }
        };
        // Every pair's row is there, also one whose token names none of the table: its sum goes nowhere.
        int64_t i0 = begin;
        for (; i0 + kEmbedAhead <= end; i0 += kEmbedAhead) {
            P pair[kEmbedAhead];
            RawChunk<In> x[kEmbedAhead];
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u)
                pair[u] = list[i0 + u];
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u)
                x[u].load(row_at(pair[u]), n);
            add(pair, x);
        }
        if (i0 < end) {
            P pair[kEmbedAhead];
            RawChunk<In> x[kEmbedAhead];
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u)
                pair[u] = list[min(i0 + u, end - 1)];
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u)
                x[u].load(row_at(pair[u]), i0 + u < end ? n : 0);
            add(pair, x);
        }
        done(true);
    } else if (h == 0) {
        slot_token[2 * unit] = slot_token[2 * unit + 1] = kNoToken;
    }
    __syncthreads();
    // A long run's sums would be one lane's after the other: blocks of them that are all of one run become one sum first.
    if (unit % (kBlockSlots / 2) == 0) {
        const int s = 2 * unit;
        uint32_t met[kBlockSlots];
#pragma unroll
        for (int u = 0; u < kBlockSlots; ++u)
            met[u] = slot_token[s + u];
        bool same = met[0] != kNoToken;
#pragma unroll
        for (int u = 1; u < kBlockSlots; ++u)
            same = same && met[u] >> 1 == met[0] >> 1;
        if (same) {
            double all[N];
#pragma unroll
            for (int i = 0; i < N; ++i)
                all[i] = 0.0;
            bool some = false;
#pragma unroll
            for (int u = 0; u < kBlockSlots; ++u)
                if (!(met[u] & 1)) {
                    some = true;
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        all[i] += (double)slot_sum[(((s + u) << ll) + h) * N + i];
                }
#pragma unroll
            for (int i = 0; i < N; ++i)
                slot_sum[((s << ll) + h) * N + i] = (float)all[i];
            if (h == 0)
                slot_token[s] = (met[0] & ~1u) | (some ? 0u : 1u);
        }
        if (h == 0)
            whole[s / kBlockSlots] = same;
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        const int s = 2 * unit + which;
        const uint32_t token = slot_token[s] >> 1;
        if (s > 0 && slot_token[s - 1] >> 1 == token)
            continue;                                            // not a run's first sum
        if (token == kNoToken >> 1) {                            // the list has ended: from here on nobody's
            if (h == 0 && blockIdx.y == 0)
                a.part_token[2 * group + 1] = kNoToken;
            continue;
        }
        double all[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            all[i] = 0.0;
        bool some = false;
        int e = s;
        do {
            if (!(slot_token[e] & 1)) {
                some = true;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    all[i] += (double)slot_sum[((e << ll) + h) * N + i];
            }
            e += e % kBlockSlots == 0 && whole[e / kBlockSlots] ? kBlockSlots : 1;
        } while (e < slots && slot_token[e] >> 1 == token);
        const bool left = s == 0 && group_before == (int)token, right = e == slots && group_behind == (int)token;
        float sum[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[i] = (float)all[i];
        if (!left && !right && some)
            put_row<Out>(a, (int)token, c, n, sum);
        const auto mark = [&](int at, bool partial) {
            const int64_t slot = 2 * group + at;
            if (h == 0 && blockIdx.y == 0)
                a.part_token[slot] = token * 2u + (partial ? 0u : 1u);
            if (partial)
                store_chunk<N>(a.part + slot * a.part_stride + c, n, sum);
        };
        if (s == 0)
            mark(0, (left || right) && some);
        if (e == slots)
            mark(1, s != 0 && right && some);
    }
}

// The partial sums of a run, mostly two, are added by the lanes of the first, in 64 bits.
template <int OUT>
__global__ void __launch_bounds__(kEmbedWaves * 64)
embed_join_kernel(SumArgs a)
{
    typedef typename Element<OUT>::type Out;
    constexpr int N = kChunk<float>;
    const int lane = threadIdx.x & 63, ll = a.ll, h = lane & ((1 << ll) - 1);
    const int64_t s = (((int64_t)blockIdx.x * kEmbedWaves + (threadIdx.x >> 6)) << (6 - ll)) + (lane >> ll);
    if (s >= a.n)
        return;
    const uint32_t token = a.part_token[s] >> 1;
    if (token == kNoToken >> 1 || plain_token(a.packing, (int)token) >= a.n_vocab || (s > 0 && a.part_token[s - 1] >> 1 == token))
        return;
    const Span at = span_of<N>(((int)blockIdx.y * 64 + h) * N, a.width, !a.accumulate);
    const int c = at.c, n = at.n;
    double all[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        all[i] = 0.0;
    bool some = false, on = true;
    for (int64_t e = s; on; e += kJoinAhead) {
        uint32_t met[kJoinAhead];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            met[u] = e + u < a.n ? a.part_token[e + u] : kNoToken;
        RawChunk<float> x[kJoinAhead];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
            on = on && met[u] >> 1 == token;
            const bool add = on && !(met[u] & 1);
            some |= add;
            x[u].load(a.part + (e + u) * a.part_stride + c, add ? n : 0);
        }
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i)
                all[i] += (double)x[u][i];
    }
    if (!some)
        return;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        sum[i] = (float)all[i];
    put_row<Out>(a, (int)token, c, n, sum);
}

// The bands' tables become one.
template <int OUT>
__global__ void __launch_bounds__(256)
embed_bands_kernel(SumArgs a, const float *tables)
{
    typedef typename Element<OUT>::type Out;
    constexpr int N = kChunk<float>;
    const int lane = threadIdx.x & 63, h = lane & ((1 << a.ll) - 1);
    const int64_t row = (((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) << (6 - a.ll)) + (lane >> a.ll);
    if (row >= a.n_vocab)
        return;
    for (int c0 = h * N; c0 < a.width; c0 += 64 * N) {
        const Span at = span_of<N>(c0, a.width, !a.accumulate);
        const int c = at.c, n = at.n;
        float sum[N], more[kXcds][N];
#pragma unroll
        for (int b = 0; b < kXcds; ++b)
            load_chunk<N>(tables + (min(b, a.bands - 1) * (int64_t)a.n_vocab + row) * a.part_stride + c, b < a.bands ? n : 0, more[b]);
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[i] = 0.0f;
#pragma unroll
        for (int b = 0; b < kXcds; ++b)
#pragma unroll
            for (int i = 0; i < N; ++i)
                sum[i] += more[b][i];
        put_row<Out>(a, (int)row, c, n, sum);
    }
}

// Few ids: a wavefront an id, which leaves if an earlier one is the same, and else adds the rows of all that are; no sort.  The
// launch's first workgroups clear the rows that nobody names, rows_each of them each.
template <int IN, int OUT, int ID>
__global__ void __launch_bounds__(kDirectWaves * 64)
embed_direct_kernel(EmbedIds ids, SumArgs a, ClearArgs clear, int32_t clear_blocks, int32_t rows_each)
{
    typedef typename Element<IN>::type In;
    typedef typename Element<OUT>::type Out;
    constexpr int N = kChunk<In>;
    __shared__ int32_t token[kDirectIds];
    __shared__ uint32_t named[kDirectRows / 32];
    __shared__ uint32_t same_rows[kDirectWaves][kDirectIds];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_ids = (int)a.n;
    if ((int)threadIdx.x < n_ids) {
        int row[1];
        ids.template rows<ID>(row, [&](int) { return threadIdx.x; }, [&](int) { return threadIdx.x - ids.row_of(threadIdx.x) * (uint32_t)ids.n_cols; });
        token[threadIdx.x] = row[0];
    }
    if ((int)blockIdx.x < clear_blocks) {
        const int64_t first = (int64_t)blockIdx.x * rows_each, end = min(first + rows_each, clear.n_rows);
        for (int i = threadIdx.x; i < kDirectRows / 32; i += kDirectWaves * 64)
            named[i] = 0;
        __syncthreads();
        if ((int)threadIdx.x < n_ids) {
            const int64_t at = token[threadIdx.x] - first;
            if (token[threadIdx.x] >= 0 && at >= 0 && at < rows_each)
                atomicOr(&named[at >> 5], 1u << (at & 31));
        }
        __syncthreads();
        const int ll = clear.ll;
        for (int64_t r = first + (wave << (6 - ll)) + (lane >> ll); r < end; r += kDirectWaves << (6 - ll))
            if (!(named[(r - first) >> 5] >> ((r - first) & 31) & 1))
                clear_row<Out>(clear, r, lane & ((1 << ll) - 1));
        return;
    }
    __syncthreads();
    const int id = ((int)blockIdx.x - clear_blocks) * kDirectWaves + wave;
    const int mine = id < n_ids ? token[id] : -1;
    if (mine < 0)
        return;
    int count = 0;
    bool earlier = false;
#pragma unroll
    for (int b = 0; b < kDirectIds; b += 64) {
        const bool same = b + lane < n_ids && token[min(b + lane, n_ids - 1)] == mine;
        const uint64_t lanes = __ballot(same);
        if (same)
            same_rows[wave][count + lanes_before(lanes)] = ids.row_of((uint32_t)(b + lane));
        earlier |= same && b + lane < id;
        count += __popcll(lanes);
    }
    if (__ballot(earlier))
        return;
    lds_sync();
    const int ll = a.ll, h = lane & ((1 << ll) - 1), part = lane >> ll, parts = 64 >> ll;
    for (int c0 = h * N; c0 < a.width; c0 += 64 * N) {
        const Span at = span_of<N>(c0, a.width, !a.accumulate);
        float sum[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            sum[i] = 0.0f;
        for (int q0 = part; q0 < count; q0 += kEmbedAhead * parts) {
            RawChunk<In> x[kEmbedAhead];
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u) {
                const int q = q0 + u * parts;
                x[u].load((const In *)a.in + (int64_t)same_rows[wave][min(q, count - 1)] * a.in_stride + at.c, q < count ? at.n : 0);
            }
#pragma unroll
            for (int u = 0; u < kEmbedAhead; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    sum[i] += x[u][i];
        }
        for (int s = ll; s < 6; ++s)
#pragma unroll
            for (int i = 0; i < N; ++i)
                sum[i] += __shfl_xor(sum[i], 1 << s);
        if (part == 0)
            put_row<Out>(a, mine, at.c, at.n, sum);
    }
}

struct SumPlan {
    int64_t groups, part_stride;   // workgroups; elements
    int32_t chunk, ll, columns;
};
// More, shorter chunks where there are few pairs to a wavefront: down to kSumLeastChunk for kSumMostWaves.
static SumPlan sum_plan(int64_t n, int32_t width, int32_t type)
{
    SumPlan p;
    const int elements = 16 / (int)type_bytes(type);
    p.ll = row_lanes_log(width, elements);
    p.columns = column_blocks(width, elements);
    p.chunk = kSumMostChunk;
    while (p.chunk > kSumLeastChunk && ((n / p.chunk * p.columns) << p.ll) < (int64_t)kSumMostWaves * 64)
        p.chunk /= 2;
    p.part_stride = (width + 3) / 4 * 4;
    const int64_t each = ((int64_t)kSumWaves << (6 - p.ll)) * p.chunk;
    p.groups = (n + each - 1) / each;
    return p;
}

struct SortPlan {
    int token_bits, passes, bits;      // of all digits, of one
    Packing packing;
    int bands;
    bool packed;
    SlotShape shape;
    SumPlan sum;
    size_t list_bytes, token_bytes, part_bytes, table_bytes, bytes;
};
// Bands of rows: the sum reads a row once for every token that it names, in the order of the tokens, so that rows come from the
// L2 cache of an XCD only if all of them fit there.  Where they do not, but a half to an eighth of them does, the list is
// sorted by band first, every XCD sums tokens over the rows of one band, and the bands' tables are added.  32768 rows of
// 256 bytes, 100 tokens each: 102 us without bands and 65 with them; 8192 such rows with 400 each 60 (the sums alone, before
// offsets had 32 bits).  The tables are written twice and read
// once, which a thirtieth as many rows as there are pairs does not outweigh.
constexpr int64_t kBandBytes = 5 << 19, kL2Bytes = 4 << 20;
constexpr int kBandLeastRun = 30;
static int bands_for(int32_t n_vocab, int32_t width, int32_t type, int64_t n_rows, int64_t n)
{
    const int64_t bytes = n_rows * width * (int64_t)type_bytes(type);
    if (n <= kEmbedFew || n_rows <= kXcds || bytes <= kL2Bytes || bytes > kXcds * kL2Bytes)
        return 1;
    int bands = 2;
    while (bands < kXcds && bytes > bands * kBandBytes)
        bands *= 2;
    return n / n_vocab >= (int64_t)kBandLeastRun * bands ? bands : 1;
}

static SortPlan sort_plan(int32_t n_vocab, int32_t width, int32_t type, int64_t n_rows, int32_t n_cols)
{
    const int64_t n = n_rows * n_cols;
    SortPlan p;
    int bits = 1;                                  // of 0 .. n_vocab
    while (((int64_t)1 << bits) <= n_vocab)
        ++bits;
    p.packing = Packing{bits_of((int)n_rows), bits, 0};
    p.bands = bits + 3 <= 30 ? bands_for(n_vocab, width, type, n_rows, n) : 1;
    if (p.bands > 1) {
        p.packing.band_magic = (uint32_t)(((uint64_t)p.bands << 32) / (uint64_t)n_rows);
        bits += bits_of(p.bands);
    }
    p.token_bits = bits;
    p.passes = (bits + 9) / 10;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.sum = sum_plan(n, width, type);
    p.packed = p.packing.row_bits + bits <= 32 && p.packing.row_bits < 32;
    p.shape = slot_shape(n, 1 << p.bits, p.packed ? sizeof(uint32_t) : sizeof(Pair));
    p.list_bytes = ((size_t)n * (p.packed ? sizeof(uint32_t) : sizeof(Pair)) + 255) / 256 * 256;
    p.token_bytes = ((size_t)p.sum.groups * 2 * 4 + 255) / 256 * 256;
    p.part_bytes = ((size_t)p.sum.groups * 2 * p.sum.part_stride * 4 + 255) / 256 * 256;
    p.table_bytes = p.bands > 1 ? ((size_t)p.bands * n_vocab * p.sum.part_stride * 4 + 255) / 256 * 256 : 0;
    p.bytes = 2 * p.list_bytes + p.token_bytes + p.part_bytes + p.table_bytes + slot_count_bytes(p.shape, kEmbedFew);
    return p;
}

static int check_embed(const char *who, int32_t n_vocab, int32_t width, int64_t n_rows, int32_t n_cols)
{
    if (n_vocab < 1 || n_vocab == 2147483647)
        return fail(FS_EINVAL, "%s: n_vocab %d outside [1, 2^31 - 2]", who, n_vocab);
    FS_TRY(check_width(who, width));
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
    const int chunk = 16 / (int)type_bytes(table_type), ll = row_lanes_log(width, chunk), blocks = column_blocks(width, chunk);
    int split = 0;                 // a long bag of few rows: its parts in neighbouring lanes, down to four ids each
    while (split < 6 - ll && (n_cols >> (split + 1)) >= 4 && (((n_rows * blocks) << (ll + split)) >> 6) < kEmbedFewWaves)
        ++split;
    EmbedArgs a = {embed_ids(ids, col_base, n_cols, n_vocab), table, table_stride, out_stride, n_rows, width, ll, split, blocks, scale, out, 0};
    const int64_t rows = ((int64_t)(n_cols == 1 ? kLookupRows : 1)) << (6 - ll - split);       // of a wavefront
    const int64_t waves = (n_rows + rows - 1) / rows * blocks;
    prof_start(kKernPack, stream);
    with_types(table_type, out_type, [&](auto i, auto o) {
        with_id_type(id_type, [&](auto d) {
            constexpr int in = decltype(i)::value, to = decltype(o)::value, id = decltype(d)::value;
            in_pieces((waves + kEmbedWaves - 1) / kEmbedWaves, [&](int64_t at, unsigned n) {
                a.block0 = at;
                const auto kernel = (n_cols - 1) >> split >= kEmbedMostFp32 ? embed_kernel<in, to, id, true>
                                    : n_cols > 1                            ? embed_kernel<in, to, id, false>
                                    : past_caches(n_rows, width, out_type)  ? embed_lookup_kernel<in, to, id, true>
                                                                            : embed_lookup_kernel<in, to, id, false>;
                hipLaunchKernelGGL(kernel, dim3(n), dim3(kEmbedWaves * 64), 0, stream, a);
            });
        });
    });
    prof_stop(stream);
    return launched("embedding kernel launch");
}

extern "C" size_t fs_embed_backward_workspace_bytes(int32_t n_vocab, int32_t width, int32_t d_out_type, int64_t n_rows, int32_t n_cols)
{
    static const char who[] = "fs_embed_backward_workspace_bytes";
    if (check_embed(who, n_vocab, width, n_rows, n_cols) != FS_OK)
        return 0;
    if (!type_ok(d_out_type)) {
        fail(FS_EINVAL, "%s: unknown element type %d of d_out", who, d_out_type);
        return 0;
    }
    return sort_plan(n_vocab, width, d_out_type, n_rows, n_cols).bytes;
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
    const SortPlan p = sort_plan(n_vocab, width, d_out_type, n_rows, n_cols);
    FS_TRY(check_array(who, "work", work, (int64_t)p.bytes, 256));
    if (work_bytes < p.bytes)
        return fail(FS_EINVAL, "%s: %zu bytes of working memory, %zu are needed", who, work_bytes, p.bytes);
    char *at = (char *)work;
    const auto take = [&](size_t bytes) {
        char *const here = at;
        at += bytes;
        return here;
    };
    void *const list[2] = {take(p.list_bytes), take(p.list_bytes)};
    uint32_t *const part_token = (uint32_t *)take(p.token_bytes);
    float *const part = (float *)take(p.part_bytes), *const tables = (float *)take(p.table_bytes);
    int32_t *const count = (int32_t *)at;
    prof_start(kKernTrainOther, stream);
    ClearArgs clear = {d_table, n_vocab, d_table_stride, d_table_type, width, row_lanes_log(width, 16 / (int)type_bytes(d_table_type))};
    if (p.bands > 1)
        clear = ClearArgs{tables, (int64_t)p.bands * n_vocab, p.sum.part_stride, FS_F32, width, row_lanes_log(width, kChunk<float>)};
    const bool keep = p.bands == 1 && accumulate;
    const bool few = n > 0 && sort_in_one(n, keep ? 0 : clear.n_rows * width * (int64_t)type_bytes(clear.type));
    // Part `which` of `parts` of what is to be cleared, and the workgroups for it.
    const auto clear_part = [&](int which, int parts, int32_t &blocks) {
        const int64_t begin = clear.n_rows * which / parts, end = clear.n_rows * (which + 1) / parts, rows = (int64_t)kSlotWaves << (6 - clear.ll);
        ClearArgs part = clear;
        part.table = (char *)clear.table + begin * clear.stride * (int64_t)type_bytes(clear.type);
        part.n_rows = end - begin;
        blocks = keep ? 0 : (int32_t)min((end - begin + rows - 1) / rows, (int64_t)kClearBlocks);
        return part;
    };
    const auto beside = [&](int pass) {
        ClearBeside c;
        c.counting = clear_part(few ? 0 : 2 * pass, few ? 1 : 2 * p.passes, c.count_blocks);
        c.placing = clear_part(few ? 0 : 2 * pass + 1, few ? 1 : 2 * p.passes, c.place_blocks);
        return c;
    };
    const int64_t rows_once = (int64_t)kDirectWaves << (6 - clear.ll), apart = min((n_vocab + rows_once - 1) / rows_once, (int64_t)kClearBlocks);
    const int64_t rows_each = (n_vocab + apart - 1) / apart;
    if (n > 0 && n <= kDirectIds && rows_each <= kDirectRows) {
        const int clear_blocks = accumulate ? 0 : (int)((n_vocab + rows_each - 1) / rows_each);
        const SumArgs a = {nullptr, p.packing, d_out, d_out_stride, d_table_stride, n, width, p.sum.ll, 0, n_vocab, accumulate, scale, d_table,
                           nullptr, nullptr, 0, 0, 1};
        with_types(d_out_type, d_table_type, [&](auto i, auto o) {
            with_id_type(id_type, [&](auto d) {
                hipLaunchKernelGGL((embed_direct_kernel<decltype(i)::value, decltype(o)::value, decltype(d)::value>),
                                   dim3((unsigned)(clear_blocks + (n + kDirectWaves - 1) / kDirectWaves)), dim3(kDirectWaves * 64), 0, stream,
                                   embed_ids(ids, col_base, n_cols, n_vocab), a, clear, clear_blocks, (int32_t)rows_each);
            });
        });
        prof_stop(stream);
        return launched("embedding gradient kernel launch");
    }
    if (n == 0 && !keep) {
        int32_t blocks;
        const ClearArgs all = clear_part(0, 1, blocks);
        hipLaunchKernelGGL(embed_clear_kernel, dim3((unsigned)blocks), dim3(kSlotThreads), 0, stream, all);
    }
    if (n > 0) {
        const int mask = (1 << p.bits) - 1;
        int now = 0;
        const auto sort = [&](auto pair) {
            typedef decltype(pair) P;
            P *const lists[2] = {(P *)list[0], (P *)list[1]};
            with_id_type(id_type, [&](auto type) {
                constexpr int id = decltype(type)::value;
                const IdDigit<id, P> of = {beside(0), embed_ids(ids, col_base, n_cols, n_vocab), lists[0], mask, p.packing};
                if (few)
                    hipLaunchKernelGGL((n <= kEmbedFew ? embed_sort_few_kernel<id, P, kEmbedFew / 1024> : embed_sort_few_kernel<id, P, kEmbedFew / 512>),
                                       dim3((unsigned)(1 + of.count_blocks)), dim3(kSlotFewWaves * 64), 0, stream, of, (int32_t)n, p.token_bits);
                else
                    launch_slots(of, p.shape, count, stream);
            });
            if (!few)
                for (int pass = 1; pass < p.passes; ++pass, now ^= 1)
                    launch_slots(PairDigit<P>{beside(pass), lists[now], lists[now ^ 1], pass * p.bits, mask, p.packing}, p.shape, count, stream);
        };
        if (p.packed)
            sort(uint32_t());
        else
            sort(Pair());
        SumArgs a = {list[now], p.packing, d_out, d_out_stride, d_table_stride, n, width, p.sum.ll, p.sum.chunk, n_vocab, accumulate, scale,
                     d_table, part_token, part, p.sum.part_stride, (int32_t)p.sum.groups, p.bands};
        SumArgs to = a;                // of what adds the bands' tables
        if (p.bands > 1) {
            a.out = tables;
            a.out_stride = p.sum.part_stride;
            a.accumulate = 0;
            a.scale = 1.0f;
        }
        with_types(d_out_type, p.bands > 1 ? FS_F32 : d_table_type, [&](auto i, auto o) {
            constexpr int in = decltype(i)::value, out = decltype(o)::value;
            const int64_t each = (p.sum.groups + p.bands - 1) / p.bands, per = kXcds / p.bands;
            const dim3 grid((unsigned)(p.bands > 1 ? (each + per - 1) / per * kXcds : p.sum.groups), (unsigned)p.sum.columns);
            const bool near = d_out_stride < ((int64_t)1 << 31) && n_rows * d_out_stride * (int64_t)type_bytes(d_out_type) < ((int64_t)1 << 32);
            const auto kernel = p.packed ? near ? embed_sum_kernel<in, out, uint32_t, true> : embed_sum_kernel<in, out, uint32_t, false>
                                         : near ? embed_sum_kernel<in, out, Pair, true> : embed_sum_kernel<in, out, Pair, false>;
            hipLaunchKernelGGL(kernel, grid, dim3(kSumWaves * 64), 0, stream, a);
            a.ll = to.ll = row_lanes_log(width, kChunk<float>);
            if (p.sum.groups > 1) {
                a.n = 2 * p.sum.groups;
                const int64_t rows = (int64_t)kEmbedWaves << (6 - a.ll);
                hipLaunchKernelGGL(embed_join_kernel<out>, dim3((unsigned)((a.n + rows - 1) / rows), (unsigned)column_blocks(width, kChunk<float>)),
                                   dim3(kEmbedWaves * 64), 0, stream, a);
            }
        });
        if (p.bands > 1)
            with_type(d_table_type, [&](auto t) {
                const int64_t each = (int64_t)4 << (6 - to.ll);
                to.packing.token_bits = 31;             // rows of one table
                hipLaunchKernelGGL(embed_bands_kernel<decltype(t)::value>, dim3((unsigned)((n_vocab + each - 1) / each)), dim3(256), 0, stream, to,
                                   (const float *)tables);
            });
    }
    prof_stop(stream);
    return launched("embedding gradient kernels launch");
}
