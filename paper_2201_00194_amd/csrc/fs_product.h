// Tiles of matrix products on the matrix units: operands through LDS, sums in registers.
//
// sum over k of a[m][k] b[n][k], of operands whose rows lie along the sum or across it (ALONG: row k has all m, or all n).  Fragments are
// 16 bytes a lane; across 16-bit operands LDS turns them as they are read.  A wavefront of 256 x 256 tiles holds 128 x 64 results, so that
// of a fragment's read from LDS four or eight products come and LDS keeps up with the matrix units.
#ifndef FS_PRODUCT_H
#define FS_PRODUCT_H

#include "fs_mixture.h"
#include "familyseer_experts.h"

namespace fs {

constexpr int kI8 = 3;      // beside FS_F32, FS_BF16 and FS_F16: an operand's type, not a result's

typedef float F4 __attribute__((ext_vector_type(4)));
typedef int I4 __attribute__((ext_vector_type(4)));
typedef short S4 __attribute__((ext_vector_type(4)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));

// What a type's tiles are made of.  A fragment is 16 bytes a lane: lane l holds, of row l % 16 of sixteen, the l / 16th 16 bytes of
// 64 along the sum.  One step of the matrix units takes 64 bytes of the sum of 16 rows and 16 columns; for fp32 that is four
// instructions, the i-th of which takes the i-th float of every lane.
template <int TYPE> struct Unit16;
template <> struct Unit16<FS_BF16> {
    typedef F4 Acc;
    static constexpr int size = 2;
    static __device__ __forceinline__ Acc step(I4 a, I4 b, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    }
};
template <> struct Unit16<FS_F16> {
    typedef F4 Acc;
    static constexpr int size = 2;
    static __device__ __forceinline__ Acc step(I4 a, I4 b, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a), __builtin_bit_cast(H8, b), c, 0, 0, 0);
    }
};
template <> struct Unit16<FS_F32> {
    typedef F4 Acc;
    static constexpr int size = 4;
    static __device__ __forceinline__ Acc step(I4 a, I4 b, Acc c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[i]), __int_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
};
template <> struct Unit16<kI8> {
    typedef I4 Acc;
    static constexpr int size = 1;
    static __device__ __forceinline__ Acc step(I4 a, I4 b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

// An operand of a tile.  `along` false: rows of elements along the sum (p at the tile's first row); true: rows of elements across
// it, one row for each term of the sum (p at the tile's first column).
struct Operand {
    const char *p;
    int64_t stride;      // bytes from row to row
    int count;           // rows, or columns, of the tile that are there
};

// The thread's number, as one that the compiler cannot know: what follows from it is computed where it is needed, and not kept in
// registers beside the sums of all tiles.
__device__ __forceinline__ int thread_here()
{
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

constexpr int kUnitBytes = 64;      // of the sum, of 1, 2 or 4 bytes an element: a step of the matrix units

// Where 16 bytes of an operand lie in LDS.  The xor spreads what sixteen lanes, or 32 with a transposing read, take at a time over the
// banks.
template <int TYPE, bool ALONG, int ROWS, int STEP, int FOUR>
struct Place {
    static constexpr int size = Unit16<TYPE>::size;
    static constexpr int chunks = ROWS * STEP / 16;
    static constexpr int per_row = ALONG ? ROWS * size / 16 : STEP / 16;     // 16-byte chunks
    static __device__ __forceinline__ int turn(int row)
    {
        constexpr int shift = FOUR == 4 ? 4 : 3;
        if constexpr (!ALONG && STEP == 128)
            return (row >> 1 & 1) | (row >> shift & 3) << 1;
        else if constexpr (!ALONG)
            return -(row >> shift) & 3;      // the four lanes of sixteen or 32 that a read takes together: 0 3 of one fragment half, 1 2 of its neighbour
        else if constexpr (size == 2 && per_row == 8)
            return (row >> 3 & 1) << 1 | (row >> 1 & 1) << 2;
        else if constexpr (size == 2)
            return (row & 1) | (row >> 3 & 1) << 1 | (row >> 1 & 1) << 3;
        else
            return 0;
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return (row * per_row + (chunk ^ turn(row))) * 16; }
};
// Which of an operand's 64 rows (columns) lane r of sixteen has in fragment f of four: such that a lane's results lie side by side.
// FOUR = 2: of 32, two fragments.
template <int TYPE, bool ALONG, int FOUR>
__device__ __forceinline__ int member(int f, int r)
{
    static_assert(FOUR == 4 || (FOUR == 2 && !ALONG), "");
    if constexpr (!ALONG)
        return (r >> 2) * (4 * FOUR) + f * 4 + (r & 3);
    else if constexpr (Unit16<TYPE>::size == 2)
        return (r >> 2) * 16 + (f ^ (r >> 2 & 1)) * 4 + (r & 3);      // both halves of 16 bytes are read at a time
    else
        return 4 * r + f;
}

// 16 bytes of which n elements are there.
template <int ALIGNED, class E = int> struct Bytes16 {
    typedef E type __attribute__((ext_vector_type(4), aligned(ALIGNED)));
};
template <int SIZE>
__device__ __forceinline__ I4 some_bytes(const char *p, int n)
{
    constexpr int N = 16 / SIZE;
    I4 v = {0, 0, 0, 0};
    if (n >= N) {
        v = *(const typename Bytes16<SIZE>::type *)p;
    } else if (n > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = i < n ? i : n - 1;
            unsigned e;
            if constexpr (SIZE == 1)
                e = ((const uint8_t *)p)[at];
            else if constexpr (SIZE == 2)
                e = ((const uint16_t *)p)[at];
            else
                e = ((const uint32_t *)p)[at];
            e = i < n ? e : 0;
            v[i * SIZE / 4] |= (int)(e << (i * SIZE % 4 * 8));
        }
    }
    return v;
}

// The bytes behind the first n, and zeros.
__device__ __forceinline__ I4 without_first(I4 v, int n)
{
    if (n & 4)
        v = I4{v[1], v[2], v[3], 0};
    if (n & 8)
        v = I4{v[2], v[3], 0, 0};
    const I4 moved = {(int)__builtin_amdgcn_alignbyte(v[1], v[0], n & 3), (int)__builtin_amdgcn_alignbyte(v[2], v[1], n & 3),
                      (int)__builtin_amdgcn_alignbyte(v[3], v[2], n & 3), (int)__builtin_amdgcn_alignbyte(0, v[3], n & 3)};
    return n >= 16 ? I4{0, 0, 0, 0} : moved;
}

// A tile's shape: BM x BN results by WM x WN wavefronts, each (BM / WM) x (BN / WN) of them, multiples of 64 (of rows along the
// sum, 32 too); STEP bytes of the sum (64 or 128) at a time, STAGES steps in LDS.
template <int BM_, int BN_, int WM_, int WN_, int STEP_, int STAGES_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STEP = STEP_, STAGES = STAGES_, threads = WM_ * WN_ * 64;
};
template <int TYPE, class SHAPE, bool AT, bool BT>
struct Tile {
    static constexpr int BM = SHAPE::BM, BN = SHAPE::BN, WM = SHAPE::WM, WN = SHAPE::WN, STEP = SHAPE::STEP, kStages = SHAPE::STAGES;
    typedef Unit16<TYPE> U;
    typedef typename U::Acc Acc;
    static constexpr int threads = WM * WN * 64;
    static constexpr int MF = BM / WM / 16, NF = BN / WN / 16;      // fragments of a wavefront
    static constexpr int MFOUR = MF < 4 ? MF : 4;
    static constexpr int a_bytes = BM * STEP, b_bytes = BN * STEP, stage_bytes = a_bytes + b_bytes;
    static constexpr int lds_bytes = kStages * stage_bytes;
    static constexpr int units = STEP / kUnitBytes;
    static constexpr int step = STEP / U::size;               // elements of the sum
    Acc acc[MF][NF];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j)
                acc[i][j] = Acc{0, 0, 0, 0};
    }

    // ---- operands through registers: any alignment, any sizes ----
    // A chunk that is not whole is loaded element by element, or, of rows of at least 16 bytes, where it ends with its row, and moved on its
    // way to LDS, so that no load waits for another.  32 768 slots of 16 experts, 1001 x 1001 bf16, us, by elements and moved: products 118 and 108,
    // turned 215 and 131 with the weights moved alone (both: 188), the weights' gradient 321 and 134.
    template <bool ALONG, int ROWS, int FOUR = 4>
    struct Fetched {
        typedef Place<TYPE, ALONG, ROWS, STEP, FOUR> P;
        static constexpr int N = P::chunks / threads, E = 16 / U::size;
        static constexpr bool kMoves = ALONG || !BT;
        I4 v[N];
        static __device__ __forceinline__ int row_of(int i) { return (threadIdx.x + i * threads) / P::per_row; }
        static __device__ __forceinline__ int first_of(int i) { return (threadIdx.x + i * threads) % P::per_row * E; }
        __device__ __forceinline__ void load(const Operand &o, int k0, int k_count, int width)
        {
            if (!kMoves || width < E) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int row = row_of(i), first = first_of(i);
                    if constexpr (ALONG)
                        v[i] = some_bytes<U::size>(o.p + (k0 + row) * o.stride + first * U::size, k0 + row < k_count ? o.count - first : 0);
                    else
                        v[i] = some_bytes<U::size>(o.p + row * o.stride + (int64_t)(k0 + first) * U::size, row < o.count ? k_count - k0 - first : 0);
                }
                return;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int row = row_of(i), first = first_of(i);
                const int64_t at = ALONG ? (k0 + row) * o.stride + min(first, o.count - E) * U::size
                                         : row * o.stride + (int64_t)min(k0 + first, k_count - E) * U::size;
                v[i] = I4{0, 0, 0, 0};
                if (ALONG ? k0 + row < k_count && first < o.count : row < o.count && k0 + first < k_count)
                    v[i] = *(const typename Bytes16<U::size>::type *)(o.p + at);
            }
        }
        __device__ __forceinline__ void store(char *lds, const Operand &o, int k0, int k_count, int width)
        {
            if (kMoves && width >= E && (ALONG ? o.count < ROWS : k0 + step > k_count)) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    v[i] = without_first(v[i], max(ALONG ? first_of(i) + E - o.count : k0 + first_of(i) + E - k_count, 0) * U::size);
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
                *(I4 *)(lds + P::at(row_of(i), first_of(i) / E)) = v[i];
        }
    };

    // ---- operands straight into LDS: rows and their 16-byte chunks aligned and whole ----
    // A wavefront's load writes 64 chunks side by side, so it is the lanes' sources that are turned.  A lane whose chunk is not there
    // has an offset past the buffer's end, and zeros come.
    template <bool ALONG, int ROWS, int FOUR = 4>
    struct Streamed {
        typedef Place<TYPE, ALONG, ROWS, STEP, FOUR> P;
        static constexpr int N = P::chunks / threads;
        static constexpr unsigned kNowhere = 0x80000000u;
        unsigned from[N];
        uint64_t base;
        int64_t stride;
        __device__ __forceinline__ Streamed() {}
        static __device__ __forceinline__ int row_of(unsigned t, int i) { return (t + i * threads) / P::per_row; }
        static __device__ __forceinline__ int chunk_of(unsigned t, int i) { return (t + i * threads) % P::per_row ^ P::turn(row_of(t, i)); }
        __device__ __forceinline__ Streamed(const Operand &o) : base((uint64_t)o.p), stride(o.stride)
        {
            const int t = thread_here();
#pragma unroll
            for (int i = 0; i < N; ++i)
                from[i] = (ALONG ? chunk_of(t, i) * (16 / U::size) : row_of(t, i)) < o.count ? row_of(t, i) * (unsigned)stride + chunk_of(t, i) * 16 : kNowhere;
        }
        // Of the next step `left` elements of the sum are there; its chunks go to `lds`.
        unsigned to;
        __device__ __forceinline__ void prepare(char *lds, int left)
        {
            if (left < step) {
                const int t = thread_here();
#pragma unroll
                for (int i = 0; i < N; ++i)
                    from[i] = (ALONG ? row_of(t, i) : chunk_of(t, i) * (16 / U::size)) < left ? from[i] : kNowhere;
            }
            to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds + (threadIdx.x >> 6) * 1024);
        }
        __device__ __forceinline__ void load(int i) const
        {
            const I4 buffer = {__builtin_amdgcn_readfirstlane((int)base), __builtin_amdgcn_readfirstlane((int)(base >> 32) & 0xffff), (int)kNowhere, 0x00020000};
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to + i * threads * 16), "v"(from[i]), "s"(buffer)
                         : "memory");
        }
        __device__ __forceinline__ void advance() { base += ALONG ? (uint64_t)step * stride : STEP; }
        // Nothing more: zeros come.
        __device__ __forceinline__ void end()
        {
#pragma unroll
            for (int i = 0; i < N; ++i)
                from[i] = kNowhere;
            stride = 0;
        }
    };

    // ---- fragments ----
    // `base`: the wavefront's first row or column.  Fragment f is of block f / 4 of 64 rows; fp32 along: v[4 * block + i][f % 4]
    // are the i-th terms of its lanes instead of v[f][i].
    template <bool ALONG, int ROWS, int FOUR>
    static __device__ __forceinline__ I4 fragment(const char *lds, int base, int f, int unit)
    {
        typedef Place<TYPE, ALONG, ROWS, STEP, FOUR> P;
        const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, block = base + f / FOUR * (16 * FOUR);
        if constexpr (!ALONG) {
            return *(const I4 *)(lds + P::at(block + member<TYPE, false, FOUR>(f % FOUR, r), unit * 4 + g));
        } else if constexpr (U::size == 4) {
            return *(const I4 *)(lds + P::at(unit * 16 + g * 4 + (f & 3), block / 4 + r));
        } else {
            // Lane r brings four elements for lanes 4 (r % 4) to 4 (r % 4) + 3, of row r / 4 of four.
            const int at = block + member<TYPE, true, 4>(f & 3, (r & 3) * 4), k = unit * 32 + g * 8 + (r >> 2);
            typedef __attribute__((address_space(3))) S4 *Read;
            const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read)(lds + P::at(k, at >> 3) + (at & 4) * 2));
            const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read)(lds + P::at(k + 4, at >> 3) + (at & 4) * 2));
            typedef short S8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(I4, S8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        }
    }
    static __device__ __forceinline__ I4 fragment_a(const char *lds, int i, int unit)
    {
        return fragment<AT, BM, MFOUR>(lds, (threadIdx.x >> 6) / WN * (BM / WM), i, unit);
    }
    static __device__ __forceinline__ I4 fragment_b(const char *lds, int j, int unit)
    {
        return fragment<BT, BN, 4>(lds + a_bytes, (threadIdx.x >> 6) % WN * (BN / WN), j, unit);
    }
    __device__ __forceinline__ void multiply(const char *lds)
    {
#pragma unroll
        for (int unit = 0; unit < units; ++unit)
            multiply(lds, unit);
    }
    __device__ __forceinline__ void multiply(const char *lds, int unit)
    {
        I4 a[MF], b[NF];
#pragma unroll
        for (int j = 0; j < NF; ++j)
            b[j] = fragment_b(lds, j, unit);
#pragma unroll
        for (int i = 0; i < MF; ++i)
            a[i] = fragment_a(lds, i, unit);
        if constexpr (TYPE == FS_F32) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < MF; ++i)
#pragma unroll
                    for (int j = 0; j < NF; ++j) {
                        const int x = AT ? a[(i & ~3) + t][i & 3] : a[i][t], y = BT ? b[(j & ~3) + t][j & 3] : b[j][t];
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(y), __int_as_float(x), acc[i][j], 0, 0, 0);
                    }
        } else {
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    acc[i][j] = U::step(b[j], a[i], acc[i][j]);
        }
    }

    // ---- one tile after the other ----
    // Loads run kAhead steps ahead of the products, across tiles.  Counted are steps since the kernel's start: step n is in place n % kStages.
    template <int STORES>
    struct Stream {
        static constexpr bool kHalves = MF == 8 && TYPE != FS_F32;
        static constexpr int kAhead = kHalves ? kStages : kStages - 1;
        static constexpr int kLoads = Streamed<AT, BM, MFOUR>::N + Streamed<BT, BN>::N;      // of a wavefront and a step
        char *lds;
        Streamed<AT, BM, MFOUR> sa;
        Streamed<BT, BN> sb;
        int left = 0;                   // elements of the sum that the tile being loaded has left
        int issued = 0, used = 0;       // steps
        int mark = 0;                   // steps that were issued before the youngest stores, of which there are STORES at least
        I4 lo[4], b[NF];                // fragments of the step that comes next
        // next() sets sa, sb and left to another tile's; false if there is none: then steps of zeros are loaded.
        template <class F>
        __device__ __forceinline__ void prepare(F next)
        {
            if (left <= 0 && !next()) {
                sa.end();
                sb.end();
                left = INT32_MAX;
            }
            char *const to = lds + (issued & (kStages - 1)) * stage_bytes;
            sa.prepare(to, left);
            sb.prepare(to + a_bytes, left);
        }
        __device__ __forceinline__ void load(int i) const
        {
            constexpr int of_a = Streamed<AT, BM, MFOUR>::N;
            if (i < of_a)
                sa.load(i);
            else
                sb.load(i - of_a);
        }
        __device__ __forceinline__ void advance()
        {
            sa.advance();
            sb.advance();
            left -= step;
            ++issued;
        }
        template <class F>
        __device__ __forceinline__ void issue(F next)
        {
            prepare(next);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                load(i);
            advance();
        }
        // Before the kernel's end: LDS is written no more.
        __device__ __forceinline__ void end() const { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
        // Step n has arrived in all wavefronts; loads return in their order, so that what is younger may be on its way.
        template <int MORE>
        static __device__ __forceinline__ void wait(int younger)
        {
            if (younger >= 3)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(3 * kLoads + MORE) : "memory");
            else if (younger == 2)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * kLoads + MORE) : "memory");
            else if (younger == 1)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads + MORE) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(MORE) : "memory");
        }
        __device__ __forceinline__ void await(int n) const
        {
            if (n < mark)
                wait<STORES>(issued - n - 1);
            else
                wait<0>(issued - n - 1);
        }
        // Begins: the first steps on their way.
        template <class F>
        __device__ __forceinline__ void begin(F next)
        {
#pragma unroll 1
            for (int i = 0; i < kAhead; ++i)
                issue(next);
            if constexpr (kHalves) {
                await(0);
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    b[j] = fragment_b(lds, j, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    lo[i] = fragment_a(lds, i, 0);
            }
        }
        __device__ __forceinline__ const char *place() const { return lds + (used & (kStages - 1)) * stage_bytes; }
        // The sums of the tile whose steps come next.
        template <class F>
        __device__ __forceinline__ void sum(Tile &t, int k_count, F next)
        {
            int steps = (k_count + step - 1) / step;
            if (steps <= 0)
                return;
            if constexpr (kHalves) {
                // Eight fragments of rows, four of columns.  The second four of rows are read while the first four are multiplied; the next
                // step's first four, and its columns one after the other, while the second four are.
                // Loads go out one by one between products: all at once, they would hold the products up behind them until the others'
                // have been taken too.
                bool some = false;                   // of a step's loads are left
#pragma unroll 1
                do {
                    const char *then = place();
#pragma unroll
                    for (int unit = 0; unit < units; ++unit) {
                        I4 hi[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            hi[i] = fragment_a(then, 4 + i, unit);
#pragma unroll
                        for (int j = 0; j < NF; ++j) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                t.acc[i][j] = U::step(b[j], lo[i], t.acc[i][j]);
                            if (unit == 0 && kLoads > NF && some) {
                                __builtin_amdgcn_sched_barrier(0);
                                load(NF + j);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                        if (unit == 0 && kLoads > NF && some)
                            advance();
                        const int next_unit = (unit + 1) % units;
                        if (next_unit == 0) {
                            await(used + 1);
                            prepare(next);           // to where this step was, which all have read
                            ++used;
                            then = place();          // behind the last step of all: read, and not used
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            lo[i] = fragment_a(then, i, next_unit);
#pragma unroll
                        for (int j = 0; j < NF; ++j) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                t.acc[4 + i][j] = U::step(b[j], hi[i], t.acc[4 + i][j]);
                            b[j] = fragment_b(then, j, next_unit);
                            if (next_unit == 0) {
                                __builtin_amdgcn_sched_barrier(0);
                                load(j);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                        if (next_unit == 0 && kLoads <= NF)
                            advance();
                    }
                    some = true;
                } while (--steps > 0);
                if (kLoads > NF) {
#pragma unroll
                    for (int j = 0; j < NF; ++j)
                        load(NF + j);
                    advance();
                }
            } else {
#pragma unroll 1
                do {
                    await(used);
                    issue(next);
                    t.multiply(place());
                    ++used;
                } while (--steps > 0);
            }
        }
        // A tile's results have been stored: by `whole`, with STORES instructions a wavefront at least.
        __device__ __forceinline__ void stored(bool whole) { mark = whole ? issued : 0; }
    };

    // The sums over k_count terms, through registers; the operands' rows have so many elements in memory.
    __device__ __forceinline__ void run(char *lds, const Operand &a, const Operand &b, int k_count, int a_width, int b_width)
    {
        if (k_count <= 0)
            return;
        Fetched<AT, BM, MFOUR> fa;
        Fetched<BT, BN> fb;
        fa.load(a, 0, k_count, a_width);
        fb.load(b, 0, k_count, b_width);
        for (int k0 = 0, half = 0; k0 < k_count; k0 += step, half ^= 1) {
            static_assert(kStages >= 2, "");
            char *const now = lds + half * stage_bytes;
            fa.store(now, a, k0, k_count, a_width);
            fb.store(now + a_bytes, b, k0, k_count, b_width);
            if (k0 + step < k_count) {
                fa.load(a, k0 + step, k_count, a_width);
                fb.load(b, k0 + step, k_count, b_width);
            }
            __syncthreads();      // the other half was read before the last one of these
            multiply(now);
        }
    }

    // ---- results ----
    // A lane has, of one row a fragment, sixteen results side by side for each block of 64 columns, and sixteen lanes have sixteen
    // rows.  They change places in `rows` bytes of LDS of the wavefront's own, sixteen rows of 128 bytes at a time, so that eight lanes
    // store a line together: where each lane stored its own results, a tile of 256 x 256 took 10 us for it.
    // make(fragment, values, what of_column(column) gave, sixteen numbers): the results as numbers; put(row, column, chunk): 16 bytes
    // of them, as S.
    static constexpr int rows_bytes = 2048;
    static __device__ __forceinline__ int row_of(int t, int r, int i)
    {
        return (t >> 6) / WN * (BM / WM) + i / MFOUR * (16 * MFOUR) + member<TYPE, AT, MFOUR>(i % MFOUR, r);
    }
    template <class S, class G, class M, class P>
    __device__ __forceinline__ void results(char *rows, int t, G of_column, M make, P put) const
    {
        typedef S Chunk __attribute__((ext_vector_type(16 / sizeof(S))));
        constexpr int passes = sizeof(S) == 4 ? 2 : 1, N = 16 / sizeof(S);      // 32 or 64 columns a pass
        char *const own = rows + (t >> 6) * rows_bytes;
        const int n0 = (t >> 6) % WN * (BN / WN), lane = t & 63, g = lane >> 4, r = lane & 15;
#pragma unroll
        for (int block = 0; block < NF / 4; ++block) {
            const auto c = of_column(n0 + block * 64 + g * 16);
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                decltype(Acc{}[0] + 0) v[16];
                float y[16];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if constexpr (BT && TYPE == FS_F32)
                            v[4 * e + j] = acc[i][block * 4 + j][e];
                        else if constexpr (BT)
                            v[4 * j + e] = g & 1 ? acc[i][block * 4 + (j ^ 1)][e] : acc[i][block * 4 + j][e];
                        else
                            v[4 * j + e] = acc[i][block * 4 + j][e];
                make(i, v, c, y);
#pragma unroll
                for (int pass = 0; pass < passes; ++pass) {
                    if (passes == 1 || g >> 1 == pass) {
#pragma unroll
                        for (int h = 0; h < 16 / N; ++h) {
                            Chunk part;
#pragma unroll
                            for (int e = 0; e < N; ++e)
                                part[e] = (S)y[h * N + e];
                            const int chunk = (g & (4 / passes - 1)) * (16 / N) + h;
                            *(Chunk *)(own + r * 128 + (chunk ^ (r >> 1)) * 16) = part;
                        }
                    }
                    lds_sync();
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int rr = u * 8 + (lane >> 3), chunk = lane & 7;
                        const Chunk part = *(const Chunk *)(own + rr * 128 + (chunk ^ (rr >> 1)) * 16);
                        put(row_of(t, rr, i), n0 + block * 64 + pass * 32 + chunk * N, part);
                    }
                    lds_sync();
                }
            }
        }
    }
};

// A chunk of results of which n are wanted.
template <class S, int N>
__device__ __forceinline__ void store_part(S *p, int n, const S __attribute__((ext_vector_type(N))) &v)
{
    if (n >= N) {
        *(typename ChunkOf<S, N>::type *)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n)
                p[i] = v[i];
    }
}

// ---- whose rows a workgroup works on ---------------------------------------------------------------
// Experts' slots are cut into pieces of `per`; a piece is of one expert.
struct Piece {
    int expert, first, count;      // its slots
    int number, of;                // which of its expert's pieces, and of how many
};
struct Bounds {
    const int32_t *first;
    int n_experts, n_slots, per;
    // The pieces of an expert (none behind the last one).
    __device__ __forceinline__ int pieces(int e, int &begin, int &end) const
    {
        begin = end = 0;
        if (e >= n_experts)
            return 0;
        begin = min(max(first[e], 0), n_slots);
        end = max(min(first[e + 1], n_slots), begin);
        return (int)(((int64_t)end - begin + per - 1) / per);
    }
    // Every lane's sum of the lanes up to it.
    static __device__ __forceinline__ int sum_to(int v)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(v, d);
            v += lane >= d ? other : 0;
        }
        return v;
    }
};

// The pieces of all experts in a row, listed once by a workgroup.  SORTED: the experts with the most slots first, and an expert without
// slots has an empty piece.
template <bool SORTED>
struct PieceTable {
    int upto[FS_MAX_EXPERTS + 1];                        // pieces of the experts before
    int16_t order[SORTED ? FS_MAX_EXPERTS : 1];
    int waves[16];
    __device__ __forceinline__ int expert_at(int place) const { return SORTED ? order[place] : place; }
    // By all THREADS of the workgroup; the number of pieces, none if bounds descend: their pieces could be more than 32 bits count.
    template <int THREADS>
    __device__ __forceinline__ int fill(const Bounds &b)
    {
        constexpr int most = (FS_MAX_EXPERTS + THREADS - 1) / THREADS;
        const int each = (b.n_experts + THREADS - 1) / THREADS, e0 = threadIdx.x * each, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        static_assert(THREADS <= 512, "");
        int n[most], sum = 0;
        bool descends = false;
        if constexpr (SORTED) {
            int begin, end;
#pragma unroll
            for (int u = 0; u < most; ++u)
                if (u < each && e0 + u < b.n_experts) {
                    b.pieces(e0 + u, begin, end);
                    n[u] = upto[e0 + u] = end - begin;
                }
            __syncthreads();
            int before[most] = {};
            for (int e = 0; e < b.n_experts; ++e) {
                const int other = upto[e];
#pragma unroll
                for (int u = 0; u < most; ++u)
                    before[u] += u < each && (other > n[u] || (other == n[u] && e < e0 + u)) ? 1 : 0;
            }
#pragma unroll
            for (int u = 0; u < most; ++u)
                if (u < each && e0 + u < b.n_experts)
                    order[before[u]] = (int16_t)(e0 + u);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < most; ++u) {
            n[u] = 0;
            if (u < each && e0 + u < b.n_experts) {
                int begin, end;
                n[u] = b.pieces(expert_at(e0 + u), begin, end);
                descends |= b.first[e0 + u + 1] < b.first[e0 + u];
                if constexpr (SORTED)
                    n[u] = max(n[u], 1);
            }
            sum += n[u];
        }
        const int to_here = Bounds::sum_to(sum);
        descends = __any(descends);
        if (lane == 63) {
            waves[wave] = to_here;
            waves[8 + wave] = descends;
        }
        __syncthreads();
        int before = to_here - sum, all = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            before += w < wave ? waves[w] : 0;
            all += waves[w];
            descends |= waves[8 + w] != 0;
        }
#pragma unroll
        for (int u = 0; u < most; ++u)
            if (u < each && e0 + u < b.n_experts) {
                upto[e0 + u] = before;
                before += n[u];
            }
        if (threadIdx.x == 0)
            upto[b.n_experts] = all;
        __syncthreads();
        return __builtin_amdgcn_readfirstlane(descends ? 0 : all);
    }
    // Piece `id`, which is there: the last expert with no more than `id` before it, by 64 lanes twice.
    __device__ __forceinline__ Piece find(const Bounds &b, int id) const
    {
        const int lane = threadIdx.x & 63, each = (b.n_experts + 63) >> 6;
        const int block = __popcll(__ballot(lane * each < b.n_experts && upto[min(lane * each, b.n_experts)] <= id)) - 1;
        const int e = block * each + lane, in_block = __popcll(__ballot(lane < each && e < b.n_experts && upto[min(e, b.n_experts)] <= id)) - 1;
        const int place = __builtin_amdgcn_readfirstlane(block * each + in_block);
        Piece p;
        p.expert = __builtin_amdgcn_readfirstlane(expert_at(place));
        const int before = __builtin_amdgcn_readfirstlane(upto[place]);
        p.of = __builtin_amdgcn_readfirstlane(upto[place + 1]) - before;
        p.number = id - before;
        // Through the scalar cache: a vector load's wait would be one for all operands that are on their way.
        typedef const __attribute__((address_space(4))) int32_t *Constant;
        const Constant first = (Constant)(uintptr_t)b.first + p.expert;
        const int begin = min(max(first[0], 0), b.n_slots), end = max(min(first[1], b.n_slots), begin);
        p.first = begin + p.number * b.per;
        p.count = min(b.per, end - p.first);
        return p;
    }
};

}  // namespace fs
#endif
