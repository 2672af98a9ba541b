// Device code of the scan with matrix states that its forward and backward kernels share: q and k as fp16 operands, the block's matrices, and
// products with them.
#pragma once
#include "ssam_scan_delta.h"
#include "ssam_scan_delta_layout.h"

namespace ssam {

template <class T> constexpr bool kSplit = sizeof(T) == 4;      // q and k are pairs of fp16 too

// Eight elements of a row as fp16, `to` a power of two; the low parts where T has more bits than fp16.  With the row's largest at 2^10 .. 2^11, eight bits of
// bf16 fit fp16 down to 2^-17, 2^-27 of the largest; below, bits under fp16's last place, 2^-24, are cut off: at most 2^-34 of the largest.
template <class T>
__device__ __forceinline__ void to_halves(const RowVec<T, 8>& v, float to, Half8& hi, Half8& lo)
{
    if constexpr (__is_same(T, _Float16)) {
        hi = v;
    } else if constexpr (kSplit<T>) {
        const HalfPair p = split(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], to);
        hi = p.hi;
        lo = p.lo;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const auto h = __builtin_amdgcn_cvt_pkrtz((float)v[i] * to, (float)v[i + 1] * to);
            hi[i] = (_Float16)h[0];
            hi[i + 1] = (_Float16)h[1];
        }
    }
}

// ---- what follows the sequence: operands in LDS ----------------------------------------------------------------------------
// A row's eight elements are put where the lane reads them that needs them, all 64 lanes' entries of an operand side by side; within 16
// entries their places are permuted by the operand's number, so that the writes of a wave, which go to many operands, spread over the banks.
template <class T, int KT>
struct WalkRoom {
    static constexpr int kParts = kSplit<T> ? 2 : 1;
    // fp32 keys of more than 128 elements leave no room for the queries' operands: those follow the keys' in their place
    static constexpr bool kOnePlace = kSplit<T> && KT > 4;
    Block m;
    Half8 keys[kParts][4 * KT][kWave];                                      // rows t (tile_row), 32 elements
    Half8 turned_keys[kParts][4 * KT][kWave];                               // elements (tile_row), 32 rows
    Half8 more[kOnePlace ? 1 : kParts][kOnePlace ? 1 : 4 * KT][kWave];      // the queries in one of the two forms

    __device__ __forceinline__ auto& queries()
    {
        if constexpr (kOnePlace) return keys;
        else return more;
    }
};
template <int KT> __device__ __forceinline__ int row_operand(int m, int k) { return m * KT + k; }
__device__ __forceinline__ int row_entry(int k, int g, int r) { return 16 * g + (r ^ ((4 * g + k) & 15)); }
__device__ __forceinline__ int turned_operand(int j, int k) { return j * 2 + k; }
__device__ __forceinline__ int turned_entry(int j, int g, int r) { return 16 * g + (r ^ ((j >> 1) & 3)); }
template <int KT> __device__ __forceinline__ Half8 row_of(const Half8 (&a)[4 * KT][kWave], int m, int k, int lane)
{
    return a[row_operand<KT>(m, k)][row_entry(k, lane >> 4, lane & 15)];
}
template <int KT> __device__ __forceinline__ Half8 turned_of(const Half8 (&a)[4 * KT][kWave], int j, int k, int lane)
{
    return a[turned_operand(j, k)][turned_entry(j, lane >> 4, lane & 15)];
}

// Operands are read from LDS a step ahead of the products that take them, and products on several results alternate: one waits for its own last sum.
// (Left to itself the compiler reads an operand, waits for it and uses it, one after the other.)
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// A value, the same for all lanes, that the compiler takes for a new one here: what is made from it is not kept in registers over a loop.  (Rows' distances,
// 16 to 64 of them, would be, and push everything else out.)
__device__ __forceinline__ unsigned afresh(unsigned v)
{
    v = __builtin_amdgcn_readfirstlane(v);
    asm volatile("" : "+s"(v));
    return v;
}

// Eight elements of a row of fewer: copies of the last one behind it.  One after the other: a rare case that is to cost the others no registers.
template <class T>
__device__ __forceinline__ RowVec<T, 8> load_few(const T* __restrict__ row, int dim)
{
    RowVec<T, 8> v(T(0));
#pragma unroll 1
    for (int i = 7; i >= 0; --i) {
        v = __builtin_shufflevector(v, v, 0, 0, 1, 2, 3, 4, 5, 6);
        v[0] = row[i < dim ? i : dim - 1];
    }
    return v;
}

// N rows of eight elements, rows row0, row0 + step .. and elements from 8 e on; rows >= 1, `base` and `stride` the same for all lanes of a wave.  There are no branches on what is
// there: a load that waits for its turn in one costs its latency by itself.  clear_eights() makes zeros of what was not there, where the values are used.
// Where all rows are there, their distances are the same for all lanes too and cost no vector instructions.
template <class T, int N>
__device__ __forceinline__ void load_eights(const T* __restrict__ base, unsigned stride, int row0, int step, int rows, int e, int dim, RowVec<T, 8> (&v)[N])
{
    stride = afresh(stride);
    const unsigned at = dim < 8 ? 0 : eights_at(e, dim);
    if (dim >= 8 && rows == kDeltaRows) {
        const unsigned lane_at = (unsigned)row0 * stride + at;
#pragma unroll
        for (int i = 0; i < N; ++i) __builtin_memcpy(&v[i], base + (unsigned)(i * step) * stride + lane_at, sizeof(v[i]));
    } else if (dim >= 8) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = row0 + i * step;
            __builtin_memcpy(&v[i], base + ((unsigned)eights_row(row, rows) * stride + at), sizeof(v[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = row0 + i * step;
            v[i] = load_few(base + (unsigned)eights_row(row, rows) * stride, dim);
        }
    }
}
// Of eight elements that lie `by` places further left than they should: those to their places (copies of something behind them).
template <class T>
__device__ __forceinline__ RowVec<T, 8> shifted(RowVec<T, 8> w, int by)
{
    if (by & 4) w = __builtin_shufflevector(w, w, 4, 5, 6, 7, 4, 5, 6, 7);
    if (by & 2) w = __builtin_shufflevector(w, w, 2, 3, 4, 5, 6, 7, 6, 7);
    if (by & 1) w = __builtin_shufflevector(w, w, 1, 2, 3, 4, 5, 6, 7, 7);
    return w;
}
// Eight floats in two registers of four (arrays of eight that are filled as a whole are left in memory by the compiler).
struct Eight {
    Float4 lo, hi;
    __device__ __forceinline__ void load(const float* p)
    {
        typedef Float4 Loose __attribute__((aligned(4)));
        lo = *reinterpret_cast<const Loose*>(p);
        hi = *reinterpret_cast<const Loose*>(p + 4);
    }
    __device__ __forceinline__ void load(const float* p, int dim)      // of fewer than eight
    {
        lo = hi = Float4(0.0f);
#pragma unroll 1
        for (int i = 7; i >= 0; --i) {      // one after the other: a rare case that is to cost the others no registers
            const float v = p[i < dim ? i : dim - 1];
            hi = Float4{lo[3], hi[0], hi[1], hi[2]};
            lo = Float4{v, lo[0], lo[1], lo[2]};
        }
    }
    __device__ __forceinline__ void shift(int by)
    {
        if (by & 4) lo = hi;
        if (by & 2) {
            lo = Float4{lo[2], lo[3], hi[0], hi[1]};
            hi = Float4{hi[2], hi[3], hi[2], hi[3]};
        }
        if (by & 1) {
            lo = Float4{lo[1], lo[2], lo[3], hi[0]};
            hi = Float4{hi[1], hi[2], hi[3], hi[3]};
        }
    }
    __device__ __forceinline__ void clear(int from)      // elements from there on
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = i < from ? lo[i] : 0.0f;
            hi[i] = i + 4 < from ? hi[i] : 0.0f;
        }
    }
};
// How far left of `at` eight elements of a row of `dim` start.
__device__ __forceinline__ int shift_of(int at, int dim) { return dim < 8 ? at : at + 8 <= dim ? 0 : at - (dim - 8); }

// Brings the elements to their places, and clears what is not there.
template <class T, int N>
__device__ __forceinline__ void clear_eights(int row0, int step, int rows, int e, int dim, RowVec<T, 8> (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (dim % 8 && dim >= 8) v[i] = shifted(v[i], shift_of(8 * e, dim));
        if (!(8 * e < dim && row0 + i * step < rows)) v[i] = RowVec<T, 8>(T(0));
        if (dim % 8)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (8 * e + k >= dim) v[i][k] = T(0);
    }
}
// 8 rows x 8 elements, rows 8 b .. and elements 8 e ..
template <class T>
__device__ __forceinline__ void load_square(const T* __restrict__ base, unsigned stride, int rows, int dim, int b, int e, RowVec<T, 8> (&v)[8])
{
    load_eights<T, 8>(base, stride, 8 * b, 1, rows, e, dim, v);
}

// A wave's columns of 64 rows on their way between memory and result tiles: 16 bytes a lane from row to row, by way of a room in LDS that is the wave's own,
// where the tiles' values lie one by one.  (Element by element from and to memory, 16 loads and 16 stores a block cost a wave 3000 cycles.)
// kDirect: without the room.
template <class T, int NT, bool kDirect>
struct Columns {
    static constexpr int kWide = 16 * NT, E = 16 / (int)sizeof(T), kOfRow = kWide / E, kOfLane = kOfRow;
    struct Room {
        RowVec<T, E> rows[kDirect ? 1 : kDeltaRows][kDirect ? 1 : kOfRow + 1];
    };
    RowVec<T, E> v[kOfLane];

    static __device__ __forceinline__ void place(int i, int& row, int& part)
    {
        const int at = i * kWave + (int)(threadIdx.x & (kWave - 1));
        row = at / kOfRow;
        part = at % kOfRow;
    }
    // `base`: the rows' first, the same for all lanes; col0: the wave's first column of `dim`.  Rows that are not there are the last one's copies until values()
    // takes them, columns the last one's.
    __device__ __forceinline__ void load(const T* __restrict__ base, unsigned stride, int rows, int col0, int dim)
    {
        const bool whole = col0 + kWide <= dim;
        if (whole && rows == kDeltaRows) {
            int row, part;
            place(0, row, part);
            const unsigned lane_at = (unsigned)row * stride + (unsigned)(col0 + part * E);
            const unsigned step = (unsigned)(kWave / kOfRow) * afresh(stride);
#pragma unroll
            for (int i = 0; i < kOfLane; ++i) __builtin_memcpy(&v[i], base + i * step + lane_at, 16);
        } else {
#pragma unroll
            for (int i = 0; i < kOfLane; ++i) {
                int row, part;
                place(i, row, part);
                const T* const at = base + (unsigned)(row < rows ? row : rows - 1) * stride;
                const int c = col0 + part * E;
                if (whole) {
                    __builtin_memcpy(&v[i], at + c, 16);
                } else {
#pragma unroll
                    for (int k = 0; k < E; ++k) v[i][k] = at[c + k < dim ? c + k : dim - 1];
                }
            }
        }
    }
    __device__ __forceinline__ void values(Room& room, int rows, Float4 (&x)[4][NT]) const
    {
        const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, r = lane & 15;
#pragma unroll
        for (int i = 0; i < kOfLane; ++i) {
            int row, part;
            place(i, row, part);
            room.rows[row][part] = v[i];
        }
        __builtin_amdgcn_wave_barrier();       // (a wave's LDS instructions are done in their order)
        const T* const at = reinterpret_cast<const T*>(&room.rows[8 * g][0]) + r;
        constexpr int kPitch = (kOfRow + 1) * E;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[m][n][i] = (float)at[tile_row(m, i) * kPitch + 16 * n];
        if (rows < kDeltaRows) {
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[m][n][i] = tile_row(m, 4 * g + i) < rows ? x[m][n][i] : 0.0f;
        }
    }
    static __device__ __forceinline__ void store(Room& room, T* __restrict__ base, unsigned stride, int rows, int col0, int dim, const Float4 (&x)[4][NT])
    {
        const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, r = lane & 15;
        constexpr int kPitch = (kOfRow + 1) * E;
        __builtin_amdgcn_wave_barrier();
        T* const to = reinterpret_cast<T*>(&room.rows[8 * g][0]) + r;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) to[tile_row(m, i) * kPitch + 16 * n] = (T)x[m][n][i];
        __builtin_amdgcn_wave_barrier();
        const unsigned step = (unsigned)(kWave / kOfRow) * afresh(stride);
        int row0, part;
        place(0, row0, part);
        const unsigned lane_at = (unsigned)row0 * stride + (unsigned)(col0 + part * E);
        const int have = dim - (col0 + part * E);
#pragma unroll
        for (int i = 0; i < kOfLane; ++i) {
            const int row = row0 + i * (kWave / kOfRow);
            const RowVec<T, E> w = room.rows[row][part];
            if (rows == kDeltaRows || row < rows) {
                if (have >= E) __builtin_memcpy(base + i * step + lane_at, &w, 16);
                else if (have > 0) store_row_vec<T, E>(base + i * step + lane_at, have, w);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
};
// Without the room; an element on its way in a register of its own: two of them packed into one would have to be waited for in turn.
template <class T, int NT>
struct Columns<T, NT, true> {
    struct Room {};
    T v[4][NT][4];
    __device__ __forceinline__ void load(const T* __restrict__ base, unsigned stride, int rows, int col0, int dim)
    {
        stride = afresh(stride);
        const int g = (threadIdx.x & (kWave - 1)) >> 4, col = col0 + (threadIdx.x & 15);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const unsigned c = (unsigned)(col + 16 * n < dim ? col + 16 * n : dim - 1);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = tile_row(m, 4 * g + i);
                    v[m][n][i] = base[(unsigned)(t < rows ? t : rows - 1) * stride + c];
                }
        }
    }
    __device__ __forceinline__ void values(Room&, int rows, Float4 (&x)[4][NT]) const
    {
        const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[m][n][i] = tile_row(m, 4 * g + i) < rows ? (float)v[m][n][i] : 0.0f;
    }
    static __device__ __forceinline__ void store(Room&, T* __restrict__ base, unsigned stride, int rows, int col0, int dim, const Float4 (&x)[4][NT])
    {
        stride = afresh(stride);
        const int g = (threadIdx.x & (kWave - 1)) >> 4, col = col0 + (threadIdx.x & 15);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (col + 16 * n >= dim) continue;
            const unsigned lane_at = 8u * g * stride + (unsigned)(col + 16 * n);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (tile_row(m, 4 * g + i) < rows) *(base + (unsigned)tile_row(m, i) * stride + lane_at) = (T)x[m][n][i];
        }
    }
};

// A wave's columns of a matrix [32 KT rows, of which `dim`] of floats.
template <int KT, int NT>
__device__ __forceinline__ void load_state(const float* __restrict__ base, unsigned stride, int dim, int col, Float4 (&s)[2 * KT][NT])
{
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const unsigned c = (unsigned)(col + 16 * n < (int)stride ? col + 16 * n : (int)stride - 1);
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = tile_row(j, 4 * g + i);
                const float x = base[(size_t)(d < dim ? d : dim - 1) * stride + c];
                s[j][n][i] = d < dim ? x : 0.0f;
            }
    }
}
template <int KT, int NT>
__device__ __forceinline__ void store_state(float* __restrict__ base, unsigned stride, int dim, int col, const Float4 (&s)[2 * KT][NT])
{
    stride = afresh(stride);
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (col + 16 * n >= (int)stride) continue;
        const unsigned lane_at = 8u * g * stride + (unsigned)(col + 16 * n);
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (dim == 32 * KT || tile_row(j, 4 * g + i) < dim) *(base + (unsigned)tile_row(j, i) * stride + lane_at) = s[j][n][i];
    }
}
// 64 rows of floats, all of them.
template <int NT>
__device__ __forceinline__ void store_tiles(float* __restrict__ base, unsigned stride, int col, const Float4 (&v)[4][NT])
{
    stride = afresh(stride);
    const int g = (threadIdx.x & (kWave - 1)) >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (col + 16 * n >= (int)stride) continue;
        const unsigned lane_at = 8u * g * stride + (unsigned)(col + 16 * n);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) *(base + (unsigned)tile_row(m, i) * stride + lane_at) = v[m][n][i];
    }
}

template <class T, int KT, int kParts>
__device__ __forceinline__ void put_rows(const Half8 (&hi)[8], const Half8 (&lo)[8], int b, int e, Half8 (&to)[kParts][4 * KT][kWave])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = row_operand<KT>(2 * (b >> 2) + (i >> 2), e >> 2), entry = row_entry(e >> 2, e & 3, 4 * (b & 3) + (i & 3));
        to[0][at][entry] = hi[i];
        if constexpr (kParts > 1) to[1][at][entry] = lo[i];
    }
}
template <class T, int KT, int kParts>
__device__ __forceinline__ void put_turned(const Half8 (&hi)[8], const Half8 (&lo)[8], int b, int e, Half8 (&to)[kParts][4 * KT][kWave])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        Half8 th, tl;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            th[k] = hi[k][i];
            if constexpr (kParts > 1) tl[k] = lo[k][i];
        }
        const int j = 2 * (e >> 2) + (i >> 2), at = turned_operand(j, b >> 2), entry = turned_entry(j, b & 3, 4 * (e & 3) + (i & 3));
        to[0][at][entry] = th;
        if constexpr (kParts > 1) to[1][at][entry] = tl;
    }
}

// kBlock threads, the last ones of a block of more, stage.
__device__ __forceinline__ int stage_thread() { return (int)(threadIdx.x & (kBlock - 1)); }

// What a block of threads brings in of a block of rows: k's rows as operands in both forms, q's as rows (kTurn: turned), the block's matrices and factors.
// load() requests it, put() writes it into LDS; kAhead: into registers, so that the loads of the next block's pass behind the work on this one.
template <class T, int KT, bool kTurn>
struct Stage {
    static constexpr bool kOnePlace = WalkRoom<T, KT>::kOnePlace;
    typedef StageLanes<KT> Lanes;
    static constexpr int kSquares = Lanes::kSquares;
    static constexpr bool kAhead = (kSplit<T> ? 2 : 1) * KT <= 4;
    static constexpr int kVecs = (int)(sizeof(Block) / 16), kOfThread = (kVecs + kBlock - 1) / kBlock;
    static_assert(sizeof(Block) % 16 == 0);
    RowVec<T, 8> square[kAhead ? 8 : 1];
    Float4 block[kAhead ? kOfThread : 1], scale[2];

    static __device__ __forceinline__ void put_square(WalkRoom<T, KT>& room, bool query, int b, int e, int rows, int dim, RowVec<T, 8> (&v)[8], const Float4 (&to)[2])
    {
        if (rows < kDeltaRows || dim < 32 * KT) clear_eights<T, 8>(8 * b, 1, rows, e, dim, v);
        Half8 hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) to_halves<T>(v[i], to[i >> 2][i & 3], hi[i], lo[i]);
        if (query) {
            if constexpr (kTurn) put_turned<T, KT>(hi, lo, b, e, room.queries());
            else put_rows<T, KT>(hi, lo, b, e, room.queries());
        } else {
            put_rows<T, KT>(hi, lo, b, e, room.keys);
            put_turned<T, KT>(hi, lo, b, e, room.turned_keys);
        }
    }
    static __device__ __forceinline__ void load_scale(const BlockFactors& f, bool query, int b, Float4 (&to)[2])
    {
        const Float4* at = reinterpret_cast<const Float4*>((query ? f.query : f.key) + 8 * b);
        to[0] = at[0];
        to[1] = at[1];
    }
    // ks, qs: the block's first row
    __device__ __forceinline__ void load(const Block& from, const T* ks, unsigned kstride, const T* qs, unsigned qstride, int rows, int dim)
    {
        if constexpr (kAhead) {
            const int job = stage_thread();
            const bool query = Lanes::query(__builtin_amdgcn_readfirstlane(job));
            if (Lanes::has(job)) {
                load_square<T>(query ? qs : ks, query ? qstride : kstride, rows, dim, Lanes::rows(job), Lanes::elements(job), square);
                load_scale(from.f, query, Lanes::rows(job), scale);
            }
#pragma unroll
            for (int i = 0; i < kOfThread; ++i) {
                const int behind = (i + 1) * kBlock - kVecs;      // threads of the last round that have none: copies of others
                block[i] = *(reinterpret_cast<const Float4*>(&from) + (behind > 0 ? i * kBlock - behind : i * kBlock) + stage_thread());
            }
        }
    }
    __device__ __forceinline__ void put(WalkRoom<T, KT>& room, const Block& from, const T* ks, unsigned kstride, const T* qs, unsigned qstride, int rows, int dim)
    {
        Float4* const to = reinterpret_cast<Float4*>(&room.m);
        if constexpr (kAhead) {
            const int job = stage_thread();
            if (Lanes::has(job)) put_square(room, Lanes::query(job), Lanes::rows(job), Lanes::elements(job), rows, dim, square, scale);
#pragma unroll
            for (int i = 0; i < kOfThread; ++i) {
                const int behind = (i + 1) * kBlock - kVecs;
                to[(behind > 0 ? i * kBlock - behind : i * kBlock) + stage_thread()] = block[i];
            }
        } else {
            put_now(room, from, ks, kstride, qs, qstride, rows, dim, 0, kOnePlace ? kSquares : 2 * kSquares);
            for (int at = stage_thread(); at < kVecs; at += kBlock) to[at] = reinterpret_cast<const Float4*>(&from)[at];
        }
    }
    // Squares first .. last - 1: the keys', then the queries'.
    static __device__ __forceinline__ void put_now(WalkRoom<T, KT>& room, const Block& from, const T* ks, unsigned kstride, const T* qs, unsigned qstride, int rows,
                                                   int dim, int first, int last)
    {
        static_assert(kSquares % kWave == 0);      // a wave's are of one side
        for (int job = first + stage_thread(); job < last; job += kBlock) {
            const bool query = Lanes::query(job);
            RowVec<T, 8> v[8];
            Float4 to[2];
            load_square<T>(query ? qs : ks, query ? qstride : kstride, rows, dim, Lanes::rows(job), Lanes::elements(job), v);
            load_scale(from.f, query, Lanes::rows(job), to);
            put_square(room, query, Lanes::rows(job), Lanes::elements(job), rows, dim, v, to);
        }
    }
};

template <int KT, int P>
__device__ __forceinline__ void read_rows(const Half8 (&a)[P][4 * KT][kWave], int m, int lane, Half8 (&to)[P][KT])
{
#pragma unroll
    for (int h = 0; h < P; ++h)
#pragma unroll
        for (int k = 0; k < KT; ++k) to[h][k] = row_of<KT>(a[h], m, k, lane);
}
template <int KT, int P>
__device__ __forceinline__ void read_turned(const Half8 (&a)[P][4 * KT][kWave], int j, int lane, Half8 (&to)[P][2])
{
#pragma unroll
    for (int h = 0; h < P; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k) to[h][k] = turned_of<KT>(a[h], j, k, lane);
}
// y = a f and z = b e: 32 K elements of the sum, a's and b's low parts where they have any.
template <int K, int NT, int P>
__device__ __forceinline__ void products_of(const Half8 (&a)[P][K], const HalfPair (&f)[K][NT], const Half8 (&b)[P][K], const HalfPair (&e)[K][NT], Float4 (&y)[NT],
                                            Float4 (&z)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) y[n] = z[n] = Float4(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int term = 0; term < (P > 1 ? 3 : 2); ++term)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                y[n] = mfma(a[term == 2 ? P - 1 : 0][k], term == 1 ? f[k][n].lo : f[k][n].hi, y[n]);
                z[n] = mfma(b[term == 2 ? P - 1 : 0][k], term == 1 ? e[k][n].lo : e[k][n].hi, z[n]);
            }
}
template <int K, int NT, int P>
__device__ __forceinline__ void products(const Half8 (&a)[P][K], const Half8 (&b)[P][K], const HalfPair (&f)[K][NT], Float4 (&y)[NT], Float4 (&z)[NT])
{
    products_of<K, NT, P>(a, f, b, f, y, z);
}

// y = a triangular matrix times the columns f (of 64 rows); kUpper: the transposed form; kExact: f has no low parts.
template <int NT, bool kUpper, bool kExact = false>
__device__ __forceinline__ void tri_products(const Half8 (&matrix)[2][kTriOperands][kWave], int lane, const HalfPair (&f)[2][NT], Float4 (&y)[4][NT])
{
    Half8 a[2][kTriOperands];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < kTriOperands; ++k) a[h][k] = matrix[h][k][lane];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) y[m][n] = Float4(0.0f);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int term = 0; term < 3; ++term)
#pragma unroll
            for (int m = 0; m < 4; ++m)
                if ((kUpper ? s >= m >> 1 : s <= m >> 1) && !(kExact && term == 1))
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        y[m][n] = mfma(a[term == 2][kUpper ? upper_operand(m, s) : lower_operand(m, s)], term == 1 ? f[s][n].lo : f[s][n].hi, y[m][n]);
}

// Walks whose operands fit into LDS twice leave the staging to four waves of their own: the next block's operands are made while this one's are used, one
// barrier a block, and loads, conversions and LDS writes (4300 cycles a block, where each wave makes its share) pass beside the products: 304 -> 239 us for 1 x 4096 rows of 32 heads.
template <class T, int KT> constexpr bool kHelped = !kSplit<T> && KT <= 4;
template <class T, int KT> constexpr int kWalkThreads = kHelped<T, KT> ? 2 * kBlock : kBlock;

// Where a sequence's blocks are, for staging.
template <class T>
struct StageFrom {
    const Block* blocks;
    const T *ks, *qs;
    long long krow, qrow;
    int heads, len, dim;

    template <class S> __device__ __forceinline__ void load(S& stage, int c) const
    {
        const int rows = len - c * kDeltaRows;
        stage.load(blocks[(long long)c * heads], ks + (long long)c * kDeltaRows * krow, (unsigned)krow, qs + (long long)c * kDeltaRows * qrow, (unsigned)qrow,
                   rows < kDeltaRows ? rows : kDeltaRows, dim);
    }
    template <class S, class Room> __device__ __forceinline__ void put(S& stage, Room& room, int c) const
    {
        const int rows = len - c * kDeltaRows;
        stage.put(room, blocks[(long long)c * heads], ks + (long long)c * kDeltaRows * krow, (unsigned)krow, qs + (long long)c * kDeltaRows * qrow, (unsigned)qrow,
                  rows < kDeltaRows ? rows : kDeltaRows, dim);
    }
    template <class S, class Room> __device__ __forceinline__ void put_queries(Room& room, int c) const
    {
        const int rows = len - c * kDeltaRows;
        S::put_now(room, blocks[(long long)c * heads], ks + (long long)c * kDeltaRows * krow, (unsigned)krow, qs + (long long)c * kDeltaRows * qrow, (unsigned)qrow,
                   rows < kDeltaRows ? rows : kDeltaRows, dim, S::kSquares, 2 * S::kSquares);
    }
};

// The staging waves' part: blocks from, from + step .. (n of them), each into the room that the others are not reading.
template <class S, class T, class Room>
__device__ __forceinline__ void stage_all(const StageFrom<T>& source, Room* rooms, int from, int step, int n)
{
    S stage;
    source.load(stage, from);
    source.put(stage, rooms[0], from);
    if (n > 1) source.load(stage, from + step);
    __syncthreads();
    for (int k = 1; k <= n; ++k) {
        if (k < n) {
            source.put(stage, rooms[k & 1], from + k * step);
            if (k + 1 < n) source.load(stage, from + (k + 1) * step);
        }
        __syncthreads();
    }
}

// 64 rows of a wave's columns as B operands; their power of two, per column.
template <int NT>
__device__ __forceinline__ void split_rows(const Float4 (&x)[4][NT], HalfPair (&f)[2][NT], float (&back)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const Scale by(over_column(larger(larger(larger(larger(0.0f, x[0][n]), x[1][n]), x[2][n]), x[3][n])));
        back[n] = by.back;
        f[0][n] = split(x[0][n], x[1][n], by.to);
        f[1][n] = split(x[2][n], x[3][n], by.to);
    }
}
// A state's.
template <int KT, int NT>
__device__ __forceinline__ void split_state(const Float4 (&s)[2 * KT][NT], HalfPair (&f)[KT][NT], float (&back)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j) m = larger(m, s[j][n]);
        const Scale by(over_column(m));
        back[n] = by.back;
#pragma unroll
        for (int k = 0; k < KT; ++k) f[k][n] = split(s[2 * k][n], s[2 * k + 1][n], by.to);
    }
}

// ---- delta_prepare -----------------------------------------------------------------------------------------------------------
constexpr int kTriStride = kDeltaRows + 4;      // floats of a row in LDS: rows and columns alike meet all banks

template <class T, int KT>
struct PrepareRoom {
    static constexpr int kParts = kSplit<T> ? 2 : 1;
    union {
        struct {
            Half8 keys[kParts][4 * KT][kDeltaRows], queries[kParts][4 * KT][kDeltaRows];      // 8 elements of every row
        };
        struct {
            float system[kDeltaRows][kTriStride], inverse[kDeltaRows][kTriStride];
        };
    };
    double sum[kDeltaRows];                       // G
    float key[kDeltaRows], query[kDeltaRows];     // factors of the fp16 operands: 2^e, over the row's length
    float beta[kDeltaRows], most[2][kWavesPerBlock];
    BlockFactors f;
};

// q's or k's rows as fp16, each with its largest magnitude's power of two taken out; sizes: what makes it up again.
template <class T, int KT, int kThreads>
struct RowLoad {
    typedef RowLanes<KT, kThreads> Lanes;
    static constexpr int kLanes = Lanes::kLanes, kAtOnce = Lanes::kAtOnce, kPasses = Lanes::kPasses;
    RowVec<T, 8> v[kPasses];

    __device__ __forceinline__ void load(const T* __restrict__ base, unsigned stride, int rows, int dim)
    {
        load_eights<T, kPasses>(base, stride, Lanes::row((int)threadIdx.x), kAtOnce, rows, threadIdx.x % kLanes, dim, v);
    }
    __device__ __forceinline__ void put(bool unit, int rows, int dim, Half8 (&to)[kSplit<T> ? 2 : 1][4 * KT][kDeltaRows], float* factor, float* scale)
    {
        const int e = threadIdx.x % kLanes;
        clear_eights<T, kPasses>(Lanes::place((int)threadIdx.x), kAtOnce, rows, e, dim, v);
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int t = Lanes::place((int)threadIdx.x) + k * kAtOnce;
            float m = 0.0f, squares = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m = larger(m, (float)v[k][i]);
                squares = __builtin_fmaf((float)v[k][i], (float)v[k][i], squares);
            }
            m = over_few(m, kLanes, Max());
            squares = over_few(squares, kLanes, Add());
            if (kLanes > 16) {
                m = __builtin_fmaxf(m, __shfl_xor(m, 16));
                squares += __shfl_xor(squares, 16);
            }
            Scale by(m);
            if (__is_same(T, _Float16)) by.to = by.back = 1.0f;
            Half8 hi, lo;
            to_halves<T>(v[k], by.to, hi, lo);
            if (kAtOnce > kDeltaRows && t >= kDeltaRows) continue;
            to[0][e][t ^ (e & 15)] = hi;
            if constexpr (kSplit<T>) to[1][e][t ^ (e & 15)] = lo;
            if (e == 0) {
                scale[t] = by.to;
                factor[t] = by.back * (unit ? 1.0f / __builtin_sqrtf(squares + 1e-6f) : 1.0f);
            }
        }
    }
};

// K K^T and Q K^T, without their factors: N tiles of columns from tile n0 on (those up to the rows' own), against the rows of tile m.  kTiles: tiles are tile_row's,
// otherwise rows 16 m ..
template <class T, int KT, bool kTiles, int N, int kParts>
__device__ __forceinline__ void key_products(const Half8 (&keys)[kParts][4 * KT][kDeltaRows], const Half8 (&queries)[kParts][4 * KT][kDeltaRows], int m, int n0,
                                             Float4 (&kk)[N], Float4 (&qk)[N])
{
    const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, r = lane & 15;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        kk[j] = qk[j] = Float4(0.0f);
        if (n0 + j <= (kTiles ? m | 1 : m))
#pragma unroll
            for (int s = 0; s < KT; ++s) {
                const int e = 4 * s + g, row = (kTiles ? tile_row(m, r) : 16 * m + r) ^ (e & 15), col = (kTiles ? tile_row(n0 + j, r) : 16 * (n0 + j) + r) ^ (e & 15);
                const Half8 b = keys[0][e][col];
                kk[j] = mfma(keys[0][e][row], b, kk[j]);
                qk[j] = mfma(queries[0][e][row], b, qk[j]);
                if constexpr (kParts == 2) {
                    const Half8 c = keys[1][e][col];
                    kk[j] = mfma(keys[0][e][row], c, kk[j]);
                    qk[j] = mfma(queries[0][e][row], c, qk[j]);
                    kk[j] = mfma(keys[1][e][row], b, kk[j]);
                    qk[j] = mfma(queries[1][e][row], b, qk[j]);
                }
            }
    }
}

// -(x y) for blocks of 16 x 16 of matrices in LDS: a result tile's rows are in the order that the next product's sum takes them.
__device__ __forceinline__ Float4 mfma_f32(float a, float b, Float4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// The inverse of I + system (strictly lower), 16 x 16 blocks: those of the diagonal by substitution, a column a lane; below it block (i, j) is
// -inverse(i, i) times the sum over k of system(i, k) inverse(k, j), one diagonal after the other.  All in fp32.  What lies above the diagonal in `inverse` is
// zero before and after.  Returns the largest magnitude that the lane has seen.
template <class Room>
__device__ __forceinline__ float invert(Room& room)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r = lane & 15;
    float most = 1.0f;
    {
        const int at = 16 * wave;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == r ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; j += 4) {
                const Float4 row = *reinterpret_cast<const Float4*>(&room.system[at + i][at + j]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j + k < i) s = __builtin_fmaf(-row[k], x[j + k], s);
            }
            x[i] = s;
            most = larger(most, s);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (g == i >> 2) room.inverse[at + i][at + r] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int d = 1; d < 4; ++d) {
        const int i = wave + d, j = wave;
        if (i < 4) {
            Float4 s(0.0f), y(0.0f);
            for (int k = j; k < i; ++k) {
                const Float4 row = *reinterpret_cast<const Float4*>(&room.system[16 * i + r][16 * k + 4 * g]);
#pragma unroll
                for (int q = 0; q < 4; ++q) s = mfma_f32(row[q], room.inverse[16 * k + 4 * g + q][16 * j + r], s);
            }
            const Float4 row = *reinterpret_cast<const Float4*>(&room.inverse[16 * i + r][16 * i + 4 * g]);
#pragma unroll
            for (int q = 0; q < 4; ++q) y = mfma_f32(row[q], s[q], y);
#pragma unroll
            for (int q = 0; q < 4; ++q) room.inverse[16 * i + 4 * g + q][16 * j + r] = -y[q];
            most = larger(most, y);
        }
        __syncthreads();
    }
    return most;
}

// A triangular matrix in LDS, zeros above its diagonal, as operands, hi and lo; kUpper: its transpose.
template <bool kUpper, int kWaves = kWavesPerBlock>
__device__ __forceinline__ void store_operands(const float (&a)[kDeltaRows][kTriStride], float to, Half8 (&out)[2][kTriOperands][kWave])
{
    const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, r = lane & 15;
    for (int k = threadIdx.x >> 6; k < kTriOperands; k += kWaves) {
        // lower: (0, 0) (1, 0) (2, 0) (2, 1) (3, 0) (3, 1); upper: (0, 0) (0, 1) (1, 0) (1, 1) (2, 1) (3, 1)
        const int m = kUpper ? (k < 4 ? k >> 1 : k - 2) : (k < 2 ? k : 1 + (k >> 1)), s = kUpper ? (k < 4 ? k & 1 : 1) : (k < 2 ? 0 : k & 1);
        const int row = tile_row(m, r), col = 32 * s + 8 * g;
        float v[8];
        if constexpr (kUpper) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = a[col + i][row];
        } else {
            const Float4 u = *reinterpret_cast<const Float4*>(&a[row][col]), w = *reinterpret_cast<const Float4*>(&a[row][col + 4]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = u[i];
                v[i + 4] = w[i];
            }
        }
        const HalfPair p = split(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], to);
        out[0][k][lane] = p.hi;
        out[1][k][lane] = p.lo;
    }
}

// Over the block; `room`: a float a wave.
template <int kWaves = kWavesPerBlock>
__device__ __forceinline__ float over_block(float m, float* room)
{
    m = over_column(over_few(m, 16, Max()));
    if ((threadIdx.x & (kWave - 1)) == 0) room[threadIdx.x >> 6] = m;
    __syncthreads();
    m = room[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = __builtin_fmaxf(m, room[w]);
    return m;
}

// The block's matrices and factors for every head of a key head.  kBack: for the gradients, the inverse of I + diag(b) A and both transposed.
template <class T, int KT, bool kBack>
__device__ __forceinline__ void prepare_block(const DeltaParams& p, const Piece& piece, long long slot, int key_head, PrepareRoom<T, KT>& room)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r = lane & 15, many = p.heads / p.key_heads;
    {
        RowLoad<T, KT, kBlock> k, q;
        k.load(sequence_base<const T>(p.k, p.pieces, piece) + piece.row0 * p.k.row + key_head * p.k_head, (unsigned)p.k.row, piece.n, p.key_dim);
        q.load(sequence_base<const T>(p.q, p.pieces, piece) + piece.row0 * p.q.row + key_head * p.q_head, (unsigned)p.q.row, piece.n, p.key_dim);
        k.put(p.unit, piece.n, p.key_dim, room.keys, room.key, room.f.key);
        q.put(p.unit, piece.n, p.key_dim, room.queries, room.query, room.f.query);
    }
    __syncthreads();
    Float4 kk[4], qk[4];
    key_products<T, KT, false, 4>(room.keys, room.queries, wave, 0, kk, qk);
    for (int h = key_head * many; h < (key_head + 1) * many; ++h) {
        __syncthreads();                          // the operands, or the last head's matrices, are done with
        if (wave == 0) {
            const bool there = lane < piece.n;
            const long long at = piece.row0 + (there ? lane : 0);
            float gate = 0.0f, beta = 0.0f;
            if (there && p.g.d) gate = sequence_base<const float>(p.g, p.pieces, piece)[at * p.g.row + h];
            if (there) beta = sequence_base<const float>(p.beta, p.pieces, piece)[at * p.beta.row + h];
            // sums in 64 bits: a row that forgets nearly all must not cost the others' differences their digits
            double sum = gate < -1000.0f ? -1000.0 : (double)gate;
#pragma unroll
            for (int x = 1; x < kWave; x *= 2) {
                const double before = __shfl_up(sum, x);
                if (lane >= x) sum += before;
            }
            const double all = __shfl(sum, kWave - 1);
            room.sum[lane] = sum;
            room.beta[lane] = beta;
            const float up = exp2_fast(kLog2e * (float)sum);
            room.f.reads[lane] = up * room.key[lane];
            room.f.beta[lane] = beta;
            room.f.writes[lane] = exp2_fast(kLog2e * (float)(all - sum)) * room.key[lane];
            room.f.asks[lane] = p.scale * up * room.query[lane];
            if (lane == 0) room.f.total = exp2_fast(kLog2e * (float)all);
        }
        __syncthreads();
        float most = 0.0f, query[4], key[4];
        double sum[4];
        const int row0 = 16 * wave + 4 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum[i] = room.sum[row0 + i];
            query[i] = p.scale * room.query[row0 + i];
            key[i] = room.key[row0 + i] * (kBack ? room.beta[row0 + i] : 1.0f);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = 16 * j + r;
            if (j > wave) {
#pragma unroll
                for (int i = 0; i < 4; ++i) room.inverse[row0 + i][col] = 0.0f;
                continue;
            }
            const double before = room.sum[col];
            const float own = room.key[col], beta = kBack ? 1.0f : room.beta[col];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = col <= row0 + i ? exp2_fast(kLog2e * (float)(sum[i] - before)) * own : 0.0f;
                const float m = query[i] * qk[j][i] * d;
                most = larger(most, m);
                room.system[row0 + i][col] = col < row0 + i ? key[i] * kk[j][i] * (d * beta) : 0.0f;
                room.inverse[row0 + i][col] = col <= row0 + i ? m : 0.0f;
            }
        }
        most = over_block(most, room.most[0]);
        Block& out = p.blocks[slot * p.heads + h];
        const Scale mix(most);
        store_operands<kBack>(room.inverse, mix.to, out.mix);
        __syncthreads();
        most = over_block(invert(room), room.most[1]);
        const Scale solve(most);
        store_operands<kBack>(room.inverse, solve.to, out.solve);
        if (tid == 0) {
            room.f.solve_back = solve.back;
            room.f.mix_back = mix.back;
        }
        __syncthreads();
        const float* from = reinterpret_cast<const float*>(&room.f);
        float* to = reinterpret_cast<float*>(&out.f);
        for (int i = tid; i < (int)(sizeof(BlockFactors) / 4); i += kBlock) to[i] = from[i];
    }
}

}  // namespace ssam
