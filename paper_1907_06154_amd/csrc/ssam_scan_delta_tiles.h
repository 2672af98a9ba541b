// Device code of the scan with matrix states that its forward and backward kernels share: q and k as fp16 operands, the block's matrices, and
// products with them.
#pragma once
#include "ssam_scan_delta.h"

namespace ssam {

template <class T> constexpr bool kSplit = sizeof(T) == 4;      // q and k are pairs of fp16 too

// Eight elements of a row as fp16, `to` a power of two; the low parts where T has more bits than fp16.
template <class T>
__device__ __forceinline__ void to_halves(const RowVec<T, 8>& v, float to, Half8& hi, Half8& lo)
{
    if constexpr (__is_same(T, _Float16)) {
        hi = v;
    } else if constexpr (kSplit<T>) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) split2(v[i] * to, v[i + 1] * to, hi, lo, i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const auto h = __builtin_amdgcn_cvt_pkrtz((float)v[i] * to, (float)v[i + 1] * to);      // eight bits: exact
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

// 8 rows x 8 elements, rows 8 b .. and elements 8 e .., zeros outside.
template <class T>
__device__ __forceinline__ void load_square(const T* __restrict__ base, long long stride, int row0, int rows, int dim, int b, int e, RowVec<T, 8> (&v)[8])
{
    const int have = dim - 8 * e;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = 8 * b + i < rows && have > 0 ? load_row_vec<T, 8>(base + (long long)(row0 + 8 * b + i) * stride + 8 * e, have) : RowVec<T, 8>(T(0));
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

// The rows of a block as operands: k's in both forms, q's as rows (kTurn: turned).  kKeys, kQueries: which of them.
template <class T, int KT, bool kKeys, bool kQueries, bool kTurn>
__device__ __forceinline__ void stage_rows(WalkRoom<T, KT>& room, const BlockFactors& f, const T* __restrict__ ks, long long kstride, const T* __restrict__ qs,
                                           long long qstride, int row0, int rows, int dim)
{
    constexpr int kAcross = 4 * KT, kSquares = 8 * kAcross;      // squares of 8 x 8 in a block's keys
    for (int job = threadIdx.x; job < (kKeys && kQueries ? 2 : 1) * kSquares; job += kBlock) {
        const bool query = kKeys && kQueries ? job >= kSquares : kQueries;
        const int b = (job % kSquares) / kAcross, e = job % kAcross;
        RowVec<T, 8> v[8];
        load_square(query ? qs : ks, query ? qstride : kstride, row0, rows, dim, b, e, v);
        const float* to = query ? f.query : f.key;
        Half8 hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) to_halves<T>(v[i], __is_same(T, _Float16) ? 1.0f : to[8 * b + i], hi[i], lo[i]);
        if (query) {
            if constexpr (kQueries && kTurn) put_turned<T, KT>(hi, lo, b, e, room.queries());
            else if constexpr (kQueries) put_rows<T, KT>(hi, lo, b, e, room.queries());
        } else if constexpr (kKeys) {
            put_rows<T, KT>(hi, lo, b, e, room.keys);
            put_turned<T, KT>(hi, lo, b, e, room.turned_keys);
        }
    }
}

__device__ __forceinline__ void stage_block(Block& to, const Block& from)
{
    constexpr int kVecs = sizeof(Block) / 16;
    static_assert(sizeof(Block) % 16 == 0);
    const Float4* a = reinterpret_cast<const Float4*>(&from);
    Float4* b = reinterpret_cast<Float4*>(&to);
    for (int i = threadIdx.x; i < kVecs; i += kBlock) b[i] = a[i];
}

// y = a times the columns f: rows of tile m (32 KT elements each), or the turned ones of tile j (64 rows).
template <int KT, int NT, int kParts>
__device__ __forceinline__ void rows_product(const Half8 (&a)[kParts][4 * KT][kWave], int m, int lane, const HalfPair (&f)[KT][NT], Float4 (&y)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) y[n] = Float4(0.0f);
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        const Half8 hi = row_of<KT>(a[0], m, k, lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            y[n] = mfma(hi, f[k][n].hi, y[n]);
            y[n] = mfma(hi, f[k][n].lo, y[n]);
        }
        if constexpr (kParts > 1) {
            const Half8 lo = row_of<KT>(a[1], m, k, lane);
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n] = mfma(lo, f[k][n].hi, y[n]);
        }
    }
}
template <int KT, int NT, int kParts>
__device__ __forceinline__ void turned_product(const Half8 (&a)[kParts][4 * KT][kWave], int j, int lane, const HalfPair (&f)[2][NT], Float4 (&y)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) y[n] = Float4(0.0f);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const Half8 hi = turned_of<KT>(a[0], j, k, lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            y[n] = mfma(hi, f[k][n].hi, y[n]);
            y[n] = mfma(hi, f[k][n].lo, y[n]);
        }
        if constexpr (kParts > 1) {
            const Half8 lo = turned_of<KT>(a[1], j, k, lane);
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n] = mfma(lo, f[k][n].hi, y[n]);
        }
    }
}

// y = rows of tile m of a lower triangular matrix times the columns f (of 64 rows).
template <int NT>
__device__ __forceinline__ void lower_product(const Half8 (&matrix)[2][kTriOperands][kWave], int m, int lane, const HalfPair (&f)[2][NT], Float4 (&y)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) y[n] = Float4(0.0f);
#pragma unroll
    for (int s = 0; s < 2; ++s)
        if (s <= m >> 1) {
            const Half8 hi = matrix[0][lower_operand(m, s)][lane], lo = matrix[1][lower_operand(m, s)][lane];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                y[n] = mfma(hi, f[s][n].hi, y[n]);
                y[n] = mfma(hi, f[s][n].lo, y[n]);
                y[n] = mfma(lo, f[s][n].hi, y[n]);
            }
        }
}

// The same for rows of tile m of an upper one.
template <int NT>
__device__ __forceinline__ void upper_product(const Half8 (&matrix)[2][kTriOperands][kWave], int m, int lane, const HalfPair (&f)[2][NT], Float4 (&y)[NT])
{
#pragma unroll
    for (int n = 0; n < NT; ++n) y[n] = Float4(0.0f);
#pragma unroll
    for (int s = 0; s < 2; ++s)
        if (s >= m >> 1) {
            const Half8 hi = matrix[0][upper_operand(m, s)][lane], lo = matrix[1][upper_operand(m, s)][lane];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                y[n] = mfma(hi, f[s][n].hi, y[n]);
                y[n] = mfma(hi, f[s][n].lo, y[n]);
                y[n] = mfma(lo, f[s][n].hi, y[n]);
            }
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
constexpr int kTriStride = kDeltaRows + 1;      // floats of a row in LDS

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
template <class T, int KT>
__device__ __forceinline__ void load_rows(const T* __restrict__ base, long long stride, int rows, int dim, bool unit, Half8 (&to)[kSplit<T> ? 2 : 1][4 * KT][kDeltaRows],
                                          float* factor, float* scale)
{
    constexpr int kLanes = 4 * KT;                // of a row
    const int e = threadIdx.x % kLanes, have = dim - 8 * e;
#pragma unroll
    for (int t = threadIdx.x / kLanes; t < kDeltaRows; t += kBlock / kLanes) {
        const RowVec<T, 8> v = t < rows && have > 0 ? load_row_vec<T, 8>(base + (long long)t * stride + 8 * e, have) : RowVec<T, 8>(T(0));
        float m = 0.0f, squares = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m = larger(m, (float)v[i]);
            squares = __builtin_fmaf((float)v[i], (float)v[i], squares);
        }
#pragma unroll
        for (int x = 1; x < kLanes; x *= 2) {
            m = __builtin_fmaxf(m, __shfl_xor(m, x));
            squares += __shfl_xor(squares, x);
        }
        Scale by(m);
        if (__is_same(T, _Float16)) by.to = by.back = 1.0f;
        Half8 hi, lo;
        to_halves<T>(v, by.to, hi, lo);
        to[0][e][t ^ (e & 15)] = hi;
        if constexpr (kSplit<T>) to[1][e][t ^ (e & 15)] = lo;
        if (e == 0) {
            scale[t] = by.to;
            factor[t] = by.back * (unit ? 1.0f / __builtin_sqrtf(squares + 1e-6f) : 1.0f);
        }
    }
}

// K K^T and Q K^T, without their factors: wave w has the rows of tile w (kTiles: tile_row, otherwise 16 w ..) and the columns up to them.
template <class T, int KT, bool kTiles, int kParts>
__device__ __forceinline__ void key_products(const Half8 (&keys)[kParts][4 * KT][kDeltaRows], const Half8 (&queries)[kParts][4 * KT][kDeltaRows],
                                             Float4 (&kk)[4], Float4 (&qk)[4])
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        kk[j] = qk[j] = Float4(0.0f);
        if (j <= (kTiles ? wave | 1 : wave))
#pragma unroll
            for (int s = 0; s < KT; ++s) {
                const int e = 4 * s + g, row = (kTiles ? tile_row(wave, r) : 16 * wave + r) ^ (e & 15), col = (kTiles ? tile_row(j, r) : 16 * j + r) ^ (e & 15);
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
// -inverse(i, i) times the sum over k of system(i, k) inverse(k, j), one diagonal after the other.  All in fp32.
template <class Room>
__device__ __forceinline__ void invert(Room& room)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r = lane & 15;
    {
        const int at = 16 * wave;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == r ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; ++j) s = __builtin_fmaf(-room.system[at + i][at + j], x[j], s);
            x[i] = s;
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
            for (int k = j; k < i; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) s = mfma_f32(room.system[16 * i + r][16 * k + 4 * g + q], room.inverse[16 * k + 4 * g + q][16 * j + r], s);
#pragma unroll
            for (int q = 0; q < 4; ++q) y = mfma_f32(room.inverse[16 * i + r][16 * i + 4 * g + q], s[q], y);
#pragma unroll
            for (int q = 0; q < 4; ++q) room.inverse[16 * i + 4 * g + q][16 * j + r] = -y[q];
        }
        __syncthreads();
    }
}

// A triangular matrix in LDS as operands, hi and lo; kUpper: its transpose.
template <bool kUpper>
__device__ __forceinline__ void store_operands(const float (&a)[kDeltaRows][kTriStride], float to, Half8 (&out)[2][kTriOperands][kWave])
{
    const int lane = threadIdx.x & (kWave - 1), g = lane >> 4, r = lane & 15;
    for (int k = threadIdx.x >> 6; k < kTriOperands; k += kWavesPerBlock) {
        // lower: (0, 0) (1, 0) (2, 0) (2, 1) (3, 0) (3, 1); upper: (0, 0) (0, 1) (1, 0) (1, 1) (2, 1) (3, 1)
        const int m = kUpper ? (k < 4 ? k >> 1 : k - 2) : (k < 2 ? k : 1 + (k >> 1)), s = kUpper ? (k < 4 ? k & 1 : 1) : (k < 2 ? 0 : k & 1);
        const int row = tile_row(m, r), col = 32 * s + 8 * g;
        Half8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float u = kUpper ? (col + i >= row ? a[col + i][row] : 0.0f) : col + i <= row ? a[row][col + i] : 0.0f;
            const float v = kUpper ? (col + i + 1 >= row ? a[col + i + 1][row] : 0.0f) : col + i + 1 <= row ? a[row][col + i + 1] : 0.0f;
            split2(u * to, v * to, hi, lo, i);
        }
        out[0][k][lane] = hi;
        out[1][k][lane] = lo;
    }
}

// Over the block; `room`: a float a wave.
__device__ __forceinline__ float over_block(float m, float* room)
{
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, x));
    if ((threadIdx.x & (kWave - 1)) == 0) room[threadIdx.x >> 6] = m;
    __syncthreads();
    m = room[0];
#pragma unroll
    for (int w = 1; w < kWavesPerBlock; ++w) m = __builtin_fmaxf(m, room[w]);
    return m;
}

// The block's matrices and factors for every head of a key head.  kBack: for the gradients, the inverse of I + diag(b) A and both transposed.
template <class T, int KT, bool kBack>
__device__ __forceinline__ void prepare_block(const DeltaParams& p, const Piece& piece, long long slot, int key_head, PrepareRoom<T, KT>& room)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r = lane & 15, many = p.heads / p.key_heads;
    load_rows<T, KT>(sequence_base<const T>(p.k, p.pieces, piece) + piece.row0 * p.k.row + key_head * p.k_head, p.k.row, piece.n, p.key_dim, p.unit, room.keys,
                     room.key, room.f.key);
    load_rows<T, KT>(sequence_base<const T>(p.q, p.pieces, piece) + piece.row0 * p.q.row + key_head * p.q_head, p.q.row, piece.n, p.key_dim, p.unit, room.queries,
                     room.query, room.f.query);
    __syncthreads();
    Float4 kk[4], qk[4];
    key_products<T, KT, false>(room.keys, room.queries, kk, qk);
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
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 16 * wave + 4 * g + i, col = 16 * j + r;
                float a = 0.0f, m = 0.0f;
                if (col <= row) {
                    const float d = exp2_fast(kLog2e * (float)(room.sum[row] - room.sum[col])) * room.key[col];
                    m = p.scale * room.query[row] * qk[j][i] * d;
                    if (col < row) a = room.key[row] * kk[j][i] * d * room.beta[kBack ? row : col];
                }
                most = larger(most, m);
                room.system[row][col] = a;
                room.inverse[row][col] = m;
            }
        most = over_block(most, room.most[0]);
        Block& out = p.blocks[slot * p.heads + h];
        const Scale mix(most);
        store_operands<kBack>(room.inverse, mix.to, out.mix);
        __syncthreads();
        invert(room);
        most = 0.0f;
        for (int i = tid; i < kDeltaRows * kDeltaRows; i += kBlock)
            if (i / kDeltaRows >= i % kDeltaRows) most = larger(most, room.inverse[i / kDeltaRows][i % kDeltaRows]);
        most = over_block(most, room.most[1]);
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
