// Gradients of the scan with matrix states (ssam_scan_delta_backward).  In a block of 64 rows, with the notation of ssam_scan_delta.h, P = scale
// (Q K^T o D), T = (I + diag(b) A)^-1, dO the gradient of O and dS1 that of the state behind the block:
//     dU = P^T dO + (exp(G_C - G) K) dS1,   dY = T^T dU,   dV = dX = b dY,
//     dS0 = exp(G_C) dS1 + scale (exp(G) Q)^T dO - (exp(G) K)^T dX                                      (delta_back_walk, block after block)
//     dbeta = rows of dY . R,   dP = scale (dO U^T) o D,   dA = -(dX U^T) o D, strictly lower,
//     dQ = scale exp(G) (dO S0^T) + dP K,   reads = dA K - exp(G) (dX S0^T),
//     last = exp(G_C - G) (U dS1^T),        writes = dP^T Q + dA^T K + last,   dK = reads + writes    (delta_back_rows, all blocks at once)
// The decay of row t lies between every write j < t and every read i >= t, so dg_t is the sum over these pairs of dP P + dA A (their parts before
// the keys' products), of what the rows i >= t have from S0, of the k.last of the rows j < t, and of exp(G_C) <S0, dS1>: no differences.
// bf16, 4 x 2048 rows of 16 heads of 128 x 128: 45 us for the blocks' matrices, 184 for the walk (bound as the forward one), 376 for the rows, one block
// of eight waves a compute unit (125 KB of LDS) whose phases wait for memory and for one another: some 100000 cycles a block, of which the two
// states' products take about 13, the products between rows 14, the turned products and what leaves 22, the first loads 12 %.
#include "ssam_scan_delta_tiles.h"

namespace ssam {
namespace {

struct DeltaBackParams {
    DeltaParams f;               // final and out unused; marks: what the forward call left; state: the gradient of the last state
    ssam_rows grad_out, grad_q, grad_k, grad_v, grad_g, grad_beta;
    long long grad_out_head, grad_v_head, grad_key_head;
    float* grad_state;
    float* behind;               // as marks: dS1 and dY of every block and head
};

template <class T, int KT>
__global__ __launch_bounds__(kBlock) void delta_back_prepare(DeltaParams p)
{
    __shared__ PrepareRoom<T, KT> room;
    const int slot = (int)(blockIdx.x / p.key_heads), key_head = (int)(blockIdx.x % p.key_heads);
    const Piece piece = find_piece(p.pieces, slot);
    if (piece.seq < 0 || piece.n <= 0) return;
    prepare_block<T, KT, true>(p, piece, slot, key_head, room);
}

// One wave: 16 NT columns of the gradient of a head's state, from the last block to the first.  (Blocks in the launch's order: with those of one XCD next to one
// another, as in delta_walk, 4 x 2048 rows of 16 heads take the same 803 us, both walks and the rows together.)
template <class T, int KT, int NT>
__global__ __launch_bounds__((kWalkThreads<T, KT>)) void delta_back_walk(DeltaBackParams b)
{
    const DeltaParams& p = b.f;
    constexpr bool kHelp = kHelped<T, KT>;
    __shared__ WalkRoom<T, KT> rooms[kHelp ? 2 : 1];
    typedef Stage<T, KT, true> S;
    typedef Columns<T, NT, kSplit<T> && (KT > 4)> Cols;
    __shared__ typename Cols::Room columns[kWavesPerBlock];
    constexpr int kParts = kSplit<T> ? 2 : 1;       // of q and k
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r16 = lane & 15;
    const int tile = (int)(blockIdx.x % p.tiles), head = (int)(blockIdx.x / p.tiles % p.heads), seq = (int)(blockIdx.x / p.tiles / p.heads);
    const int key_head = head / (p.heads / p.key_heads);
    int first, len;
    span_of(p.pieces, seq, first, len);
    const int blocks = (len + kDeltaRows - 1) / kDeltaRows;
    const long long slot0 = p.pieces.begin ? first_slot(p.pieces, seq) : (long long)seq * p.pieces.per;
    const int col0 = (tile * kWavesPerBlock + __builtin_amdgcn_readfirstlane(wave)) * 16 * NT, c0 = col0 + r16;
    const Piece whole{seq, first, len, 0, len};
    const long long end = (long long)(blocks - 1) * kDeltaRows;                                  // first row of the last block
    const StageFrom<T> source{p.blocks + slot0 * p.heads + head, sequence_base<const T>(p.k, p.pieces, whole) + key_head * p.k_head,
                              sequence_base<const T>(p.q, p.pieces, whole) + key_head * p.q_head, p.k.row, p.q.row, p.heads, len, p.key_dim};
    if (kHelp && wave >= kWavesPerBlock) {
        if (blocks > 0) stage_all<S>(source, rooms, blocks - 1, -1, blocks);
        return;
    }
    if (kHelp && col0 >= p.value_dim) {        // no columns: the barriers alone, as many as stage_all has
        if (blocks > 0)
            for (int c = 0; c <= blocks; ++c) __syncthreads();
        return;
    }
    const T* dos = sequence_base<const T>(b.grad_out, p.pieces, whole) + head * b.grad_out_head + end * b.grad_out.row;
    T* dvs = b.grad_v.d ? sequence_base<T>(b.grad_v, p.pieces, whole) + head * b.grad_v_head + end * b.grad_v.row : nullptr;
    const long long state_at = ((long long)seq * p.heads + head) * p.key_dim * p.value_dim;
    const unsigned ostride = (unsigned)b.grad_out.row, vstride = (unsigned)b.grad_v.row;

    Float4 s[2 * KT][NT];
    if (p.state) {
        load_state<KT, NT>(p.state + state_at, p.value_dim, p.key_dim, c0, s);
    } else {
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n) s[j][n] = Float4(0.0f);
    }
    S stage;
    Cols v;
    int rows = len - (blocks - 1) * kDeltaRows;
    if (blocks > 0) {
        if (!kHelp) source.load(stage, blocks - 1);
        v.load(dos, ostride, rows, col0, p.value_dim);
        if (kHelp) __syncthreads();
    }
    for (int c = blocks - 1; c >= 0; --c) {
        WalkRoom<T, KT>& room = rooms[kHelp ? (blocks - 1 - c) & 1 : 0];
        if (!kHelp) {
            __syncthreads();
            source.put(stage, room, c);
        }
        float* const behind = mark_of(b.behind, p, slot0 + c, head);
        store_state<KT, NT>(behind, p.value_dim, p.key_dim, c0, s);
        Float4 o[4][NT], x[4][NT];       // dO; dU, dY, dX
        v.values(columns[wave], rows, o);
        if (!kHelp) __syncthreads();
        const int this_rows = rows;
        if (c > 0) {
            dos -= (long long)kDeltaRows * b.grad_out.row;
            rows = kDeltaRows;
            if (!kHelp) source.load(stage, c - 1);
            v.load(dos, ostride, rows, col0, p.value_dim);
        }
        {
            HalfPair f[KT][NT];
            float back[NT];
            Half8 key[2][2][kParts][KT];
            read_rows<KT, kParts>(room.keys, 0, lane, key[0][0]);
            read_rows<KT, kParts>(room.keys, 1, lane, key[0][1]);
            split_state<KT, NT>(s, f, back);
#pragma unroll
            for (int m = 0; m < 4; m += 2) {
                if (m == 0 && !S::kOnePlace) {
                    read_rows<KT, kParts>(room.keys, 2, lane, key[1][0]);
                    read_rows<KT, kParts>(room.keys, 3, lane, key[1][1]);
                }
                in_order();
                if (m == 2 && S::kOnePlace) {       // (pairs of long keys: no registers for two steps)
                    read_rows<KT, kParts>(room.keys, 2, lane, key[0][0]);
                    read_rows<KT, kParts>(room.keys, 3, lane, key[0][1]);
                }
                const int now = S::kOnePlace ? 0 : m >> 1;
                products<KT, NT, kParts>(key[now][0], key[now][1], f, x[m], x[m + 1]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const Float4 writes = *reinterpret_cast<const Float4*>(&room.m.f.writes[tile_row(m + k, 4 * g)]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) x[m + k][n] *= writes * back[n];
                }
            }
        }
        if constexpr (S::kOnePlace) {
            __syncthreads();
            source.template put_queries<S>(room, c);
            __syncthreads();
        }
        HalfPair f[2][NT];
        float back[NT];
        split_rows<NT>(o, f, back);
        {
            Float4 a[4][NT];
            tri_products<NT, true>(room.m.mix, lane, f, a);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) x[m][n] += a[m][n] * (back[n] * room.m.f.mix_back);
        }
        split_rows<NT>(x, f, back);
        tri_products<NT, true>(room.m.solve, lane, f, x);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) x[m][n] *= back[n] * room.m.f.solve_back;
        store_tiles<NT>(behind + (size_t)p.key_dim * p.value_dim, p.value_dim, c0, x);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const Float4 beta = *reinterpret_cast<const Float4*>(&room.m.f.beta[tile_row(m, 4 * g)]);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[m][n] *= beta;
        }
        if (dvs) Cols::store(columns[wave], dvs, vstride, this_rows, col0, p.value_dim, x);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const Float4 reads = *reinterpret_cast<const Float4*>(&room.m.f.reads[tile_row(m, 4 * g)]),
                         asks = *reinterpret_cast<const Float4*>(&room.m.f.asks[tile_row(m, 4 * g)]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                x[m][n] *= -reads;
                o[m][n] *= asks;
            }
        }
        if (dvs) dvs -= (long long)kDeltaRows * b.grad_v.row;
        HalfPair fo[2][NT];
        float back_o[NT];
        Half8 key[2][kParts][2], query[2][kParts][2];
        read_turned<KT, kParts>(room.turned_keys, 0, lane, key[0]);
        read_turned<KT, kParts>(room.queries(), 0, lane, query[0]);
        split_rows<NT>(x, f, back);
        split_rows<NT>(o, fo, back_o);
        const float total = room.m.f.total;
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j) {
            const int now = j & 1;
            if (j + 1 < 2 * KT) {
                read_turned<KT, kParts>(room.turned_keys, j + 1, lane, key[now ^ 1]);
                read_turned<KT, kParts>(room.queries(), j + 1, lane, query[now ^ 1]);
            }
            in_order();
            Float4 a[NT], q[NT];
            products_of<2, NT, kParts>(key[now], f, query[now], fo, a, q);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j][n][i] = __builtin_fmaf(total, s[j][n][i], __builtin_fmaf(a[n][i], back[n], q[n][i] * back_o[n]));
        }
        if (kHelp) __syncthreads();
    }
    if (b.grad_state) store_state<KT, NT>(b.grad_state + state_at, p.value_dim, p.key_dim, c0, s);
}

// ---- gradients of q, k, g and beta ----------------------------------------------------------------------------------------
constexpr int kAcross = 128;               // values taken together
constexpr int kAcrossSteps = kAcross / 32;
constexpr int kRowWaves = 8, kRowThreads = kRowWaves * kWave;      // half the registers of sums a wave, and two of them on a SIMD

template <class T, int KT>
struct RowsRoom {
    static constexpr int kParts = kSplit<T> ? 2 : 1;
    static constexpr bool kKept = kParts * KT <= 4;      // q's and k's rows stay in LDS beside everything else
    typedef Half8 Rows[kParts][4 * KT][kDeltaRows];      // 8 elements of every row
    struct Operands {                                    // rows t (tile_row), 32 values
        Half8 grad[kParts][4 * kAcrossSteps][kWave], x[2][4 * kAcrossSteps][kWave], u[2][4 * kAcrossSteps][kWave];
    };
    struct Triangles {
        Half8 turned[kParts][4 * KT][kWave];
        Half8 tri[4][2][kTriOperands][kWave];
        float matrix[kDeltaRows][kTriStride];
    };
    struct Both {
        Rows keys, queries;
    };
    struct Nothing {};
    union {
        std::conditional_t<kKept, Nothing, Both> first;
        Operands o;
        Triangles t;
    };
    std::conditional_t<kKept, Both, Nothing> kept;
    double sum[kDeltaRows];
    float back[3][kDeltaRows];             // powers of two of grad's, x's and u's rows
    float up[kDeltaRows], rest[kDeltaRows], beta[kDeltaRows], dbeta[kDeltaRows];
    float key[kDeltaRows], query[kDeltaRows], key_back[kDeltaRows], query_back[kDeltaRows];
    float dots[2][kRowWaves][kDeltaRows], pairs[kRowWaves][kDeltaRows];
    float most[2][kRowWaves], inner[kRowWaves], total;

    __device__ __forceinline__ Both& rows()
    {
        if constexpr (kKept) return kept;
        else return first;
    }
};

// Tile and row in it of row t: the inverse of tile_row.
__device__ __forceinline__ int tile_of(int t) { return 2 * (t >> 5) + (t >> 2 & 1); }
__device__ __forceinline__ int row_in_tile(int t) { return 4 * (t >> 3 & 3) + (t & 3); }

// Rows' sums over the lanes and waves of v[m][i], what a lane has for row tile_row(m, 4 g + i); to be read after a barrier.
__device__ __forceinline__ void put_dots(const float (&v)[4][4], float (&to)[kRowWaves][kDeltaRows])
{
    const int lane = threadIdx.x & (kWave - 1), g = lane >> 4;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float s = over_few(v[m][i], 16, Add());
            if ((lane & 15) == 0) to[threadIdx.x >> 6][tile_row(m, 4 * g + i)] = s;
        }
}
__device__ __forceinline__ float dot_of(const float (&from)[kRowWaves][kDeltaRows], int t)
{
    float s = from[0][t];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) s += from[w][t];
    return s;
}

// dO, dY and R of a block's rows, 8 of kAcross values a lane, 16 lanes a row.
template <class T>
struct RowData {
    static constexpr int kPasses = kDeltaRows * 16 / kRowThreads;
    RowVec<T, 8> o[kPasses];
    Eight y[kPasses], u[kPasses];

    __device__ __forceinline__ void load(int tid, const T* dos, unsigned stride, const float* ys, const float* us, int dim, int rows, int v0)
    {
        const int at = v0 + 8 * (tid & 15), row = (tid >> 4);
        if (dim >= 8) {
            const unsigned c = (unsigned)(at + 8 <= dim ? at : dim - 8);
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const int t = row + k * (kRowThreads / 16);
                __builtin_memcpy(&o[k], dos + ((unsigned)(t < rows ? t : rows - 1) * stride + c), sizeof(o[k]));
                y[k].load(ys + ((unsigned)(t * dim) + c));
                u[k].load(us + ((unsigned)(t * dim) + c));
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const int t = row + k * (kRowThreads / 16);
                o[k] = load_few(dos + (unsigned)(t < rows ? t : rows - 1) * stride, dim);
                y[k].load(ys + (unsigned)(t * dim), dim);
                u[k].load(us + (unsigned)(t * dim), dim);
            }
        }
    }
    // What pass k has, zeros where nothing is.
    __device__ __forceinline__ void take(int tid, int k, int rows, int dim, int v0)
    {
        const int at = v0 + 8 * (tid & 15);
        if ((tid >> 4) + k * (kRowThreads / 16) >= rows) o[k] = RowVec<T, 8>(T(0));
        if (v0 + kAcross <= dim) return;
        if (dim % 8) {
            o[k] = shifted(o[k], shift_of(at, dim));
            y[k].shift(shift_of(at, dim));
            u[k].shift(shift_of(at, dim));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i >= dim) o[k][i] = T(0);
        y[k].clear(dim - at);
        u[k].clear(dim - at);
    }
};
// Some of a state's rows, 8 of 32 values a lane and step.
struct StateRow {
    Eight v[kAcrossSteps];
    __device__ __forceinline__ void load(const float* state, int d, int key_dim, int dim, int v0)
    {
        const int g = (threadIdx.x & (kWave - 1)) >> 4;
        const float* const row = state + (size_t)(d < key_dim ? d : key_dim - 1) * dim;
        if (dim >= 8) {
#pragma unroll
            for (int s = 0; s < kAcrossSteps; ++s) {
                const int at = v0 + 32 * s + 8 * g;
                v[s].load(row + (unsigned)(at + 8 <= dim ? at : dim - 8));
            }
        } else {
#pragma unroll
            for (int s = 0; s < kAcrossSteps; ++s) v[s].load(row, dim);
        }
    }
    __device__ __forceinline__ float clear(int d, int key_dim, int dim, int v0)      // and the largest magnitude
    {
        const int g = (threadIdx.x & (kWave - 1)) >> 4;
        if (v0 + kAcross > dim) {
#pragma unroll
            for (int s = 0; s < kAcrossSteps; ++s) {
                const int at = v0 + 32 * s + 8 * g;
                if (dim % 8) v[s].shift(shift_of(at, dim));
                v[s].clear(dim - at);
            }
        }
        float m = 0.0f;
#pragma unroll
        for (int s = 0; s < kAcrossSteps; ++s) {
            if (d >= key_dim) v[s].lo = v[s].hi = Float4(0.0f);
            m = larger(larger(m, v[s].lo), v[s].hi);
        }
        return m;
    }
};

// kShared: several heads share a key, whose gradients are summed.
template <class T, int KT, bool kShared>
__global__ __launch_bounds__(kRowThreads) void delta_back_rows(DeltaBackParams b)
{
    const DeltaParams& p = b.f;
    typedef RowsRoom<T, KT> Room;
    constexpr int kParts = kSplit<T> ? 2 : 1, kTiles = (2 * KT + kRowWaves - 1) / kRowWaves;      // of a wave, along the keys
    __shared__ Room room;
    int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int lane = tid & (kWave - 1), g = lane >> 4, r = lane & 15;
    const int slot = (int)(blockIdx.x / p.key_heads), key_head = (int)(blockIdx.x % p.key_heads), many = kShared ? p.heads / p.key_heads : 1;
    const Piece piece = find_piece(p.pieces, slot);
    if (piece.seq < 0 || piece.n <= 0) return;
    const T* const ks = sequence_base<const T>(p.k, p.pieces, piece) + piece.row0 * p.k.row + key_head * p.k_head;
    const T* const qs = sequence_base<const T>(p.q, p.pieces, piece) + piece.row0 * p.q.row + key_head * p.q_head;
    const size_t below = (size_t)p.key_dim * p.value_dim;      // a mark's second part
    const T* const grads = sequence_base<const T>(b.grad_out, p.pieces, piece) + piece.row0 * b.grad_out.row;
    RowData<T> data;
    float gate = 0.0f, beta_ = 0.0f;
    auto load_head = [&](int h) {
        const bool there = wave == 0 && lane < piece.n;
        const long long at = piece.row0 + (there ? lane : 0);
        if (wave == 0) {
            gate = p.g.d ? sequence_base<const float>(p.g, p.pieces, piece)[at * p.g.row + h] : 0.0f;
            beta_ = sequence_base<const float>(p.beta, p.pieces, piece)[at * p.beta.row + h];
        }
        data.load(tid, grads + h * b.grad_out_head, (unsigned)b.grad_out.row, mark_of(b.behind, p, slot, h) + below, mark_of(p.marks, p, slot, h) + below, p.value_dim,
                  piece.n, 0);
    };
    const int tile = wave & 3, col0 = wave >> 2 << 1;      // of the 64 x 64 products: a wave's tile of rows and its two of columns
    Float4 kk[2], qk[2];                      // K K^T and Q K^T
    {
        RowLoad<T, KT, kRowThreads> k, q;
        k.load(ks, (unsigned)p.k.row, piece.n, p.key_dim);
        q.load(qs, (unsigned)p.q.row, piece.n, p.key_dim);
        load_head(key_head * many);
        k.put(p.unit, piece.n, p.key_dim, room.rows().keys, room.key_back, room.key);
        q.put(p.unit, piece.n, p.key_dim, room.rows().queries, room.query_back, room.query);
    }
    __syncthreads();
    if constexpr (!Room::kKept) key_products<T, KT, true, 2>(room.rows().keys, room.rows().queries, tile, col0, kk, qk);
    // Elements of the key's or query's row t that the wave's tiles have, as the rule takes them.
    auto row_elements = [&](bool query, int t, float (&v)[kTiles]) {
        const float per = query ? room.query_back[t] : room.key_back[t];
#pragma unroll
        for (int jj = 0; jj < kTiles; ++jj) {
            const int d = tile_row(wave * kTiles + jj, r);
            if constexpr (Room::kKept) {
                v[jj] = 0.0f;
                if (wave * kTiles + jj >= 2 * KT) continue;
                const auto& from = query ? room.rows().queries : room.rows().keys;
                auto element = [&](const Half8& eight) { return (float)reinterpret_cast<const _Float16*>(&eight)[d & 7]; };
                v[jj] = element(from[0][d >> 3][t ^ (d >> 3 & 15)]);
                if constexpr (kParts > 1) v[jj] += element(from[1][d >> 3][t ^ (d >> 3 & 15)]);
                v[jj] *= per;
            } else {
                const T* const x = query ? qs : ks;
                const float e = (float)x[(unsigned)(t < piece.n ? t : piece.n - 1) * (unsigned)(query ? p.q.row : p.k.row) + (unsigned)(d < p.key_dim ? d : p.key_dim - 1)];
                v[jj] = t < piece.n && d < p.key_dim ? e * (per * (query ? room.query[t] : room.key[t])) : 0.0f;
            }
        }
    };
    // Addresses in LDS are made anew for every step of the work: all of them together, kept over the loops, would take the registers of everything else.
    auto fresh_lane = [&] { asm volatile("" : "+v"(tid), "+v"(lane), "+v"(g), "+v"(r)); };
    Float4 dq[4][kTiles], dk[4][kTiles];      // sums over the heads that share the key
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int j = 0; j < kTiles; ++j) dq[m][j] = dk[m][j] = Float4(0.0f);

    for (int h = key_head * many; h < (key_head + 1) * many; ++h) {
        fresh_lane();
        const float* const mark = mark_of(p.marks, p, slot, h);
        const float* const behind = mark_of(b.behind, p, slot, h);
        if (kShared && h > key_head * many) load_head(h);
        __syncthreads();
        if (wave == 0) {
            if (lane >= piece.n) gate = beta_ = 0.0f;
            double sum = gate < -1000.0f ? -1000.0 : (double)gate;
#pragma unroll
            for (int x = 1; x < kWave; x *= 2) {
                const double before = __shfl_up(sum, x);
                if (lane >= x) sum += before;
            }
            const double all = __shfl(sum, kWave - 1);
            room.sum[lane] = sum;
            room.beta[lane] = beta_;
            room.dbeta[lane] = 0.0f;
            room.up[lane] = exp2_fast(kLog2e * (float)sum);
            room.rest[lane] = exp2_fast(kLog2e * (float)(all - sum));
            if (lane == 0) room.total = exp2_fast(kLog2e * (float)all);
        }
        Float4 asked[4][kTiles], reads[4][kTiles], last[4][kTiles], pd[2], nd[2];
        float inner = 0.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            pd[m & 1] = nd[m & 1] = Float4(0.0f);
#pragma unroll
            for (int j = 0; j < kTiles; ++j) asked[m][j] = reads[m][j] = last[m][j] = Float4(0.0f);
        }
        for (int v0 = 0; v0 < p.value_dim; v0 += kAcross) {
            fresh_lane();
            if (v0) data.load(tid, grads + h * b.grad_out_head, (unsigned)b.grad_out.row, behind + below, mark + below, p.value_dim, piece.n, v0);
            __syncthreads();
            // dO, dX = b dY and U = b R as operands
            const int e = tid & 15;
#pragma unroll
            for (int k = 0; k < RowData<T>::kPasses; ++k) {
                const int t = (tid >> 4) + k * (kRowThreads / 16);
                const float beta = room.beta[t];
                data.take(tid, k, piece.n, p.value_dim, v0);
                RowVec<T, 8>& o = data.o[k];
                Eight &y = data.y[k], &u = data.u[k];
                float dot = 0.0f, mo = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) dot = __builtin_fmaf(y.lo[i], u.lo[i], __builtin_fmaf(y.hi[i], u.hi[i], dot));
#pragma unroll
                for (int i = 0; i < 8; ++i) mo = larger(mo, (float)o[i]);
                y.lo *= beta;
                y.hi *= beta;
                u.lo *= beta;
                u.hi *= beta;
                float mx = larger(larger(0.0f, y.lo), y.hi), mu = larger(larger(0.0f, u.lo), u.hi);
                dot = over_few(dot, 16, Add());
                mo = over_few(mo, 16, Max());
                mx = over_few(mx, 16, Max());
                mu = over_few(mu, 16, Max());
                Scale so(mo);
                const Scale sx(mx), su(mu);
                if (__is_same(T, _Float16)) so.to = so.back = 1.0f;
                if (e == 0) {
                    room.back[0][t] = so.back;
                    room.back[1][t] = sx.back;
                    room.back[2][t] = su.back;
                    room.dbeta[t] += dot;
                }
                const int operand = tile_of(t) * kAcrossSteps + (e >> 2), entry = row_entry(e >> 2, e & 3, row_in_tile(t));
                Half8 hi, lo;
                to_halves<T>(o, so.to, hi, lo);
                room.o.grad[0][operand][entry] = hi;
                if constexpr (kParts > 1) room.o.grad[1][operand][entry] = lo;
                const HalfPair py = split(y.lo, y.hi, sx.to), pu = split(u.lo, u.hi, su.to);
                room.o.x[0][operand][entry] = py.hi;
                room.o.x[1][operand][entry] = py.lo;
                room.o.u[0][operand][entry] = pu.hi;
                room.o.u[1][operand][entry] = pu.lo;
            }
            StateRow s0, s1;
            s0.load(mark, tile_row(wave * kTiles, r), p.key_dim, p.value_dim, v0);
            __syncthreads();
            auto operand = [&](const Half8 (&a)[4 * kAcrossSteps][kWave], int m, int s) { return a[m * kAcrossSteps + s][row_entry(s, g, r)]; };
            // dO U^T and dX U^T
            fresh_lane();
#pragma unroll
            for (int k0 = 0; k0 < 2; ++k0)
                if (const int n = col0 + k0; n <= (tile | 1)) {
                    Float4 a(0.0f), c(0.0f);
#pragma unroll
                    for (int s = 0; s < kAcrossSteps; ++s) {
                        const Half8 uh = operand(room.o.u[0], n, s), ul = operand(room.o.u[1], n, s), xh = operand(room.o.x[0], tile, s);
#pragma unroll
                        for (int k = 0; k < kParts; ++k) {
                            const Half8 o = operand(room.o.grad[k], tile, s);
                            a = mfma(o, uh, a);
                            if (k == 0) a = mfma(o, ul, a);
                        }
                        c = mfma(xh, uh, c);
                        c = mfma(xh, ul, c);
                        c = mfma(operand(room.o.x[1], tile, s), uh, c);
                    }
                    const float col = room.back[2][tile_row(n, r)];
                    const Float4 ro = *reinterpret_cast<const Float4*>(&room.back[0][tile_row(tile, 4 * g)]), rx = *reinterpret_cast<const Float4*>(&room.back[1][tile_row(tile, 4 * g)]);
                    pd[k0] += a * (ro * col);
                    nd[k0] += c * (rx * col);
                }
            in_order();
            // dO S0^T, dX S0^T and U dS1^T: a wave has some of the keys' elements, for all rows
#pragma unroll
            for (int jj = 0; jj < kTiles; ++jj) {
                fresh_lane();
                const int j = wave * kTiles + jj, d = tile_row(j, r);
                if (jj) in_order();
                const int row = j < 2 * KT ? d : p.key_dim;
                HalfPair f[kAcrossSteps];
                float back;
                auto to_operands = [&](StateRow& s) {
                    const Scale by(over_column(s.clear(row, p.key_dim, p.value_dim, v0)));
                    back = by.back;
#pragma unroll
                    for (int k = 0; k < kAcrossSteps; ++k) f[k] = split(s.v[k].lo, s.v[k].hi, by.to);
                };
                to_operands(s0);
                s1.load(behind, d, p.key_dim, p.value_dim, v0);
                in_order();
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (m) in_order();
                    Float4 a(0.0f), c(0.0f);
#pragma unroll
                    for (int s = 0; s < kAcrossSteps; ++s) {
                        const Half8 xh = operand(room.o.x[0], m, s);
                        c = mfma(xh, f[s].hi, c);
#pragma unroll
                        for (int k = 0; k < kParts; ++k) {
                            const Half8 o = operand(room.o.grad[k], m, s);
                            a = mfma(o, f[s].hi, a);
                            if (k == 0) a = mfma(o, f[s].lo, a);
                        }
                        c = mfma(xh, f[s].lo, c);
                        c = mfma(operand(room.o.x[1], m, s), f[s].hi, c);
                    }
                    const int t0 = tile_row(m, 4 * g);
                    const Float4 up = *reinterpret_cast<const Float4*>(&room.up[t0]), ro = *reinterpret_cast<const Float4*>(&room.back[0][t0]),
                                 rx = *reinterpret_cast<const Float4*>(&room.back[1][t0]);
                    asked[m][jj] += a * (up * ro * (p.scale * back));
                    reads[m][jj] -= c * (up * rx * back);
                }
                in_order();
                to_operands(s1);
#pragma unroll
                for (int s = 0; s < kAcrossSteps; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) inner = __builtin_fmaf(s0.v[s].lo[i], s1.v[s].lo[i], __builtin_fmaf(s0.v[s].hi[i], s1.v[s].hi[i], inner));
                if (jj + 1 < kTiles) s0.load(mark, tile_row(j + 1, r), p.key_dim, p.value_dim, v0);
                in_order();
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (m) in_order();
                    Float4 w(0.0f);
#pragma unroll
                    for (int s = 0; s < kAcrossSteps; ++s) {
                        const Half8 uh = operand(room.o.u[0], m, s);
                        w = mfma(uh, f[s].hi, w);
                        w = mfma(uh, f[s].lo, w);
                        w = mfma(operand(room.o.u[1], m, s), f[s].hi, w);
                    }
                    const int t0 = tile_row(m, 4 * g);
                    const Float4 rest = *reinterpret_cast<const Float4*>(&room.rest[t0]), ru = *reinterpret_cast<const Float4*>(&room.back[2][t0]);
                    last[m][jj] += w * (rest * ru * back);
                }
            }
        }
        // what the rows' decays have of S0, of dS1 and of one another's products
        {
            fresh_lane();
            float dots[4][4], lasts[4][4];
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = tile_row(m, 4 * g + i);
                    float k[kTiles], q[kTiles], s = 0.0f, l = 0.0f;
                    row_elements(false, t, k);
                    row_elements(true, t, q);
#pragma unroll
                    for (int jj = 0; jj < kTiles; ++jj) {
                        s = __builtin_fmaf(q[jj], asked[m][jj][i], s);
                        s = __builtin_fmaf(k[jj], reads[m][jj][i], s);
                        l = __builtin_fmaf(k[jj], last[m][jj][i], l);
                    }
                    dots[m][i] = s;
                    lasts[m][i] = l;
                }
            put_dots(dots, room.dots[0]);
            put_dots(lasts, room.dots[1]);
        }
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) inner += __shfl_xor(inner, x);
        if (lane == 0) room.inner[wave] = inner;
        if constexpr (Room::kKept) key_products<T, KT, true, 2>(room.rows().keys, room.rows().queries, tile, col0, kk, qk);
        __syncthreads();                          // the matrix lies over the operands
        fresh_lane();
        // dP and dA without their keys' and queries' factors: in place
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = tile_row(tile, 4 * g + i), col = tile_row(col0 + n, r);
                const float d = col <= row ? exp2_fast(kLog2e * (float)(room.sum[row] - room.sum[col])) : 0.0f;
                pd[n][i] = col <= row ? p.scale * pd[n][i] * d : 0.0f;
                nd[n][i] = col < row ? -nd[n][i] * d : 0.0f;
                const float both = pd[n][i] * qk[n][i] * room.query_back[row] + nd[n][i] * kk[n][i] * room.key_back[row];
                room.t.matrix[row][col] = col < row ? both * room.key_back[col] : 0.0f;
            }
        __syncthreads();
        {                                         // each row's sums up to a column: 8 columns a lane, then the lanes before it
            const int row = 8 * wave + (lane & 7), part = lane >> 3;
            float s = 0.0f, before = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s += room.t.matrix[row][8 * part + i];
                room.t.matrix[row][8 * part + i] = s;
            }
#pragma unroll
            for (int k = 0; k < 7; ++k) {
                const float one = __shfl(s, 8 * k + (lane & 7));
                if (k < part) before += one;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) room.t.matrix[row][8 * part + i] += before;
        }
        __syncthreads();
        {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = room.t.matrix[8 * wave + i][lane > 0 ? lane - 1 : 0];
                if (8 * wave + i >= lane && lane > 0) s += v;
            }
            room.pairs[wave][lane] = s;
        }
        __syncthreads();
        if (wave == 0) {
            float from = dot_of(room.dots[0], lane), up_to = dot_of(room.dots[1], lane);
#pragma unroll
            for (int x = 1; x < kWave; x *= 2) {
                const float a = __shfl_down(from, x), c = __shfl_up(up_to, x);
                if (lane + x < kWave) from += a;
                if (lane >= x) up_to += c;
            }
            const float before = __shfl_up(up_to, 1);
            float inner_ = room.inner[0];
#pragma unroll
            for (int w = 1; w < kRowWaves; ++w) inner_ += room.inner[w];
            const float dg = dot_of(room.pairs, lane) + from + (lane ? before : 0.0f) + room.total * inner_;
            const long long at = piece.row0 + lane;
            if (lane < piece.n) {
                if (b.grad_g.d) sequence_base<float>(b.grad_g, p.pieces, piece)[at * b.grad_g.row + h] = dg;
                if (b.grad_beta.d) sequence_base<float>(b.grad_beta, p.pieces, piece)[at * b.grad_beta.row + h] = room.dbeta[lane];
            }
        }
        // as operands: their columns, transposed their rows, with the factor of the key or query that they meet
        float back[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k) __syncthreads();
            fresh_lane();
            float most = 0.0f;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = tile_row(tile, 4 * g + i), col = tile_row(col0 + n, r);
                    const float v = (k % 2 ? nd[n][i] : pd[n][i]) * (k < 2 ? room.key_back[col] : k == 2 ? room.query_back[row] : room.key_back[row]);
                    most = larger(most, v);
                    room.t.matrix[row][col] = v;
                }
            const Scale by(over_block<kRowWaves>(most, room.most[k % 2]));
            back[k] = by.back;
            if (k < 2) store_operands<false, kRowWaves>(room.t.matrix, by.to, room.t.tri[k]);
            else store_operands<true, kRowWaves>(room.t.matrix, by.to, room.t.tri[k]);
        }
#pragma unroll
        for (int query = 0; query < 2; ++query) {
            if (query) __syncthreads();
            fresh_lane();
            for (int job = tid; job < 32 * KT; job += kRowThreads) {
                const int sq = job / (4 * KT), e = job % (4 * KT);
                Half8 hi[8], lo[8];
                if constexpr (Room::kKept) {
                    const auto& from = query ? room.rows().queries : room.rows().keys;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        hi[i] = from[0][e][(8 * sq + i) ^ (e & 15)];
                        if constexpr (kParts > 1) lo[i] = from[1][e][(8 * sq + i) ^ (e & 15)];
                    }
                } else {
                    RowVec<T, 8> v[8];
                    load_square<T>(query ? qs : ks, (unsigned)(query ? p.q.row : p.k.row), piece.n, p.key_dim, sq, e, v);
                    clear_eights<T, 8>(8 * sq, 1, piece.n, e, p.key_dim, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) to_halves<T>(v[i], __is_same(T, _Float16) ? 1.0f : (query ? room.query : room.key)[8 * sq + i], hi[i], lo[i]);
                }
                put_turned<T, KT>(hi, lo, sq, e, room.t.turned);
            }
            __syncthreads();
#pragma unroll
            for (int jj = 0; jj < kTiles; ++jj) {
                const int j = wave * kTiles + jj;
                if (j >= 2 * KT) continue;
                HalfPair f[2][1];
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    f[s][0].hi = turned_of<KT>(room.t.turned[0], j, s, lane);
                    f[s][0].lo = kParts > 1 ? turned_of<KT>(room.t.turned[kParts - 1], j, s, lane) : Half8((_Float16)0.0f);
                }
                in_order();
                Float4 a[4][1];
                if (!query) {
                    tri_products<1, false, kParts == 1>(room.t.tri[0], lane, f, a);
#pragma unroll
                    for (int m = 0; m < 4; ++m) asked[m][jj] += a[m][0] * back[0];
                    in_order();
                    tri_products<1, false, kParts == 1>(room.t.tri[1], lane, f, a);
#pragma unroll
                    for (int m = 0; m < 4; ++m) reads[m][jj] += a[m][0] * back[1];
                    in_order();
                    tri_products<1, true, kParts == 1>(room.t.tri[3], lane, f, a);
#pragma unroll
                    for (int m = 0; m < 4; ++m) last[m][jj] += a[m][0] * back[3];
                } else {
                    tri_products<1, true, kParts == 1>(room.t.tri[2], lane, f, a);
#pragma unroll
                    for (int m = 0; m < 4; ++m) last[m][jj] += a[m][0] * back[2];
                }
            }
        }
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                dq[m][j] += asked[m][j];
                dk[m][j] += reads[m][j] + last[m][j];
            }
    }
    // through the rows' lengths: d - e (e . d) over the length, e the row at unit length
#pragma unroll
    for (int query = 0; query < 2; ++query) {
        const ssam_rows& to = query ? b.grad_q : b.grad_k;
        if (!to.d) continue;
        Float4(&d)[4][kTiles] = query ? dq : dk;
        fresh_lane();
        if (p.unit) {
            float dots[4][4];
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float e[kTiles], s = 0.0f;
                    row_elements(query, tile_row(m, 4 * g + i), e);
#pragma unroll
                    for (int jj = 0; jj < kTiles; ++jj) s = __builtin_fmaf(e[jj], d[m][jj][i], s);
                    dots[m][i] = s;
                }
            __syncthreads();
            put_dots(dots, room.dots[0]);
            __syncthreads();
        }
        else __syncthreads();
        // by way of LDS, so that whole rows leave
        constexpr int E = 16 / (int)sizeof(T), kOfRow = 32 * KT / E;
        RowVec<T, E>(*const out)[kOfRow] = reinterpret_cast<RowVec<T, E>(*)[kOfRow]>(&room.t.turned[0][0][0]);
        static_assert(sizeof(room.t.turned) >= sizeof(T) * kDeltaRows * 32 * KT);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = tile_row(m, 4 * g + i);
                float e[kTiles], per = 1.0f, dot = 0.0f;
                if (p.unit) {
                    row_elements(query, t, e);
                    per = query ? room.query[t] * room.query_back[t] : room.key[t] * room.key_back[t];
                    dot = dot_of(room.dots[0], t);
                }
#pragma unroll
                for (int jj = 0; jj < kTiles; ++jj) {
                    const int at = tile_row(wave * kTiles + jj, r);
                    if (wave * kTiles + jj >= 2 * KT) continue;
                    reinterpret_cast<T*>(&out[t][0])[at] = (T)(p.unit ? per * (d[m][jj][i] - e[jj] * dot) : d[m][jj][i]);
                }
            }
        __syncthreads();
        T* const rows = sequence_base<T>(to, p.pieces, piece) + piece.row0 * to.row + key_head * b.grad_key_head;
        for (int at = tid; at < kDeltaRows * kOfRow; at += kRowThreads) {
            const int t = at / kOfRow, part = at % kOfRow;
            if (t < piece.n && part * E < p.key_dim) store_row_vec<T, E>(rows + ((unsigned)t * (unsigned)to.row + (unsigned)(part * E)), p.key_dim - part * E, out[t][part]);
        }
        __syncthreads();
    }
}

struct BackPlan {
    long long slots;
    size_t blocks, behind;      // bytes
};
BackPlan back_plan(const ssam_scan_delta_backward_args& a)
{
    BackPlan p;
    p.slots = piece_slots(a.seq, kDeltaRows);
    p.blocks = (size_t)product(product(p.slots, a.heads), sizeof(Block));
    p.behind = (size_t)product(product(p.slots, a.heads), (long long)(a.key_dim + kDeltaRows) * a.value_dim * 4);
    return p;
}

}  // namespace
}  // namespace ssam

extern "C" {

size_t ssam_scan_delta_backward_workspace_bytes(const ssam_scan_delta_backward_args* a)
{
    using namespace ssam;
    if (!a || check_delta(*a) || check_sequences(a->seq) || a->seq.sequences == 0) return 0;
    const BackPlan p = back_plan(*a);
    return (size_t)held_to_62((__int128)p.blocks + p.behind);
}

int ssam_scan_delta_backward(const ssam_scan_delta_backward_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_delta(*a)) return e;
    if (int e = check_sequences(a->seq)) return e;
    if (a->seq.sequences == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype);
    if (int e = check_delta_rows(*a, a->seq)) return e;
    const long long keys = (long long)a->key_heads * a->key_dim, values = (long long)a->heads * a->value_dim;
    if (a->grad_out_head < 0 || a->grad_out_head > kMaxStride) return SSAM_ERR_DIM;
    for (const ssam_rows* r : {&a->grad_out, &a->grad_q, &a->grad_k, &a->grad_v})
        if (int e = check_tile_rows(*r, a->seq)) return e;
    if (int e = check_rows(a->grad_out, a->seq, heads_width(a->heads, a->grad_out_head, a->value_dim), esz, false)) return e;
    for (const ssam_rows* r : {&a->grad_q, &a->grad_k})
        if (int e = check_out_rows(*r, a->seq, keys, esz, true)) return e;
    if (int e = check_out_rows(a->grad_v, a->seq, values, esz, true)) return e;
    for (const ssam_rows* r : {&a->grad_g, &a->grad_beta})
        if (int e = check_out_rows(*r, a->seq, a->heads, 4, true)) return e;
    for (const void* f : {(const void*)a->d_marks, (const void*)a->d_grad_final, (const void*)a->d_grad_state})
        if ((uintptr_t)f % 4) return SSAM_ERR_DIM;
    if (!a->d_marks || !a->d_work) return SSAM_ERR_NULL;
    const BackPlan plan = back_plan(*a);
    const size_t bytes = ssam_scan_delta_backward_workspace_bytes(a);
    if ((long long)bytes > kMaxExtent || a->work_bytes < bytes || (uintptr_t)a->d_work % 16) return SSAM_ERR_DIM;
    const long long state_bytes = product(a->seq.sequences, values * a->key_dim * 4);
    if (state_bytes > 4 * kMaxExtent) return SSAM_ERR_DIM;
    const Cover outs[] = {cover_rows(a->grad_q, a->seq, keys, esz), cover_rows(a->grad_k, a->seq, keys, esz), cover_rows(a->grad_v, a->seq, values, esz),
                          cover_rows(a->grad_g, a->seq, a->heads, 4), cover_rows(a->grad_beta, a->seq, a->heads, 4),
                          cover_plain(a->d_grad_state, state_bytes), cover_plain(a->d_work, (long long)bytes)};
    const Cover ins[] = {cover_rows(a->q, a->seq, heads_width(a->key_heads, a->q_head, a->key_dim), esz),
                         cover_rows(a->k, a->seq, heads_width(a->key_heads, a->k_head, a->key_dim), esz),
                         cover_rows(a->v, a->seq, heads_width(a->heads, a->v_head, a->value_dim), esz), cover_rows(a->g, a->seq, a->heads, 4),
                         cover_rows(a->beta, a->seq, a->heads, 4), cover_rows(a->grad_out, a->seq, heads_width(a->heads, a->grad_out_head, a->value_dim), esz),
                         cover_plain(a->d_grad_final, state_bytes), cover_plain(a->d_marks, (long long)plan.behind)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;

    const WalkPlan walk = walk_plan(*a);
    DeltaBackParams b{};
    b.f = DeltaParams{make_pieces(a->seq, kDeltaRows), a->q, a->k, a->v, ssam_rows{nullptr, 0, 0}, a->g, a->beta, a->q_head, a->k_head, a->v_head, 0,
                      a->d_grad_final, nullptr, const_cast<float*>(a->d_marks), static_cast<Block*>(a->d_work), a->heads, a->key_heads, a->key_dim,
                      a->value_dim, a->unit != 0, a->scale, walk.tiles};
    b.grad_out = a->grad_out;
    b.grad_q = a->grad_q;
    b.grad_k = a->grad_k;
    b.grad_v = a->grad_v;
    b.grad_g = a->grad_g;
    b.grad_beta = a->grad_beta;
    b.grad_out_head = a->grad_out_head;
    b.grad_v_head = a->value_dim;
    b.grad_key_head = a->key_dim;
    b.grad_state = a->d_grad_state;
    b.behind = reinterpret_cast<float*>(static_cast<char*>(a->d_work) + plan.blocks);
    const long long walks = product((long long)a->seq.sequences * a->heads, b.f.tiles), rows = product(plan.slots, a->key_heads);
    const bool all = a->grad_q.d || a->grad_k.d || a->grad_g.d || a->grad_beta.d;      // or the state's and the values' alone
    if (rows > max_grid(all ? kRowThreads : kBlock)) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    return with_delta_type(a->dtype, [&](auto t) {
        return with_key(a->key_dim, [&](auto kt) {
            using T = decltype(t);
            constexpr int KT = decltype(kt)::value;
            if (walks > max_grid(kWalkThreads<T, KT>)) return (int)SSAM_ERR_DIM;
            hipLaunchKernelGGL((delta_back_prepare<T, KT>), dim3((unsigned)rows), dim3(kBlock), 0, st, b.f);
            if (int e = launched()) return e;
            if constexpr (kSplit<T> && KT <= 4)
                if (walk.wide) hipLaunchKernelGGL((delta_back_walk<T, KT, 2>), dim3((unsigned)walks), dim3(kWalkThreads<T, KT>), 0, st, b);
            if (!walk.wide) hipLaunchKernelGGL((delta_back_walk<T, KT, 1>), dim3((unsigned)walks), dim3(kWalkThreads<T, KT>), 0, st, b);
            if (int e = launched()) return e;
            if (!all) return (int)SSAM_OK;
            if (a->heads > a->key_heads) hipLaunchKernelGGL((delta_back_rows<T, KT, true>), dim3((unsigned)rows), dim3(kRowThreads), 0, st, b);
            else hipLaunchKernelGGL((delta_back_rows<T, KT, false>), dim3((unsigned)rows), dim3(kRowThreads), 0, st, b);
            return launched();
        });
    });
}

}  // extern "C"
