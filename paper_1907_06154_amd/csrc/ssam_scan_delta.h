// What the kernels of the scan with matrix states (ssam_scan_delta) share.
//
// Rows are taken C = 64 at a time.  With G_t the sum of g over the block's rows up to t, D_ij = exp(G_i - G_j) for i >= j, 0 otherwise,
// A = strictly lower part of (K K^T o D), S the state before the block and b = beta:
//     X = V - exp(G) K S,    R = (I + A diag(b))^-1 X,    U = b R,    O = scale (exp(G) Q S + (Q K^T o D) U),
//     state behind it = exp(G_C) S + (exp(G_C - G) K)^T U
// R is what each row's value misses of what the state holds for its key.  Everything but S and V is known without the state, so it is made for all
// blocks at once (delta_prepare); the rest follows the sequence.
//
// Matrix products run on v_mfma_f32_16x16x32_f16.  q, k of 16 bits are one fp16 operand: fp16 as it is, bf16 with a power of two per row taken
// out (to_halves says how exact that is).  Everything else is a pair hi + lo of fp16 under a power of two that brings the largest of what shares it, a column's
// 64 rows, a state's column, a triangular matrix, a row of fp32 q or k, to 2^10 .. 2^11.  hi is within 2^-11 of a value and lo within 2^-11 of the rest, so that
// the pair is 2^-22 of the value off, until lo is subnormal, 2^13 below the largest: from there on it is 2^-25 off, 2^-35 of the largest.  Two products
// against q or k, three between two such pairs (lo lo is below 2^-22).  bf16 pairs keep 16 bits, which the state's fp32 would show.
//
// Operand layout: lane (g = lane / 16, r = lane % 16) of an A operand holds row r, elements 8 g .. 8 g + 7 of 32 along the sum; of a B
// operand column r and the same elements; of a result rows 4 g .. 4 g + 3, column r.  What a row of a result tile stands for is free:
// tiles 2 p and 2 p + 1 stand for indices 32 p + 8 g + (0 .. 3) and + (4 .. 7), so that a lane's eight values of both are the eight that
// it holds of the next product's B operand, in order.  So S -> X -> R -> U -> S stays in a wave's registers, 16 columns of the values a
// tile; only operands made from q, k and the block's matrices are loaded, and those are the same for every column.
#pragma once
#include "ssam_rows.h"

namespace ssam {

constexpr int kDeltaRows = SSAM_DELTA_ROWS;

typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
typedef RowVec<float, 4> Float4;

__device__ __forceinline__ Float4 mfma(Half8 a, Half8 b, Float4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

struct HalfPair {
    Half8 hi, lo;
};

// A power of two that brings m (the largest magnitude of what it scales) to 2^10 .. 2^11, and its reciprocal; infinities and NaN pass.
struct Scale {
    float to, back;
    __device__ __forceinline__ Scale() {}
    __device__ __forceinline__ explicit Scale(float m)
    {
        unsigned e = (__builtin_bit_cast(unsigned, m) >> 23) & 255u;
        e = e < 11u ? 11u : e;
        to = __builtin_bit_cast(float, (264u - e) << 23);
        back = __builtin_bit_cast(float, (e - 10u) << 23);
    }
};

// Two values as hi + lo, each rounded to nearest: two mixed-precision multiply-adds a value, to v and to v - hi.  (The empty statements keep the halves of a
// register where they are: without them the compiler makes fp32 values first and converts those.  Instructions in them would be unsafe: a matrix instruction
// reads what it adds to up to three wait states after its issue, which the compiler keeps free for its own instructions and not for such.)
typedef _Float16 Half2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split(float a, float b, float to, unsigned& hi, unsigned& lo)
{
    _Float16 first = (_Float16)__builtin_fmaf(a, to, 0.0f);
    asm("" : "+v"(first));
    Half2 h{first, (_Float16)__builtin_fmaf(b, to, 0.0f)};
    asm("" : "+v"(h));
    first = (_Float16)__builtin_fmaf(a, to, -(float)h[0]);
    asm("" : "+v"(first));
    hi = __builtin_bit_cast(unsigned, h);
    lo = __builtin_bit_cast(unsigned, Half2{first, (_Float16)__builtin_fmaf(b, to, -(float)h[1])});
}
__device__ __forceinline__ HalfPair split(float a0, float a1, float a2, float a3, float a4, float a5, float a6, float a7, float to)
{
    typedef unsigned Four __attribute__((ext_vector_type(4)));
    unsigned h0, h1, h2, h3, l0, l1, l2, l3;
    split(a0, a1, to, h0, l0);
    split(a2, a3, to, h1, l1);
    split(a4, a5, to, h2, l2);
    split(a6, a7, to, h3, l3);
    HalfPair p;
    p.hi = __builtin_bit_cast(Half8, Four{h0, h1, h2, h3});
    p.lo = __builtin_bit_cast(Half8, Four{l0, l1, l2, l3});
    return p;
}
// The values of two result tiles as a B operand.
__device__ __forceinline__ HalfPair split(const Float4& a, const Float4& b, float to) { return split(a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3], to); }

// The larger of two magnitudes; a NaN may be passed over, as it reaches the products by itself.
__device__ __forceinline__ float larger(float m, float v) { return __builtin_fmaxf(m, __builtin_fabsf(v)); }
__device__ __forceinline__ float larger(float m, const Float4& v) { return larger(larger(larger(larger(m, v[0]), v[1]), v[2]), v[3]); }
// Over the four lanes of a column, lane, lane ^ 16, ^ 32 and ^ 48: the instructions swap halves of two registers, of the wave or of its pairs of rows
// of 16 lanes, which lie two wait states behind the write of either: `m` comes from a vector instruction, and so does its copy, so that no matrix instruction
// is still at either register.  (The builtins' second result is the first one's copy in this compiler.)
__device__ __forceinline__ float over_column(float m)
{
    float a = m, b = m;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    a = b = __builtin_fmaxf(a, b);
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return __builtin_fmaxf(a, b);
}

// What row r of result tile m stands for.
__device__ __forceinline__ int tile_row(int m, int r) { return 32 * (m >> 1) + 8 * (r >> 2) + 4 * (m & 1) + (r & 3); }

// ---- a block's matrices and factors, from delta_prepare --------------------------------------------------------------------
// Lower triangular [64][64] as A operands: tile m's rows against 32 columns s, those with s <= m / 2; the transposed ones s >= m / 2.
constexpr int kTriOperands = 6;
__device__ __forceinline__ int lower_operand(int m, int s) { return m < 2 ? m : 2 * (m - 1) + s; }
__device__ __forceinline__ int upper_operand(int m, int s) { return m < 2 ? 2 * m + s : 2 + m; }

struct BlockFactors {
    float reads[kDeltaRows];     // exp(G_t) x the key's factor
    float beta[kDeltaRows];
    float writes[kDeltaRows];    // exp(G_C - G_t) x the key's factor
    float asks[kDeltaRows];      // scale x exp(G_t) x the query's factor
    float key[kDeltaRows], query[kDeltaRows];   // what an element is multiplied by to become its fp16 operand
    float total;                 // exp(G_C)
    float solve_back, mix_back;  // what the two matrices' operands are to be multiplied by
    float pad;
};
struct Block {
    Half8 solve[2][kTriOperands][kWave];        // hi and lo of the system's inverse
    Half8 mix[2][kTriOperands][kWave];          // and of scale (Q K^T o D)
    BlockFactors f;
};

struct DeltaParams {
    Pieces pieces;
    ssam_rows q, k, v, out, g, beta;
    long long q_head, k_head, v_head, out_head;
    const float *state;
    float *final, *marks;
    Block* blocks;               // [slots][heads]
    int heads, key_heads, key_dim, value_dim, unit;
    float scale;
    int tiles;                   // of the walk: blocks along the values
};

// A mark: the state before a block, [key_dim][value_dim], and its R, [64][value_dim].
__device__ __forceinline__ float* mark_of(float* marks, const DeltaParams& p, long long slot, int head)
{
    return marks + (slot * p.heads + head) * (long long)(p.key_dim + kDeltaRows) * p.value_dim;
}

// Blocks go to the eight XCDs in turn; neighbours, which read the same rows of q and k, are made those of one XCD and its L2.
__device__ __forceinline__ unsigned near_block()
{
    constexpr unsigned kXcds = 8;
    const unsigned each = gridDim.x / kXcds, whole = each * kXcds;
    return blockIdx.x < whole ? blockIdx.x % kXcds * each + blockIdx.x / kXcds : blockIdx.x;
}

// ---- checks ----------------------------------------------------------------------------------------------------------------
template <class Args>
int check_delta(const Args& a)
{
    if (!type_bytes(a.dtype)) return SSAM_ERR_ENUM;
    if (a.heads < 1 || a.key_heads < 1 || a.heads % a.key_heads || a.key_dim < 1 || a.key_dim > SSAM_MAX_KEY || a.value_dim < 1) return SSAM_ERR_SHAPE;
    if (a.heads > kMaxChannels || a.value_dim > kMaxChannels || (long long)a.heads * a.value_dim > kMaxChannels) return SSAM_ERR_DIM;
    return SSAM_OK;
}
inline long long heads_width(int heads, long long apart, int dim) { return run_extent(heads, apart, dim); }

template <class Args>
int check_delta_rows(const Args& a, const ssam_sequences& q)
{
    const int esz = type_bytes(a.dtype);
    for (long long s : {a.q_head, a.k_head, a.v_head})
        if (s < 0 || s > kMaxStride) return SSAM_ERR_DIM;
    if (int e = check_rows(a.q, q, heads_width(a.key_heads, a.q_head, a.key_dim), esz, false)) return e;
    if (int e = check_rows(a.k, q, heads_width(a.key_heads, a.k_head, a.key_dim), esz, false)) return e;
    if (int e = check_rows(a.v, q, heads_width(a.heads, a.v_head, a.value_dim), esz, false)) return e;
    for (const ssam_rows* r : {&a.q, &a.k, &a.v, &a.g, &a.beta})
        if (int e = check_tile_rows(*r, q)) return e;
    if (int e = check_rows(a.g, q, a.heads, 4, true)) return e;
    return check_rows(a.beta, q, a.heads, 4, false);
}
// A result's heads must not share elements either.
inline int check_out_heads(const ssam_rows& r, const ssam_sequences& q, int heads, long long apart, int dim, int esz, bool optional)
{
    if (apart < 0 || apart > kMaxStride || (r.d && heads > 1 && apart < dim)) return SSAM_ERR_DIM;
    if (int e = check_tile_rows(r, q)) return e;
    return check_out_rows(r, q, heads_width(heads, apart, dim), esz, optional);
}

// fp32: with two walks a compute unit or more, a wave takes 32 columns, so that half as many blocks make the same operands: 16 x 512 rows of 32
// heads of 128 x 128 451 -> 360 us, their gradients 1777 -> 1660, but 4 x 1024 rows (256 walks) 199 -> 247.  16 bits have staging waves in place of it (778 and 793 us for
// 8 x 4096 rows); fewer columns a block, on more of them, gave 16 bits 4 % at 64 walks and cost the gradients' 6 %.  Keys beyond 128 leave no registers for it.
struct WalkPlan {
    bool wide;
    int tiles;
};
template <class Args>
WalkPlan walk_plan(const Args& a)
{
    const int tiles = (a.value_dim + 63) / 64;
    const bool wide = a.dtype == SSAM_F32 && (long long)a.seq.sequences * a.heads * tiles >= 512 && a.value_dim > 64 && a.key_dim <= 128;
    return {wide, wide ? (a.value_dim + 127) / 128 : tiles};
}

template <class F>
int with_delta_type(int dtype, F f)
{
    if (dtype == SSAM_F32) return f(float());
    if (dtype == SSAM_F16) return f(_Float16());
    return f(__bf16());
}
// f gets the 32s of a key, rounded up to a power of two, as a compile-time constant.
template <class F>
int with_key(int key_dim, F f)
{
    if (key_dim <= 32) return f(std::integral_constant<int, 1>{});
    if (key_dim <= 64) return f(std::integral_constant<int, 2>{});
    if (key_dim <= 128) return f(std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 8>{});
}

}  // namespace ssam
