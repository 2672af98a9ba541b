// What the selective scan's kernels share: how channels and states lie over the lanes of a wave, and the tensors.
//
// A wave holds 64 / GL channels; the GL lane groups of a channel hold NS states each, in registers.  Lane bits: the low bits
// are channels, so that the four lanes of a quad (DPP quad_perm) work on four channels with the SAME states: a quad needs NS
// values of b (and c) per row, every lane of it loads NS / 4 of them, and the multiply-add takes the other three from its
// neighbours by DPP -- one 32-bit LDS read per four states instead of four.  The groups are bits 2-3 of the lane (GL = 4), bit 3
// (GL = 2) or none, so that the sum over a channel's states is completed by rotations inside the row of 16 lanes.
#pragma once
#include "ssam_rows.h"

namespace ssam {

template <int GL_, int NS_>
struct ScanShape {
    static constexpr int GL = GL_, NS = NS_;
    static constexpr int kStates = GL * NS;                       // states held: those of the call, some more than once (state_at)
    static constexpr int kWaveChannels = kWave / GL;
    static constexpr int kChannels = kWavesPerBlock * kWaveChannels;   // of a block
};

template <int GL> __device__ __forceinline__ int lane_group(int lane) { return GL == 4 ? (lane >> 2) & 3 : GL == 2 ? (lane >> 3) & 1 : 0; }
template <int GL> __device__ __forceinline__ int lane_channel(int lane)
{
    return GL == 4 ? (lane & 3) + ((lane >> 4) << 2) : GL == 2 ? (lane & 7) + ((lane >> 4) << 3) : lane;
}

// The value of lane Q of the quad.
template <int Q>
__device__ __forceinline__ float quad_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), Q * 0x55, 0xf, 0xf, true));
}
// v[i] + b(lane i of the quad) x, i = 0 .. 3: the 4x4 matrix instruction with K = 1, sixteen outer products side by side whose lanes lie
// as the quads do.  It takes 8 cycles where four products by DPP take 16 (full fp32; 1 x 4096 rows 140 -> 136 us, the
// gradients of 4 x 2048 rows of 2048 channels 501 -> 478).
__device__ __forceinline__ RowVec<float, 4> quad_outer(float b, float x, RowVec<float, 4> v) { return __builtin_amdgcn_mfma_f32_4x4x1f32(b, x, v, 0, 0, 0); }

// Four rows' y += c0 h0 + c1 h1 + c2 h2 + c3 h3 (kFirst: y = ..), with cQ the value of lane Q of the quad: multiply-adds that take it by
// DPP themselves (the compiler moves it into a register first, twice the instructions).  A DPP read must lie two wait states behind
// the write of its register, a read of what the 4x4 matrix instruction wrote five, and the compiler counts neither into nor out of
// these blocks: hence the s_nop, of eight wait states, and the order row by row.  y leaves only through another of these blocks or
// into memory, never into a DPP of the compiler's.
template <bool kFirst>
__device__ __forceinline__ void quad_dots(float (&y)[4], const float (&c)[4], const float (&h)[4][4])
{
#define SSAM_DOT(OP, Q, A, B, C, D)                                                                                \
    OP " %0, %4, %" #A " quad_perm:[" #Q "," #Q "," #Q "," #Q "] row_mask:0xf bank_mask:0xf\n\t"                     \
    OP " %1, %5, %" #B " quad_perm:[" #Q "," #Q "," #Q "," #Q "] row_mask:0xf bank_mask:0xf\n\t"                     \
    OP " %2, %6, %" #C " quad_perm:[" #Q "," #Q "," #Q "," #Q "] row_mask:0xf bank_mask:0xf\n\t"                     \
    OP " %3, %7, %" #D " quad_perm:[" #Q "," #Q "," #Q "," #Q "] row_mask:0xf bank_mask:0xf\n\t"
#define SSAM_INPUTS                                                                                                \
    "v"(c[0]), "v"(c[1]), "v"(c[2]), "v"(c[3]), "v"(h[0][0]), "v"(h[1][0]), "v"(h[2][0]), "v"(h[3][0]), "v"(h[0][1]), \
        "v"(h[1][1]), "v"(h[2][1]), "v"(h[3][1]), "v"(h[0][2]), "v"(h[1][2]), "v"(h[2][2]), "v"(h[3][2]), "v"(h[0][3]), \
        "v"(h[1][3]), "v"(h[2][3]), "v"(h[3][3])
    if constexpr (kFirst)
        asm("s_nop 7\n\t" SSAM_DOT("v_mul_f32_dpp", 0, 8, 9, 10, 11) SSAM_DOT("v_fmac_f32_dpp", 1, 12, 13, 14, 15)
                SSAM_DOT("v_fmac_f32_dpp", 2, 16, 17, 18, 19) SSAM_DOT("v_fmac_f32_dpp", 3, 20, 21, 22, 23)
            : "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
            : SSAM_INPUTS);
    else
        asm("s_nop 7\n\t" SSAM_DOT("v_fmac_f32_dpp", 0, 8, 9, 10, 11) SSAM_DOT("v_fmac_f32_dpp", 1, 12, 13, 14, 15)
                SSAM_DOT("v_fmac_f32_dpp", 2, 16, 17, 18, 19) SSAM_DOT("v_fmac_f32_dpp", 3, 20, 21, 22, 23)
            : "+&v"(y[0]), "+&v"(y[1]), "+&v"(y[2]), "+&v"(y[3])
            : SSAM_INPUTS);
#undef SSAM_DOT
#undef SSAM_INPUTS
}
// Sums over the lane groups of a channel of four rows' values that quad_dots made.  Each group is left with one row's sum (GL = 4) or
// two (GL = 2): y[j], j a multiple of GL, is row j + sum_row.  The adds write only the groups (banks of four lanes) that keep that
// row: six in place of the eight that leave every sum everywhere, and a quarter of the stores.
template <int GL> __device__ __forceinline__ int sum_row(int lane) { return GL == 4 ? 0x1302 >> lane_group<4>(lane) * 4 & 3 : lane_group<GL>(lane); }
template <int GL>
__device__ __forceinline__ void group_sums(float (&y)[4])
{
    if constexpr (GL == 4)
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"      // rows 0, 1 in two groups each
            "v_add_f32_dpp %1, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"      // rows 2, 3
            "s_nop 0\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
            "v_add_f32_dpp %0, %1, %1 row_ror:12 row_mask:0xf bank_mask:0x5"
            : "+v"(y[0]), "+v"(y[2])
            : "v"(y[1]), "v"(y[3]));
    if constexpr (GL == 2)
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %1, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xc"
            : "+v"(y[0]), "+v"(y[2])
            : "v"(y[1]), "v"(y[3]));
}

// One row's sum of cQ h[Q]; h may come from the matrix instruction, hence five wait states.
__device__ __forceinline__ float quad_dot(float c, float h0, float h1, float h2, float h3)
{
    float y;
    asm("s_nop 4\n\t"
        "v_mul_f32_dpp %0, %1, %2 quad_perm:[0,0,0,0] row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %3 quad_perm:[1,1,1,1] row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %4 quad_perm:[2,2,2,2] row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %5 quad_perm:[3,3,3,3] row_mask:0xf bank_mask:0xf"
        : "=&v"(y)
        : "v"(c), "v"(h0), "v"(h1), "v"(h2), "v"(h3));
    return y;
}
// Two values' sums over the lane groups of a channel; these blocks may have made either.
template <int GL>
__device__ __forceinline__ void group_sums(float& r, float& s)
{
    if constexpr (GL == 4)
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "s_nop 0\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:4 row_mask:0xf bank_mask:0xf"
            : "+v"(r), "+v"(s));
    if constexpr (GL == 2)
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf"
            : "+v"(r), "+v"(s));
}

// Where the values of a row's b and c lie in LDS: the NS / 4 that a lane loads side by side.  Lane (group, quad lane j) needs states
// group * NS + 4 m + j.
template <class Shape> __device__ __forceinline__ int pair_place(int n) { return (n / Shape::NS * 4 + n % 4) * (Shape::NS / 4) + n % Shape::NS / 4; }
template <class Shape> __device__ __forceinline__ int own_pairs(int lane) { return (lane_group<Shape::GL>(lane) * 4 + (lane & 3)) * (Shape::NS / 4); }

// Where the channels of a tile lie in LDS: a thread loads E neighbours and spreads them over the row in steps of CB / E (channel c at
// c % E * (CB / E) + c / E), so that the lanes of a wave, each with its e-th value, write one run.  A lane works on the channel at its place.
template <int CB, int E> __device__ __forceinline__ int placed_channel(int at) { return at % (CB / E) * E + at / (CB / E); }

// A layout's places for states lie in blocks of four, one vector each.  The last block with states of its own starts further left where it
// would pass their end, and the blocks behind hold the first ones' again, so that some states are held two times (counts below four: element
// by element, up to eight times).  Their copies run alike; c's value is shared out between them, a power of two of them, so that nothing is
// rounded and their terms add up to the one.  Zeros for b and c in the places left over would not do: an infinite input or gradient times zero
// is NaN, and NaN times zero would reach y.  (4 x 2048 rows of 2048 channels, forward and gradients: 13 states 127 and 344 us, 50 states 396
// and 1711; with zeros kept by selections 139 and 389, 465 and 1963; with nothing against NaN 129 and 352, 401 and 1752.)  In the gradients
// the copies of g are shares too; what leaves is multiplied by their number.
__device__ __forceinline__ int state_block(int j, int states)      // first state of block j; at least four states
{
    const int blocks = (states + 3) / 4, first = 4 * (j < blocks ? j : j - blocks);
    return first < states - 4 ? first : states - 4;
}
__device__ __forceinline__ int state_at(int place, int states)
{
    if (states >= 4) return state_block(place / 4, states) + place % 4;
    return states == 3 ? (place % 4 < 2 ? place % 4 : 2) : place & (states - 1);
}
// How many of `held` places hold what place i of block j holds.  More than half of the places have a state of their own, or there are at most
// four states, so of four and more it is two below `lo` and from `hi` on, else one.
struct StateCopies {
    int states, held, lo, hi;
    __device__ __forceinline__ StateCopies(int j, int states_, int held_) : states(states_), held(held_)
    {
        const int blocks = (states + 3) / 4, again = held / 4 - blocks, b = j < blocks ? j : j - blocks, over = 4 * blocks - states;
        lo = b < again ? 4 : b == blocks - 1 ? over : 0;
        hi = b == blocks - 2 ? 4 - over : 4;
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if (states < 4) return (float)(held / 4 * (states == 1 ? 4 : states == 2 || i >= 2 ? 2 : 1));
        return i < lo || i >= hi ? 2.0f : 1.0f;
    }
};

// A channel's NS states of this lane, places n0 .. , in an array [..][channels][states]; zeros / not stored where it is not there.
// kShared: there may be more places than states.
template <int NS, bool kShared = true>
__device__ __forceinline__ void load_states(const float* __restrict__ a, int n0, int states, bool there, float (&h)[NS])
{
#pragma unroll
    for (int m = 0; m < NS; m += 4) {
        RowVec<float, 4> v(0.0f);
        if (!kShared) {
            v = load_row_vec<float, 4>(a + n0 + m, there ? states - n0 - m : 0);
        } else if (states < 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (there) v[i] = a[state_at(i, states)];
        } else if (there) {
            v = load_row_vec<float, 4>(a + state_block((n0 + m) / 4, states), 4);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) h[m + i] = v[i];
    }
}
template <int NS, bool kShared = true>
__device__ __forceinline__ void store_states(float* __restrict__ a, int n0, int states, bool there, const float (&h)[NS])
{
#pragma unroll
    for (int m = 0; m < NS; m += 4) {
        const RowVec<float, 4> v = {h[m], h[m + 1], h[m + 2], h[m + 3]};
        if (!kShared) {
            if (there) store_row_vec<float, 4>(a + n0 + m, 4, v);
        } else if (states >= 4) {
            if (there && n0 + m < states) store_row_vec<float, 4>(a + state_block((n0 + m) / 4, states), 4, v);
        } else if (n0 + m == 0) {
            store_row_vec<float, 4>(a, there ? states : 0, v);
        }
    }
}

// A decay rate for exp2.  An infinity (-inf: a state that forgets at once) becomes the last finite value, so that a time step of zero
// leaves the state alone there too: rows behind a sequence pass as such.
__device__ __forceinline__ float decay_rate(float a)
{
    const float r = a * kLog2e;
    return __builtin_fabsf(r) == __builtin_inff() ? __builtin_copysignf(3.402823466e38f, r) : r;
}
template <int NS, bool kShared = true>
__device__ __forceinline__ void load_rates(const float* __restrict__ a, int n0, int states, bool there, float (&a2)[NS])
{
    load_states<NS, kShared>(a, n0, states, there, a2);
#pragma unroll
    for (int i = 0; i < NS; ++i) a2[i] = decay_rate(a2[i]);
}

// The tile of channels of a block: blocks never span two groups of b and c.
struct ChannelTile {
    int group, c0, n;     // group, first channel, channels
};
__device__ __forceinline__ ChannelTile channel_tile(int tile, int per_group, int group_channels, int wide)
{
    ChannelTile t;
    t.group = tile / per_group;
    const int at = (tile - t.group * per_group) * wide;
    t.c0 = t.group * group_channels + at;
    t.n = group_channels - at < wide ? group_channels - at : wide;
    return t;
}

// What a thread loads of a tile of K rows x CB channels: E neighbours of one row.  There are no branches on it: a vector that would
// pass the tile's last channel starts further left instead (its channels are then another thread's too; both write the same values
// to the same places), a row behind the piece is read as the piece's last.  Only tiles of fewer than E channels go by elements.
template <class T, int K, int CB, int E>
struct TileLane {
    int row, col, wide;          // row of the tile; first channel; channels of the tile
    bool narrow;

    __device__ __forceinline__ TileLane(int tid, int n)
        : row(tid * E / CB), col(tid * E % CB), wide(n), narrow(n < E)
    {
        if (col + E > n) col = narrow ? 0 : n - E;
    }
    // `base`: the tile's row 0, channel 0 (the same for all threads); `left`: rows from there to the piece's end, at least 1
    __device__ __forceinline__ unsigned offset(long long stride, int left) const
    {
        return (unsigned)(row < left ? row : left - 1) * (unsigned)stride + (unsigned)col;
    }
    __device__ __forceinline__ RowVec<T, E> load(const T* __restrict__ base, long long stride, int left) const
    {
        return load_row_vec<T, E>(base + offset(stride, left), narrow ? wide : E, narrow);
    }
    __device__ __forceinline__ void store(T* __restrict__ base, long long stride, int left, const RowVec<T, E>& v) const
    {
        if (row < left) store_row_vec<T, E>(base + offset(stride, left), narrow ? wide : E, v, narrow);
    }
    // LDS place of its e-th channel
    __device__ __forceinline__ int place(int e) const
    {
        const int c = col + e;
        return (c % E) * (CB / E) + c / E;
    }
};

// f gets the lane layout for a number of states as a compile-time constant.
template <class F>
int with_shape(int states, F f)
{
    if (states <= 4) return f(ScanShape<1, 4>{});
    if (states <= 8) return f(ScanShape<2, 4>{});
    if (states <= 16) return f(ScanShape<4, 4>{});
    if (states <= 32) return f(ScanShape<4, 8>{});
    return f(ScanShape<4, 16>{});
}
// f gets whether there are more places than states as a compile-time constant.
template <int kPlaces, class F>
int with_shared(int states, F f)
{
    return states < kPlaces ? f(std::true_type{}) : f(std::false_type{});
}
template <class F>
int with_row_type(int dtype, F f)
{
    if (dtype == SSAM_F32) return f(float());
    if (dtype == SSAM_F16) return f(_Float16());
    return f(__bf16());
}

inline int check_scan(int dtype, int channels, int states, int groups)
{
    if (dtype != SSAM_F32 && dtype != SSAM_F16 && dtype != SSAM_BF16) return SSAM_ERR_ENUM;
    if (channels <= 0 || channels > kMaxChannels) return SSAM_ERR_DIM;
    if (states < 1 || states > SSAM_MAX_STATES || groups < 1 || channels % groups) return SSAM_ERR_SHAPE;
    return SSAM_OK;
}

// Blocks along the channels, and the widest channel tile.
inline int tile_channels(int states) { return states <= 4 ? 256 : states <= 8 ? 128 : 64; }
inline int tiles_per_group(int channels, int states, int groups)
{
    const int w = tile_channels(states);
    return (channels / groups + w - 1) / w;
}

// b and c: groups x states elements, `apart` from group to group.
inline long long group_width(int groups, int states, long long apart) { return run_extent(groups, apart, states); }

// b and c of a call, whichever.
template <class Args>
int check_group_rows(const Args& a, const ssam_sequences& q, int esz)
{
    if (a.b_group < 0 || a.b_group > kMaxStride || a.c_group < 0 || a.c_group > kMaxStride) return SSAM_ERR_DIM;
    if (int e = check_rows(a.b, q, group_width(a.groups, a.states, a.b_group), esz, false)) return e;
    return check_rows(a.c, q, group_width(a.groups, a.states, a.c_group), esz, false);
}

// ---- sequences in pieces ------------------------------------------------------------------------------------------------
// Rows of a piece, a multiple of 32, so that sequences x channel tiles x pieces come to about `blocks` blocks; one piece a sequence
// where `alone` sequences x channel tiles are there without.
int scan_piece_rows(const ssam_sequences& q, int tiles, int blocks, int alone);

// Pieces that another follows, at most rows / piece of them in the packed form however many sequences there are, have an entry of
// [channels][states] in `ends` and of [channels] in `sums`: the piece in slot `slot` of sequence `seq` this one.
__device__ __forceinline__ int end_entry(const Pieces& q, int slot, int seq) { return q.begin ? slot - seq : slot; }
// The forward direction keeps the states before cut sequences too: of the sequence whose first piece is in slot `slot` here.
__device__ __forceinline__ int start_entry(const Pieces& q, int slot, int seq)
{
    if (!q.begin) return slot + q.per - 1;
    const int followed = q.rows / q.piece;
    return followed + (q.sequences <= followed ? seq : slot - seq);
}
inline long long end_entries(const ssam_sequences& q, int piece, bool starts)
{
    if (!q.d_begin) return piece_slots(q, piece);
    const long long followed = q.rows / piece;
    return followed + (starts ? q.sequences < followed ? q.sequences : followed : 0);
}

// Turns what each piece adds to the state into the states between the pieces: `ends` and `sums`, the time steps of a piece added up (its
// decay is exp(a * sum)), by entries.
//   forward:  the entry of a piece becomes the state behind it, from `initial` (zeros without) before the first, which itself goes into
//             the sequence's start entry
//   backward: the entry of a piece holds what the NEXT one lets out at its first row, and becomes all of that, from `initial` (the gradient
//             of the last state) behind the last piece
int launch_join(const Pieces& p, float* ends, const float* sums, const float* a, const float* initial, int channels, int states, bool backward,
                hipStream_t stream);

}  // namespace ssam
