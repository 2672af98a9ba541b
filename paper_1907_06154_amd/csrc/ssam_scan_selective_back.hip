// Gradients of the selective scan.  With dy the gradient at y, per channel and state
//     g_t = c_t dy_t + a_{t+1} g_{t+1}                     (a_t = exp(d_t a), x_t = a_t h_{t-1}, q_t = g_t x_t)
//     db_t = sum over channels g_t d_t u_t,  dc_t = sum over channels h_t dy_t
//     du_t = skip dy_t + d_t s_t,  dd_t = r_t + u_t s_t    with s_t = sum_n g_t b_t, r_t = sum_n a q_t
//     da = sum_t d_t q_t,  dskip = sum_t dy_t u_t,  ddt_t = dd_t sigmoid(dt_t + bias),  dbias = sum_t ddt_t
// The rows run backwards, in tiles of 16; a tile starts from the forward call's mark (the state before its first row) and makes its
// states again, part of a tile at a time: 8 rows' states and decays in registers (up to 16 states), 64 of them, and back over those.
// (Marks every 8 rows would save the second half's way to its first row, 9 of 72 cycles a state, for 4 bytes more per row, channel and
// 16 states, written and read; keeping 16 rows takes 128 registers and spills.)
// Bound by vector issue: 22 instructions per row, channel and state, two waves a SIMD, which 233 registers leave; 4 x 2048 rows of 2048
// channels and 16 states 270 us, what the pieces let out 61, the forward call 135.  With 16 states nothing spills; the kernels that do, by bytes
// of scratch a lane: 8 states in 16 bits 52 and 80 (fewer than 8: 72 and 100), 32 states in fp32 28 (fewer: 48), fewer than 32 in 16 bits 16 - 24.
//
// The sums over channels: a wave's and the block's waves' through LDS, the blocks of a group through the workspace and a launch that
// adds them in order.
#include "ssam_scan_selective.h"

namespace ssam {
namespace {

constexpr int kTile = SSAM_MARK_ROWS;
constexpr int kBackBlocks = 1024;     // two rounds of the two blocks per compute unit that 256 registers leave
// The parameters' gradients of every slot are a workspace: of more blocks than this at once, launch after launch (32 to a compute unit are
// enough for its ends not to matter; 4096 sequences of 8 rows, 4096 channels, 16 states: 151 MB for 1.2 GB).
constexpr long long kPartBlocks = 1 << 15;
constexpr long long kMaxGroupStates = 1 << 27;   // groups x states: offsets in a tile's rows of both then have 32 bits
constexpr int kBackAlone = 512;       // sequences x channel tiles that are enough without cutting (8 x 8192 rows of 2048 channels, 256 of them: 505 us cut, 551 whole)

struct BackParams {
    Pieces pieces, mark_slots;
    ssam_rows in, dt, gate, b, c, grad_out;
    long long b_group, c_group;
    const float *a, *skip, *dt_bias, *marks, *grad_final;
    ssam_rows grad_in, grad_dt, grad_gate, grad_b, grad_c;
    float* grad_state;
    float *ends, *sums;               // pieces: what reaches each from behind
    float* part_bc;                   // [tile of the group][row][group][2][states]
    float* part_param;                // [slot of the launch][channels x states, channels (skip), channels (bias)]
    int slot0;                        // of the launch
    long long rows_total;
    int channels, states, groups, group_channels, per_group, tiles, softplus;
};

template <int CTRL>
__device__ __forceinline__ float quad_moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// Sums over a wave's channels of four states' terms of b's and of c's gradient.  The lanes put their terms into LDS, one vector
// each, and every output -- 4 GL states of b, as many of c -- is added up by LP lanes, eight channels each: 8 vector instructions
// where swaps between rows of lanes and DPP took 22.  A wave reads what itself wrote (the LDS keeps a wave's order), one step later,
// so no barrier and no wait is needed.  The vectors lie so that eight lanes' writes and 32 lanes' reads each meet every bank once.
// A lane without a channel writes beside them: its terms are zeros, or NaN where b or c is infinite, and the zeros in its own vectors stay.
template <int GL>
struct ChannelSums {
    static constexpr int kOutputs = 8 * GL, LP = kWave / kOutputs;
    static constexpr int kApart = 92 * 4;                // b's terms, then c's
    static constexpr int kFloats = 2 * kApart;           // of one step

    float* at;           // this wave's two steps
    int to, from, which, i, group;

    // channel c of group g
    static __device__ __forceinline__ int vector(int c, int g) { return c % LP + LP * g + 12 * (c / LP % 2) + 24 * (c / (2 * LP)); }
    __device__ __forceinline__ ChannelSums(float* buffer, int lane, bool live)
    {
        const int o = lane / LP, part = lane % LP;
        i = o % 4;
        group = o / 4 % GL;
        which = o / (4 * GL);
        at = buffer;
        to = (live ? vector(lane_channel<GL>(lane), lane_group<GL>(lane)) : 8 + lane % 4) * 4;      // (8 .. 11 are no lane's)
        from = which * kApart + vector(part, group) * 4 + i;
    }
    __device__ __forceinline__ void put(int step, const float (&vb)[4], const float (&vc)[4]) const
    {
        float* p = at + (step & 1) * kFloats + to;
        *reinterpret_cast<RowVec<float, 4>*>(p) = RowVec<float, 4>{vb[0], vb[1], vb[2], vb[3]};
        *reinterpret_cast<RowVec<float, 4>*>(p + kApart) = RowVec<float, 4>{vc[0], vc[1], vc[2], vc[3]};
        __builtin_amdgcn_wave_barrier();     // no instruction: the compiler keeps the other lanes' reads behind it
    }
    // channels part, part + LP, ..
    __device__ __forceinline__ void take(int step, float (&t)[8]) const
    {
        const float* p = at + (step & 1) * kFloats + from;
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = p[(12 * (k & 1) + 24 * (k >> 1)) * 4];
    }
    static __device__ __forceinline__ float sum(const float (&t)[8])
    {
        float v = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        if (LP >= 2) v += quad_moved<0xB1>(v);
        if (LP >= 4) v += quad_moved<0x4E>(v);
        return v;
    }
    // the state of this lane's output, for the vector of number m
    template <int NS> __device__ __forceinline__ int state(int m) const { return group * NS + 4 * m + i; }
};

// kWhole: everything.  !kWhole: only what a piece lets out at its first row when nothing reaches it from behind.
template <class T, class Shape, bool kWhole, bool kShared>
__global__ __launch_bounds__(kBlock, Shape::NS <= 8 ? 2 : 1) void scan_back(BackParams p)
{
    constexpr int GL = Shape::GL, NS = Shape::NS, NP = Shape::kStates, CB = Shape::kChannels, K = kTile;
    constexpr int E = K * CB / kBlock;                   // values of a thread
    constexpr int kPairs = (K * NP + kBlock - 1) / kBlock;
    // Rows whose states and decays are kept at a time, half of what spills much more (fp32 with eight values a thread: 456 us, 377 with four rows).
    constexpr int kKept = NS == 16 || (E >= 8 && sizeof(T) == 4) ? 4 : 32 / NS;
    constexpr bool kMarkAhead = NS < 16;                 // the next tile's mark is requested with its rows
    // Whether a row counts for the rates' gradient is a branch behind the row, with more states a lane a selection each, whose values need
    // not be held so long (8 states 235 us, by selections 239; 20 states fp32 674 and 654).
    constexpr bool kRowBranch = NS == 4;
    constexpr int kRow = CB + CB / E;                    // a row in LDS, padded: see scan_rows
    // A thread's eight values' parameters, 16 registers, come from LDS: those would spill too (8 states 396 -> 330 us; four values' do not, and are held).
    constexpr bool kFromLds = E >= 8;
    using Pair = RowVec<float, 2>;
    __shared__ Pair dx[K][kRow];                         // d, d u
    __shared__ float dys[K][kRow];                       // dy; from a row's turn on its y, read and written by one wave
    __shared__ Pair bc[K][NP];
    __shared__ float per_channel[2][kFromLds ? CB : 1];  // bias of dt, skip
    __shared__ Pair rs[kWhole ? K : 1][kRow];            // r, s
    __shared__ float sum_bc[kWhole ? kWavesPerBlock : 1][K][2][NP];
    __shared__ __attribute__((aligned(16))) float terms[kWhole ? kWavesPerBlock : 1][2 * ChannelSums<GL>::kFloats];

    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
    const int slot = blockIdx.x / p.tiles + p.slot0;
    const ChannelTile ct = channel_tile(blockIdx.x % p.tiles, p.per_group, p.group_channels, CB);
    const Piece q = find_piece(p.pieces, slot);
    const long long plane = (long long)p.channels * p.states;
    const int place = wave * Shape::kWaveChannels + lane_channel<GL>(lane);
    const int ch = placed_channel<CB, E>(place);
    const bool live = ch < ct.n;
    const int n0 = lane_group<GL>(lane) * NS;
    const long long cell = (long long)(ct.c0 + ch) * p.states;
    float* part_param = kWhole && p.part_param ? p.part_param + (slot - p.slot0) * (plane + 2LL * p.channels) : nullptr;
    if (q.seq < 0) {
        if (part_param) {       // an empty slot adds zeros
            float none[NS] = {};
            store_states<NS, kShared>(part_param + cell, n0, p.states, live, none);
            if (tid < ct.n) part_param[plane + ct.c0 + tid] = part_param[plane + p.channels + ct.c0 + tid] = 0.0f;
        }
        return;
    }
    if (!kWhole && q.row0 == 0) return;                  // nothing lies before it

    float a2[NS], g[NS], da[NS];
    load_rates<NS, kShared>(p.a + cell, n0, p.states, live, a2);
    const bool last = q.row0 + q.n >= q.len;
    if (!kWhole) load_states<NS, kShared>(nullptr, 0, 0, false, g);
    else if (!last) load_states<NS, kShared>(p.ends + end_entry(p.pieces, slot, q.seq) * plane + cell, n0, p.states, live, g);
    else load_states<NS, kShared>(p.grad_final + q.seq * plane + cell, n0, p.states, live && p.grad_final, g);
    // !kWhole: the states do not meet, and every copy has the whole of g.
    auto state_of = [&](int place) { return kShared ? state_at(place, p.states) : place; };
    auto copies = [&](int place) { return kWhole && kShared ? StateCopies(place / 4, p.states, NP)[place % 4] : 1.0f; };
#pragma unroll
    for (int i = 0; i < NS; ++i) da[i] = 0.0f;
    float sum = 0.0f;
    const float* marks = nullptr;
    if (kWhole) {
        const long long s0 = p.mark_slots.begin ? first_slot(p.mark_slots, q.seq) : (long long)q.seq * p.mark_slots.per;
        marks = p.marks + (s0 + q.row0 / K) * plane + cell;
    }

    const TileLane<T, K, CB, E> mine(tid, ct.n);
    const bool gated = p.gate.d;
    const T* in = sequence_base<T>(p.in, p.pieces, q) + (long long)q.row0 * p.in.row + ct.c0;
    const T* dt = sequence_base<T>(p.dt, p.pieces, q) + (long long)q.row0 * p.dt.row + ct.c0;
    const T* gate = gated ? sequence_base<T>(p.gate, p.pieces, q) + (long long)q.row0 * p.gate.row + ct.c0 : nullptr;
    const T* dout = sequence_base<T>(p.grad_out, p.pieces, q) + (long long)q.row0 * p.grad_out.row + ct.c0;
    const T* pb = sequence_base<T>(p.b, p.pieces, q) + (long long)q.row0 * p.b.row + ct.group * p.b_group;
    const T* pc = sequence_base<T>(p.c, p.pieces, q) + (long long)q.row0 * p.c.row + ct.group * p.c_group;
    T* grad_in = kWhole && p.grad_in.d ? sequence_base<T>(p.grad_in, p.pieces, q) + (long long)q.row0 * p.grad_in.row + ct.c0 : nullptr;
    T* grad_dt = kWhole && p.grad_dt.d ? sequence_base<T>(p.grad_dt, p.pieces, q) + (long long)q.row0 * p.grad_dt.row + ct.c0 : nullptr;
    T* grad_gate = kWhole && p.grad_gate.d && gated ? sequence_base<T>(p.grad_gate, p.pieces, q) + (long long)q.row0 * p.grad_gate.row + ct.c0 : nullptr;
    const long long row_total = (p.pieces.begin ? (long long)q.first : (long long)q.seq * p.pieces.rows) + q.row0;
    float* part_bc = kWhole && p.part_bc
                         ? p.part_bc + (((long long)(blockIdx.x % p.tiles - ct.group * p.per_group) * p.rows_total + row_total) * p.groups + ct.group) *
                                           2 * p.states
                         : nullptr;
    float bias_held[E], skip_held[E], dskip[E], dbias[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dskip[e] = dbias[e] = 0.0f;
    auto bias_of = [&](int c) { return p.dt_bias && c < ct.n ? p.dt_bias[ct.c0 + c] : 0.0f; };
    auto skip_of = [&](int c) { return kWhole && p.skip && c < ct.n ? p.skip[ct.c0 + c] : 0.0f; };
    if constexpr (kFromLds) {
        if (tid < CB) {
            per_channel[0][tid] = bias_of(tid);
            per_channel[1][tid] = skip_of(tid);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            bias_held[e] = bias_of(mine.col + e);
            skip_held[e] = skip_of(mine.col + e);
        }
    }
    auto bias = [&](int e) { return kFromLds ? per_channel[0][mine.col + e] : bias_held[e]; };
    auto skip = [&](int e) { return kFromLds ? per_channel[1][mine.col + e] : skip_held[e]; };
    // Channels behind the tile keep d = 0, d u = 0, dy = 0 throughout.
    if (ct.n < CB)
        for (int i = tid; i < K * kRow; i += kBlock) {
            dx[i / kRow][i % kRow] = Pair{0.0f, 0.0f};
            dys[i / kRow][i % kRow] = 0.0f;
        }
    if (kWhole && ct.n < CB)
        for (int i = lane; i < 2 * ChannelSums<GL>::kFloats; i += kWave) terms[wave][i] = 0.0f;
    __syncthreads();                                     // before the first tile's values go there

    using Vec = RowVec<T, E>;
    Vec u, dr, z, go, u_next, d_next, z_next, g_next;
    T b_next[kPairs], c_next[kPairs];
    static_assert(kBlock % (2 * NP) == 0, "a thread's values of b and c are all of one state, its sums for their gradients too");
    float mark[NS], mark_next[NS];
    auto request = [&](int row) {
        const int left = q.n - row;
        if (kWhole) u_next = mine.load(in + (long long)row * p.in.row, p.in.row, left);
        d_next = mine.load(dt + (long long)row * p.dt.row, p.dt.row, left);
        g_next = mine.load(dout + (long long)row * p.grad_out.row, p.grad_out.row, left);
        if (gated) z_next = mine.load(gate + (long long)row * p.gate.row, p.gate.row, left);
        const T* b0 = kWhole ? pb + (long long)row * p.b.row : nullptr;
        const T* c0 = pc + (long long)row * p.c.row;
        const int state = state_of(tid % NP);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const int i = tid + e * kBlock;
            const unsigned r = i / NP < left ? i / NP : left - 1;
            if (kWhole) b_next[e] = b0[r * (unsigned)p.b.row + state];
            c_next[e] = c0[r * (unsigned)p.c.row + state];
        }
        if (kWhole && kMarkAhead) load_states<NS, kShared>(marks + (row / K) * plane, n0, p.states, live, mark_next);
    };
    const int pairs = own_pairs<Shape>(lane), sum_at = sum_row<GL>(lane);
    const ChannelSums<GL> across(terms[kWhole ? wave : 0], lane, live);

    const int tiles = (q.n + K - 1) / K;
    if (tiles > 0) request((tiles - 1) * K);
#pragma unroll
    for (int i = 0; i < NS; ++i) g[i] *= 1.0f / copies(n0 + i);        // (waits for g, so behind the first tile's requests)
    for (int tile = tiles - 1; tile >= 0; --tile) {
        const int row = tile * K;
        const bool behind = row + mine.row >= q.n;       // a row behind the piece: d = 0, dy = 0, b = c = 0, it passes states and gradients unchanged
        u = u_next;
        dr = d_next;
        z = z_next;
        go = g_next;
        if (kWhole && kMarkAhead)
#pragma unroll
            for (int i = 0; i < NS; ++i) mark[i] = mark_next[i];
        float dy[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float raw = (float)dr[e] + bias(e);
            float v = p.softplus ? softplus(raw) : raw;
            dy[e] = (float)go[e];
            if (gated) dy[e] *= silu((float)z[e]);
            const bool is = !behind && (!mine.narrow || e < mine.wide);
            v = is ? v : 0.0f;
            dy[e] = is ? dy[e] : 0.0f;
            dx[mine.row][mine.place(e)] = Pair{v, is && kWhole ? v * (float)u[e] : 0.0f};
            dys[mine.row][mine.place(e)] = dy[e];
        }
        const float share = 1.0f / copies(tid % NP);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const int i = tid + e * kBlock, n = i % NP;
            const bool is = row + i / NP < q.n;
            if (kPairs * kBlock <= K * NP || i < K * NP)
                bc[i / NP][pair_place<Shape>(n)] = Pair{kWhole && is ? (float)b_next[e] : 0.0f, is ? (float)c_next[e] * share : 0.0f};
        }
        __syncthreads();
        if (tile > 0) request(row - K);

        if constexpr (!kWhole) {
#pragma unroll 1
            for (int t0 = K - 4; t0 >= 0; t0 -= 4) {
                float d4[4], dy4[4], c4[4][NS / 4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    d4[k] = dx[t0 + k][place][0];
                    dy4[k] = dys[t0 + k][place];
#pragma unroll
                    for (int m = 0; m < NS / 4; ++m) c4[k][m] = bc[t0 + k][pairs + m][1];
                }
#pragma unroll
                for (int m = 0; m < NS / 4; ++m) {
                    float e[4][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[k][i] = exp2_fast(d4[k] * a2[4 * m + i]);
#pragma unroll
                    for (int k = 3; k >= 0; --k) {
                        const RowVec<float, 4> gv = quad_outer(c4[k][m], dy4[k], RowVec<float, 4>{g[4 * m], g[4 * m + 1], g[4 * m + 2], g[4 * m + 3]});
#pragma unroll
                        for (int i = 0; i < 4; ++i) g[4 * m + i] = gv[i] * e[k][i];
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) sum += d4[k];
            }
        } else {
#pragma unroll 1
            for (int part = K / kKept - 1; part >= 0; --part) {
                // the states again, from the mark: those before this part's rows in passing, then each row's
                float h[NS], hs[kKept][NS], as[kKept][NS], dyr[kKept];
                Pair dv[kKept], w[kKept][NS / 4];
                if (!kMarkAhead) load_states<NS, kShared>(marks + tile * plane, n0, p.states, live, mark);
#pragma unroll
                for (int k = 0; k < kKept; ++k) {
                    dv[k] = dx[part * kKept + k][place];
                    dyr[k] = dys[part * kKept + k][place];
#pragma unroll
                    for (int m = 0; m < NS / 4; ++m) w[k][m] = bc[part * kKept + k][pairs + m];
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) h[i] = mark[i];
                for (int t0 = 0; t0 < part * kKept; t0 += 4) {
#pragma unroll
                    for (int t = t0; t < t0 + 4; ++t) {
                        const Pair d = dx[t][place];
#pragma unroll
                        for (int m = 0; m < NS / 4; ++m) {
                            const float b = bc[t][pairs + m][0];
                            const RowVec<float, 4> v = quad_outer(b, d[1], RowVec<float, 4>{});
#pragma unroll
                            for (int i = 0; i < 4; ++i) h[4 * m + i] = __builtin_fmaf(exp2_fast(d[0] * a2[4 * m + i]), h[4 * m + i], v[i]);
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < kKept; ++k) {
                    const float* before = k ? hs[k - 1] : h;
#pragma unroll
                    for (int m = 0; m < NS / 4; ++m) {
                        const float b = w[k][m][0], x = dv[k][1];
                        const RowVec<float, 4> v = quad_outer(b, x, RowVec<float, 4>{});
#pragma unroll
                        for (int i = 4 * m; i < 4 * m + 4; ++i) {
                            as[k][i] = exp2_fast(dv[k][0] * a2[i]);
                            hs[k][i] = __builtin_fmaf(as[k][i], before[i], v[i - 4 * m]);
                        }
                    }
                }
                if (gated) {             // y, for the gate's gradient
#pragma unroll
                    for (int k = 0; k < kKept; k += 4) {
                        float y[4];
#pragma unroll
                        for (int m = 0; m < NS / 4; ++m) {
                            float c[4], hm[4][4];
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                c[r] = w[k + r][m][1];
#pragma unroll
                                for (int i = 0; i < 4; ++i) hm[r][i] = hs[k + r][4 * m + i];
                            }
                            if (m == 0) quad_dots<true>(y, c, hm);
                            else quad_dots<false>(y, c, hm);
                        }
                        group_sums<GL>(y);
#pragma unroll
                        for (int r = 0; r < 4; r += GL) dys[part * kKept + k + r + sum_at][place] = y[r];
                    }
                }
                float terms_of[8];
#pragma unroll
                for (int k = kKept - 1; k >= 0; --k) {
                    const int t = part * kKept + k;
                    const float* before = k ? hs[k - 1] : h;
                    const bool own = row + t < q.n;       // of a row behind the piece, `before` is the last state, which may be infinite
                    float r = 0.0f, s = 0.0f, qs[kRowBranch ? NS : 1];
#pragma unroll
                    for (int m = 0; m < NS / 4; ++m) {
                        const int step = (kKept - 1 - k) * (NS / 4) + m;
                        if (step > 0) across.take(step - 1, terms_of);       // added up below: their reads pass this step's arithmetic
                        float *gm = g + 4 * m, vb[4], vc[4];
                        const RowVec<float, 4> gv = quad_outer(w[k][m][1], dyr[k], RowVec<float, 4>{gm[0], gm[1], gm[2], gm[3]});
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            gm[j] = gv[j];
                            vc[j] = hs[k][4 * m + j] * dyr[k];
                            vb[j] = gm[j] * dv[k][1];
                        }
                        const float sm = quad_dot(w[k][m][0], gm[0], gm[1], gm[2], gm[3]);
                        s = m ? s + sm : sm;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int i = 4 * m + j;
                            g[i] *= as[k][i];                      // what reaches the row before
                            const float qi = g[i] * before[i];
                            if constexpr (kRowBranch) qs[i] = qi;
                            else da[i] = own ? __builtin_fmaf(dv[k][0], qi, da[i]) : da[i];
                            r = i ? __builtin_fmaf(a2[i], qi, r) : a2[i] * qi;
                        }
                        across.put(step, vb, vc);
                        if (step > 0) {
                            const int tp = m ? t : t + 1, mp = m ? m - 1 : NS / 4 - 1;
                            sum_bc[wave][tp][across.which][across.template state<NS>(mp)] = across.sum(terms_of);
                        }
                    }
                    group_sums<GL>(r, s);
                    rs[t][place] = Pair{r, s};
                    if constexpr (kRowBranch) {
                        if (own) {
                            asm volatile("");           // (else the compiler makes selections of it)
#pragma unroll
                            for (int i = 0; i < NS; ++i) da[i] = __builtin_fmaf(dv[k][0], qs[i], da[i]);
                        }
                    }
                }
                across.take(kKept * (NS / 4) - 1, terms_of);
                sum_bc[wave][part * kKept][across.which][across.template state<NS>(NS / 4 - 1)] = across.sum(terms_of);
            }
        }
        __syncthreads();
        if constexpr (kWhole) {
            float du[E], ddt[E], dz[E];
            const int left = q.n - row;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int at = mine.place(e);
                const Pair v = rs[mine.row][at];
                const float ue = (float)u[e];
                du[e] = dx[mine.row][at][0] * v[1];
                if (p.skip) du[e] = __builtin_fmaf(skip(e), dy[e], du[e]);
                float dd = __builtin_fmaf(ue, v[1], v[0] * 0.693147180559945f);   // r was made with rates for exp2
                if (p.softplus) dd *= sigmoid((float)dr[e] + bias(e));
                ddt[e] = dd;
                dskip[e] += behind ? 0.0f : dy[e] * ue;
                dbias[e] += behind ? 0.0f : dd;
                if (gated) {
                    const float ze = (float)z[e], sig = sigmoid(ze);
                    const float y = dys[mine.row][at];
                    dz[e] = (float)go[e] * (p.skip ? __builtin_fmaf(skip(e), ue, y) : y) * (sig * __builtin_fmaf(ze, 1.0f - sig, 1.0f));
                } else {
                    dz[e] = 0.0f;
                }
            }
            if (grad_in) mine.store(grad_in + (long long)row * p.grad_in.row, p.grad_in.row, left, rounded<T, E>(du));
            if (grad_dt) mine.store(grad_dt + (long long)row * p.grad_dt.row, p.grad_dt.row, left, rounded<T, E>(ddt));
            if (grad_gate) mine.store(grad_gate + (long long)row * p.grad_gate.row, p.grad_gate.row, left, rounded<T, E>(dz));
            if (part_bc) {
                float* to = part_bc + (long long)row * p.groups * 2 * p.states;
                const unsigned wide = p.groups * 2 * p.states;
                const int state = state_of(tid % NP);
                const float parts = tid / NP % 2 ? 1.0f : copies(tid % NP);      // of the gradient of b
                for (int i = tid; i < K * 2 * NP; i += kBlock) {
                    const int r = i / (2 * NP), w = i / NP % 2, n = i % NP;
                    float v = sum_bc[0][r][w][n];
#pragma unroll
                    for (int k = 1; k < kWavesPerBlock; ++k) v += sum_bc[k][r][w][n];
                    if (r < left && (!kShared || n < (p.states + 3) / 4 * 4)) to[r * wide + w * p.states + state] = v * parts;
                }
            }
            __syncthreads();      // the next tile's values go where these were read
        }
    }
    if constexpr (kWhole) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            g[i] *= copies(n0 + i);
            da[i] *= copies(n0 + i);
        }
        if (p.grad_state && q.row0 == 0) store_states<NS, kShared>(p.grad_state + q.seq * plane + cell, n0, p.states, live, g);
        if (!part_param) return;
        store_states<NS, kShared>(part_param + cell, n0, p.states, live, da);
        // the tile's rows of every channel, added in order
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (!mine.narrow || e < mine.wide) rs[mine.row][mine.place(e)] = Pair{dskip[e], dbias[e]};
        __syncthreads();
        if (tid < ct.n) {
            const int at = tid % E * (CB / E) + tid / E;
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int r = 0; r < K; ++r) {
                s0 += rs[r][at][0];
                s1 += rs[r][at][1];
            }
            part_param[plane + ct.c0 + tid] = s0;
            part_param[plane + p.channels + ct.c0 + tid] = s1;
        }
    } else {
        const long long entry = end_entry(p.pieces, slot - 1, q.seq);
        store_states<NS, kShared>(p.ends + entry * plane + cell, n0, p.states, live, g);
        if (live && n0 == 0) p.sums[entry * p.channels + ct.c0 + ch] = sum;
    }
}

// Gradients of b and c: the tiles of a group added up, in order.  A block takes kSumRows rows, a thread values 256 apart, and keeps
// eight tiles' requests in flight (1537 rows of 32 states forward and back: 108 us, with eight rows a block 111).
constexpr int kSumRows = 4;
template <class T>
__global__ __launch_bounds__(kBlock) void back_sum_bc(BackParams p, Pieces rows)
{
    const Piece q = find_piece(rows, blockIdx.x);
    if (q.seq < 0) return;
    const long long row_total = (rows.begin ? (long long)q.first : (long long)q.seq * rows.rows) + q.row0;
    const int wide = p.groups * 2 * p.states;
    const long long apart = p.rows_total * wide;
    const float* __restrict__ from = p.part_bc + row_total * wide;
    for (int i = threadIdx.x; i < q.n * wide; i += kBlock) {
        float v = 0.0f;
#pragma unroll 8
        for (int k = 0; k < p.per_group; ++k) v += from[k * apart + i];
        const int r = i / wide, at = i % wide, grp = at / (2 * p.states), n = at % (2 * p.states);
        const ssam_rows& to = n < p.states ? p.grad_b : p.grad_c;
        if (to.d)
            sequence_base<T>(to, rows, q)[(long long)(q.row0 + r) * to.row + grp * p.states + (n < p.states ? n : n - p.states)] = (T)v;
    }
}

// Sums over a launch's slots, 16 interleaved runs of them and then the runs, always in the same order; `more`: on top of the launches before.
constexpr int kRuns = 16;
__global__ __launch_bounds__(kWave* kRuns) void back_sum_params(const float* __restrict__ parts, long long slots, long long plane, int channels,
                                                                float* grad_a, float* grad_skip, float* grad_dt_bias, bool more)
{
    __shared__ float run[kRuns][kWave];
    const int lane = threadIdx.x & (kWave - 1), r = threadIdx.x >> 6;
    const long long wide = plane + 2LL * channels;
    const long long i = (long long)blockIdx.x * kWave + lane;
    float s = 0.0f;
    if (i < wide)
        for (long long k = r; k < slots; k += kRuns) s += parts[k * wide + i];
    run[r][lane] = s;
    __syncthreads();
    if (r != 0 || i >= wide) return;
#pragma unroll
    for (int k = 1; k < kRuns; ++k) s += run[k][lane];
    float* to = i < plane ? grad_a ? grad_a + i : nullptr : i < plane + channels ? grad_skip ? grad_skip + (i - plane) : nullptr
                                                          : grad_dt_bias ? grad_dt_bias + (i - plane - channels) : nullptr;
    if (to) *to = more ? *to + s : s;
}

// As with_shape, but for eight states from one on: a tile of 256 channels would not fit the LDS twice.
template <class F>
int with_back_shape(int states, F f)
{
    if (states <= 8) return f(ScanShape<2, 4>{});
    if (states <= 16) return f(ScanShape<4, 4>{});
    if (states <= 32) return f(ScanShape<4, 8>{});
    return f(ScanShape<4, 16>{});
}

struct BackPlan {
    int per_group, tiles, piece;
    long long slots, slots_each, rows_total, blocks, sum_blocks;     // slots_each: of a launch of the main kernel
    bool fits, cut, params, bc;       // fits: no launch has more blocks than it may (without, the call is refused and needs no workspace)
    size_t ends, sums, part_bc, part_param, bytes;
};

size_t whole_lines(size_t bytes) { return (bytes + 127) / 128 * 128; }

BackPlan plan_of(const ssam_scan_selective_backward_args& a)
{
    BackPlan p{};
    const int wide = a.states <= 8 ? 128 : 64;
    p.per_group = (a.channels / a.groups + wide - 1) / wide;
    p.tiles = p.per_group * a.groups;
    p.piece = scan_piece_rows(a.seq, p.tiles, kBackBlocks, kBackAlone);
    p.slots = piece_slots(a.seq, p.piece);
    p.rows_total = a.seq.d_begin ? a.seq.rows : (long long)a.seq.rows * a.seq.sequences;
    p.blocks = p.slots * p.tiles;
    p.params = a.d_grad_a || a.d_grad_skip || a.d_grad_dt_bias;
    p.bc = a.grad_b.d || a.grad_c.d;
    p.slots_each = p.params && p.blocks > kPartBlocks ? (kPartBlocks + p.tiles - 1) / p.tiles : p.slots;
    p.sum_blocks = p.bc ? piece_slots(a.seq, kSumRows) : 0;
    p.fits = p.blocks <= kMaxGrid && p.sum_blocks <= kMaxGrid;
    if (!p.fits) return p;
    p.cut = a.seq.rows > p.piece;
    const size_t plane = (size_t)a.channels * a.states;
    const size_t entries = p.cut ? end_entries(a.seq, p.piece, false) : 0;
    p.ends = whole_lines(entries * plane * 4);
    p.sums = whole_lines(entries * a.channels * 4);
    p.part_bc = p.bc ? whole_lines((size_t)p.per_group * p.rows_total * a.groups * 2 * a.states * 4) : 0;
    p.part_param = p.params ? whole_lines((size_t)p.slots_each * (plane + 2 * (size_t)a.channels) * 4) : 0;
    p.bytes = p.ends + p.sums + p.part_bc + p.part_param;
    return p;
}

}  // namespace
}  // namespace ssam

extern "C" {

size_t ssam_scan_selective_backward_workspace_bytes(const ssam_scan_selective_backward_args* a)
{
    using namespace ssam;
    if (!a || check_scan(a->dtype, a->channels, a->states, a->groups) || check_sequences(a->seq)) return 0;
    return plan_of(*a).bytes;
}

int ssam_scan_selective_backward(const ssam_scan_selective_backward_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_scan(a->dtype, a->channels, a->states, a->groups)) return e;
    if (int e = check_sequences(a->seq)) return e;
    const BackPlan plan = plan_of(*a);
    if (a->seq.sequences == 0 && !plan.params) return SSAM_OK;
    const int esz = type_bytes(a->dtype);
    if (!a->d_a || (!a->d_marks && a->seq.sequences > 0)) return SSAM_ERR_NULL;
    if (int e = check_group_rows(*a, a->seq, esz)) return e;
    for (const ssam_rows* r : {&a->in, &a->dt, &a->grad_out})
        if (int e = check_rows(*r, a->seq, a->channels, esz, false)) return e;
    if (int e = check_rows(a->gate, a->seq, a->channels, esz, true)) return e;
    for (const ssam_rows* r : {&a->grad_in, &a->grad_dt, &a->grad_gate})
        if (int e = check_out_rows(*r, a->seq, a->channels, esz, true)) return e;
    for (const ssam_rows* r : {&a->in, &a->dt, &a->gate, &a->b, &a->c, &a->grad_out, &a->grad_in, &a->grad_dt, &a->grad_gate})
        if (int e = check_tile_rows(*r, a->seq)) return e;
    const long long bc_width = (long long)a->groups * a->states;
    if (bc_width >= kMaxGroupStates) return SSAM_ERR_DIM;
    for (const ssam_rows* r : {&a->grad_b, &a->grad_c})
        if (int e = check_out_rows(*r, a->seq, bc_width, esz, true)) return e;
    for (const void* f : {(const void*)a->d_a, (const void*)a->d_skip, (const void*)a->d_dt_bias, (const void*)a->d_marks, (const void*)a->d_grad_final,
                          (const void*)a->d_grad_a, (const void*)a->d_grad_skip, (const void*)a->d_grad_dt_bias, (const void*)a->d_grad_state})
        if ((uintptr_t)f % 4) return SSAM_ERR_DIM;
    if (plan.bytes && !a->d_work) return SSAM_ERR_NULL;
    if (plan.bytes && (a->work_bytes < plan.bytes || (uintptr_t)a->d_work % 16)) return SSAM_ERR_DIM;
    const long long plane = (long long)a->channels * a->states * 4, state_bytes = a->seq.sequences * plane, wide = a->channels * 4LL;
    const long long mark_bytes = product(piece_slots(a->seq, SSAM_MARK_ROWS), plane);
    if (mark_bytes > 4 * kMaxExtent) return SSAM_ERR_DIM;
    const Cover outs[] = {cover_rows(a->grad_in, a->seq, a->channels, esz), cover_rows(a->grad_dt, a->seq, a->channels, esz),
                          cover_rows(a->grad_gate, a->seq, a->channels, esz), cover_rows(a->grad_b, a->seq, bc_width, esz),
                          cover_rows(a->grad_c, a->seq, bc_width, esz), cover_plain(a->d_grad_a, plane), cover_plain(a->d_grad_skip, wide),
                          cover_plain(a->d_grad_dt_bias, wide), cover_plain(a->d_grad_state, state_bytes),
                          cover_plain(plan.bytes ? a->d_work : nullptr, (long long)plan.bytes)};
    const Cover ins[] = {cover_rows(a->in, a->seq, a->channels, esz), cover_rows(a->dt, a->seq, a->channels, esz),
                         cover_rows(a->gate, a->seq, a->channels, esz), cover_rows(a->grad_out, a->seq, a->channels, esz),
                         cover_rows(a->b, a->seq, group_width(a->groups, a->states, a->b_group), esz),
                         cover_rows(a->c, a->seq, group_width(a->groups, a->states, a->c_group), esz), cover_plain(a->d_a, plane),
                         cover_plain(a->d_skip, wide), cover_plain(a->d_dt_bias, wide),
                         cover_plain(a->d_marks, mark_bytes), cover_plain(a->d_grad_final, state_bytes)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;

    BackParams p{};
    p.pieces = make_pieces(a->seq, plan.piece);
    p.mark_slots = make_pieces(a->seq, SSAM_MARK_ROWS);
    p.in = a->in;
    p.dt = a->dt;
    p.gate = a->gate;
    p.b = a->b;
    p.c = a->c;
    p.grad_out = a->grad_out;
    p.b_group = a->b_group;
    p.c_group = a->c_group;
    p.a = a->d_a;
    p.skip = a->d_skip;
    p.dt_bias = a->d_dt_bias;
    p.marks = a->d_marks;
    p.grad_final = a->d_grad_final;
    p.grad_in = a->grad_in;
    p.grad_dt = a->grad_dt;
    p.grad_gate = a->grad_gate;
    p.grad_b = a->grad_b;
    p.grad_c = a->grad_c;
    p.grad_state = a->d_grad_state;
    char* work = static_cast<char*>(a->d_work);
    if (plan.cut) {
        p.ends = reinterpret_cast<float*>(work);
        p.sums = reinterpret_cast<float*>(work + plan.ends);
    }
    if (plan.bc) p.part_bc = reinterpret_cast<float*>(work + plan.ends + plan.sums);
    if (plan.params) p.part_param = reinterpret_cast<float*>(work + plan.ends + plan.sums + plan.part_bc);
    p.rows_total = plan.rows_total;
    p.channels = a->channels;
    p.states = a->states;
    p.groups = a->groups;
    p.group_channels = a->channels / a->groups;
    p.per_group = plan.per_group;
    p.tiles = plan.tiles;
    p.softplus = a->softplus != 0;
    const long long blocks = plan.blocks, sum_blocks = plan.sum_blocks;
    const long long param_blocks = (plane / 4 + 2LL * a->channels + kWave - 1) / kWave;
    if (!plan.fits || param_blocks > kMaxGrid / 4) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    auto sum_params = [&](long long slots, bool more) {
        hipLaunchKernelGGL(back_sum_params, dim3((unsigned)param_blocks), dim3(kWave * kRuns), 0, st, p.part_param, slots, plane / 4, a->channels,
                           a->d_grad_a, a->d_grad_skip, a->d_grad_dt_bias, more);
    };
    return with_row_type(a->dtype, [&](auto t) {
        return with_back_shape(a->states, [&](auto shape) {
            using T = decltype(t);
            using S = decltype(shape);
            if (blocks) {
                const int e = with_shared<S::kStates>(a->states, [&](auto shared) -> int {
                    constexpr bool kShared = decltype(shared)::value;
                    if (plan.cut) {
                        hipLaunchKernelGGL((scan_back<T, S, false, kShared>), dim3((unsigned)blocks), dim3(kBlock), 0, st, p);
                        if (int e = launch_join(p.pieces, p.ends, p.sums, a->d_a, a->d_grad_final, a->channels, a->states, true, st)) return e;
                    }
                    for (long long slot0 = 0; slot0 < plan.slots; slot0 += plan.slots_each) {
                        const long long slots = plan.slots - slot0 < plan.slots_each ? plan.slots - slot0 : plan.slots_each;
                        p.slot0 = (int)slot0;
                        hipLaunchKernelGGL((scan_back<T, S, true, kShared>), dim3((unsigned)(slots * plan.tiles)), dim3(kBlock), 0, st, p);
                        if (plan.params) sum_params(slots, slot0 > 0);
                    }
                    return SSAM_OK;
                });
                if (e) return e;
                if (plan.bc)
                    hipLaunchKernelGGL((back_sum_bc<T>), dim3((unsigned)sum_blocks), dim3(kBlock), 0, st, p, make_pieces(a->seq, kSumRows));
            }
            if (plan.params && !blocks) sum_params(0, false);
            return launched();
        });
    });
}

}  // extern "C"
