// Scan with decay chosen by the input (ssam_scan_selective):
//     h_t[n] = exp(d_t a[n]) h_{t-1}[n] + d_t u_t b_t[n],    y_t = sum_n c_t[n] h_t[n] + skip u_t
// one channel's recurrence per group of lanes (ssam_scan_selective.h), 64 .. 256 channels to a block, states in registers.
//
// A block walks its rows in tiles of 2048 values: the tile's time steps, inputs and gates are requested one tile ahead, 16 bytes a
// lane; every thread turns its eight values into (d, d u) once and puts them into LDS with the rows' b and c, the waves run the
// recurrence from there, leave y in LDS, and the threads that loaded the values finish them (skip, gate) and store them.
//
// Per state and row that is one exp, three products and two sums; the exp (8 cycles of a SIMD against 2.5 - 4 of the others) makes the
// vector unit the bound, not memory (8 bytes a value): 8 x 4096 rows of 4096 channels, 16 states, bf16 590 us, of which the unit
// is busy 71 - 79 % with the two waves per SIMD that there are, at 4.5 cycles an instruction; the bytes alone would take 211, the exps 119.
#include "ssam_scan_selective.h"

namespace ssam {
namespace {

constexpr int kElems = 8;                    // values of a tile that a thread loads, and stores
constexpr int kBlocks = 1024;                // four blocks of four waves per compute unit
constexpr int kAlone = 256;                  // sequences x channel tiles that are enough without cutting (4 sequences of 4096 rows, 4096 channels: 425 us, cut 472)

struct ScanParams {
    Pieces pieces;
    ssam_rows in, dt, gate, out, b, c;
    long long b_group, c_group;
    const float *a, *skip, *dt_bias, *state;
    float *final, *marks, *ends, *sums;   // ends: [entry][channels][states], sums: [entry][channels]
    Pieces mark_slots;
    int channels, states, group_channels, per_group, tiles, softplus;
};

// Rows whose operands are read from LDS together, one group ahead of the arithmetic.
constexpr int kAhead = 4;

// kWhole: all rows, outputs and the last state.  !kWhole: only the state that a piece adds (from zero) and its time steps' sum.
template <class T, class Shape, bool kWhole>
__global__ __launch_bounds__(kBlock, Shape::NS > 4 ? 2 : sizeof(T) == 4 ? 3 : 4) void scan_rows(ScanParams p)
{
    constexpr int GL = Shape::GL, NS = Shape::NS, NP = Shape::kStates, CB = Shape::kChannels, E = kElems;
    constexpr int K = kBlock * E / CB;                   // rows of a tile
    constexpr int kPairs = (K * NP + kBlock - 1) / kBlock;
    constexpr int kRow = CB + CB / E;                    // a row in LDS: padded so that the rows of a wave's writes miss one another's banks
    using Pair = RowVec<float, 2>;
    __shared__ Pair dx[K][kRow];                         // d, d u
    __shared__ Pair bc[K][NP];
    __shared__ float ys[kWhole ? K : 1][kRow];
    __shared__ float per_channel[kWhole ? 2 : 1][CB];    // bias of dt, skip

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int slot = blockIdx.x / p.tiles;
    const Piece q = find_piece(p.pieces, slot);
    if (q.seq < 0) return;
    const bool last = q.row0 + q.n >= q.len;
    if (!kWhole && last) return;                         // nothing follows it
    const ChannelTile ct = channel_tile(blockIdx.x % p.tiles, p.per_group, p.group_channels, CB);

    // this lane's channel and states
    const int place = (tid >> 6) * Shape::kWaveChannels + lane_channel<GL>(lane);
    const int ch = placed_channel<CB, E>(place);
    const bool live = ch < ct.n;
    const int n0 = lane_group<GL>(lane) * NS;
    const long long cell = (long long)(ct.c0 + ch) * p.states;    // its row of [channels][states]
    const long long plane = (long long)p.channels * p.states;
    float a2[NS], h[NS];
    load_rates<NS>(p.a + cell, n0, p.states, live, a2);
    if (!kWhole) load_states<NS>(nullptr, 0, 0, false, h);
    else if (q.row0 > 0) load_states<NS>(p.ends + end_entry(p.pieces, slot - 1, q.seq) * plane + cell, n0, p.states, live, h);
    else if (q.n < q.len)   // not from p.state: the last piece's block may have stored p.final over it by now
        load_states<NS>(p.ends + start_entry(p.pieces, slot, q.seq) * plane + cell, n0, p.states, live, h);
    else load_states<NS>(p.state + q.seq * plane + cell, n0, p.states, live && p.state, h);
    float sum = 0.0f;
    float* marks = nullptr;
    if (kWhole && p.marks) {
        const long long s0 = p.mark_slots.begin ? first_slot(p.mark_slots, q.seq) : (long long)q.seq * p.mark_slots.per;
        marks = p.marks + (s0 + q.row0 / SSAM_MARK_ROWS) * plane + cell;
    }

    // this thread's eight values of a tile
    const TileLane<T, K, CB, E> mine(tid, ct.n);
    const T* in = sequence_base<T>(p.in, p.pieces, q) + (long long)q.row0 * p.in.row + ct.c0;
    const T* dt = sequence_base<T>(p.dt, p.pieces, q) + (long long)q.row0 * p.dt.row + ct.c0;
    const bool gated = kWhole && p.gate.d;
    const T* gate = gated ? sequence_base<T>(p.gate, p.pieces, q) + (long long)q.row0 * p.gate.row + ct.c0 : nullptr;
    T* out = kWhole ? sequence_base<T>(p.out, p.pieces, q) + (long long)q.row0 * p.out.row + ct.c0 : nullptr;
    const T* pb = sequence_base<T>(p.b, p.pieces, q) + (long long)q.row0 * p.b.row + ct.group * p.b_group;
    const T* pc = kWhole ? sequence_base<T>(p.c, p.pieces, q) + (long long)q.row0 * p.c.row + ct.group * p.c_group : nullptr;
    if (tid < CB) {
        per_channel[0][tid] = p.dt_bias && tid < ct.n ? p.dt_bias[ct.c0 + tid] : 0.0f;
        if (kWhole) per_channel[1][tid] = p.skip && tid < ct.n ? p.skip[ct.c0 + tid] : 0.0f;
    }
    // Channels behind the tile keep d = 0, d u = 0 throughout.
    if (ct.n < CB)
        for (int i = tid; i < K * kRow; i += kBlock) dx[i / kRow][i % kRow] = Pair{0.0f, 0.0f};
    __syncthreads();                                     // before the first tile's values go there

    using Vec = RowVec<T, E>;
    Vec u, z, u_next, d_next, z_next;
    T b_next[kPairs], c_next[kPairs];
    static_assert(kBlock % NP == 0, "a thread's values of b and c are all of one state");
    const int state = state_at(tid % NP, p.states);
    const float share = 1.0f / StateCopies(tid % NP / 4, p.states, NP)[tid % 4];
    auto request = [&](int row) {
        const int left = q.n - row;
        u_next = mine.load(in + (long long)row * p.in.row, p.in.row, left);
        d_next = mine.load(dt + (long long)row * p.dt.row, p.dt.row, left);
        if (gated) z_next = mine.load(gate + (long long)row * p.gate.row, p.gate.row, left);
        const T* b0 = pb + (long long)row * p.b.row;
        const T* c0 = kWhole ? pc + (long long)row * p.c.row : nullptr;
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const int i = tid + e * kBlock;
            const unsigned r = i / NP < left ? i / NP : left - 1;
            b_next[e] = b0[r * (unsigned)p.b.row + state];
            if (kWhole) c_next[e] = c0[r * (unsigned)p.c.row + state];
        }
    };
    // Rows behind the piece get d = 0, d u = 0, b = 0: the state passes them unchanged, an infinite one too.
    auto stage = [&](int row) {
        u = u_next;
        z = z_next;
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (float)d_next[e] + per_channel[0][mine.col + e];
        if (p.softplus)
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = softplus(v[e]);
#pragma unroll
        for (int e = 0; e < E; ++e) dx[mine.row][mine.place(e)] = Pair{v[e], v[e] * (float)u[e]};
        if (row + mine.row >= q.n || mine.narrow) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (row + mine.row >= q.n || e >= mine.wide) dx[mine.row][mine.place(e)] = Pair{0.0f, 0.0f};
        }
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const int i = tid + e * kBlock, n = i % NP;
            const bool is = row + i / NP < q.n;
            if (kPairs * kBlock <= K * NP || i < K * NP)
                bc[i / NP][pair_place<Shape>(n)] = Pair{is ? (float)b_next[e] : 0.0f, kWhole && is ? (float)c_next[e] * share : 0.0f};
        }
    };
    struct Operands {
        Pair dv[kAhead], w[kAhead][NS / 4];
    };
    const int pairs = own_pairs<Shape>(lane), sum_at = sum_row<GL>(lane);
    auto fetch = [&](int t, Operands& o) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            o.dv[k] = dx[t + k][place];
#pragma unroll
            for (int m = 0; m < NS / 4; ++m) o.w[k][m] = bc[t + k][pairs + m];
        }
    };
    auto advance = [&](int t, const Operands& o) {
        float y[kAhead];
        if (!kWhole)
#pragma unroll
            for (int k = 0; k < kAhead; ++k) sum += o.dv[k][0];
#pragma unroll
        for (int m = 0; m < NS / 4; ++m) {
            float e[kAhead][4], c[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                c[k] = o.w[k][m][1];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[k][i] = exp2_fast(o.dv[k][0] * a2[4 * m + i]);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                RowVec<float, 4> v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = e[k][i] * h[4 * m + i];
                v = quad_outer(o.w[k][m][0], o.dv[k][1], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[k][i] = h[4 * m + i] = v[i];
            }
            if (kWhole) {
                if (m == 0) quad_dots<true>(y, c, e);
                else quad_dots<false>(y, c, e);
            }
        }
        if (kWhole) {
            group_sums<GL>(y);
#pragma unroll
            for (int k = 0; k < kAhead; k += GL) ys[t + k + sum_at][place] = y[k];
        }
    };

    if (q.n > 0) request(0);                             // (an empty sequence has no row to hold to)
    for (int row = 0; row < q.n; row += K) {
        stage(row);
        __syncthreads();
        if (row + K < q.n) request(row + K);
        if (kWhole && p.marks && K < SSAM_MARK_ROWS && row % SSAM_MARK_ROWS == 0)
            store_states<NS>(marks + (row / SSAM_MARK_ROWS) * plane, n0, p.states, live, h);
        Operands now, next;
        fetch(0, now);
#pragma unroll 1
        for (int t = 0; t < K; t += 2 * kAhead) {
            if (row + t >= q.n) break;
            if (kWhole && p.marks && K >= SSAM_MARK_ROWS && t % SSAM_MARK_ROWS == 0)
                store_states<NS>(marks + ((row + t) / SSAM_MARK_ROWS) * plane, n0, p.states, live, h);
            fetch(t + kAhead, next);
            advance(t, now);
            if (t + 2 * kAhead < K) fetch(t + 2 * kAhead, now);
            advance(t + kAhead, next);
        }
        __syncthreads();
        if (kWhole) {
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = ys[mine.row][mine.place(e)];
            if (p.skip)         // (without one there is no such term, not one of zero times an input that may be infinite)
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(per_channel[1][mine.col + e], (float)u[e], o[e]);
            if (gated)
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] *= silu((float)z[e]);
            mine.store(out + (long long)row * p.out.row, p.out.row, q.n - row, rounded<T, E>(o));
        }
    }
    if (kWhole) {
        if (p.final && last) store_states<NS>(p.final + q.seq * plane + cell, n0, p.states, live, h);
    } else {
        const long long entry = end_entry(p.pieces, slot, q.seq);
        store_states<NS>(p.ends + entry * plane + cell, n0, p.states, live, h);
        if (live && n0 == 0) p.sums[entry * p.channels + ct.c0 + ch] = sum;
    }
}

// One thread per channel and state walks a sequence's pieces; their values are requested eight pieces at a time
// (1 x 16384 rows of 512 channels, 128 pieces: 84 us with all else, four at a time 87, 32 at a time 92).  A block takes every
// `seqs_apart`-th sequence.
template <bool kBackward>
__global__ __launch_bounds__(kBlock) void join_pieces(Pieces pc, float* ends, const float* __restrict__ sums, const float* __restrict__ a,
                                                      const float* initial, int channels, int states, unsigned blocks_each, int seqs_apart)
{
    const long long plane = (long long)channels * states;
    const long long i = (long long)(blockIdx.x % blocks_each) * kBlock + threadIdx.x;
    if (i >= plane) return;
    for (int seq = blockIdx.x / blocks_each; seq < pc.sequences; seq += seqs_apart) {
        int begin, len;
        span_of(pc, seq, begin, len);
        const int n = len > pc.piece ? (len + pc.piece - 1) / pc.piece : 1;
        if (n == 1) continue;
        const int slot0 = pc.begin ? first_slot(pc, seq) : seq * pc.per;
        const long long entry0 = end_entry(pc, slot0, seq);
        const int c = (int)(i / states);
        const float a2 = decay_rate(a[i]);
        float h = initial ? initial[seq * plane + i] : 0.0f;
        if (!kBackward) ends[start_entry(pc, slot0, seq) * plane + i] = h;
        constexpr int kAtOnce = 8;
        for (int k = 0; k < n - 1; k += kAtOnce) {          // what the last adds nothing follows
            float e[kAtOnce], s[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const bool there = k + j < n - 1;
                const long long at = entry0 + (kBackward ? n - 2 - (k + j) : k + j);
                e[j] = there ? ends[at * plane + i] : 0.0f;
                s[j] = there ? sums[at * channels + c] : 0.0f;
            }
            // The decay of many rows may come out as 0 though no row's is: an infinity passes it as it passes them.  Where that makes NaN of
            // it, the pieces are gone over again.
            const float before = h;
            float out[kAtOnce];
            auto pass = [&](bool infinite) {
                h = before;
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    if (k + j >= n - 1) break;
                    const float x = a2 * s[j], decay = exp2_fast(x);
                    const bool passes = infinite && __builtin_fabsf(h) == __builtin_inff() && x > -__builtin_inff();
                    out[j] = h = __builtin_fmaf(passes ? __builtin_fmaxf(decay, 0x1p-126f) : decay, h, e[j]);
                }
            };
            pass(false);
            if (h != h) pass(true);
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (k + j < n - 1) ends[(entry0 + (kBackward ? n - 2 - (k + j) : k + j)) * plane + i] = out[j];
        }
    }
}

struct Plan {
    int tiles, piece;
    long long slots, blocks;
    bool cut;              // sequences may be more than one piece
    size_t ends, bytes;    // bytes of the pieces' states, and of the whole workspace (none for more blocks than a launch holds, which are refused)
};

Plan plan_of(const ssam_scan_selective_args& a)
{
    Plan p;
    p.tiles = tiles_per_group(a.channels, a.states, a.groups) * a.groups;
    p.piece = scan_piece_rows(a.seq, p.tiles, kBlocks, kAlone);
    p.slots = piece_slots(a.seq, p.piece);
    p.blocks = p.slots * p.tiles;
    p.cut = a.seq.rows > p.piece && p.blocks <= kMaxGrid;
    const size_t entries = p.cut ? end_entries(a.seq, p.piece, true) : 0;
    p.ends = entries * a.channels * a.states * sizeof(float);
    p.bytes = p.ends + entries * a.channels * sizeof(float);
    return p;
}

// ---- one row per sequence ----------------------------------------------------------------------------------------------
struct ScanStepParams {
    int rows, slots, channels, states, group_channels, per_group, tiles, softplus;
    const int* slot_of;
    ssam_rows in, dt, gate, out, b, c;
    long long b_group, c_group;
    const float *a, *skip, *dt_bias;
    float* state;
    long long slot_stride;
};

// The value of lane K of the P lanes around this one, and the sum over them.
template <int P, int K>
__device__ __forceinline__ float from_part(float v)
{
    if constexpr (P == 1) return v;
    else if constexpr (P == 2)
        return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), K == 0 ? 0xA0 : 0xF5, 0xf, 0xf, true));   // [0,0,2,2], [1,1,3,3]
    else if constexpr (P == 4) return quad_lane<K>(v);
    else return __shfl(v, (int)(threadIdx.x & (kWave - 1) & ~(P - 1)) | K);
}
template <int P>
__device__ __forceinline__ float part_sum(float v)
{
    auto moved = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if constexpr (P >= 2) v += moved(v, std::integral_constant<int, 0xB1>{});    // [1,0,3,2]
    if constexpr (P >= 4) v += moved(v, std::integral_constant<int, 0x4E>{});    // [2,3,0,1]
    if constexpr (P >= 8) v += moved(v, std::integral_constant<int, 0x141>{});   // eight lanes mirrored: the other quad
    if constexpr (P >= 16) v += moved(v, std::integral_constant<int, 0x128>{});  // the row of 16 turned by 8
    return v;
}

template <int... K, class F>
__device__ __forceinline__ void for_each(std::integer_sequence<int, K...>, F f)
{
    (f(std::integral_constant<int, K>{}), ...);
}

// Channels that P lanes with four states each go through one after the other, and those of a wave.
constexpr int step_each(int P) { return P < 4 ? P : 4; }
constexpr int step_channels(int P) { return kWave / P * step_each(P); }

// P lanes share a channel, four states each, so that every load of states is a run of whole lines; what belongs to a channel alone
// (time step, gate, output) is made once, by the lane of that number, and handed round.  A block's waves take the same channels of four rows, so
// that the rates come from the L1.  Bound by the state: 8 bytes per value of it (256 rows of 4096 channels, 16 states: 31 us, 4.5 TB/s).
template <class T, int P, bool kShared>
__global__ __launch_bounds__(kBlock) void scan_step(ScanStepParams p)
{
    const int lane = threadIdx.x & (kWave - 1);
    const int row_blocks = (p.rows + kWavesPerBlock - 1) / kWavesPerBlock;
    const int row = (int)(blockIdx.x % row_blocks) * kWavesPerBlock + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    constexpr int KC = step_each(P);
    const ChannelTile ct = channel_tile((int)(blockIdx.x / row_blocks), p.per_group, p.group_channels, step_channels(P));
    constexpr int kApart = kWave / P;            // the k-th of a lane's channels is k * kApart + lane / P: a load of the k-th is one run
    const int part = lane & (P - 1), first = lane / P, n0 = part * 4;
    const StateCopies copies(part, p.states, 4 * P);
    float share[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) share[i] = kShared ? 1.0f / copies[i] : 1.0f;
    const bool own = part < KC && part * kApart + first < ct.n;
    const int c = ct.c0 + part * kApart + first; // the channel whose time step and output are this lane's
    struct Row {
        float u, d, z;
        RowVec<T, 4> b, w;
    };
    auto request = [&](int r) {
        Row x;
        x.u = own ? (float)static_cast<const T*>(p.in.d)[r * p.in.row + c] : 0.0f;
        x.d = own ? (float)static_cast<const T*>(p.dt.d)[r * p.dt.row + c] : 0.0f;
        x.z = own && p.gate.d ? (float)static_cast<const T*>(p.gate.d)[r * p.gate.row + c] : 0.0f;
        const T* b = static_cast<const T*>(p.b.d) + r * p.b.row + ct.group * p.b_group;
        const T* w = static_cast<const T*>(p.c.d) + r * p.c.row + ct.group * p.c_group;
        if (!kShared || p.states >= 4) {
            const int n = kShared ? state_block(part, p.states) : n0;
            x.b = load_row_vec<T, 4>(b + n, 4);
            x.w = load_row_vec<T, 4>(w + n, 4);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x.b[i] = b[state_at(i, p.states)];
                x.w[i] = w[state_at(i, p.states)];
            }
        }
        return x;
    };
    Row x = request(row);
    const float bias = own && p.dt_bias ? p.dt_bias[c] : 0.0f;
    const float skip = own && p.skip ? p.skip[c] : 0.0f;
    SlotRows same(p.slot_of, p.rows, p.slots, row);
    if (!same.leads()) return;
    float* __restrict__ state = p.state + (long long)same.slot() * p.slot_stride;
    float h[KC][4], a2[KC][4];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const long long cell = (long long)(ct.c0 + k * kApart + first) * p.states;
        const bool there = k * kApart + first < ct.n;
        load_states<4, kShared>(state + cell, n0, p.states, there, h[k]);
        load_rates<4, kShared>(p.a + cell, n0, p.states, there, a2[k]);
    }
    for (int r = row;;) {
        float d = x.d + bias;
        if (p.softplus) d = softplus(d);
        const float du = d * x.u;
        float y = 0.0f;
        for_each(std::make_integer_sequence<int, KC>{}, [&](auto k) {
            constexpr int kk = decltype(k)::value;
            const float dk = from_part<P, kk>(d), xk = from_part<P, kk>(du);
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[kk][i] = __builtin_fmaf(exp2_fast(dk * a2[kk][i]), h[kk][i], (float)x.b[i] * xk);
                s = __builtin_fmaf((float)x.w[i] * share[i], h[kk][i], s);
            }
            s = part_sum<P>(s);
            y = part == kk ? s : y;
        });
        if (p.skip) y = __builtin_fmaf(skip, x.u, y);
        if (p.gate.d) y *= silu(x.z);
        if (own) static_cast<T*>(p.out.d)[r * p.out.row + c] = (T)y;
        r = same.next();
        if (r < 0) break;
        x = request(r);
    }
#pragma unroll
    for (int k = 0; k < KC; ++k)
        store_states<4, kShared>(state + (long long)(ct.c0 + k * kApart + first) * p.states, n0, p.states, k * kApart + first < ct.n, h[k]);
}

}  // namespace

int scan_piece_rows(const ssam_sequences& q, int tiles, int blocks, int alone)
{
    constexpr long long kShortest = 32;   // shorter ones wait for the join (369 rows of 518 channels forward and back: 69 us, with 64: 84)
    constexpr long long kWhole = 128;     // not worth the join (128 rows of 4096 channels: 17.6 us, cut 18.7; 256 rows: 30.7, cut 22.9)
    constexpr long long kLongest = 1 << 30;
    const long long total = q.d_begin ? q.rows : (long long)q.rows * q.sequences, whole = (long long)q.sequences * tiles;
    // Packed sequences end inside pieces: shorter ones even that out where there are few (37 in 8191 rows: 119 us, 139 without; 12 in
    // 16384 rows of 4096 channels: 446, 465 with 1.5 times as many), and are too many where there are not (64 in 8192 rows of 4096
    // channels with 1.5 times: 237, 206 without).
    if (q.d_begin && whole < blocks) blocks *= 2;
    long long piece = (product(total, tiles) + blocks - 1) / blocks;
    if (q.rows <= kWhole) piece = kWhole;
    else if (!q.d_begin && whole >= alone) piece = q.rows;
    piece = (piece + 31) / 32 * 32;
    return (int)(piece < kShortest ? kShortest : piece > kLongest ? kLongest : piece);
}

int launch_join(const Pieces& p, float* ends, const float* sums, const float* a, const float* initial, int channels, int states, bool backward,
                hipStream_t stream)
{
    const unsigned each = (unsigned)(((long long)channels * states + kBlock - 1) / kBlock);
    const int apart = (int)(p.sequences < kMaxGrid / each ? p.sequences : kMaxGrid / each);
    const dim3 grid(each * (unsigned)apart);
    if (backward) hipLaunchKernelGGL((join_pieces<true>), grid, dim3(kBlock), 0, stream, p, ends, sums, a, initial, channels, states, each, apart);
    else hipLaunchKernelGGL((join_pieces<false>), grid, dim3(kBlock), 0, stream, p, ends, sums, a, initial, channels, states, each, apart);
    return launched();
}

}  // namespace ssam

extern "C" {

size_t ssam_scan_selective_workspace_bytes(const ssam_scan_selective_args* a)
{
    using namespace ssam;
    if (!a || check_scan(a->dtype, a->channels, a->states, a->groups) || check_sequences(a->seq) || a->seq.sequences == 0) return 0;
    return plan_of(*a).bytes;
}

long long ssam_scan_selective_marks(const ssam_scan_selective_args* a)
{
    using namespace ssam;
    if (!a || check_scan(a->dtype, a->channels, a->states, a->groups) || check_sequences(a->seq)) return 0;
    return piece_slots(a->seq, SSAM_MARK_ROWS);
}

int ssam_scan_selective(const ssam_scan_selective_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_scan(a->dtype, a->channels, a->states, a->groups)) return e;
    if (int e = check_sequences(a->seq)) return e;
    if (a->seq.sequences == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype);
    if (!a->d_a) return SSAM_ERR_NULL;
    if (int e = check_group_rows(*a, a->seq, esz)) return e;
    for (const ssam_rows* r : {&a->in, &a->dt})
        if (int e = check_rows(*r, a->seq, a->channels, esz, false)) return e;
    if (int e = check_rows(a->gate, a->seq, a->channels, esz, true)) return e;
    if (int e = check_out_rows(a->out, a->seq, a->channels, esz, false)) return e;
    for (const ssam_rows* r : {&a->in, &a->dt, &a->gate, &a->out, &a->b, &a->c})
        if (int e = check_tile_rows(*r, a->seq)) return e;
    for (const void* f : {(const void*)a->d_a, (const void*)a->d_skip, (const void*)a->d_dt_bias, (const void*)a->d_state, (const void*)a->d_final,
                          (const void*)a->d_marks})
        if ((uintptr_t)f % 4) return SSAM_ERR_DIM;
    const Plan plan = plan_of(*a);
    if (plan.bytes && !a->d_work) return SSAM_ERR_NULL;
    if (plan.bytes && (a->work_bytes < plan.bytes || (uintptr_t)a->d_work % 16)) return SSAM_ERR_DIM;
    const long long plane = (long long)a->channels * a->states * 4, state_bytes = a->seq.sequences * plane;
    const long long mark_bytes = product(piece_slots(a->seq, SSAM_MARK_ROWS), plane);
    if (a->d_marks && mark_bytes > 4 * kMaxExtent) return SSAM_ERR_DIM;
    const Cover state = cover_plain(a->d_state, state_bytes);
    const Cover outs[] = {cover_rows(a->out, a->seq, a->channels, esz), cover_plain(a->d_final, state_bytes),
                          cover_plain(a->d_marks, mark_bytes),
                          cover_plain(plan.bytes ? a->d_work : nullptr, (long long)plan.bytes)};
    const Cover ins[] = {cover_rows(a->in, a->seq, a->channels, esz), cover_rows(a->dt, a->seq, a->channels, esz),
                         cover_rows(a->gate, a->seq, a->channels, esz),
                         cover_rows(a->b, a->seq, group_width(a->groups, a->states, a->b_group), esz),
                         cover_rows(a->c, a->seq, group_width(a->groups, a->states, a->c_group), esz), cover_plain(a->d_a, plane),
                         cover_plain(a->d_skip, a->channels * 4LL), cover_plain(a->d_dt_bias, a->channels * 4LL)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    for (int i = 0; i < 4; ++i)
        if (overlaps(outs[i], state) && !(i == 1 && a->d_final == a->d_state)) return SSAM_ERR_ALIAS;

    ScanParams p{};
    p.pieces = make_pieces(a->seq, plan.piece);
    p.mark_slots = make_pieces(a->seq, SSAM_MARK_ROWS);
    p.in = a->in;
    p.dt = a->dt;
    p.gate = a->gate;
    p.out = a->out;
    p.b = a->b;
    p.c = a->c;
    p.b_group = a->b_group;
    p.c_group = a->c_group;
    p.a = a->d_a;
    p.skip = a->d_skip;
    p.dt_bias = a->d_dt_bias;
    p.state = a->d_state;
    p.final = a->d_final;
    p.marks = a->d_marks;
    p.channels = a->channels;
    p.states = a->states;
    p.group_channels = a->channels / a->groups;
    p.per_group = tiles_per_group(a->channels, a->states, a->groups);
    p.tiles = plan.tiles;
    p.softplus = a->softplus != 0;
    const long long blocks = plan.blocks;
    if (blocks > kMaxGrid) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    return with_row_type(a->dtype, [&](auto t) {
        return with_shape(a->states, [&](auto shape) {
            using T = decltype(t);
            using S = decltype(shape);
            if (plan.cut) {
                p.ends = static_cast<float*>(a->d_work);
                p.sums = reinterpret_cast<float*>(static_cast<char*>(a->d_work) + plan.ends);
                hipLaunchKernelGGL((scan_rows<T, S, false>), dim3((unsigned)blocks), dim3(kBlock), 0, st, p);
                if (int e = launch_join(p.pieces, p.ends, p.sums, a->d_a, a->d_state, a->channels, a->states, false, st)) return e;
            }
            hipLaunchKernelGGL((scan_rows<T, S, true>), dim3((unsigned)blocks), dim3(kBlock), 0, st, p);
            return launched();
        });
    });
}

int ssam_scan_selective_step(const ssam_scan_selective_step_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_scan(a->dtype, a->channels, a->states, a->groups)) return e;
    if (int e = check_slots(a->rows, a->slots, a->d_slots)) return e;
    if (a->rows == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype);
    const ssam_sequences q{1, a->rows, nullptr, nullptr};
    if (!a->d_a || !a->d_state) return SSAM_ERR_NULL;
    if (int e = check_group_rows(*a, q, esz)) return e;
    for (const ssam_rows* r : {&a->in, &a->dt})
        if (int e = check_rows(*r, q, a->channels, esz, false)) return e;
    if (int e = check_rows(a->gate, q, a->channels, esz, true)) return e;
    if (int e = check_out_rows(a->out, q, a->channels, esz, false)) return e;
    for (const void* f : {(const void*)a->d_a, (const void*)a->d_skip, (const void*)a->d_dt_bias, (const void*)a->d_state})
        if ((uintptr_t)f % 4) return SSAM_ERR_DIM;
    const long long slot = (long long)a->channels * a->states;
    if (int e = check_pool(a->slots, a->slot_stride, slot)) return e;
    const Cover outs[] = {cover_rows(a->out, q, a->channels, esz), cover_slots(a->d_state, a->slots, a->slot_stride, slot, 4)};
    const Cover ins[] = {cover_rows(a->in, q, a->channels, esz), cover_rows(a->dt, q, a->channels, esz), cover_rows(a->gate, q, a->channels, esz),
                         cover_rows(a->b, q, group_width(a->groups, a->states, a->b_group), esz),
                         cover_rows(a->c, q, group_width(a->groups, a->states, a->c_group), esz), cover_plain(a->d_a, slot * 4),
                         cover_plain(a->d_skip, a->channels * 4LL), cover_plain(a->d_dt_bias, a->channels * 4LL),
                         cover_plain(a->d_slots, a->rows * 4LL)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    ScanStepParams p{};
    p.rows = a->rows;
    p.slots = a->slots;
    p.channels = a->channels;
    p.states = a->states;
    p.group_channels = a->channels / a->groups;
    const int lanes = a->states <= 4 ? 1 : a->states <= 8 ? 2 : a->states <= 16 ? 4 : a->states <= 32 ? 8 : 16;
    p.per_group = (p.group_channels + step_channels(lanes) - 1) / step_channels(lanes);
    p.tiles = p.per_group * a->groups;
    p.softplus = a->softplus != 0;
    p.slot_of = a->d_slots;
    p.in = a->in;
    p.dt = a->dt;
    p.gate = a->gate;
    p.out = a->out;
    p.b = a->b;
    p.c = a->c;
    p.b_group = a->b_group;
    p.c_group = a->c_group;
    p.a = a->d_a;
    p.skip = a->d_skip;
    p.dt_bias = a->d_dt_bias;
    p.state = a->d_state;
    p.slot_stride = a->slot_stride;
    const long long blocks = ((long long)a->rows + kWavesPerBlock - 1) / kWavesPerBlock * p.tiles;
    if (blocks > kMaxGrid) return SSAM_ERR_DIM;
    return with_row_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        const dim3 grid((unsigned)blocks), block(kBlock);
        hipStream_t st = (hipStream_t)hip_stream;
        auto launch = [&](auto parts) {
            constexpr int P = decltype(parts)::value;
            return with_shared<4 * P>(a->states, [&](auto shared) {
                hipLaunchKernelGGL((scan_step<T, P, decltype(shared)::value>), grid, block, 0, st, p);
                return launched();
            });
        };
        if (lanes == 1) return launch(std::integral_constant<int, 1>{});
        if (lanes == 2) return launch(std::integral_constant<int, 2>{});
        if (lanes == 4) return launch(std::integral_constant<int, 4>{});
        if (lanes == 8) return launch(std::integral_constant<int, 8>{});
        return launch(std::integral_constant<int, 16>{});
    });
}

}  // extern "C"
