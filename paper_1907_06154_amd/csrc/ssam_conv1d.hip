// Per-channel causal filter along time (ssam_conv1d), its gradients and its single-row form: the register cache and the
// sliding window of the 2D filters turned so that the window slides along rows.  A lane owns the V channels of one 16-byte
// vector and marches over its piece of a sequence with the last taps-1 rows in registers; channels never meet, so there is no
// shift between lanes and no LDS.  Every row is read once per piece, and taps-1 rows more above a piece (from the L2).  Bound
// by memory: 2 x taps operations on the 2 x 2 bytes of a value.
#include "ssam_rows.h"

namespace ssam {
namespace {

constexpr int kMarch = 4;          // rows requested together

template <class T> constexpr int kChan = 16 / sizeof(T);   // channels of a lane
constexpr int kBackChan = 4;                               // and in the backward march, which holds more of each

struct Conv1dParams {
    Pieces pieces;
    ssam_rows in, out;
    const void *weight, *bias, *state;
    void* final;
    int channels, strips, silu, params_f32;
    long long waves;
};

// A lane's V channels.  A vector that would pass the last channel starts further left instead: its channels are then also those of the
// lane before, and both make and store the same values.  The two are always lanes of one wave, whose loads of a state that is
// updated in place come before its stores.  A strip of fewer than V channels is one lane's, by elements.
template <int V>
struct Channels {
    int first, have;
    bool narrow, there;
    __device__ __forceinline__ Channels(int strip, int lane, int channels)
    {
        const int c0 = strip * (kWave * V), left = channels - c0;
        first = c0 + lane * V;
        there = first < channels;
        narrow = left < V;
        have = narrow ? left : V;
        if (first + V > channels) first = narrow ? c0 : channels - V;      // lanes that have none repeat the last as well
    }
    template <class T> __device__ __forceinline__ RowVec<T, V> load(const T* __restrict__ p) const { return load_row_vec<T, V>(p, have, narrow); }
    template <class T, bool kStream> __device__ __forceinline__ void store(T* __restrict__ p, const RowVec<T, V>& v) const
    {
        store_row_vec<T, V, kStream>(p, have, v, narrow);
    }
};

// The taps of V channels are V * W consecutive values: W whole vectors.
template <class P, int W, int V>
__device__ __forceinline__ void load_taps_as(const void* weight, const Channels<V>& ch, float (&w)[W][V])
{
    RowVec<P, V> r[W];
#pragma unroll
    for (int k = 0; k < W; ++k) r[k] = load_row_vec<P, V>(static_cast<const P*>(weight) + (long long)ch.first * W + k * V, ch.have * W - k * V, ch.narrow);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][v] = (float)r[(v * W + j) / V][(v * W + j) % V];
}
template <class T, int W, int V>
__device__ __forceinline__ void load_taps(const void* weight, bool f32, const Channels<V>& ch, float (&w)[W][V])
{
    if (f32) load_taps_as<float, W, V>(weight, ch, w);
    else load_taps_as<T, W, V>(weight, ch, w);
}

template <class T, int V>
__device__ __forceinline__ void load_bias(const void* bias, bool f32, const Channels<V>& ch, float (&b)[V])
{
    if (!bias) {
#pragma unroll
        for (int v = 0; v < V; ++v) b[v] = 0.0f;
    } else if (f32) {
        const RowVec<float, V> r = ch.load(static_cast<const float*>(bias) + ch.first);
#pragma unroll
        for (int v = 0; v < V; ++v) b[v] = r[v];
    } else {
        const RowVec<T, V> r = ch.load(static_cast<const T*>(bias) + ch.first);
#pragma unroll
        for (int v = 0; v < V; ++v) b[v] = (float)r[v];
    }
}

// Row t < 0 of sequence s: from its carried state, zeros without one.
template <class T, int W, int V>
__device__ __forceinline__ RowVec<T, V> carried_row(const void* state, int s, int t, int channels, const Channels<V>& ch)
{
    if (!state) return RowVec<T, V>(T(0));
    return ch.load(static_cast<const T*>(state) + ((long long)s * (W - 1) + (W - 1 + t)) * channels + ch.first);
}

template <class T, int W>
__global__ __launch_bounds__(kBlock) void conv1d_rows(Conv1dParams p)
{
    constexpr int V = kChan<T>;
    const int lane = threadIdx.x & (kWave - 1);
    const long long wave = (long long)blockIdx.x * kWavesPerBlock + (threadIdx.x >> 6);
    if (wave >= p.waves) return;
    const int strip = (int)(wave % p.strips);
    const Piece q = find_piece(p.pieces, (int)(wave / p.strips));
    if (q.seq < 0) return;
    const Channels<V> ch(strip, lane, p.channels);
    if (!ch.there) return;
    const T* __restrict__ in = sequence_base<T>(p.in, p.pieces, q) + ch.first;
    T* __restrict__ out = sequence_base<T>(p.out, p.pieces, q) + ch.first;
    RowVec<T, V> win[W], next[kMarch];        // rows t - W + 1 .. t, and the rows after those in work
    auto request = [&](int k) {               // rows behind the piece are read as its last, and not used
#pragma unroll
        for (int u = 0; u < kMarch; ++u) next[u] = ch.load(in + (long long)(q.row0 + (k + u < q.n ? k + u : q.n - 1)) * p.in.row);
    };
    if (q.n > 0) request(0);
    float w[W][V], b[V];
    load_taps<T, W, V>(p.weight, p.params_f32, ch, w);
    load_bias<T, V>(p.bias, p.params_f32, ch, b);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int t = q.row0 - (W - 1) + j;
        win[j + 1] = t >= 0 ? ch.load(in + (long long)t * p.in.row) : carried_row<T, W, V>(p.state, q.seq, t, p.channels, ch);
    }
    for (int k = 0; k < q.n; k += kMarch) {
        RowVec<T, V> x[kMarch];
#pragma unroll
        for (int u = 0; u < kMarch; ++u) x[u] = next[u];
        if (k + kMarch < q.n) request(k + kMarch);
#pragma unroll
        for (int u = 0; u < kMarch; ++u) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
            win[W - 1] = x[u];
            float y[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s = b[v];
#pragma unroll
                for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][v], (float)win[j][v], s);
                y[v] = s;
            }
            if (p.silu)
#pragma unroll
                for (int v = 0; v < V; ++v) y[v] = silu(y[v]);
            if (k + u < q.n) ch.template store<T, true>(out + (long long)(q.row0 + k + u) * p.out.row, rounded<T, V>(y));
        }
    }
    // The first piece's wave also hands on the state: it is the only one that reads the old one, so that both may be the same
    // array (row j of the new state is row len + j of the old one, never below j).
    if (W > 1 && p.final && q.row0 == 0) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = q.len - (W - 1) + j;
            const RowVec<T, V> x = t >= 0 ? ch.load(in + (long long)t * p.in.row) : carried_row<T, W, V>(p.state, q.seq, t, p.channels, ch);
            ch.template store<T, false>(static_cast<T*>(p.final) + ((long long)q.seq * (W - 1) + j) * p.channels + ch.first, x);
        }
    }
}

// ---- gradients ---------------------------------------------------------------------------------------------------------
struct Conv1dBackParams {
    Pieces pieces;
    ssam_rows in, grad_out, grad_in;
    const void *weight, *bias, *state, *grad_final;
    void* grad_state;
    float* parts;               // [four slots][W + 1][channels]: their sums for the weight's and the bias's gradient, or null
    int channels, strips, silu, params_f32;
    long long slots;
};

template <class T, int V>
__device__ __forceinline__ void widened(const RowVec<T, V>& x, float (&f)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = (float)x[v];
}

// q_t = dy_t silu'(p_t), dx_t = sum_j w[j] q_{t + W - 1 - j}, dw[j] = sum_t q_t x_{t - W + 1 + j}, db = sum_t q_t.  One march over
// the rows of the piece and the W-1 behind it: p_t comes again from the window of inputs, and a second window holds the last W
// q's.  dx runs W-1 rows behind the march, so the first piece also meets rows -(W-1) .. -1, the gradient of the carried rows.
// The sums over rows stay in registers; a block's four waves, four slots of one strip, add theirs in LDS, and what a block has goes
// to `parts`, to be added block after block.  8 x 2048 rows of 4096 channels, four taps, bf16: 84 us for three tensors, 4.8 TB/s; the
// sums over the blocks 5 us.
template <class T, int W>
__global__ __launch_bounds__(kBlock) void conv1d_back(Conv1dBackParams p)
{
    constexpr int V = kBackChan;
    __shared__ RowVec<float, V> block_sums[kWavesPerBlock - 1][W + 1][kWave];
    // The wave's number as a scalar, so that what depends on its rows is a scalar branch (8 x 2048 rows of 4096 channels, with the forward
    // call: 139 us, with vector ones 158).
    const int lane = threadIdx.x & (kWave - 1), in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int strip = blockIdx.x % p.strips;
    const long long slot = (long long)(blockIdx.x / p.strips) * kWavesPerBlock + in_block;
    Piece q = find_piece(p.pieces, (int)(slot < p.slots ? slot : 0));
    const Channels<V> ch(strip, lane, p.channels);
    if (slot >= p.slots || !ch.there) q.seq = -1;       // stays for the sums
    float dw[W + 1][V];         // the last: the bias's
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) dw[j][v] = 0.0f;
    if (q.seq >= 0) {
        const T* __restrict__ in = sequence_base<T>(p.in, p.pieces, q) + ch.first;
        const T* __restrict__ dy = sequence_base<T>(p.grad_out, p.pieces, q) + ch.first;
        T* __restrict__ dx = p.grad_in.d ? sequence_base<T>(p.grad_in, p.pieces, q) + ch.first : nullptr;
        const int rows = q.n + W - 1;       // the march: rows row0 .. row0 + rows - 1
        RowVec<T, V> x_next[kMarch], g_next[kMarch];
        float win[W][V];                    // widened once, not at each of its 2 W uses (fp16, three taps 152 -> 136 us with the forward call)
        auto request = [&](int k) {         // rows behind the sequence are read as its last, and their q is not used
#pragma unroll
            for (int u = 0; u < kMarch; ++u) {
                const int t = q.row0 + k + u < q.len ? q.row0 + k + u : q.len - 1;
                x_next[u] = ch.load(in + (long long)t * p.in.row);
                g_next[u] = ch.load(dy + (long long)t * p.grad_out.row);
            }
        };
#pragma unroll
        for (int u = 0; u < kMarch; ++u) x_next[u] = g_next[u] = RowVec<T, V>(T(0));
        if (q.len > 0) request(0);
        float w[W][V], b[V], qs[W][V];
        load_taps<T, W, V>(p.weight, p.params_f32, ch, w);
        load_bias<T, V>(p.bias, p.params_f32, ch, b);
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) qs[j][v] = 0.0f;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = q.row0 - (W - 1) + j;
            widened<T, V>(t >= 0 ? ch.load(in + (long long)t * p.in.row) : carried_row<T, W, V>(p.state, q.seq, t, p.channels, ch), win[j + 1]);
        }
        for (int k = 0; k < rows; k += kMarch) {
            RowVec<T, V> x[kMarch], g[kMarch];
#pragma unroll
            for (int u = 0; u < kMarch; ++u) {
                x[u] = x_next[u];
                g[u] = g_next[u];
            }
            if (q.len > 0 && k + kMarch < rows) request(k + kMarch);
#pragma unroll
            for (int u = 0; u < kMarch; ++u) {
                const int t = q.row0 + k + u;
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) win[j][v] = win[j + 1][v];
                widened<T, V>(x[u], win[W - 1]);
#pragma unroll
                for (int j = W - 1; j > 0; --j)
#pragma unroll
                    for (int v = 0; v < V; ++v) qs[j][v] = qs[j - 1][v];
#pragma unroll
                for (int v = 0; v < V; ++v) qs[0][v] = (float)g[u][v];
                if (p.silu) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float s = b[v];
#pragma unroll
                        for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][v], win[j][v], s);
                        const float sig = sigmoid(s);
                        qs[0][v] *= sig * __builtin_fmaf(s, 1.0f - sig, 1.0f);
                    }
                }
                // The piece's own rows alone: those behind it, and the carried ones of an empty sequence, may hold an infinity, which
                // times zero is not zero.
                if (k + u < q.n) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j][v] = __builtin_fmaf(qs[0][v], win[j][v], dw[j][v]);
                        dw[W][v] += qs[0][v];
                    }
                }
                const int o = t - (W - 1);  // the row whose gradient is complete
                const bool carried = o < 0;
                if (k + u >= rows || (o < q.row0 && !carried) || (carried ? !p.grad_state : !dx)) continue;
                float d[V];
                if (t < q.len && t >= W - 1) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        d[v] = w[0][v] * qs[0][v];
#pragma unroll
                        for (int j = 1; j < W; ++j) d[v] = __builtin_fmaf(w[j][v], qs[j][v], d[v]);
                    }
                } else {        // only the taps that rows of the sequence lie under: another's may be infinite
#pragma unroll
                    for (int v = 0; v < V; ++v) d[v] = 0.0f;
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        if (t - j >= 0 && t - j < q.len)
#pragma unroll
                            for (int v = 0; v < V; ++v) d[v] = __builtin_fmaf(w[j][v], qs[j][v], d[v]);
                }
                const int tail = o - (q.len - (W - 1));
                if (p.grad_final && tail >= 0) {
                    const RowVec<T, V> f =
                        ch.load(static_cast<const T*>(p.grad_final) + ((long long)q.seq * (W - 1) + tail) * p.channels + ch.first);
#pragma unroll
                    for (int v = 0; v < V; ++v) d[v] += (float)f[v];
                }
                T* to = carried ? static_cast<T*>(p.grad_state) + ((long long)q.seq * (W - 1) + t) * p.channels + ch.first
                                : dx + (long long)o * p.grad_in.row;
                ch.template store<T, true>(to, rounded<T, V>(d));
            }
        }
    }
    if (!p.parts) return;
    RowVec<float, V> f[W + 1];
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) f[j][v] = dw[j][v];
    if (in_block > 0)
#pragma unroll
        for (int j = 0; j <= W; ++j) block_sums[in_block - 1][j][lane] = f[j];
    __syncthreads();
    if (in_block > 0 || !ch.there) return;
#pragma unroll
    for (int j = 0; j <= W; ++j) {
#pragma unroll
        for (int k = 0; k < kWavesPerBlock - 1; ++k) f[j] += block_sums[k][j][lane];
        ch.template store<float, false>(p.parts + ((long long)(blockIdx.x / p.strips) * (W + 1) + j) * p.channels + ch.first, f[j]);
    }
}

// parts summed over the blocks' slots, 16 interleaved runs of them and then the runs, always in the same order.
constexpr int kRuns = 16;
template <class T>
__global__ __launch_bounds__(kWave* kRuns) void conv1d_back_sums(const float* __restrict__ parts, long long slots, int W, int channels,
                                                                 void* grad_weight, void* grad_bias, int params_f32)
{
    __shared__ float run[kRuns][kWave];
    const int lane = threadIdx.x & (kWave - 1), r = threadIdx.x >> 6;
    const int strips = (channels + kWave - 1) / kWave;
    const int j = blockIdx.x / strips;
    const int c = (blockIdx.x % strips) * kWave + lane;
    float s = 0.0f;
    if (c < channels)
#pragma unroll 4
        for (long long i = r; i < slots; i += kRuns) s += parts[(i * (W + 1) + j) * channels + c];
    run[r][lane] = s;
    __syncthreads();
    if (r != 0 || c >= channels) return;
#pragma unroll
    for (int k = 1; k < kRuns; ++k) s += run[k][lane];
    void* to = j < W ? grad_weight : grad_bias;
    const long long at = j < W ? (long long)c * W + j : c;
    if (!to) return;
    if (params_f32) static_cast<float*>(to)[at] = s;
    else static_cast<T*>(to)[at] = (T)s;
}

// ---- one row per sequence ----------------------------------------------------------------------------------------------
struct Conv1dStepParams {
    int rows, slots, channels, strips, silu, params_f32;
    const int* slot_of;
    ssam_rows in, out;
    const void *weight, *bias;
    void* state;
    long long slot_stride;
};

// The window is the state: read, shifted, written.  384 rows of 8192 channels, four taps, bf16: 13.0 us for 50 MB, 3.9 TB/s; one row of
// 2048 channels 3.6 us, a launch.
template <class T, int W>
__global__ __launch_bounds__(kBlock) void conv1d_step(Conv1dStepParams p)
{
    constexpr int V = kChan<T>;
    const int lane = threadIdx.x & (kWave - 1);
    const int row_blocks = (p.rows + kWavesPerBlock - 1) / kWavesPerBlock;      // a block's waves: the same channels of four rows
    const int row = (int)(blockIdx.x % row_blocks) * kWavesPerBlock + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const Channels<V> ch((int)(blockIdx.x / row_blocks), lane, p.channels);
    const T* in = static_cast<const T*>(p.in.d) + ch.first;
    RowVec<T, V> x = ch.load(in + (long long)row * p.in.row);
    float w[W][V], b[V];
    load_taps<T, W, V>(p.weight, p.params_f32, ch, w);
    load_bias<T, V>(p.bias, p.params_f32, ch, b);
    SlotRows same(p.slot_of, p.rows, p.slots, row);      // every lane takes part to the end: the rows of a slot are found by ballots
    if (!same.leads()) return;
    T* __restrict__ state = static_cast<T*>(p.state) + (long long)same.slot() * p.slot_stride + ch.first;
    RowVec<T, V> win[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j + 1] = ch.load(state + (long long)j * p.channels);
    for (int r = row;;) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
        win[W - 1] = x;
        float y[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float s = b[v];
#pragma unroll
            for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][v], (float)win[j][v], s);
            y[v] = p.silu ? silu(s) : s;
        }
        ch.template store<T, false>(static_cast<T*>(p.out.d) + (long long)r * p.out.row + ch.first, rounded<T, V>(y));
        r = same.next();
        if (r < 0) break;
        x = ch.load(in + (long long)r * p.in.row);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) ch.template store<T, false>(state + (long long)j * p.channels, win[j + 1]);
}

// ---- host --------------------------------------------------------------------------------------------------------------
template <class T, class F>
int with_taps(int taps, F f)
{
    switch (taps) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
    }
}

// f gets the element type's code and the filter's length as compile-time constants.
template <class F>
int with_type_and_taps(int dtype, int taps, F f)
{
    if (dtype == SSAM_F32) return with_taps<float>(taps, [&](auto w) { return f(float(), w); });
    if (dtype == SSAM_F16) return with_taps<_Float16>(taps, [&](auto w) { return f(_Float16(), w); });
    return with_taps<__bf16>(taps, [&](auto w) { return f(__bf16(), w); });
}

int check_filter(int dtype, int param_dtype, int channels, int taps)
{
    if (!type_bytes(dtype) || (param_dtype != dtype && param_dtype != SSAM_F32)) return SSAM_ERR_ENUM;
    if (channels <= 0 || channels > kMaxChannels) return SSAM_ERR_DIM;
    if (taps < 1 || taps > SSAM_MAX_TAPS) return SSAM_ERR_SHAPE;
    return SSAM_OK;
}

bool misaligned(const void* p, int bytes) { return (uintptr_t)p % bytes != 0; }

int strips_of(int channels, int each) { return (channels + kWave * each - 1) / (kWave * each); }
int forward_strips(int channels, int dtype) { return strips_of(channels, 16 / type_bytes(dtype)); }

// Rows of a piece: long pieces read fewer rows twice, short ones give more waves; 4096 waves (four per SIMD) are enough (2048 and
// 8192 are within 1 %).  At least 8, more than the rows a piece reads above itself; fewer than 16 where that gives too few waves
// (512 rows of 4096 channels: 6.7 us, with 16: 9.6).
int piece_rows(const ssam_sequences& q, int strips, int longest)
{
    int rows = longest;
    while (rows > 8 && piece_slots(q, rows) * strips < 4096) rows /= 2;
    return rows;
}

// Rows of a piece of the backward march (4 x 4096 rows of 4096 channels, eight taps, forward and back: 287 us, of 32 rows 320; with four
// taps 32 rows gain 2 % or lose it), and the slots of its partial sums.
int back_piece_rows(const ssam_conv1d_backward_args& a) { return piece_rows(a.seq, strips_of(a.channels, kBackChan), 64); }
long long back_parts(const ssam_conv1d_backward_args& a) { return (piece_slots(a.seq, back_piece_rows(a)) + kWavesPerBlock - 1) / kWavesPerBlock; }

// Blocks of the march: more than a launch holds are refused, and need no workspace.
long long back_blocks(const ssam_conv1d_backward_args& a) { return back_parts(a) * strips_of(a.channels, kBackChan); }

size_t back_bytes(const ssam_conv1d_backward_args& a)
{
    if ((!a.d_grad_weight && !a.d_grad_bias) || back_blocks(a) > kMaxGrid) return 0;
    return (size_t)back_parts(a) * (a.taps + 1) * a.channels * sizeof(float);
}

}  // namespace
}  // namespace ssam

extern "C" {

int ssam_conv1d(const ssam_conv1d_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_filter(a->dtype, a->param_dtype, a->channels, a->taps)) return e;
    if (int e = check_sequences(a->seq)) return e;
    if (a->seq.sequences == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype), psz = type_bytes(a->param_dtype);
    if (!a->d_weight) return SSAM_ERR_NULL;
    if (int e = check_rows(a->in, a->seq, a->channels, esz, false)) return e;
    if (int e = check_out_rows(a->out, a->seq, a->channels, esz, false)) return e;
    if (misaligned(a->d_weight, psz) || misaligned(a->d_bias, psz) || misaligned(a->d_state, esz) || misaligned(a->d_final, esz)) return SSAM_ERR_DIM;
    const long long state_bytes = (long long)a->seq.sequences * (a->taps - 1) * a->channels * esz;
    const Cover outs[] = {cover_rows(a->out, a->seq, a->channels, esz), cover_plain(a->d_final, state_bytes)};
    const Cover ins[] = {cover_rows(a->in, a->seq, a->channels, esz), cover_plain(a->d_weight, (long long)a->channels * a->taps * psz),
                         cover_plain(a->d_bias, (long long)a->channels * psz),
                         cover_plain(a->d_state == a->d_final ? nullptr : a->d_state, state_bytes)};
    if (any_overlap(outs, ins) || (a->d_state && overlaps(outs[0], cover_plain(a->d_state, state_bytes)))) return SSAM_ERR_ALIAS;
    Conv1dParams p{};
    p.strips = forward_strips(a->channels, a->dtype);
    // 32768 rows of 8192 channels, four taps: 197 us (5.45 TB/s), in pieces of 32 rows 215; 65000 rows of 5000, eight taps: 312, of 16 rows 351.
    const int piece = piece_rows(a->seq, p.strips, a->taps <= 4 ? 16 : 32);
    p.pieces = make_pieces(a->seq, piece);
    p.in = a->in;
    p.out = a->out;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    p.state = a->d_state;
    p.final = a->d_final;
    p.channels = a->channels;
    p.silu = a->silu != 0;
    p.params_f32 = a->param_dtype == SSAM_F32;
    p.waves = piece_slots(a->seq, piece) * p.strips;
    const long long blocks = (p.waves + kWavesPerBlock - 1) / kWavesPerBlock;
    if (blocks > kMaxGrid) return SSAM_ERR_DIM;
    return with_type_and_taps(a->dtype, a->taps, [&](auto t, auto w) {
        hipLaunchKernelGGL((conv1d_rows<decltype(t), decltype(w)::value>), dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)hip_stream, p);
        return launched();
    });
}

size_t ssam_conv1d_backward_workspace_bytes(const ssam_conv1d_backward_args* a)
{
    using namespace ssam;
    if (!a || check_filter(a->dtype, a->param_dtype, a->channels, a->taps) || check_sequences(a->seq)) return 0;
    return back_bytes(*a);
}

int ssam_conv1d_backward(const ssam_conv1d_backward_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_filter(a->dtype, a->param_dtype, a->channels, a->taps)) return e;
    if (int e = check_sequences(a->seq)) return e;
    const int esz = type_bytes(a->dtype), psz = type_bytes(a->param_dtype);
    const bool sums = a->d_grad_weight || a->d_grad_bias;
    const bool none = a->seq.sequences == 0;
    if (none && !sums) return SSAM_OK;
    if (!a->d_weight) return SSAM_ERR_NULL;
    if (int e = check_rows(a->in, a->seq, a->channels, esz, false)) return e;
    if (int e = check_rows(a->grad_out, a->seq, a->channels, esz, false)) return e;
    if (int e = check_out_rows(a->grad_in, a->seq, a->channels, esz, true)) return e;
    if (misaligned(a->d_weight, psz) || misaligned(a->d_bias, psz) || misaligned(a->d_state, esz) || misaligned(a->d_grad_final, esz) ||
        misaligned(a->d_grad_weight, psz) || misaligned(a->d_grad_bias, psz) || misaligned(a->d_grad_state, esz))
        return SSAM_ERR_DIM;
    const long long state_bytes = (long long)a->seq.sequences * (a->taps - 1) * a->channels * esz;
    const size_t need = back_bytes(*a);
    if (need && !a->d_work) return SSAM_ERR_NULL;
    if (need && (a->work_bytes < need || misaligned(a->d_work, 16))) return SSAM_ERR_DIM;
    const Cover outs[] = {cover_rows(a->grad_in, a->seq, a->channels, esz), cover_plain(a->d_grad_weight, (long long)a->channels * a->taps * psz),
                          cover_plain(a->d_grad_bias, (long long)a->channels * psz), cover_plain(a->d_grad_state, state_bytes),
                          cover_plain(need ? a->d_work : nullptr, (long long)need)};
    const Cover ins[] = {cover_rows(a->in, a->seq, a->channels, esz), cover_rows(a->grad_out, a->seq, a->channels, esz),
                         cover_plain(a->d_weight, (long long)a->channels * a->taps * psz), cover_plain(a->d_bias, (long long)a->channels * psz),
                         cover_plain(a->d_state, state_bytes), cover_plain(a->d_grad_final, state_bytes)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    Conv1dBackParams p{};
    p.strips = strips_of(a->channels, kBackChan);
    const int piece = back_piece_rows(*a);
    p.pieces = make_pieces(a->seq, piece);
    p.in = a->in;
    p.grad_out = a->grad_out;
    p.grad_in = a->grad_in;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    p.state = a->d_state;
    p.grad_final = a->d_grad_final;
    p.grad_state = a->d_grad_state;
    p.parts = sums ? static_cast<float*>(a->d_work) : nullptr;
    p.channels = a->channels;
    p.silu = a->silu != 0;
    p.params_f32 = a->param_dtype == SSAM_F32;
    p.slots = piece_slots(a->seq, piece);
    const long long parts = back_parts(*a), blocks = back_blocks(*a);
    const long long sum_blocks = (long long)((a->channels + kWave - 1) / kWave) * (a->taps + 1);
    if (blocks > kMaxGrid || sum_blocks > kMaxGrid / 4) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    return with_type_and_taps(a->dtype, a->taps, [&](auto t, auto w) {
        if (blocks) hipLaunchKernelGGL((conv1d_back<decltype(t), decltype(w)::value>), dim3((unsigned)blocks), dim3(kBlock), 0, st, p);
        if (sums)
            hipLaunchKernelGGL((conv1d_back_sums<decltype(t)>), dim3((unsigned)sum_blocks), dim3(kWave * kRuns), 0, st, p.parts, parts, a->taps,
                               a->channels, a->d_grad_weight, a->d_grad_bias, p.params_f32);
        return launched();
    });
}

int ssam_conv1d_step(const ssam_conv1d_step_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_filter(a->dtype, a->param_dtype, a->channels, a->taps)) return e;
    if (int e = check_slots(a->rows, a->slots, a->d_slots)) return e;
    if (a->rows == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype), psz = type_bytes(a->param_dtype);
    const ssam_sequences q{1, a->rows, nullptr, nullptr};
    if (!a->d_weight || (!a->d_state && a->taps > 1)) return SSAM_ERR_NULL;
    if (int e = check_rows(a->in, q, a->channels, esz, false)) return e;
    if (int e = check_out_rows(a->out, q, a->channels, esz, false)) return e;
    const long long slot = (long long)(a->taps - 1) * a->channels;
    if (int e = check_pool(a->slots, a->slot_stride, slot)) return e;
    if (misaligned(a->d_weight, psz) || misaligned(a->d_bias, psz) || misaligned(a->d_state, esz)) return SSAM_ERR_DIM;
    const Cover outs[] = {cover_rows(a->out, q, a->channels, esz), cover_slots(a->d_state, a->slots, a->slot_stride, slot, esz)};
    const Cover ins[] = {cover_rows(a->in, q, a->channels, esz), cover_plain(a->d_weight, (long long)a->channels * a->taps * psz),
                         cover_plain(a->d_bias, (long long)a->channels * psz), cover_plain(a->d_slots, (long long)a->rows * 4)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    Conv1dStepParams p{};
    p.rows = a->rows;
    p.slots = a->slots;
    p.channels = a->channels;
    p.strips = forward_strips(a->channels, a->dtype);
    p.silu = a->silu != 0;
    p.params_f32 = a->param_dtype == SSAM_F32;
    p.slot_of = a->d_slots;
    p.in = a->in;
    p.out = a->out;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    p.state = a->d_state;
    p.slot_stride = a->slot_stride;
    const long long blocks = ((long long)a->rows + kWavesPerBlock - 1) / kWavesPerBlock * p.strips;
    if (blocks > kMaxGrid) return SSAM_ERR_DIM;
    return with_type_and_taps(a->dtype, a->taps, [&](auto t, auto w) {
        hipLaunchKernelGGL((conv1d_step<decltype(t), decltype(w)::value>), dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)hip_stream, p);
        return launched();
    });
}

}  // extern "C"
