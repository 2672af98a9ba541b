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

struct Conv1dParams {
    Pieces pieces;
    ssam_rows in, out;
    const void *weight, *bias, *state;
    void* final;
    int channels, strips, silu, params_f32;
    long long waves;
};

template <class T, int W>
__device__ __forceinline__ void load_taps(const void* weight, bool f32, int c, int have, float (&w)[W][kChan<T>])
{
#pragma unroll
    for (int v = 0; v < kChan<T>; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][v] = v < have ? param_at<T>(weight, f32, (long long)(c + v) * W + j) : 0.0f;
}

template <class T>
__device__ __forceinline__ void load_bias(const void* bias, bool f32, int c, int have, float (&b)[kChan<T>])
{
#pragma unroll
    for (int v = 0; v < kChan<T>; ++v) b[v] = bias && v < have ? param_at<T>(bias, f32, c + v) : 0.0f;
}

// Row t < 0 of sequence s: from its carried state, zeros without one.
template <class T, int W>
__device__ __forceinline__ RowVec<T, kChan<T>> carried_row(const void* state, int s, int t, int channels, int c, int have)
{
    if (!state) return load_row_vec<T, kChan<T>>(nullptr, 0);
    return load_row_vec<T, kChan<T>>(static_cast<const T*>(state) + ((long long)s * (W - 1) + (W - 1 + t)) * channels + c, have);
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
    const int c = (strip * kWave + lane) * V;
    const int have = p.channels - c;
    if (have <= 0) return;
    const T* __restrict__ in = sequence_base<T>(p.in, p.pieces, q) + c;
    T* __restrict__ out = sequence_base<T>(p.out, p.pieces, q) + c;
    float w[W][V], b[V];
    load_taps<T, W>(p.weight, p.params_f32, c, have, w);
    load_bias<T>(p.bias, p.params_f32, c, have, b);
    RowVec<T, V> win[W];        // rows t - W + 1 .. t
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int t = q.row0 - (W - 1) + j;
        win[j + 1] = t >= 0 ? load_row_vec<T, V>(in + (long long)t * p.in.row, q.n > 0 ? have : 0)
                            : carried_row<T, W>(p.state, q.seq, t, p.channels, c, have);
    }
    for (int k = 0; k < q.n; k += kMarch) {
        RowVec<T, V> x[kMarch];
#pragma unroll
        for (int u = 0; u < kMarch; ++u)
            x[u] = load_row_vec<T, V>(in + (long long)(q.row0 + k + u) * p.in.row, k + u < q.n ? have : 0);
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
                y[v] = p.silu ? silu(s) : s;
            }
            if (k + u < q.n) store_row_vec<T, V>(out + (long long)(q.row0 + k + u) * p.out.row, have, rounded<T, V>(y));
        }
    }
    // The first piece's wave also hands on the state: it is the only one that reads the old one, so that both may be the same
    // array (row j of the new state is row len + j of the old one, never below j).
    if (W > 1 && p.final && q.row0 == 0) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = q.len - (W - 1) + j;
            const RowVec<T, V> x = t >= 0 ? load_row_vec<T, V>(in + (long long)t * p.in.row, have)
                                          : carried_row<T, W>(p.state, q.seq, t, p.channels, c, have);
            store_row_vec<T, V>(static_cast<T*>(p.final) + ((long long)q.seq * (W - 1) + j) * p.channels + c, have, x);
        }
    }
}

// ---- gradients ---------------------------------------------------------------------------------------------------------
struct Conv1dBackParams {
    Pieces pieces;
    ssam_rows in, grad_out, grad_in;
    const void *weight, *bias, *state, *grad_final;
    void* grad_state;
    float* parts;               // [slot][W + 1][channels]: this slot's sums for the weight's and the bias's gradient, or null
    int channels, strips, silu, params_f32;
    long long waves;
};

// q_t = dy_t silu'(p_t), dx_t = sum_j w[j] q_{t + W - 1 - j}, dw[j] = sum_t q_t x_{t - W + 1 + j}, db = sum_t q_t.  One march over
// the rows of the piece and the W-1 behind it: p_t comes again from the window of inputs, and a second window holds the last W
// q's.  dx runs W-1 rows behind the march, so the first piece also meets rows -(W-1) .. -1, the gradient of the carried rows.
// The sums over rows stay in registers and go to `parts`, to be added slot after slot.
template <class T, int W>
__global__ __launch_bounds__(kBlock) void conv1d_back(Conv1dBackParams p)
{
    constexpr int V = kChan<T>;
    const int lane = threadIdx.x & (kWave - 1);
    const long long wave = (long long)blockIdx.x * kWavesPerBlock + (threadIdx.x >> 6);
    if (wave >= p.waves) return;
    const int strip = (int)(wave % p.strips);
    const int slot = (int)(wave / p.strips);
    const Piece q = find_piece(p.pieces, slot);
    const int c = (strip * kWave + lane) * V;
    const int have = p.channels - c;
    if (have <= 0) return;
    float dw[W + 1][V];         // the last: the bias's
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) dw[j][v] = 0.0f;
    if (q.seq >= 0) {
        const T* __restrict__ in = sequence_base<T>(p.in, p.pieces, q) + c;
        const T* __restrict__ dy = sequence_base<T>(p.grad_out, p.pieces, q) + c;
        T* __restrict__ dx = p.grad_in.d ? sequence_base<T>(p.grad_in, p.pieces, q) + c : nullptr;
        float w[W][V], b[V], qs[W][V];
        load_taps<T, W>(p.weight, p.params_f32, c, have, w);
        load_bias<T>(p.bias, p.params_f32, c, have, b);
        RowVec<T, V> win[W];
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) qs[j][v] = 0.0f;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = q.row0 - (W - 1) + j;
            win[j + 1] = t >= 0 ? load_row_vec<T, V>(in + (long long)t * p.in.row, have)
                                : carried_row<T, W>(p.state, q.seq, t, p.channels, c, have);
        }
        const int rows = q.n + W - 1;       // the march: rows row0 .. row0 + rows - 1, zeros from len on
        for (int k = 0; k < rows; k += kMarch) {
            RowVec<T, V> x[kMarch], g[kMarch];
#pragma unroll
            for (int u = 0; u < kMarch; ++u) {
                const int t = q.row0 + k + u;
                const int there = k + u < rows && t < q.len ? have : 0;
                x[u] = load_row_vec<T, V>(in + (long long)t * p.in.row, there);
                g[u] = load_row_vec<T, V>(dy + (long long)t * p.grad_out.row, there);
            }
#pragma unroll
            for (int u = 0; u < kMarch; ++u) {
                const int t = q.row0 + k + u;
                if (k + u >= rows) continue;
#pragma unroll
                for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
                win[W - 1] = x[u];
#pragma unroll
                for (int v = 0; v < V; ++v) {
#pragma unroll
                    for (int j = W - 1; j > 0; --j) qs[j][v] = qs[j - 1][v];
                    float d = (float)g[u][v];
                    if (p.silu) {
                        float s = b[v];
#pragma unroll
                        for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][v], (float)win[j][v], s);
                        const float sig = sigmoid(s);
                        d *= sig * __builtin_fmaf(s, 1.0f - sig, 1.0f);
                    }
                    qs[0][v] = t < q.len ? d : 0.0f;
                }
                if (k + u < q.n) {          // rows of this piece; those behind it are another's
#pragma unroll
                    for (int v = 0; v < V; ++v) {
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j][v] = __builtin_fmaf(qs[0][v], (float)win[j][v], dw[j][v]);
                        dw[W][v] += qs[0][v];
                    }
                }
                const int o = t - (W - 1);  // the row whose gradient is complete
                const bool carried = o < 0;
                if (o < q.row0 && !carried) continue;
                if (carried ? !p.grad_state : !dx) continue;
                float d[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    d[v] = 0.0f;
#pragma unroll
                    for (int j = 0; j < W; ++j) d[v] = __builtin_fmaf(w[j][v], qs[j][v], d[v]);
                }
                const int tail = o - (q.len - (W - 1));
                if (p.grad_final && tail >= 0) {
                    const RowVec<T, V> f = load_row_vec<T, V>(
                        static_cast<const T*>(p.grad_final) + ((long long)q.seq * (W - 1) + tail) * p.channels + c, have);
#pragma unroll
                    for (int v = 0; v < V; ++v) d[v] += (float)f[v];
                }
                T* to = carried ? static_cast<T*>(p.grad_state) + ((long long)q.seq * (W - 1) + t) * p.channels + c
                                : dx + (long long)o * p.grad_in.row;
                store_row_vec<T, V>(to, have, rounded<T, V>(d));
            }
        }
    }
    if (p.parts) {
#pragma unroll
        for (int j = 0; j <= W; ++j) {
            RowVec<float, V> f;
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = dw[j][v];
            store_row_vec<float, V>(p.parts + ((long long)slot * (W + 1) + j) * p.channels + c, have, f);
        }
    }
}

// parts summed over the slots, 16 interleaved runs of them and then the runs, always in the same order.
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
    long long slot_stride, waves;
};

template <class T, int W>
__global__ __launch_bounds__(kBlock) void conv1d_step(Conv1dStepParams p)
{
    constexpr int V = kChan<T>;
    const int lane = threadIdx.x & (kWave - 1);
    const long long wave = (long long)blockIdx.x * kWavesPerBlock + (threadIdx.x >> 6);
    if (wave >= p.waves) return;
    const int row = (int)(wave / p.strips);
    const int c = ((int)(wave % p.strips) * kWave + lane) * V;
    const int have = p.channels - c;
    SlotRows same(p.slot_of, p.rows, p.slots, row);
    if (!same.leads()) return;
    T* __restrict__ state = static_cast<T*>(p.state) + (long long)same.slot() * p.slot_stride + c;
    float w[W][V], b[V];
    load_taps<T, W>(p.weight, p.params_f32, c, have, w);
    load_bias<T>(p.bias, p.params_f32, c, have, b);
    RowVec<T, V> win[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j + 1] = load_row_vec<T, V>(state + (long long)j * p.channels, have);
    for (int r = row; r >= 0; r = same.next()) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
        win[W - 1] = load_row_vec<T, V>(static_cast<const T*>(p.in.d) + (long long)r * p.in.row + c, have);
        float y[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float s = b[v];
#pragma unroll
            for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][v], (float)win[j][v], s);
            y[v] = p.silu ? silu(s) : s;
        }
        if (have > 0) store_row_vec<T, V>(static_cast<T*>(p.out.d) + (long long)r * p.out.row + c, have, rounded<T, V>(y));
    }
    if (have > 0) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) store_row_vec<T, V>(state + (long long)j * p.channels, have, win[j + 1]);
    }
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

int strips_of(int channels, int dtype) { const int wide = kWave * 16 / type_bytes(dtype); return (channels + wide - 1) / wide; }

// Rows of a piece: long pieces read fewer rows twice, short ones give more waves; 4096 waves (four per SIMD) are enough.
int piece_rows(const ssam_sequences& q, int strips, int longest)
{
    int rows = longest;
    while (rows > 8 && piece_slots(q, rows) * strips < 4096) rows /= 2;
    return rows;
}

// Rows of a piece of the backward march, and the slots of its partial sums.
int back_piece_rows(const ssam_conv1d_backward_args& a) { return piece_rows(a.seq, strips_of(a.channels, a.dtype), 64); }

size_t back_bytes(const ssam_conv1d_backward_args& a)
{
    if (!a.d_grad_weight && !a.d_grad_bias) return 0;
    return (size_t)piece_slots(a.seq, back_piece_rows(a)) * (a.taps + 1) * a.channels * sizeof(float);
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
    if (int e = check_rows(a->in, a->seq, esz, false)) return e;
    if (int e = check_out_rows(a->out, a->seq, a->channels, esz, false)) return e;
    if (misaligned(a->d_weight, psz) || misaligned(a->d_bias, psz) || misaligned(a->d_state, esz) || misaligned(a->d_final, esz)) return SSAM_ERR_DIM;
    const long long state_bytes = (long long)a->seq.sequences * (a->taps - 1) * a->channels * esz;
    const Cover outs[] = {cover_rows(a->out, a->seq, a->channels, esz), cover_plain(a->d_final, state_bytes)};
    const Cover ins[] = {cover_rows(a->in, a->seq, a->channels, esz), cover_plain(a->d_weight, (long long)a->channels * a->taps * psz),
                         cover_plain(a->d_bias, (long long)a->channels * psz),
                         cover_plain(a->d_state == a->d_final ? nullptr : a->d_state, state_bytes)};
    if (any_overlap(outs, ins) || (a->d_state && overlaps(outs[0], cover_plain(a->d_state, state_bytes)))) return SSAM_ERR_ALIAS;
    Conv1dParams p{};
    p.strips = strips_of(a->channels, a->dtype);
    const int piece = piece_rows(a->seq, p.strips, 32);
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
    if (int e = check_rows(a->in, a->seq, esz, false)) return e;
    if (int e = check_rows(a->grad_out, a->seq, esz, false)) return e;
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
    p.strips = strips_of(a->channels, a->dtype);
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
    const long long slots = piece_slots(a->seq, piece);
    p.waves = slots * p.strips;
    const long long blocks = (p.waves + kWavesPerBlock - 1) / kWavesPerBlock;
    const long long sum_blocks = (long long)((a->channels + kWave - 1) / kWave) * (a->taps + 1);
    if (blocks > kMaxGrid || sum_blocks > kMaxGrid / 4) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    return with_type_and_taps(a->dtype, a->taps, [&](auto t, auto w) {
        if (blocks) hipLaunchKernelGGL((conv1d_back<decltype(t), decltype(w)::value>), dim3((unsigned)blocks), dim3(kBlock), 0, st, p);
        if (sums)
            hipLaunchKernelGGL((conv1d_back_sums<decltype(t)>), dim3((unsigned)sum_blocks), dim3(kWave * kRuns), 0, st, p.parts, slots, a->taps,
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
    if (int e = check_rows(a->in, q, esz, false)) return e;
    if (int e = check_out_rows(a->out, q, a->channels, esz, false)) return e;
    const long long slot = (long long)(a->taps - 1) * a->channels;
    if (misaligned(a->d_weight, psz) || misaligned(a->d_bias, psz) || misaligned(a->d_state, esz) || a->slot_stride < slot || a->slot_stride > kMaxStride)
        return SSAM_ERR_DIM;
    const Cover outs[] = {cover_rows(a->out, q, a->channels, esz), cover_slots(a->d_state, a->slots, a->slot_stride, slot, esz)};
    const Cover ins[] = {cover_rows(a->in, q, a->channels, esz), cover_plain(a->d_weight, (long long)a->channels * a->taps * psz),
                         cover_plain(a->d_bias, (long long)a->channels * psz), cover_plain(a->d_slots, (long long)a->rows * 4)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    Conv1dStepParams p{};
    p.rows = a->rows;
    p.slots = a->slots;
    p.channels = a->channels;
    p.strips = strips_of(a->channels, a->dtype);
    p.silu = a->silu != 0;
    p.params_f32 = a->param_dtype == SSAM_F32;
    p.slot_of = a->d_slots;
    p.in = a->in;
    p.out = a->out;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    p.state = a->d_state;
    p.slot_stride = a->slot_stride;
    p.waves = (long long)a->rows * p.strips;
    const long long blocks = (p.waves + kWavesPerBlock - 1) / kWavesPerBlock;
    if (blocks > kMaxGrid) return SSAM_ERR_DIM;
    return with_type_and_taps(a->dtype, a->taps, [&](auto t, auto w) {
        hipLaunchKernelGGL((conv1d_step<decltype(t), decltype(w)::value>), dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)hip_stream, p);
        return launched();
    });
}

}  // extern "C"
