// Root-mean-square norm of rows (ssam_rms_norm), with the residual's addition, a gate and an output in 8 bits, and its gradients.
// A unit, `width` values of one row that are normalised together, is held in the registers of TP lanes from its one load to its one
// store: lane i has the vectors i, i + TP, .. of 16 bytes.  Bound by memory: a few operations on the 4 to 8 bytes of a value
// (32768 rows of 4096 bf16 with residual and sum: 188 us, 5.7 TB/s).
// 8192 rows of 8192 bf16 with residual to e4m3 in blocks of 128: 103 us, 4.6 TB/s; 16 values a lane, since 32 of them left two waves a
// SIMD (159 us), and blocks of whole vectors in a kernel of their own, since the division by element of the others costs 120 registers (153).
#include "ssam_rows.h"

namespace ssam {
namespace {

constexpr int kMaxWidth = 32768;                            // values of a unit: 32 a lane of 1024
template <class T> constexpr int kVec = 16 / sizeof(T);     // values of a vector

struct NormParams {
    ssam_rows in, residual, sum, gate, out;
    const void* weight;
    float* scales;
    long long units;
    int groups, width, rows, block, params_f32;
    float eps;
};

// The larger of two values >= 0; NaN stays, as its bits are above infinity's.
struct Larger {
    __device__ __forceinline__ float operator()(float a, float b) const
    {
        const unsigned x = __builtin_bit_cast(unsigned, a), y = __builtin_bit_cast(unsigned, b);
        return __builtin_bit_cast(float, x > y ? x : y);
    }
};
// Over aligned groups of n lanes, a power of two; every lane gets the same result.
template <class Op> __device__ __forceinline__ float over_lanes(float v, int n, Op op)
{
    v = over_few(v, n, op);
    if (n > 16) v = op(v, __shfl_xor(v, 16));
    if (n > 32) v = op(v, __shfl_xor(v, 32));
    return v;
}

// Over the TP threads of a unit; `room`: a float for each wave of the block, used by one call (a barrier lies between two calls of one).
template <int TP, class Op>
__device__ __forceinline__ float over_unit(float v, float* room, Op op)
{
    v = over_lanes(v, TP < kWave ? TP : kWave, op);
    if constexpr (TP > kWave) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & (kWave - 1)) == 0) room[wave] = v;
        __syncthreads();
        v = room[0];
#pragma unroll
        for (int k = 1; k < TP / kWave; ++k) v = op(v, room[k]);
    }
    return v;
}

__device__ __forceinline__ long long row_offset(const ssam_rows& r, long long row, int rows)
{
    const long long s = row / rows;
    return s * r.batch + (row - s * rows) * r.row;
}
template <class T> __device__ __forceinline__ T* unit_of(const ssam_rows& r, long long unit, int groups, int rows, int width)
{
    const long long row = unit / groups;
    return static_cast<T*>(r.d) + row_offset(r, row, rows) + (unit - row * groups) * width;
}

// V weights from channel c on, as floats.
template <class T, int V>
__device__ __forceinline__ RowVec<float, V> load_weights(const void* w, int params_f32, int c, int have, bool part)
{
    RowVec<float, V> f(1.0f);
    if (!w) return f;
    if (params_f32) return load_row_vec<float, V>(static_cast<const float*>(w) + c, have, part);
    const RowVec<T, V> t = load_row_vec<T, V>(static_cast<const T*>(w) + c, have, part);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)t[i];
    return f;
}

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// What a block's codes are multiplied by: its largest magnitude lands on e4m3's, 448.
__device__ __forceinline__ float scale_of(float most)
{
    const float scale = most == 0.0f ? 1.0f : most / 448.0f;
    return scale < 0x1p-126f ? 0x1p-126f : scale;
}

// Codes of a block whose largest magnitude is that of y = f z for values z that have not been through the root's rounding, 1 <= f < 2: y / scale is
// 448 z / max|z|, whose halves between two codes are met exactly where z is (16 bits times a weight of 16 bits); y and scale would each be
// rounded, and which side of a half their quotient falls on would be chance.  448 = 0.875 x 2^9: the quotient of c z and b, c = 0.875, from the
// instruction's reciprocal (1 ulp) and one step of correction by the remainder: what is left is 2^-44 of the quotient, so that one that is a half comes out as
// it.  (Three operations a value more than the product with a reciprocal alone, and a division for eight of them less.)  Near the scale's least value, where y has
// fewer bits, and where the largest value is not finite: the quotient of y and the scale itself.
struct Quotient {
    float scale, per, first, less, back;
    __device__ __forceinline__ Quotient() {}
    __device__ __forceinline__ Quotient(float most, float f)      // max|z|
    {
        const float y = most * f;
        scale = scale_of(y);
        const bool plain = y > 0x1p-90f && y < __builtin_inff();
        const float c = plain ? 0.875f : f, b = plain ? most * 0x1p-9f : scale;
        per = __builtin_amdgcn_rcpf(b);
        first = c * per;
        less = c - 1.0f;
        back = __builtin_isinf(b) ? 0.0f : b;      // (finite values over an infinite scale are zero, not NaN)
    }
    __device__ __forceinline__ float of(float z) const
    {
        const float q = z * first;
        return __builtin_fmaf(__builtin_fmaf(less, z, __builtin_fmaf(-q, back, z)), per, q);
    }
};

// How a unit leaves.
constexpr int kPlain = 0;       // in its own type
constexpr int kLanes = 1;       // e4m3, a block being the unit or the vectors of an aligned group of 2^n <= 16 lanes: no division by element
constexpr int kAnyBlock = 2;    // e4m3 in other blocks, their largest magnitudes in LDS

template <class T, int TP, int NV, int kOut>
__global__ __launch_bounds__(TP > kBlock ? TP : kBlock) void rms_norm(NormParams p)
{
    constexpr int V = kVec<T>, kThreads = TP > kBlock ? TP : kBlock, kUnits = kThreads / TP;
    __shared__ float room[2][kThreads / kWave];
    extern __shared__ unsigned most_of[];
    constexpr bool kE4m3 = kOut != kPlain;
    const int at = threadIdx.x % TP, mine = threadIdx.x / TP;
    for (long long first = (long long)blockIdx.x * kUnits; first < p.units; first += (long long)gridDim.x * kUnits) {
        const long long u = first + mine;
        const bool there = u < p.units;
        const long long unit = there ? u : p.units - 1;
        const T* in = unit_of<T>(p.in, unit, p.groups, p.rows, p.width);
        RowVec<T, V> x[NV];
        float s[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TP + at) * V, have = p.width - c;
            x[j] = have > 0 ? load_row_vec<T, V>(in + c, have) : RowVec<T, V>(T(0));
        }
        if (p.residual.d) {
            const T* res = unit_of<T>(p.residual, unit, p.groups, p.rows, p.width);
            RowVec<T, V> r[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TP + at) * V, have = p.width - c;
                r[j] = have > 0 ? load_row_vec<T, V>(res + c, have) : RowVec<T, V>(T(0));
            }
            T* sum = p.sum.d ? unit_of<T>(p.sum, unit, p.groups, p.rows, p.width) : nullptr;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TP + at) * V, have = p.width - c;
#pragma unroll
                for (int i = 0; i < V; ++i) x[j][i] = (T)((float)x[j][i] + (float)r[j][i]);
                if (sum && there && have > 0) store_row_vec<T, V>(sum + c, have, x[j]);
            }
        }
        float squares = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[j][i] = (float)x[j][i];
                squares = __builtin_fmaf(s[j][i], s[j][i], squares);
            }
        squares = over_unit<TP>(squares, room[0], Add());
        float r = 1.0f / __builtin_sqrtf(squares / (float)p.width + p.eps), f = 1.0f;
        if (kE4m3 && r == r) {      // its power of two alone, exact; the rest joins the scale.  (Zero and infinity are their own, NaN stays.)
            const unsigned bits = __builtin_bit_cast(unsigned, r);
            f = __builtin_bit_cast(float, (bits & 0x7fffffu) | 0x3f800000u);
            r = __builtin_bit_cast(float, bits & 0x7f800000u);
        }
        const T* gate = p.gate.d ? unit_of<T>(p.gate, unit, p.groups, p.rows, p.width) : nullptr;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TP + at) * V, have = p.width - c;
            if (have <= 0) continue;
            const RowVec<float, V> w = load_weights<T, V>(p.weight, p.params_f32, c, have, true);
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = kE4m3 ? s[j][i] * r * w[i] : s[j][i] * (r * w[i]);
            if (gate) {
                const RowVec<T, V> z = load_row_vec<T, V>(gate + c, have);
#pragma unroll
                for (int i = 0; i < V; ++i) s[j][i] *= silu((float)z[i]);
            }
        }
        if constexpr (!kE4m3) {
            T* out = unit_of<T>(p.out, unit, p.groups, p.rows, p.width);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TP + at) * V, have = p.width - c;
                if (there && have > 0) store_row_vec<T, V>(out + c, have, rounded<T, V>(s[j]));
            }
        } else {
            uint8_t* out = unit_of<uint8_t>(p.out, unit, p.groups, p.rows, p.width);
            float* scales = p.scales + unit * (p.width / p.block);
            const int lanes = p.block / V, doublings = __builtin_ctz(lanes | 1 << 30);
            const bool whole = p.block == p.width;
            float most = 0.0f;
            if (kOut == kLanes && whole) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) most = Larger()(most, __builtin_fabsf(s[j][i]));
                most = over_unit<TP>(most, room[1], Larger());
            }
            if constexpr (kOut == kAnyBlock) {
                const int blocks = p.width / p.block;
                unsigned* m = most_of + mine * blocks;
                for (int b = at; b < blocks; b += TP) m[b] = 0;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = (j * TP + at) * V + i;
                        if (c < p.width) atomicMax(&m[c / p.block], __builtin_bit_cast(unsigned, __builtin_fabsf(s[j][i])));      // any order gives the same
                    }
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TP + at) * V, have = p.width - c;
                float q[V];
                if constexpr (kOut == kLanes) {
                    float m = most;
                    if (!whole) {
                        m = 0.0f;
#pragma unroll
                        for (int i = 0; i < V; ++i) m = Larger()(m, __builtin_fabsf(s[j][i]));
                        m = over_lanes(m, lanes, Larger());
                    }
                    const Quotient by(m, f);
                    const int first_of = whole ? c : (j * TP + at) & (lanes - 1), b = whole ? 0 : (j * TP + at) >> doublings;
                    if (there && have > 0 && first_of == 0) scales[b] = by.scale;
#pragma unroll
                    for (int i = 0; i < V; ++i) q[i] = by.of(s[j][i]);
                } else {
                    Quotient by;
                    int block = -1;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        if (c + i >= p.width) {
                            q[i] = 0.0f;
                            continue;
                        }
                        const int b = (c + i) / p.block;
                        if (b != block) {
                            block = b;
                            by = Quotient(__builtin_bit_cast(float, most_of[mine * (p.width / p.block) + b]), f);
                        }
                        q[i] = by.of(s[j][i]);
                        if (there && (c + i) % p.block == 0) scales[b] = by.scale;
                    }
                }
                if (!there || have <= 0) continue;
                if (have >= V) {
                    RowVec<uint32_t, V / 4> word;
#pragma unroll
                    for (int i = 0; i < V; i += 4) word[i / 4] = pack_e4m3(q[i], q[i + 1], q[i + 2], q[i + 3]);
                    __builtin_memcpy(out + c, &word, V);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (i < have) out[c + i] = (uint8_t)pack_e4m3(q[i], q[i], q[i], q[i]);
                }
            }
        }
        if (TP > kWave || kE4m3) __syncthreads();       // before the next unit's sums
    }
}

// ---- gradients ---------------------------------------------------------------------------------------------------------
struct NormBackParams {
    ssam_rows in, gate, grad_out, grad_sum, grad_in, grad_gate;
    const void* weight;
    float* parts;            // [blocks][width], or null
    long long units;
    int groups, width, rows, params_f32;
    float eps;
};

// With r = 1 / sqrt(mean(s^2) + eps), d = grad_out (times silu(gate)) and a = d w r:
//     grad_in = a - s r^2 mean(a s) + grad_sum,   grad_weight = sum over the units of d s r
// Both means come from one pass over the unit: mean(a s) = r mean(d w s).  The weights' sums stay in the lanes' registers over the units
// of a block and leave as one row of `parts`.  16384 rows of 4096 bf16 with the sum's gradient: 140 us, 3.8 TB/s, and 7 for the parts; the next unit's
// loads made early take 31 registers more, with three waves a SIMD in place of four 184 us, and 512 lanes a unit 167.
template <class T, int TP, int NV>
__global__ __launch_bounds__(TP > kBlock ? TP : kBlock) void rms_norm_back(NormBackParams p)
{
    constexpr int V = kVec<T>, kThreads = TP > kBlock ? TP : kBlock, kUnits = kThreads / TP;
    __shared__ float room[2][kThreads / kWave];
    __shared__ RowVec<float, V> shares[kUnits > 1 ? kThreads : 1];
    const int at = threadIdx.x % TP, mine = threadIdx.x / TP;
    float dw[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[j][i] = 0.0f;
    for (long long first = (long long)blockIdx.x * kUnits; first < p.units; first += (long long)gridDim.x * kUnits) {
        const long long u = first + mine;
        const bool there = u < p.units;
        const long long unit = there ? u : p.units - 1;
        const T* in = unit_of<T>(p.in, unit, p.groups, p.rows, p.width);
        const T* grad = unit_of<T>(p.grad_out, unit, p.groups, p.rows, p.width);
        const T* gate = p.gate.d ? unit_of<T>(p.gate, unit, p.groups, p.rows, p.width) : nullptr;
        RowVec<T, V> x[NV], d[NV];
        float squares = 0.0f, mixed = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TP + at) * V, have = p.width - c;
            x[j] = have > 0 ? load_row_vec<T, V>(in + c, have) : RowVec<T, V>(T(0));
            d[j] = have > 0 ? load_row_vec<T, V>(grad + c, have) : RowVec<T, V>(T(0));
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TP + at) * V, have = p.width - c;
            if (have <= 0) continue;
            const RowVec<float, V> w = load_weights<T, V>(p.weight, p.params_f32, c, have, true);
            RowVec<T, V> z(T(0));
            if (gate) z = load_row_vec<T, V>(gate + c, have);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = (float)x[j][i];
                float e = (float)d[j][i];
                if (gate) e *= silu((float)z[i]);
                squares = __builtin_fmaf(s, s, squares);
                mixed = __builtin_fmaf(e * w[i], s, mixed);
            }
        }
        squares = over_unit<TP>(squares, room[0], Add());
        mixed = over_unit<TP>(mixed, room[1], Add());
        const float r = 1.0f / __builtin_sqrtf(squares / (float)p.width + p.eps);
        const float back = mixed / (float)p.width * r * r * r;
        T* gx = p.grad_in.d ? unit_of<T>(p.grad_in, unit, p.groups, p.rows, p.width) : nullptr;
        T* gz = p.grad_gate.d ? unit_of<T>(p.grad_gate, unit, p.groups, p.rows, p.width) : nullptr;
        const T* more = p.grad_sum.d ? unit_of<T>(p.grad_sum, unit, p.groups, p.rows, p.width) : nullptr;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TP + at) * V, have = p.width - c;
            if (have <= 0 || !there) continue;
            const RowVec<float, V> w = load_weights<T, V>(p.weight, p.params_f32, c, have, true);
            RowVec<T, V> z(T(0)), m(T(0));
            if (gate) z = load_row_vec<T, V>(gate + c, have);
            if (more) m = load_row_vec<T, V>(more + c, have);
            float dx[V], dz[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = (float)x[j][i];
                float e = (float)d[j][i];
                if (gate) {
                    const float t = (float)z[i], sig = sigmoid(t);
                    dz[i] = e * (s * r * w[i]) * (sig * (1.0f + t * (1.0f - sig)));
                    e *= t * sig;
                }
                dw[j][i] = __builtin_fmaf(e, s * r, dw[j][i]);
                dx[i] = __builtin_fmaf(-back, s, e * w[i] * r);
                if (more) dx[i] += (float)m[i];
            }
            if (gx) store_row_vec<T, V>(gx + c, have, rounded<T, V>(dx));
            if (gz) store_row_vec<T, V>(gz + c, have, rounded<T, V>(dz));
        }
        if (TP > kWave) __syncthreads();
    }
    if (!p.parts) return;
    float* part = p.parts + (long long)blockIdx.x * p.width;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TP + at) * V, have = p.width - c;
        RowVec<float, V> f;
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = dw[j][i];
        if constexpr (kUnits > 1) {
            __syncthreads();
            shares[threadIdx.x] = f;
            __syncthreads();
            if (mine == 0)
#pragma unroll
                for (int k = 1; k < kUnits; ++k) f += shares[k * TP + at];
        }
        if (mine == 0 && have > 0) store_row_vec<float, V>(part + c, have, f);
    }
}

// parts summed over the blocks, 16 interleaved runs of them and then the runs, always in the same order.
constexpr int kRuns = 16;
template <class T>
__global__ __launch_bounds__(kWave* kRuns) void rms_norm_back_sums(const float* __restrict__ parts, int blocks, int width, void* grad_weight, int params_f32)
{
    __shared__ float run[kRuns][kWave];
    const int lane = threadIdx.x & (kWave - 1), r = threadIdx.x >> 6, c = blockIdx.x * kWave + lane;
    float s = 0.0f;
    if (c < width)
#pragma unroll 4
        for (int i = r; i < blocks; i += kRuns) s += parts[(long long)i * width + c];
    run[r][lane] = s;
    __syncthreads();
    if (r != 0 || c >= width) return;
#pragma unroll
    for (int k = 1; k < kRuns; ++k) s += run[k][lane];
    if (params_f32) static_cast<float*>(grad_weight)[c] = s;
    else static_cast<T*>(grad_weight)[c] = (T)s;
}

// ---- host --------------------------------------------------------------------------------------------------------------
template <class F>
int with_row_type(int dtype, F f)
{
    if (dtype == SSAM_F32) return f(float());
    if (dtype == SSAM_F16) return f(_Float16());
    return f(__bf16());
}

// f gets the threads of a unit and the vectors of a thread as compile-time constants: one wave a unit, whose sums need no barrier, where units fill
// the card (4096 rows of 2048 bf16 13.7 -> 12.5 us), and more lanes for it where they do not (64 rows 4.7 -> 3.6 us).
template <int V, class F>
int with_layout(int width, long long units, F f)
{
    const int vectors = (width + V - 1) / V;
#define SSAM_LAYOUT(TP, NV) \
    if (vectors <= TP * NV) return f(std::integral_constant<int, TP>{}, std::integral_constant<int, NV>{})
    SSAM_LAYOUT(16, 1);
    if (units >= 2048 || vectors <= 64) {
        SSAM_LAYOUT(64, 1);
        SSAM_LAYOUT(64, 2);
        SSAM_LAYOUT(64, 4);
    }
    SSAM_LAYOUT(256, 1);
    SSAM_LAYOUT(256, 2);
    SSAM_LAYOUT(512, 2);
    SSAM_LAYOUT(1024, 2);
    SSAM_LAYOUT(1024, 4);
    if constexpr (V == 4) SSAM_LAYOUT(1024, 8);
#undef SSAM_LAYOUT
    return SSAM_ERR_SHAPE;
}

constexpr int kBackBlocks = 1024;      // four a compute unit
// Units that a block takes at a time, as rms_norm_back's layout has them.
int back_blocks(int dtype, int width, long long units)
{
    return with_row_type(dtype, [&](auto t) {
        return with_layout<kVec<decltype(t)>>(width, units, [&](auto tp, auto) {
            constexpr int TP = decltype(tp)::value, kUnits = TP < kBlock ? kBlock / TP : 1;
            const long long need = (units + kUnits - 1) / kUnits;
            return (int)(need < kBackBlocks ? need : kBackBlocks);
        });
    });
}

template <class Args>
int check_norm(const Args& a)
{
    if (!type_bytes(a.dtype) || (a.param_dtype != a.dtype && a.param_dtype != SSAM_F32)) return SSAM_ERR_ENUM;
    if (a.channels <= 0 || a.channels > kMaxChannels || a.sequences < 0 || a.rows < 0 || a.sequences > SSAM_MAX_EXTENT || a.rows > SSAM_MAX_EXTENT) return SSAM_ERR_DIM;
    if ((long long)a.sequences * a.rows > kMaxRows) return SSAM_ERR_DIM;
    if (a.groups < 1 || a.channels % a.groups || a.channels / a.groups > kMaxWidth || !(a.eps >= 0.0f)) return SSAM_ERR_SHAPE;
    return (uintptr_t)a.d_weight % (a.param_dtype == SSAM_F32 ? 4 : 2) ? SSAM_ERR_DIM : SSAM_OK;
}

int norm(const ssam_rms_norm_args* a, void* hip_stream, bool e4m3)
{
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_norm(*a)) return e;
    const int esz = type_bytes(a->dtype), width = a->channels / a->groups, out_size = e4m3 ? 1 : esz;
    if (e4m3 && (a->block < 1 || width % a->block || (a->block < 16 && a->block != width))) return SSAM_ERR_SHAPE;
    const ssam_sequences q{a->sequences, a->rows, nullptr, nullptr};
    const bool empty = a->sequences == 0 || a->rows == 0;
    if (int e = check_rows(a->in, q, a->channels, esz, false)) return e;
    for (const ssam_rows* r : {&a->residual, &a->gate})
        if (int e = check_rows(*r, q, a->channels, esz, true)) return e;
    if (a->sum.d && !a->residual.d) return SSAM_ERR_NULL;
    if (int e = check_out_rows(a->sum, q, a->channels, esz, true)) return e;
    if (int e = check_out_rows(a->out, q, a->channels, out_size, false)) return e;
    if (e4m3 && !a->d_scales && !empty) return SSAM_ERR_NULL;
    if (e4m3 && (uintptr_t)a->d_scales % 4) return SSAM_ERR_DIM;
    if (empty) return SSAM_OK;
    const long long units = (long long)a->sequences * a->rows * a->groups;
    const bool in_place = a->sum.d && a->sum.d == a->residual.d && a->sum.row == a->residual.row && a->sum.batch == a->residual.batch;
    const Cover residual = cover_rows(a->residual, q, a->channels, esz);
    const Cover outs[] = {cover_rows(a->out, q, a->channels, out_size), cover_rows(a->sum, q, a->channels, esz),
                          cover_plain(e4m3 ? a->d_scales : nullptr, e4m3 ? product(units, width / a->block * 4LL) : 0)};
    const Cover ins[] = {cover_rows(a->in, q, a->channels, esz), cover_rows(a->gate, q, a->channels, esz),
                         cover_plain(a->d_weight, (long long)width * (a->param_dtype == SSAM_F32 ? 4 : esz))};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    for (int i = 0; i < 3; ++i)
        if (overlaps(outs[i], residual) && !(i == 1 && in_place)) return SSAM_ERR_ALIAS;
    const NormParams p{a->in, a->residual, a->sum, a->gate, a->out, a->d_weight, a->d_scales, units, a->groups, width, a->rows, a->block,
                       a->param_dtype == SSAM_F32, a->eps};
    return with_row_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        return with_layout<kVec<T>>(width, units, [&](auto tp, auto nv) {
            constexpr int TP = decltype(tp)::value, NV = decltype(nv)::value, kThreads = TP > kBlock ? TP : kBlock, kUnits = kThreads / TP;
            const long long need = (units + kUnits - 1) / kUnits, most = kMaxGrid / (kThreads / kBlock);
            const dim3 grid((unsigned)(need < most ? need : most)), block(kThreads);
            hipStream_t st = (hipStream_t)hip_stream;
            const int lanes = e4m3 && a->block % kVec<T> == 0 ? a->block / kVec<T> : 0;
            if (!e4m3) hipLaunchKernelGGL((rms_norm<T, TP, NV, kPlain>), grid, block, 0, st, p);
            else if (a->block == width || (lanes && lanes <= 16 && !(lanes & (lanes - 1)))) hipLaunchKernelGGL((rms_norm<T, TP, NV, kLanes>), grid, block, 0, st, p);
            else hipLaunchKernelGGL((rms_norm<T, TP, NV, kAnyBlock>), grid, block, (size_t)kUnits * (width / a->block) * 4, st, p);
            return launched();
        });
    });
}

}  // namespace
}  // namespace ssam

extern "C" {

int ssam_rms_norm(const ssam_rms_norm_args* a, void* hip_stream) { return ssam::norm(a, hip_stream, false); }
int ssam_rms_norm_e4m3(const ssam_rms_norm_args* a, void* hip_stream) { return ssam::norm(a, hip_stream, true); }

size_t ssam_rms_norm_backward_workspace_bytes(const ssam_rms_norm_backward_args* a)
{
    using namespace ssam;
    if (!a || check_norm(*a) || !a->d_grad_weight) return 0;
    const long long units = (long long)a->sequences * a->rows * a->groups;
    const int width = a->channels / a->groups;
    return (size_t)back_blocks(a->dtype, width, units) * width * 4;
}

int ssam_rms_norm_backward(const ssam_rms_norm_backward_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_norm(*a)) return e;
    const int esz = type_bytes(a->dtype), width = a->channels / a->groups, psz = a->param_dtype == SSAM_F32 ? 4 : esz;
    const ssam_sequences q{a->sequences, a->rows, nullptr, nullptr};
    for (const ssam_rows* r : {&a->in, &a->grad_out})
        if (int e = check_rows(*r, q, a->channels, esz, false)) return e;
    for (const ssam_rows* r : {&a->gate, &a->grad_sum})
        if (int e = check_rows(*r, q, a->channels, esz, true)) return e;
    for (const ssam_rows* r : {&a->grad_in, &a->grad_gate})
        if (int e = check_out_rows(*r, q, a->channels, esz, true)) return e;
    if (a->grad_gate.d && !a->gate.d && a->sequences && a->rows) return SSAM_ERR_NULL;
    if ((uintptr_t)a->d_grad_weight % psz) return SSAM_ERR_DIM;
    const long long units = (long long)a->sequences * a->rows * a->groups;
    const size_t bytes = ssam_rms_norm_backward_workspace_bytes(a);
    if (bytes && !a->d_work) return SSAM_ERR_NULL;
    if (bytes && (a->work_bytes < bytes || (uintptr_t)a->d_work % 16)) return SSAM_ERR_DIM;
    const Cover outs[] = {cover_rows(a->grad_in, q, a->channels, esz), cover_rows(a->grad_gate, q, a->channels, esz),
                          cover_plain(a->d_grad_weight, (long long)width * psz), cover_plain(bytes ? a->d_work : nullptr, (long long)bytes)};
    const Cover ins[] = {cover_rows(a->in, q, a->channels, esz), cover_rows(a->gate, q, a->channels, esz), cover_rows(a->grad_out, q, a->channels, esz),
                         cover_rows(a->grad_sum, q, a->channels, esz), cover_plain(a->d_weight, (long long)width * psz)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    const int blocks = back_blocks(a->dtype, width, units);
    hipStream_t st = (hipStream_t)hip_stream;
    const NormBackParams p{a->in, a->gate, a->grad_out, a->grad_sum, a->grad_in, a->grad_gate, a->d_weight, bytes ? static_cast<float*>(a->d_work) : nullptr,
                           units, a->groups, width, a->rows, a->param_dtype == SSAM_F32, a->eps};
    return with_row_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        if (blocks > 0) {
            const int e = with_layout<kVec<T>>(width, units, [&](auto tp, auto nv) {
                constexpr int TP = decltype(tp)::value, NV = decltype(nv)::value, kThreads = TP > kBlock ? TP : kBlock;
                hipLaunchKernelGGL((rms_norm_back<T, TP, NV>), dim3((unsigned)blocks), dim3(kThreads), 0, st, p);
                return launched();
            });
            if (e) return e;
        }
        if (!a->d_grad_weight) return (int)SSAM_OK;
        hipLaunchKernelGGL((rms_norm_back_sums<T>), dim3((unsigned)((width + kWave - 1) / kWave)), dim3(kWave * kRuns), 0, st, p.parts, blocks, width,
                           a->d_grad_weight, p.params_f32);
        return launched();
    });
}

}  // extern "C"
