// The scan with matrix states for one more row of many sequences (ssam_scan_delta_step).  A block holds one head's state, or a range of
// its columns, in registers between its one load and its one store.  S'^T k and S'^T q come from one pass: with S = S' + k u^T,
// S^T q = S'^T q + (k . q) u.  Bound by memory: a state is read and written for seven operations on each of its values (256 rows of 32 heads of
// 128 x 128: 217 us, 4.9 TB/s).
#include "ssam_scan_delta.h"

namespace ssam {
namespace {

struct DeltaStepParams {
    int rows, slots, heads, key_heads, key_dim, value_dim, unit, tiles;
    float scale;
    const int* slot_of;
    ssam_rows q, k, v, out, g, beta;
    long long q_head, k_head, v_head, out_head;
    float* state;
    long long slot_stride;
};

// LN lanes of four columns each; 256 / LN groups of rows, ROWS rows of a group in a thread.
template <class T, int LN, int ROWS>
__global__ __launch_bounds__(kBlock) void delta_step(DeltaStepParams p)
{
    constexpr int kGroups = kBlock / LN, kDim = kGroups * ROWS, kWide = 4 * LN;
    __shared__ float keys[kDim], queries[kDim];
    __shared__ Float4 sums[2][kWavesPerBlock][LN];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, col = tid % LN, group = tid / LN;
    const int tile = (int)(blockIdx.x % p.tiles), head = (int)(blockIdx.x / p.tiles % p.heads), row = (int)(blockIdx.x / p.tiles / p.heads);
    SlotRows same(p.slot_of, p.rows, p.slots, row);
    if (!same.leads()) return;
    const int c0 = tile * kWide + 4 * col, have = p.value_dim - c0;
    float* const state = p.state + (long long)same.slot() * p.slot_stride + (long long)head * p.key_dim * p.value_dim + c0;
    Float4 s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int d = i * kGroups + group;
        s[i] = d < p.key_dim && have > 0 ? load_row_vec<float, 4>(state + (long long)d * p.value_dim, have) : Float4(0.0f);
    }
    const int key_head = head / (p.heads / p.key_heads);
    for (int r = row;;) {
        const T* k = static_cast<const T*>(p.k.d) + (long long)r * p.k.row + key_head * p.k_head;
        const T* q = static_cast<const T*>(p.q.d) + (long long)r * p.q.row + key_head * p.q_head;
        const float g = p.g.d ? static_cast<const float*>(p.g.d)[(long long)r * p.g.row + head] : 0.0f;
        const float beta = static_cast<const float*>(p.beta.d)[(long long)r * p.beta.row + head];
        const T* vrow = static_cast<const T*>(p.v.d) + (long long)r * p.v.row + head * p.v_head + c0;
        const RowVec<T, 4> v = have > 0 ? load_row_vec<T, 4>(vrow, have) : RowVec<T, 4>(T(0));
        constexpr int kOf = (kDim + kWave - 1) / kWave;     // elements of a lane; every wave makes the sums by itself
        float kv[kOf], qv[kOf], kk = 0.0f, qq = 0.0f, kq = 0.0f;
#pragma unroll
        for (int i = 0; i < kOf; ++i) {
            const int d = i * kWave + lane;
            kv[i] = d < p.key_dim ? (float)k[d] : 0.0f;
            qv[i] = d < p.key_dim ? (float)q[d] : 0.0f;
            kk = __builtin_fmaf(kv[i], kv[i], kk);
            qq = __builtin_fmaf(qv[i], qv[i], qq);
            kq = __builtin_fmaf(kv[i], qv[i], kq);
        }
#pragma unroll
        for (int x = 1; x < kWave; x *= 2) {
            kk += __shfl_xor(kk, x);
            qq += __shfl_xor(qq, x);
            kq += __shfl_xor(kq, x);
        }
        const float fk = p.unit ? 1.0f / __builtin_sqrtf(kk + 1e-6f) : 1.0f, fq = p.unit ? 1.0f / __builtin_sqrtf(qq + 1e-6f) : 1.0f;
        if (wave == 0)
#pragma unroll
            for (int i = 0; i < kOf; ++i) {
                const int d = i * kWave + lane;
                if (d < kDim) {
                    keys[d] = kv[i] * fk;
                    queries[d] = qv[i] * fq;
                }
            }
        __syncthreads();
        const float decay = exp2_fast(kLog2e * (g < -1000.0f ? -1000.0f : g));
        float key[ROWS];
        Float4 a(0.0f), b(0.0f);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int d = i * kGroups + group;
            const float query = queries[d];
            key[i] = keys[d];
            s[i] *= decay;
            a += s[i] * key[i];
            b += s[i] * query;
        }
#pragma unroll
        for (int x = LN; x < kWave; x *= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] += __shfl_xor(a[i], x);
                b[i] += __shfl_xor(b[i], x);
            }
        if (lane < LN) {
            sums[0][wave][lane] = a;
            sums[1][wave][lane] = b;
        }
        __syncthreads();
        a = sums[0][0][col];
        b = sums[1][0][col];
#pragma unroll
        for (int w = 1; w < kWavesPerBlock; ++w) {
            a += sums[0][w][col];
            b += sums[1][w][col];
        }
        float o[4];
        Float4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] = beta * ((float)v[i] - a[i]);
            o[i] = p.scale * __builtin_fmaf(kq * fk * fq, u[i], b[i]);
        }
        if (group == 0 && have > 0)
            store_row_vec<T, 4>(static_cast<T*>(p.out.d) + (long long)r * p.out.row + head * p.out_head + c0, have, rounded<T, 4>(o));
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (i * kGroups + group < p.key_dim) s[i] += key[i] * u;      // (not zero times an infinity where there is no row)
        r = same.next();
        if (r < 0) break;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int d = i * kGroups + group;
        if (d < p.key_dim && have > 0) store_row_vec<float, 4>(state + (long long)d * p.value_dim, have, s[i]);
    }
}

}  // namespace
}  // namespace ssam

extern "C" int ssam_scan_delta_step(const ssam_scan_delta_step_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_delta(*a)) return e;
    if (int e = check_slots(a->rows, a->slots, a->d_slots)) return e;
    if (a->rows == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype);
    const ssam_sequences q{1, a->rows, nullptr, nullptr};
    if (!a->d_state) return SSAM_ERR_NULL;
    if ((uintptr_t)a->d_state % 4) return SSAM_ERR_DIM;
    if (int e = check_delta_rows(*a, q)) return e;
    if (int e = check_out_heads(a->out, q, a->heads, a->out_head, a->value_dim, esz, false)) return e;
    const long long slot = (long long)a->heads * a->key_dim * a->value_dim;
    if (int e = check_pool(a->slots, a->slot_stride, slot)) return e;
    const Cover outs[] = {cover_rows(a->out, q, heads_width(a->heads, a->out_head, a->value_dim), esz),
                          cover_slots(a->d_state, a->slots, a->slot_stride, slot, 4)};
    const Cover ins[] = {cover_rows(a->q, q, heads_width(a->key_heads, a->q_head, a->key_dim), esz),
                         cover_rows(a->k, q, heads_width(a->key_heads, a->k_head, a->key_dim), esz),
                         cover_rows(a->v, q, heads_width(a->heads, a->v_head, a->value_dim), esz), cover_rows(a->g, q, a->heads, 4),
                         cover_rows(a->beta, q, a->heads, 4), cover_plain(a->d_slots, a->rows * 4LL)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    DeltaStepParams p{a->rows, a->slots, a->heads, a->key_heads, a->key_dim, a->value_dim, a->unit != 0, 1, a->scale, a->d_slots, a->q, a->k, a->v, a->out,
                      a->g, a->beta, a->q_head, a->k_head, a->v_head, a->out_head, a->d_state, a->slot_stride};
    const long long many = (long long)a->rows * a->heads;
    // 128 columns a block, 512 contiguous bytes of a row, where that leaves a block a compute unit or more (8 rows of 32 heads of 128 x 128: 10.8 -> 9.7
    // us, 256 rows 224 -> 217), otherwise 32 (4 rows 8.3 -> 6.4 us).
    const bool wide = many * ((a->value_dim + 127) / 128) >= 256 && a->value_dim > 32;
    p.tiles = (a->value_dim + (wide ? 127 : 31)) / (wide ? 128 : 32);
    if (product(many, p.tiles) > kMaxGrid) return SSAM_ERR_DIM;
    return with_delta_type(a->dtype, [&](auto t) {
        return with_key(a->key_dim, [&](auto kt) {
            using T = decltype(t);
            constexpr int KT = decltype(kt)::value;
            const dim3 grid((unsigned)(many * p.tiles)), block(kBlock);
            hipStream_t st = (hipStream_t)hip_stream;
            if (wide) hipLaunchKernelGGL((delta_step<T, 32, 4 * KT>), grid, block, 0, st, p);
            else hipLaunchKernelGGL((delta_step<T, 8, KT>), grid, block, 0, st, p);
            return launched();
        });
    });
}
