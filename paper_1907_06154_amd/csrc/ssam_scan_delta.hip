// The scan with matrix states along time (ssam_scan_delta): what the blocks' rows have to do with one another (delta_prepare, one launch over
// all blocks), then the states from block to block and the outputs (delta_walk).
#include "ssam_scan_delta_tiles.h"

namespace ssam {
namespace {

template <class T, int KT>
__global__ __launch_bounds__(kBlock) void delta_prepare(DeltaParams p)
{
    __shared__ PrepareRoom<T, KT> room;
    const int slot = (int)(blockIdx.x / p.key_heads), key_head = (int)(blockIdx.x % p.key_heads);
    const Piece piece = find_piece(p.pieces, slot);
    if (piece.seq < 0 || piece.n <= 0) return;
    prepare_block<T, KT, false>(p, piece, slot, key_head, room);
}

// One wave: 16 NT columns of a head's state, from its sequence's first block to the last.  The operands made from q, k and the block's matrices
// are in LDS, the same for the block's four waves.
template <class T, int KT, int NT>
__global__ __launch_bounds__(kBlock) void delta_walk(DeltaParams p)
{
    __shared__ WalkRoom<T, KT> room;
    constexpr bool kOnePlace = WalkRoom<T, KT>::kOnePlace;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r16 = lane & 15;
    const int tile = (int)(blockIdx.x % p.tiles), head = (int)(blockIdx.x / p.tiles % p.heads), seq = (int)(blockIdx.x / p.tiles / p.heads);
    const int key_head = head / (p.heads / p.key_heads);
    int first, len;
    span_of(p.pieces, seq, first, len);
    const int blocks = (len + kDeltaRows - 1) / kDeltaRows;
    const long long slot0 = p.pieces.begin ? first_slot(p.pieces, seq) : (long long)seq * p.pieces.per;
    const int c0 = (tile * kWavesPerBlock + wave) * 16 * NT + r16;       // the lane's column of the first tile
    const Piece whole{seq, first, len, 0, len};
    const T* const qs = sequence_base<const T>(p.q, p.pieces, whole) + key_head * p.q_head;
    const T* const ks = sequence_base<const T>(p.k, p.pieces, whole) + key_head * p.k_head;
    const T* const vs = sequence_base<const T>(p.v, p.pieces, whole) + head * p.v_head + c0;
    T* const os = sequence_base<T>(p.out, p.pieces, whole) + head * p.out_head + c0;
    const long long state_at = ((long long)seq * p.heads + head) * p.key_dim * p.value_dim + c0;

    Float4 s[2 * KT][NT];
#pragma unroll
    for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = tile_row(j, 4 * g + i);
                s[j][n][i] = p.state && d < p.key_dim && c0 + 16 * n < p.value_dim ? p.state[state_at + (long long)d * p.value_dim + 16 * n] : 0.0f;
            }
    for (int c = 0; c < blocks; ++c) {
        const int row0 = c * kDeltaRows, rows = len - row0 < kDeltaRows ? len - row0 : kDeltaRows;
        const long long slot = slot0 + c;
        __syncthreads();
        const Block& from = p.blocks[slot * p.heads + head];
        stage_rows<T, KT, true, !kOnePlace, false>(room, from.f, ks, p.k.row, qs, p.q.row, row0, rows, p.key_dim);
        stage_block(room.m, from);
        float* const mark = p.marks ? mark_of(p.marks, p, slot, head) + c0 : nullptr;
        if (mark)
#pragma unroll
            for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = tile_row(j, 4 * g + i);
                        if (d < p.key_dim && c0 + 16 * n < p.value_dim) mark[(long long)d * p.value_dim + 16 * n] = s[j][n][i];
                    }
        __syncthreads();

        // X = V - exp(G) K S and Q S
        Float4 x[4][NT], o[4][NT];
        float back_s[NT];
        {
            HalfPair f[KT][NT];
            split_state<KT, NT>(s, f, back_s);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                Float4 a[NT];
                rows_product<KT, NT>(room.keys, m, lane, f, a);
                const int t0 = tile_row(m, 4 * g);
                const Float4 reads = *reinterpret_cast<const Float4*>(&room.m.f.reads[t0]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = t0 + i < rows && c0 + 16 * n < p.value_dim ? (float)vs[(long long)(row0 + t0 + i) * p.v.row + 16 * n] : 0.0f;
                        x[m][n][i] = v - reads[i] * (a[n][i] * back_s[n]);
                    }
            }
            if constexpr (kOnePlace) {
                __syncthreads();
                stage_rows<T, KT, false, true, false>(room, from.f, ks, p.k.row, qs, p.q.row, row0, rows, p.key_dim);
                __syncthreads();
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) rows_product<KT, NT>(room.queries(), m, lane, f, o[m]);
        }
        // R = (I + A diag(b))^-1 X;  x becomes U = b R
        float back_u[NT];
        HalfPair f[2][NT];
        split_rows<NT>(x, f, back_u);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            lower_product<NT>(room.m.solve, m, lane, f, x[m]);
            const int t0 = tile_row(m, 4 * g);
            const Float4 beta = *reinterpret_cast<const Float4*>(&room.m.f.beta[t0]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                x[m][n] *= back_u[n] * room.m.f.solve_back;
                if (mark && c0 + 16 * n < p.value_dim)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mark[(long long)(p.key_dim + t0 + i) * p.value_dim + 16 * n] = x[m][n][i];
                x[m][n] *= beta;
            }
        }
        // O = scale (exp(G) Q S + (Q K^T o D) U)
        split_rows<NT>(x, f, back_u);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            Float4 a[NT];
            lower_product<NT>(room.m.mix, m, lane, f, a);
            const int t0 = tile_row(m, 4 * g);
            const Float4 asks = *reinterpret_cast<const Float4*>(&room.m.f.asks[t0]);
            const Float4 writes = *reinterpret_cast<const Float4*>(&room.m.f.writes[t0]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t0 + i < rows && c0 + 16 * n < p.value_dim)
                        os[(long long)(row0 + t0 + i) * p.out.row + 16 * n] = (T)__builtin_fmaf(a[n][i], back_u[n] * room.m.f.mix_back, asks[i] * (o[m][n][i] * back_s[n]));
                x[m][n] *= writes;
            }
        }
        // S = exp(G_C) S + (exp(G_C - G) K)^T U
        split_rows<NT>(x, f, back_u);
        const float total = room.m.f.total;
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j) {
            Float4 a[NT];
            turned_product<KT, NT>(room.turned_keys, j, lane, f, a);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j][n][i] = __builtin_fmaf(total, s[j][n][i], a[n][i] * back_u[n]);
        }
    }
    if (p.final)
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = tile_row(j, 4 * g + i);
                    if (d < p.key_dim && c0 + 16 * n < p.value_dim) p.final[state_at + (long long)d * p.value_dim + 16 * n] = s[j][n][i];
                }
}

}  // namespace
}  // namespace ssam

extern "C" {

size_t ssam_scan_delta_workspace_bytes(const ssam_scan_delta_args* a)
{
    using namespace ssam;
    if (!a || check_delta(*a) || check_sequences(a->seq) || a->seq.sequences == 0) return 0;
    return (size_t)product(product(piece_slots(a->seq, kDeltaRows), a->heads), sizeof(Block));
}

long long ssam_scan_delta_marks(const ssam_scan_delta_args* a)
{
    using namespace ssam;
    if (!a || check_delta(*a) || check_sequences(a->seq)) return 0;
    return piece_slots(a->seq, kDeltaRows);
}

int ssam_scan_delta(const ssam_scan_delta_args* a, void* hip_stream)
{
    using namespace ssam;
    if (!a) return SSAM_ERR_NULL;
    if (int e = check_delta(*a)) return e;
    if (int e = check_sequences(a->seq)) return e;
    if (a->seq.sequences == 0) return SSAM_OK;
    const int esz = type_bytes(a->dtype);
    if (int e = check_delta_rows(*a, a->seq)) return e;
    if (int e = check_out_heads(a->out, a->seq, a->heads, a->out_head, a->value_dim, esz, false)) return e;
    for (const void* f : {(const void*)a->d_state, (const void*)a->d_final, (const void*)a->d_marks})
        if ((uintptr_t)f % 4) return SSAM_ERR_DIM;
    const size_t bytes = ssam_scan_delta_workspace_bytes(a);
    if (!a->d_work) return SSAM_ERR_NULL;
    if (a->work_bytes < bytes || (uintptr_t)a->d_work % 16) return SSAM_ERR_DIM;
    const long long slots = piece_slots(a->seq, kDeltaRows), plane = (long long)a->heads * a->key_dim * a->value_dim * 4;
    const long long mark_bytes = product(slots, (long long)a->heads * (a->key_dim + kDeltaRows) * a->value_dim * 4);
    if ((long long)bytes > kMaxExtent || (a->d_marks && mark_bytes > 4 * kMaxExtent) || product(a->seq.sequences, plane) > 4 * kMaxExtent) return SSAM_ERR_DIM;
    const Cover state = cover_plain(a->d_state, a->seq.sequences * plane);
    const Cover outs[] = {cover_rows(a->out, a->seq, heads_width(a->heads, a->out_head, a->value_dim), esz), cover_plain(a->d_final, a->seq.sequences * plane),
                          cover_plain(a->d_marks, mark_bytes), cover_plain(a->d_work, (long long)bytes)};
    const Cover ins[] = {cover_rows(a->q, a->seq, heads_width(a->key_heads, a->q_head, a->key_dim), esz),
                         cover_rows(a->k, a->seq, heads_width(a->key_heads, a->k_head, a->key_dim), esz),
                         cover_rows(a->v, a->seq, heads_width(a->heads, a->v_head, a->value_dim), esz), cover_rows(a->g, a->seq, a->heads, 4),
                         cover_rows(a->beta, a->seq, a->heads, 4)};
    if (any_overlap(outs, ins)) return SSAM_ERR_ALIAS;
    for (int i = 0; i < 4; ++i)
        if (overlaps(outs[i], state) && !(i == 1 && a->d_final == a->d_state)) return SSAM_ERR_ALIAS;

    DeltaParams p{make_pieces(a->seq, kDeltaRows), a->q, a->k, a->v, a->out, a->g, a->beta, a->q_head, a->k_head, a->v_head, a->out_head, a->d_state,
                  a->d_final, a->d_marks, static_cast<Block*>(a->d_work), a->heads, a->key_heads, a->key_dim, a->value_dim, a->unit != 0, a->scale, 1};
    const long long heads = (long long)a->seq.sequences * a->heads;
    const bool wide = false;
    p.tiles = (a->value_dim + (wide ? 127 : 63)) / (wide ? 128 : 64);
    if (product(slots, a->key_heads) > kMaxGrid || product(heads, p.tiles) > kMaxGrid) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    return with_delta_type(a->dtype, [&](auto t) {
        return with_key(a->key_dim, [&](auto kt) {
            using T = decltype(t);
            constexpr int KT = decltype(kt)::value;
            hipLaunchKernelGGL((delta_prepare<T, KT>), dim3((unsigned)(slots * a->key_heads)), dim3(kBlock), 0, st, p);
            if (int e = launched()) return e;
            hipLaunchKernelGGL((delta_walk<T, KT, 1>), dim3((unsigned)(heads * p.tiles)), dim3(kBlock), 0, st, p);
            return launched();
        });
    });
}

}  // extern "C"
