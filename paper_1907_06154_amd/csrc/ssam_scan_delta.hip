// The scan with matrix states along time (ssam_scan_delta): what the blocks' rows have to do with one another (delta_prepare, one launch over
// all blocks), then the states from block to block and the outputs (delta_walk).
// bf16, heads of 128 x 128: 1 x 4096 rows of 32 heads take 38 + 223 us, 8 x 4096 242 + 568 (653 both, once the clock has settled).  A walk is bound by one wave's
// chain, 3.5 us for 64 rows: five matrix products in line, some 130 matrix instructions (2100 of 7700 cycles), and between them the columns' largest values and the splits into
// pairs of fp16.  The bytes would take 21 and 160 us.  Waves without columns do nothing: 1 to 16 values beyond 64 cost no LDS reads of three
// more waves (heads of 96 x 80, 8191 packed rows of 6: 93 -> 71 us).
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
// are in LDS, the same for the block's four waves; the next block's are on their way in registers.
template <class T, int KT, int NT>
__global__ __launch_bounds__((kWalkThreads<T, KT>)) void delta_walk(DeltaParams p)
{
    constexpr bool kHelp = kHelped<T, KT>;
    __shared__ WalkRoom<T, KT> rooms[kHelp ? 2 : 1];
    typedef Stage<T, KT, false> S;
    typedef Columns<T, NT, kSplit<T> && (KT > 4)> Cols;
    __shared__ typename Cols::Room columns[kWavesPerBlock];
    constexpr int kParts = kSplit<T> ? 2 : 1;       // of q and k
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6, g = lane >> 4, r16 = lane & 15;
    const unsigned block = near_block();
    const int tile = (int)(block % p.tiles), head = (int)(block / p.tiles % p.heads), seq = (int)(block / p.tiles / p.heads);
    const int key_head = head / (p.heads / p.key_heads);
    int first, len;
    span_of(p.pieces, seq, first, len);
    const int blocks = (len + kDeltaRows - 1) / kDeltaRows;
    const long long slot0 = p.pieces.begin ? first_slot(p.pieces, seq) : (long long)seq * p.pieces.per;
    const int col0 = (tile * kWavesPerBlock + __builtin_amdgcn_readfirstlane(wave)) * 16 * NT, c0 = col0 + r16;      // the lane's first column
    const Piece whole{seq, first, len, 0, len};
    const StageFrom<T> source{p.blocks + slot0 * p.heads + head, sequence_base<const T>(p.k, p.pieces, whole) + key_head * p.k_head,
                              sequence_base<const T>(p.q, p.pieces, whole) + key_head * p.q_head, p.k.row, p.q.row, p.heads, len, p.key_dim};
    if (kHelp && wave >= kWavesPerBlock) {
        if (blocks > 0) stage_all<S>(source, rooms, 0, 1, blocks);
        return;
    }
    if (kHelp && col0 >= p.value_dim) {        // no columns: the barriers alone, as many as stage_all has
        if (blocks > 0)
            for (int c = 0; c <= blocks; ++c) __syncthreads();
        return;
    }
    const T* vs = sequence_base<const T>(p.v, p.pieces, whole) + head * p.v_head;
    T* os = sequence_base<T>(p.out, p.pieces, whole) + head * p.out_head;
    const long long state_at = ((long long)seq * p.heads + head) * p.key_dim * p.value_dim;
    const unsigned vstride = (unsigned)p.v.row, ostride = (unsigned)p.out.row;

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
    int rows = len < kDeltaRows ? len : kDeltaRows;
    if (blocks > 0) {
        if (!kHelp) source.load(stage, 0);
        v.load(vs, vstride, rows, col0, p.value_dim);
        if (kHelp) __syncthreads();
    }
    for (int c = 0; c < blocks; ++c) {
        WalkRoom<T, KT>& room = rooms[kHelp ? c & 1 : 0];
        if (!kHelp) {
            __syncthreads();
            source.put(stage, room, c);
        }
        float* const mark = p.marks ? mark_of(p.marks, p, slot0 + c, head) : nullptr;
        if (mark) store_state<KT, NT>(mark, p.value_dim, p.key_dim, c0, s);
        Float4 x[4][NT], o[4][NT];
        v.values(columns[wave], rows, x);
        if (!kHelp) __syncthreads();
        const int this_rows = rows;
        if (c + 1 < blocks) {
            vs += (long long)kDeltaRows * p.v.row;
            rows = len - (c + 1) * kDeltaRows;
            rows = rows < kDeltaRows ? rows : kDeltaRows;
            if (!kHelp) source.load(stage, c + 1);
            v.load(vs, vstride, rows, col0, p.value_dim);
        }

        // X = V - exp(G) K S and Q S
        float back_s[NT];
        {
            HalfPair f[KT][NT];
            Half8 key[2][kParts][KT], query[2][kParts][KT];
            read_rows<KT, kParts>(room.keys, 0, lane, key[0]);
            read_rows<KT, kParts>(S::kOnePlace ? room.keys : room.queries(), S::kOnePlace ? 1 : 0, lane, query[0]);
            split_state<KT, NT>(s, f, back_s);
            if constexpr (S::kOnePlace) {
                products<KT, NT, kParts>(key[0], query[0], f, o[0], o[1]);
                read_rows<KT, kParts>(room.keys, 2, lane, key[0]);
                read_rows<KT, kParts>(room.keys, 3, lane, query[0]);
                products<KT, NT, kParts>(key[0], query[0], f, o[2], o[3]);
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                Float4 a[NT];
                if constexpr (S::kOnePlace) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) a[n] = o[m][n];
                } else {
                    if (m < 3) {
                        read_rows<KT, kParts>(room.keys, m + 1, lane, key[(m + 1) & 1]);
                        read_rows<KT, kParts>(room.queries(), m + 1, lane, query[(m + 1) & 1]);
                    }
                    in_order();
                    products<KT, NT, kParts>(key[m & 1], query[m & 1], f, a, o[m]);
                }
                const Float4 reads = *reinterpret_cast<const Float4*>(&room.m.f.reads[tile_row(m, 4 * g)]);
#pragma unroll
                for (int n = 0; n < NT; ++n) x[m][n] -= reads * (a[n] * back_s[n]);
            }
            if constexpr (S::kOnePlace) {
                __syncthreads();
                source.template put_queries<S>(room, c);
                __syncthreads();
#pragma unroll
                for (int m = 0; m < 4; m += 2) {
                    read_rows<KT, kParts>(room.queries(), m, lane, key[0]);
                    read_rows<KT, kParts>(room.queries(), m + 1, lane, query[0]);
                    products<KT, NT, kParts>(key[0], query[0], f, o[m], o[m + 1]);
                }
            }
        }
        // R = (I + A diag(b))^-1 X;  x becomes U = b R
        float back_u[NT];
        HalfPair f[2][NT];
        split_rows<NT>(x, f, back_u);
        tri_products<NT, false>(room.m.solve, lane, f, x);
        if (mark) {
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) x[m][n] *= back_u[n] * room.m.f.solve_back;
            store_tiles<NT>(mark + (size_t)p.key_dim * p.value_dim, p.value_dim, c0, x);
#pragma unroll
            for (int n = 0; n < NT; ++n) back_u[n] = 1.0f;
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) back_u[n] *= room.m.f.solve_back;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const Float4 beta = *reinterpret_cast<const Float4*>(&room.m.f.beta[tile_row(m, 4 * g)]);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[m][n] *= beta * back_u[n];
        }
        // O = scale (exp(G) Q S + (Q K^T o D) U)
        split_rows<NT>(x, f, back_u);
        {
            Float4 a[4][NT];
            tri_products<NT, false>(room.m.mix, lane, f, a);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const Float4 asks = *reinterpret_cast<const Float4*>(&room.m.f.asks[tile_row(m, 4 * g)]);
                const Float4 writes = *reinterpret_cast<const Float4*>(&room.m.f.writes[tile_row(m, 4 * g)]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    a[m][n] = a[m][n] * (back_u[n] * room.m.f.mix_back) + asks * (o[m][n] * back_s[n]);
                    x[m][n] *= writes;
                }
            }
            Cols::store(columns[wave], os, ostride, this_rows, col0, p.value_dim, a);
        }
        os += (long long)kDeltaRows * p.out.row;
        // S = exp(G_C) S + (exp(G_C - G) K)^T U
        {
            Half8 key[2][2][kParts][2];
            read_turned<KT, kParts>(room.turned_keys, 0, lane, key[0][0]);
            read_turned<KT, kParts>(room.turned_keys, 1, lane, key[0][1]);
            split_rows<NT>(x, f, back_u);
            const float total = room.m.f.total;
#pragma unroll
            for (int j = 0; j < 2 * KT; j += 2) {
                const int now = j >> 1 & 1;
                if (j + 2 < 2 * KT) {
                    read_turned<KT, kParts>(room.turned_keys, j + 2, lane, key[now ^ 1][0]);
                    read_turned<KT, kParts>(room.turned_keys, j + 3, lane, key[now ^ 1][1]);
                }
                in_order();
                Float4 a[2][NT];
                products<2, NT, kParts>(key[now][0], key[now][1], f, a[0], a[1]);
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[j + k][n][i] = __builtin_fmaf(total, s[j + k][n][i], a[k][n][i] * back_u[n]);
            }
        }
        if (kHelp) __syncthreads();
    }
    if (p.final) store_state<KT, NT>(p.final + state_at, p.value_dim, p.key_dim, c0, s);
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

    const WalkPlan plan = walk_plan(*a);
    const DeltaParams p{make_pieces(a->seq, kDeltaRows), a->q, a->k, a->v, a->out, a->g, a->beta, a->q_head, a->k_head, a->v_head, a->out_head, a->d_state,
                  a->d_final, a->d_marks, static_cast<Block*>(a->d_work), a->heads, a->key_heads, a->key_dim, a->value_dim, a->unit != 0, a->scale, plan.tiles};
    const long long heads = (long long)a->seq.sequences * a->heads;
    if (product(slots, a->key_heads) > max_grid(kBlock)) return SSAM_ERR_DIM;
    hipStream_t st = (hipStream_t)hip_stream;
    return with_delta_type(a->dtype, [&](auto t) {
        return with_key(a->key_dim, [&](auto kt) {
            using T = decltype(t);
            constexpr int KT = decltype(kt)::value;
            if (product(heads, p.tiles) > max_grid(kWalkThreads<T, KT>)) return (int)SSAM_ERR_DIM;
            hipLaunchKernelGGL((delta_prepare<T, KT>), dim3((unsigned)(slots * a->key_heads)), dim3(kBlock), 0, st, p);
            if (int e = launched()) return e;
            const dim3 walks((unsigned)(heads * p.tiles));
            if constexpr (kSplit<T> && KT <= 4)
                if (plan.wide) {
                    hipLaunchKernelGGL((delta_walk<T, KT, 2>), walks, dim3(kWalkThreads<T, KT>), 0, st, p);
                    return launched();
                }
            hipLaunchKernelGGL((delta_walk<T, KT, 1>), walks, dim3(kWalkThreads<T, KT>), 0, st, p);
            return launched();
        });
    });
}

}  // extern "C"
