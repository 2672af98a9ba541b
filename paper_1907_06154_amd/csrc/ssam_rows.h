// What the sequence operators share: rows of channels in 32 or 16 bits, how a wave finds its piece of a sequence,
// and the host's checks of tensors of rows.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/ssam_sequence.h"
#include "ssam_device.h"

namespace ssam {

// V adjacent channels of a row, as they are in memory.
template <class T, int V> using RowVec = T __attribute__((ext_vector_type(V)));

// Channels p[0 .. have): zeros behind them.  A whole vector is one access at the element's alignment (global memory takes
// unaligned vectors on this target), so rows of any stride keep 16 bytes per lane.
// (`part`: that `have` may be less, where the caller knows it does not.)
template <class T, int V>
__device__ __forceinline__ RowVec<T, V> load_row_vec(const T* __restrict__ p, int have, bool part = true)
{
    static_assert(sizeof(RowVec<T, V>) == V * sizeof(T), "a vector type of another number of elements is longer than they are");
    RowVec<T, V> v;
    if (!part || have >= V) {
        __builtin_memcpy(&v, p, sizeof(v));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < have ? p[i] : T(0);
    }
    return v;
}

// (kStream: a result larger than the caches, not read again soon.)
template <class T, int V, bool kStream = false>
__device__ __forceinline__ void store_row_vec(T* __restrict__ p, int have, const RowVec<T, V>& v, bool part = true)
{
    if (!part || have >= V) {
        if constexpr (kStream) {
            typedef RowVec<T, V> Loose __attribute__((aligned(sizeof(T))));
            __builtin_nontemporal_store(v, reinterpret_cast<Loose*>(p));
        } else {
            __builtin_memcpy(p, &v, sizeof(v));
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < have) p[i] = v[i];
    }
}

// fp32 to T: one rounding, to nearest even.
template <class T, int V>
__device__ __forceinline__ RowVec<T, V> rounded(const float (&x)[V])
{
    RowVec<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)x[i];
    return v;
}

constexpr float kLog2e = 1.44269504088896340736f;

// 2^x by the hardware instruction (1 ulp; results below 2^-126 become 0, which only ever scales a sum).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 1 / (1 + exp(-x)): exact limits 0 and 1, NaN kept.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp2_fast(-kLog2e * x)); }
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }

// log(1 + exp(x)) = max(x, 0) + log1p(e) with e = exp(-|x|) in (0, 1].  t = 1 + e loses the low bits of a small e, and the time
// steps of a trained layer are 0.001 .. 0.1, that is e of the same size; e - (t - 1), which is exact, puts them back (log(t) changes
// by that over t, and where it matters t is 1).  e is as far off as its rounded exponent makes it, 1.3 |x| u, and exp2's 2 u; the hardware's
// log2 is within 2 u of its value near 1 too: (6 + 1.3 |x|) u in all, 15 u at a time step of 0.001.
__device__ __forceinline__ float softplus(float x)
{
    const float e = exp2_fast(-kLog2e * __builtin_fabsf(x));
    const float t = 1.0f + e;
    return __builtin_fmaxf(x, 0.0f) + __builtin_fmaf(0.693147180559945f, __builtin_amdgcn_logf(t), e - (t - 1.0f));   // NaN comes through e
}

// ---- sequences ---------------------------------------------------------------------------------------------------------
// Work along time is dealt out in slots of `piece` rows.  Batch forms: slot = s * per + c for piece c of sequence s.  Packed
// form: slot = begin / piece + s + c, which needs no prefix sum over the sequences: s's pieces end before
// end / piece + s + 1, where those of s + 1 begin.
struct Pieces {
    const int* begin;   // packed form, or null
    const int* end;     // packed form, or the lengths of a padded batch, or null
    int sequences, rows, piece;
    int per;            // batch forms: slots of a sequence
};

struct Piece {
    int seq;            // -1: nothing in this slot
    int first;          // packed form: the sequence's first row; otherwise 0
    int len;            // rows of the sequence
    int row0, n;        // the piece: rows row0 .. row0 + n - 1 of the sequence
};

inline long long piece_slots(const ssam_sequences& q, int piece)
{
    if (q.sequences <= 0) return 0;
    if (q.d_begin) return (long long)q.rows / piece + q.sequences;
    const long long per = ((long long)q.rows + piece - 1) / piece;
    return (per > 0 ? per : 1) * q.sequences;
}

inline Pieces make_pieces(const ssam_sequences& q, int piece)
{
    const long long per = ((long long)q.rows + piece - 1) / piece;
    return Pieces{q.d_begin, q.d_end, q.sequences, q.rows, piece, (int)(per > 0 ? per : 1)};
}

__device__ __forceinline__ int held(int v, int hi) { return v < 0 ? 0 : v > hi ? hi : v; }

// First slot of sequence s (packed form).
__device__ __forceinline__ int first_slot(const Pieces& q, int s) { return held(q.begin[s], q.rows) / q.piece + s; }

__device__ __forceinline__ void span_of(const Pieces& q, int s, int& first, int& len)
{
    first = q.begin ? held(q.begin[s], q.rows) : 0;
    const int end = q.end ? held(q.end[s], q.rows) : q.rows;
    len = end > first ? end - first : 0;
}

// The piece of a slot; all 64 lanes call it together with the same slot.  The packed form looks for the last sequence whose
// first slot is not behind this one, 64 candidates at a time; the last round's lanes hold its rows too, so that up to 64 sequences
// take one wait for memory.
__device__ __forceinline__ Piece find_piece(const Pieces& q, int slot)
{
    Piece p{-1, 0, 0, 0, 0};
    int s = 0, c = 0, first = 0, len = 0;
    if (q.begin) {
        const int lane = threadIdx.x & (kWave - 1);
        int n = q.sequences;
        while (true) {
            const int step = (n + kWave - 1) / kWave;
            const int i = lane * step;
            int begin = 0, end = 0;
            if (i < n) {
                begin = q.begin[s + i];
                if (step == 1) end = q.end[s + i];
            }
            begin = held(begin, q.rows);
            end = held(end, q.rows);
            const int hits = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < n && begin / q.piece + s + i <= slot));
            if (hits == 0) return p;
            const int skip = (hits - 1) * step;
            s += skip;
            if (step == 1) {
                first = __builtin_amdgcn_readlane(begin, skip);
                const int behind = __builtin_amdgcn_readlane(end, skip);
                len = behind > first ? behind - first : 0;
                break;
            }
            n = n - skip < step ? n - skip : step;
        }
        s = __builtin_amdgcn_readfirstlane(s);
        c = slot - (first / q.piece + s);
    } else {
        s = slot / q.per;
        c = slot - s * q.per;
        span_of(q, s, first, len);
    }
    const long long row0 = (long long)c * q.piece;
    if (c < 0 || (c > 0 && row0 >= len)) return p;
    p.seq = s;
    p.first = first;
    p.len = len;
    p.row0 = (int)row0;
    p.n = len - p.row0 < q.piece ? len - p.row0 : q.piece;
    return p;
}

// Address of a sequence's row 0 (batch forms: by the batch stride; packed: by its first row).
template <class T>
__device__ __forceinline__ T* sequence_base(const ssam_rows& r, const Pieces& q, const Piece& p)
{
    return static_cast<T*>(r.d) + (q.begin ? (long long)p.first * r.row : (long long)p.seq * r.batch);
}

// ---- slots -------------------------------------------------------------------------------------------------------------
// The rows of a call that name one slot, in order.  The first of them leads: its wave takes them all, one behind the other, and
// the waves of the others leave, so that a slot named twice is one sequence that gets two rows and never a race.  Every lane of
// a wave asks with the same row; one round of loads covers 512 rows, and only a slot that is named again costs more.
class SlotRows {
public:
    __device__ __forceinline__ SlotRows(const int* slot_of, int rows, int slots, int row)
        : of_(slot_of), rows_(rows), at_(row + 1), mine_(slot_of ? slot_of[row] : row), again_(false)
    {
        leads_ = mine_ >= 0 && mine_ < slots;
        if (!of_ || !leads_) return;
        const int lane = threadIdx.x & (kWave - 1);
        constexpr int kAtOnce = 8;
        for (int b = 0; b < rows; b += kAtOnce * kWave) {
            bool before = false, behind = false;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int i = b + k * kWave + lane;
                const bool same = i < rows && of_[i] == mine_;
                before |= same && i < row;
                behind |= same && i > row;
            }
            leads_ = leads_ && __builtin_amdgcn_ballot_w64(before) == 0;
            again_ = again_ || __builtin_amdgcn_ballot_w64(behind) != 0;
        }
    }
    __device__ __forceinline__ bool leads() const { return leads_; }
    __device__ __forceinline__ int slot() const { return mine_; }
    // The next row of the slot, -1 behind the last.
    __device__ __forceinline__ int next()
    {
        if (!again_) return -1;
        const int lane = threadIdx.x & (kWave - 1);
        for (; at_ < rows_; at_ += kWave) {
            const unsigned long long m = __builtin_amdgcn_ballot_w64(at_ + lane < rows_ && of_[at_ + lane < rows_ ? at_ + lane : at_] == mine_);
            if (m) {
                const int r = at_ + __builtin_ctzll(m);
                at_ = r + 1;
                return r;
            }
        }
        return -1;
    }

private:
    const int* of_;
    int rows_, at_, mine_;
    bool leads_, again_;
};

// ---- host: checks ------------------------------------------------------------------------------------------------------
inline int type_bytes(int dtype) { return dtype == SSAM_F32 ? 4 : dtype == SSAM_F16 || dtype == SSAM_BF16 ? 2 : 0; }

constexpr long long kMaxChannels = 1 << 24;
constexpr long long kMaxStride = 1LL << 40;      // elements from row to row, sequence to sequence, group to group, slot to slot
constexpr long long kMaxExtent = 1LL << 59;      // elements from a tensor's first to behind its last: offsets and bytes then fit 64 bits
constexpr long long kMaxRows = 1LL << 40;        // of a batch: their products with tiles of channels then fit 64 bits
constexpr long long kMaxTileStride = 1 << 24;    // elements from row to row where a tile's offsets (32 rows of 4 bytes) have 32 bits

// Sums and products of what the caller says, held to 2^62.
inline long long held_to_62(__int128 v) { return v > (1LL << 62) ? 1LL << 62 : (long long)v; }
inline long long product(long long a, long long b) { return held_to_62((__int128)a * b); }
// `count` runs of `width` elements, `step` apart.
inline long long run_extent(long long count, long long step, long long width) { return held_to_62((__int128)(count - 1) * step + width); }
inline long long rows_extent(const ssam_rows& r, const ssam_sequences& q, long long width)
{
    const long long rows = run_extent(q.rows, r.row, width);
    return q.d_begin ? rows : run_extent(q.sequences, r.batch, rows);
}

// What a tensor covers: `count` rows (batch after batch) of `width` bytes, `step` bytes apart; one = a plain range.
struct Cover {
    uintptr_t at;
    long long bytes;         // from the first to behind the last
    long long step, width;   // step 0: not a comb of rows, the whole range counts
};

inline Cover cover_plain(const void* p, long long bytes) { return Cover{(uintptr_t)p, p ? bytes : 0, 0, 0}; }

inline Cover cover_rows(const ssam_rows& r, const ssam_sequences& q, long long width_elems, int esz)
{
    if (!r.d || q.sequences <= 0 || q.rows <= 0) return Cover{(uintptr_t)r.d, 0, 0, 0};
    const long long width = width_elems * esz;
    // All rows lie on one comb, whose step is the shorter of the strides that count, if the longer is a multiple of it: batches of whole
    // sequences and buffers with all sequences' rows in turn alike.
    const bool both = !q.d_begin && q.sequences > 1 && q.rows > 1 && r.row > 0 && r.batch > 0;
    long long step = !q.d_begin && q.sequences > 1 && (q.rows == 1 || r.row == 0) ? r.batch : r.row;
    bool comb = true;
    if (both) {
        step = r.row < r.batch ? r.row : r.batch;
        comb = (r.row < r.batch ? r.batch : r.row) % step == 0;
    }
    comb = comb && step * esz >= width;
    return Cover{(uintptr_t)r.d, rows_extent(r, q, width_elems) * esz, comb ? step * esz : 0, width};
}

inline bool overlaps(const Cover& a, const Cover& b)
{
    if (!a.bytes || !b.bytes) return false;
    if (a.at + (uintptr_t)a.bytes <= b.at || b.at + (uintptr_t)b.bytes <= a.at) return false;
    if (a.step && a.step == b.step) {      // column ranges of one buffer
        const long long off = a.at <= b.at ? (long long)((b.at - a.at) % (uintptr_t)a.step)
                                           : a.step - 1 - (long long)((a.at - b.at - 1) % (uintptr_t)a.step);
        return off < a.width || off + b.width > a.step;
    }
    return true;
}

// 0: fine, otherwise the error.  `width`: elements of a row; `optional`: a NULL tensor is fine.
inline int check_rows(const ssam_rows& r, const ssam_sequences& q, long long width, int esz, bool optional)
{
    const bool empty = q.sequences == 0 || q.rows == 0;
    if (!r.d) return optional || empty ? SSAM_OK : SSAM_ERR_NULL;
    if ((uintptr_t)r.d % esz || r.row < 0 || r.row > kMaxStride || (!q.d_begin && (r.batch < 0 || r.batch > kMaxStride))) return SSAM_ERR_DIM;
    return !empty && rows_extent(r, q, width) > kMaxExtent ? SSAM_ERR_DIM : SSAM_OK;
}

// Rows that are read and written in tiles.
inline int check_tile_rows(const ssam_rows& r, const ssam_sequences& q) { return r.d && q.rows > 1 && r.row > kMaxTileStride ? SSAM_ERR_DIM : SSAM_OK; }

// A result's rows must not share elements with one another either.
inline int check_out_rows(const ssam_rows& r, const ssam_sequences& q, long long width, int esz, bool optional)
{
    if (int e = check_rows(r, q, width, esz, optional)) return e;
    if (!r.d) return SSAM_OK;
    if (q.rows > 1 && r.row < width) return SSAM_ERR_DIM;
    if (!q.d_begin && q.sequences > 1) {
        const bool after = r.batch >= (q.rows > 0 ? (long long)(q.rows - 1) * r.row + width : width);       // sequence behind sequence
        const bool between = r.row >= (long long)(q.sequences - 1) * r.batch + width && r.batch >= width;   // rows of the sequences in turn
        if (!after && !between) return SSAM_ERR_DIM;
    }
    return SSAM_OK;
}

inline int check_sequences(const ssam_sequences& q)
{
    if (q.sequences < 0 || q.rows < 0 || q.rows > SSAM_MAX_EXTENT || q.sequences > SSAM_MAX_EXTENT) return SSAM_ERR_DIM;
    if (!q.d_begin && (long long)q.rows * q.sequences > kMaxRows) return SSAM_ERR_DIM;
    if (q.d_begin && !q.d_end) return SSAM_ERR_NULL;
    if ((uintptr_t)q.d_begin % 4 || (uintptr_t)q.d_end % 4) return SSAM_ERR_DIM;
    return SSAM_OK;
}

inline int check_slots(int rows, int slots, const int* d_slots)
{
    return rows < 0 || rows > SSAM_MAX_EXTENT || slots < 0 || slots > SSAM_MAX_EXTENT || (uintptr_t)d_slots % 4 ? SSAM_ERR_DIM : SSAM_OK;
}
// A pool of slots of `slot` elements, `stride` apart.
inline int check_pool(int slots, long long stride, long long slot)
{
    return stride < slot || stride > kMaxStride || (slots > 0 && run_extent(slots, stride, slot) > kMaxExtent) ? SSAM_ERR_DIM : SSAM_OK;
}

inline Cover cover_slots(const void* p, int slots, long long stride, long long slot, int esz)
{
    return cover_plain(p, slots > 0 && slot > 0 ? run_extent(slots, stride, slot) * esz : 0);
}

template <int NA, int NB>
inline bool any_overlap(const Cover (&outs)[NA], const Cover (&ins)[NB])
{
    for (int i = 0; i < NA; ++i) {
        for (int j = 0; j < NB; ++j)
            if (overlaps(outs[i], ins[j])) return true;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i], outs[j])) return true;
    }
    return false;
}

constexpr long long kMaxGrid = (1LL << 24) - 1;   // blocks of 256 threads: a launch holds fewer than 2^32 threads

inline int launched() { return hipGetLastError() == hipSuccess ? SSAM_OK : SSAM_ERR_HIP; }

}  // namespace ssam
