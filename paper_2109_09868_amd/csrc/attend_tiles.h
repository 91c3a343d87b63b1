// Attention of many rows: tiles of rows against tiles of keys on the matrix cores.
//
// The rows of a sequence and one head of the cache are packed, token by token and within a token head by head of the group that shares
// the cache's head, so that a group needs its keys and values once whatever its size.  A workgroup has kWaves x 32 such rows and
// walks over the tiles of keys that any of them sees: the first tokens' and the window's.  Per tile a wave forms
//   S^T = K Q^T   [keys x 32 rows],  P = exp2(c S - c top),  O^T += V^T P^T   [Dh x 32 rows]
// with its running maximum `top` and sum per row.  Scores come transposed so that a row's scores sit in one lane and the one 32
// lanes away: a maximum is 31 local steps and one exchange; and so that a lane's scores are, after rounding, the operand of
// the second product as they stand: which 8 of 16 keys a lane holds only has to be the same for V, whose operand is read from LDS
// with the transposing load, 4 keys at a time.
//
// Keys and values go through LDS, the next tile's on their way while this one is computed: straight there where heads and pages are whole
// (else by registers), two tiles of each and one barrier a tile.  Rows of LDS are permuted in pieces of 16 bytes so that both kinds of reads spread over all banks.
//
// Bound by the matrix cores and the vector units, one after the other, at the clock that power leaves: two prompts of 4099 and 7001 tokens (32 heads of
// 128 on 8, bf16) 636 to 704 us by card, 981 to 886 TFLOP/s; 12001 tokens of 24 heads of 64 in a window of 2048 (fp16) 193 to 209 us, 715 to 661
// TFLOP/s; 192 texts of 128 tokens, 12 heads of 64 in 32 bits, 100 to 103 us, 48 TFLOP/s and 3.0 TB/s: their four waves have 1, 2, 3 and 4 tiles
// and meet after each, and wait for their first loads.
#pragma once

#include "attend_shared.h"

namespace approxifer {


// slots: tiles of rows of all sequences (single: one for each); parts: workgroups that share a tile's keys, `chunk` tiles of 64 each or
// as many more as it takes.
constexpr int kTileRows = 128;
struct TileGrid {
    int64_t slots;
    int parts, chunk;
    bool single;
    template <int kKeys>
    __device__ __forceinline__ int chunk_of(int steps) const {
        return parts == 1 ? 0x7fffffff : max(chunk * (64 / kKeys), (steps + parts - 1) / parts);
    }
};

template <class E, int DP>
struct TileShape {
    static constexpr int kSize = sizeof(typename E::Value);
    static constexpr int kPerPiece = 16 / kSize;              // elements of 16 bytes
    static constexpr int kPieces = DP * kSize / 16;           // of a row
    static constexpr int kStride = pow2_at_least(kPieces);    // pieces between rows in LDS
    // 32 keys a tile where 64 take too much LDS or too many registers, and for short 32-bit heads, where three workgroups share a CU so
    // (192 sequences of 128 tokens, 12 heads of 64: 110 us when this was chosen, 125 with 64 keys and two workgroups)
    static constexpr bool kShort = kSize == 4 && DP == 64;
    static constexpr int kKeys = kStride * 16 > 512 || DP > 128 || kShort ? 32 : 64;
    static constexpr int kWaves = 4;
    static constexpr int kRows = 32 * kWaves;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kOwn = kKeys / kWaves;               // keys of a tile that a wave loads
    static constexpr int kLoads = kOwn * kPieces / kWave;     // pieces per lane and operand
    static constexpr int kBytes = kKeys * kStride * 16;       // of one operand's tile
    static constexpr int kLds = 4 * kBytes;
    static constexpr int kAhead = 6;                          // operands in flight
    static constexpr int kGroups = kShort ? 3 : kLds <= 80 * 1024 && DP <= 128 ? 2 : 1; // workgroups that share a CU
    static_assert(kOwn * kPieces % kWave == 0, "whole pieces per lane");
    static __device__ __forceinline__ int at(int row, int piece) { return piece_at<kStride>(row, piece); }
};

// Tiles of rows are numbered over all sequences: sequence b begins at tile starts[b] group / rows + b, which leaves each room for its
// own and at most one that is empty.  (Tiles of every sequence up to the longest would leave most workgroups of a ragged batch empty;
// that costs more than their launches: workgroups go to the parts of an XCD in turn, whether they are empty or not, and where every
// second one was, half the CUs stood still.)  Returns the sequence of tile `slot` and its tile there.
__device__ __forceinline__ int slot_owner(const Sequences &s, int64_t slot, int group, int rows, int64_t *tile) {
    const auto begin_of = [&](int b) { return static_cast<int64_t>(s.starts[b]) * group / rows + b; };
    int lo = 0, span = s.B;
    while (span > 1) {                                        // 64 sequences at a time
        const int step = (span + kWave - 1) / kWave, k = lane_id() * step;
        const unsigned long long before = __ballot(k < span && begin_of(lo + k) <= slot);
        const int last = before != 0 ? (63 - __clzll(before)) * step : 0;
        span = min(step, span - last);
        lo += last;
    }
    *tile = slot - begin_of(lo);
    return lo;
}

// kWhole: Dh is DP.  kSmall: pages of fewer tokens than a wave loads of a tile.  kShared: rows are those of a group of sequences, or of one,
// and keys the ones that the group has in common, or the others; workgroup `group_index` of that call has them, g is not used, and sums
// always meet in the workspace.  lds: TileShape::kLds bytes at least, as an array: as a pointer it cost scratch memory in instances of 32 bits.
template <class E, int DP, bool kWhole, bool kSmall, int kLds>
__device__ __forceinline__ void attend_tiles_shared(const AttendCall &c, const SharedCall &shared, int64_t group_index, char (&lds)[kLds]) {
    constexpr bool kShared = true;
    const TileGrid g{};
    float *const workspace = nullptr;
#include "attend_tiles_body.h"
}

template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (TileShape<E, DP>::kGroups)) void attend_tiles_kernel(AttendCall c, TileGrid g, float *workspace) {
    constexpr bool kShared = false;
    const SharedCall shared{};
    const int64_t group_index = 0;
    __shared__ __align__(16) char lds[TileShape<E, DP>::kLds];
#include "attend_tiles_body.h"
}

template <class E, int DP, int kWaves>
__global__ __launch_bounds__(256) void attend_join_tiles_kernel(AttendCall c, TileGrid g, const float *workspace) {
    typedef TileShape<E, DP> S;
    const int group = c.Hq / c.Hkv;
    const int64_t at = kWaves == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + wave_id() : blockIdx.x;
    const int n = static_cast<int>(at % S::kRows);
    const int64_t index = at / S::kRows;
    if (index >= g.slots * c.Hkv) return;
    const int h = static_cast<int>(index % c.Hkv);
    const int64_t slot = g.slots - 1 - index / c.Hkv;
    int64_t tile = 0;
    const int b = g.single ? static_cast<int>(slot) : slot_owner(c.seq, slot, group, S::kRows, &tile);
    const Rows rows = rows_of(c.seq, b);
    const int64_t row_count = static_cast<int64_t>(rows.n) * group, first = tile * S::kRows;
    if (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || tile < 0 || first + n >= row_count) return;
    const int p0 = rows.place(static_cast<int>(first / group));
    const int p1 = rows.place(static_cast<int>(min(first + S::kRows - 1, row_count - 1) / group));
    const KeyTiles<S::kKeys> keys(c.window, c.sinks, p0, p1);
    const int chunk = g.chunk_of<S::kKeys>(keys.steps);
    if (keys.steps <= chunk) return;                          // written already
    join_row<E, DP, kWaves>(c, rows, first + n, h, workspace + index * g.parts * part_floats(S::kRows, c.Dh), S::kRows, n,
                            (keys.steps + chunk - 1) / chunk);
}

template <class E, int DP, bool kWhole, bool kSmall>
hipError_t launch_tiles(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream) {
    typedef TileShape<E, DP> S;
    static_assert(S::kRows == kTileRows, "rows of a tile");
    // late rows see most: their tiles come first.  A head of the cache keeps its XCD where there are 8 of them.
    const int64_t heads = g.slots * c.Hkv;
    const int64_t blocks = heads * g.parts + (c.status != nullptr ? (c.seq.B + S::kWaves - 1) / S::kWaves : 0);
    hipError_t e = launch_kernel(attend_tiles_kernel<E, DP, kWhole, kSmall>, dim3(static_cast<unsigned>(blocks)), dim3(S::kThreads), 0,
                                 stream, c, g, workspace);
    if (e == hipSuccess && g.parts > 1) {
        // four waves for a row of many parts, as far as they are there: rows many 77 us with one and 87 with four (128 tokens of 32 heads, 20000
        // keys), rows few 36 and 25 (8 tokens of 8 heads, 60000 keys)
        const bool many = g.parts > 8 && c.seq.T * c.Hq <= 1024;
        const int64_t all = heads * S::kRows;
        e = launch_kernel(many ? attend_join_tiles_kernel<E, DP, 4> : attend_join_tiles_kernel<E, DP, 1>,
                          dim3(static_cast<unsigned>(many ? all : (all + 3) / 4)), dim3(256), 0, stream, c, g,
                          static_cast<const float *>(workspace));
    }
    return e;
}

template <class E, bool kSmall>
hipError_t launch_tiles_of(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream) {
    if (c.Dh == 64) return launch_tiles<E, 64, true, kSmall>(c, g, workspace, stream);
    if (c.Dh == 128) return launch_tiles<E, 128, true, kSmall>(c, g, workspace, stream);
    if (c.Dh == 256) return launch_tiles<E, 256, true, kSmall>(c, g, workspace, stream);
    if (c.Dh < 64) return launch_tiles<E, 64, false, kSmall>(c, g, workspace, stream);
    if (c.Dh <= 96) return launch_tiles<E, 96, false, kSmall>(c, g, workspace, stream);
    if (c.Dh < 128) return launch_tiles<E, 128, false, kSmall>(c, g, workspace, stream);
    if (c.Dh <= 192) return launch_tiles<E, 192, false, kSmall>(c, g, workspace, stream);
    return launch_tiles<E, 256, false, kSmall>(c, g, workspace, stream);
}
template <class E>
hipError_t launch_tiles_of(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream) {
    return c.seq.page_shift >= 4 ? launch_tiles_of<E, false>(c, g, workspace, stream) : launch_tiles_of<E, true>(c, g, workspace, stream);
}

hipError_t launch_tiles_f32(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_tiles_f16(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_tiles_bf16(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream);

}  // namespace approxifer
