// Attention of few rows to long sequences: every key and value is read once, from HBM into registers, by one wave.
//
// Rows of a sequence and one head of the cache are packed as in the tiles kernel, 16 to a workgroup: the group's heads of one token, or of a
// few.  The keys that they see are cut into parts for several workgroups, and a part's tiles go to four waves in turn; waves share
// nothing until they are done, so there is no barrier in the loop.  Per tile of 32 keys a wave forms S^T = K Q^T on the 16 x 16 matrix
// instructions, K straight from memory as the operand wants it; P as it stands is the other product's operand, V takes the way through
// the wave's own piece of LDS for the transposing load (32-bit types: for values of one dimension by 16 lanes).  The next
// tile's keys and values are on their way meanwhile: 16 KB a wave at 128 x 2 bytes, 128 KB a CU.
// Bound by HBM: three sequences of up to 131072 keys (8 heads of 128, bf16) 236 us, 5.8 TB/s; 192 with windows of 1024 (2 heads of 128, fp16) 44 us,
// 4.5 TB/s; 24 of up to 129 keys (12 heads of 64, 32 bits) 11 us, of which the bytes are 3.
#pragma once

#include "attend_shared.h"

namespace approxifer {

template <class E, int DP>
struct TokenShape {
    static constexpr int kSize = sizeof(typename E::Value);
    static constexpr int kPerPiece = 16 / kSize;
    static constexpr int kPieces = DP * kSize / 16;
    static constexpr int kStride = pow2_at_least(kPieces);
    static constexpr int kBlocks = kSize == 2 || DP <= 64 ? 2 : 1;       // of 16 keys
    static constexpr int kKeys = 16 * kBlocks;
    static constexpr int kWaves = 4;
    static constexpr int kRows = 16;
    static constexpr int kSteps = kPieces / 4;                           // products per block of scores
    static constexpr int kLoads = kKeys * kPieces / kWave;               // pieces of V per lane
    static constexpr int kTile = kKeys * kStride * 16;
    static constexpr int kOutBytes = kRows * DP * 4;                     // a wave's sums, when the waves meet
    static constexpr int kBytes = kTile > kOutBytes ? kTile : kOutBytes;
    static constexpr int kLds = kWaves * kBytes;
    static_assert(kPieces % 4 == 0 && kKeys * kPieces % kWave == 0, "whole pieces per lane");
};

// parts: workgroups that share a block of rows, each with `chunk` tiles, or as many more as it takes; blocks: blocks of 16 rows of the longest sequence; rows: of those
// 16, as many as there can be.
struct TokenGrid {
    int pairs, blocks, parts, chunk, rows;
    __device__ __forceinline__ int chunk_of(int steps) const { return parts == 1 ? 0x7fffffff : max(chunk, (steps + parts - 1) / parts); }
};

// kWhole: Dh is DP.  kSmall: pages of fewer than 16 tokens.  kShared: as in attend_tiles_shared().  lds: TokenShape::kLds bytes at least.
// kScores: scores are kept, those of hidden keys as -infinity.
template <class E, int DP, bool kWhole, bool kSmall, bool kShared, bool kScores, int kLds>
__device__ __forceinline__ void attend_tokens(const AttendCall &c, const TokenGrid &g, float *workspace, const SharedCall &shared,
                                              int64_t group_index, char (&lds)[kLds]) {
#include "attend_tokens_body.h"
}

template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (DP > 128 ? 1 : 2)) void attend_tokens_kernel(AttendCall c, TokenGrid g, float *workspace) {
    constexpr bool kShared = false, kScores = false;
    const SharedCall shared{};
    const int64_t group_index = 0;
    __shared__ __align__(16) char lds[TokenShape<E, DP>::kLds];
#include "attend_tokens_body.h"
}

template <class E, int DP, int kWaves>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendCall c, TokenGrid g, const float *workspace) {
    typedef TokenShape<E, DP> S;
    const int group = c.Hq / c.Hkv;
    const int64_t index = kWaves == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + wave_id() : blockIdx.x;
    const int n = static_cast<int>(index % g.rows), block = static_cast<int>(index / g.rows % g.blocks);
    const int64_t pair64 = index / g.rows / g.blocks;
    if (pair64 >= g.pairs) return;
    const int pair = static_cast<int>(pair64);
    const Rows rows = rows_of(c.seq, pair / c.Hkv);
    const int64_t row_count = static_cast<int64_t>(rows.n) * group, first = static_cast<int64_t>(block) * S::kRows;
    if (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || first + n >= row_count) return;
    const int p0 = rows.place(static_cast<int>(first / group));
    const int p1 = rows.place(static_cast<int>(min(first + S::kRows - 1, row_count - 1) / group));
    const KeyTiles<S::kKeys> keys(c.window, c.sinks, p0, p1);
    const int chunk = g.chunk_of(keys.steps);
    if (keys.steps <= chunk) return;                          // written already
    join_row<E, DP, kWaves>(c, rows, first + n, pair % c.Hkv,
                            workspace + (static_cast<int64_t>(pair) * g.blocks + block) * g.parts * part_floats(S::kRows, c.Dh), S::kRows,
                            n, (keys.steps + chunk - 1) / chunk);
}

inline int64_t token_blocks(const AttendCall &c, const TokenGrid &g) {
    return static_cast<int64_t>(g.pairs) * g.parts * g.blocks + (c.status != nullptr ? (c.seq.B + 3) / 4 : 0);
}

template <class E, int DP>
hipError_t join_tokens(const AttendCall &c, const TokenGrid &g, const float *workspace, hipStream_t stream) {
    const int64_t all = static_cast<int64_t>(g.pairs) * g.blocks * g.rows;
    const bool many = g.parts > 8;
    if (g.parts < 2) return hipSuccess;
    return launch_kernel(many ? attend_join_kernel<E, DP, 4> : attend_join_kernel<E, DP, 1>,
                         dim3(static_cast<unsigned>(many ? all : (all + 3) / 4)), dim3(256), 0, stream, c, g, workspace);
}
template <class E>
hipError_t join_tokens_of(const AttendCall &c, const TokenGrid &g, const float *workspace, hipStream_t stream) {
    if (c.Dh <= 64) return join_tokens<E, 64>(c, g, workspace, stream);
    if (c.Dh <= 96) return join_tokens<E, 96>(c, g, workspace, stream);
    if (c.Dh <= 128) return join_tokens<E, 128>(c, g, workspace, stream);
    if (c.Dh <= 192) return join_tokens<E, 192>(c, g, workspace, stream);
    return join_tokens<E, 256>(c, g, workspace, stream);
}

template <class E, int DP, bool kWhole, bool kSmall>
hipError_t launch_tokens(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    const int64_t blocks = token_blocks(c, g);
    if (blocks == 0) return hipSuccess;                       // max_rows is 0: nothing but statuses is written
    const hipError_t e = launch_kernel(attend_tokens_kernel<E, DP, kWhole, kSmall>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, c, g, workspace);
    return e == hipSuccess ? join_tokens<E, DP>(c, g, workspace, stream) : e;
}

template <class E, bool kSmall>
hipError_t launch_tokens_of(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    if (c.Dh == 64) return launch_tokens<E, 64, true, kSmall>(c, g, workspace, stream);
    if (c.Dh == 128) return launch_tokens<E, 128, true, kSmall>(c, g, workspace, stream);
    if (c.Dh == 256) return launch_tokens<E, 256, true, kSmall>(c, g, workspace, stream);
    if (c.Dh < 64) return launch_tokens<E, 64, false, kSmall>(c, g, workspace, stream);
    if (c.Dh <= 96) return launch_tokens<E, 96, false, kSmall>(c, g, workspace, stream);
    if (c.Dh < 128) return launch_tokens<E, 128, false, kSmall>(c, g, workspace, stream);
    if (c.Dh <= 192) return launch_tokens<E, 192, false, kSmall>(c, g, workspace, stream);
    return launch_tokens<E, 256, false, kSmall>(c, g, workspace, stream);
}
template <class E>
hipError_t launch_tokens_of(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    return c.seq.page_shift >= 4 ? launch_tokens_of<E, false>(c, g, workspace, stream) : launch_tokens_of<E, true>(c, g, workspace, stream);
}

hipError_t join_tokens_f32(const AttendCall &c, const TokenGrid &g, const float *workspace, hipStream_t stream);
hipError_t join_tokens_f16(const AttendCall &c, const TokenGrid &g, const float *workspace, hipStream_t stream);
hipError_t join_tokens_bf16(const AttendCall &c, const TokenGrid &g, const float *workspace, hipStream_t stream);
// How the keys of calls of few rows are cut; ragged: for sequences of very different lengths.
bool few_rows(int64_t B, int Hq, int Hkv, int64_t max_rows, int dtype);
TokenGrid token_grid(int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks,
                     size_t workspace_bytes, bool ragged = false);
hipError_t launch_tokens_f32(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_tokens_f16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_tokens_bf16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);

}  // namespace approxifer
