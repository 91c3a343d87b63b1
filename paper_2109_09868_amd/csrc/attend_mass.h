// The weights that attention gave, added up per key: mass[j] += sum over rows and heads of exp2(c S - base) / total.
//
// A row's weights need its total, so this comes behind attention, which leaves every row's maximum and total.  For few rows it leaves the
// scores, too: 4 bytes for a key and head next to the 4 Dh and more that the key and its value are, and not read from memory
// again.  For many rows they are formed again, the other way round than there: a wave holds 64 keys (32 of long heads) as operands in
// registers and the rows of their sequence come by in tiles through LDS, so that D = Q K^T has a key's scores in one lane and the one 32
// lanes away, and a key's sum is formed where its scores are.  Each workgroup has 4 such waves, a range of the cache's heads, and a
// part of the rows; where there is more than one workgroup to a key, the sums meet in the workspace and are added in order, so that
// results do not depend on who came first.
#pragma once

#include "attend_tokens.h"

namespace approxifer {

template <class E, int DP>
struct MassShape {
    static constexpr int kSize = sizeof(typename E::Value);
    static constexpr int kPerPiece = 16 / kSize;
    static constexpr int kPieces = DP * kSize / 16;
    static constexpr int kStride = pow2_at_least(kPieces);
    static constexpr int kSteps = kPieces / 2;                           // products per block of scores
    static constexpr int kCols = kSteps <= 8 ? 2 : 1;                    // blocks of 32 keys that a wave holds
    static constexpr int kWaves = 4;
    static constexpr int kOwn = 32 * kCols;                              // keys of a wave
    static constexpr int kKeys = kOwn * kWaves;
    static constexpr int kRows = kPieces <= 16 ? 64 : 32;                // of a tile
    static constexpr int kLoads = (kRows * kPieces + 255) / 256;         // pieces of a tile of rows that a thread brings
    static constexpr int kTile = kRows * kStride * 16;
};

// blocks: blocks of keys of the longest sequence; heads, parts: workgroups to a block's heads of the cache, and to its rows.
struct MassGrid {
    int64_t blocks;
    int heads, parts;
    int64_t stride;                                           // of a sequence's sums in the workspace
    __host__ __device__ __forceinline__ int slices() const { return heads * parts; }
};
constexpr int kMassKeys = 256;                                // keys of a block are this or half of it
constexpr int64_t kMassBlocks = 1 << 20;                      // of a launch: more blocks are taken in turn

// What a tile's rows need besides themselves.
struct MassRows {
    float base[64], inverse[64];
    int place[64];
};

// One block of keys of a sequence, for one range of heads and part of the rows.
template <class E, int DP, bool kWhole>
__device__ __forceinline__ void mass_block(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, int64_t index,
                                           char (&tiles)[2][MassShape<E, DP>::kTile], MassRows (&infos)[2]) {
    typedef typename E::Value V;
    typedef MassShape<E, DP> S;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), half = lane >> 5, col = lane & 31;
    const int slices = g.slices(), slice = static_cast<int>(index % slices);
    const int b = static_cast<int>(index / slices % c.seq.B), j0 = static_cast<int>(index / slices / c.seq.B) * S::kKeys;
    const Rows rows = rows_of(c.seq, b);
    if (!rows.ok || rows.n == 0 || rows.n > c.max_rows || rows.length > c.max_len || j0 >= rows.length) return;
    const int group = c.Hq / c.Hkv, head_part = slice / g.parts, part = slice % g.parts;
    const int h0 = static_cast<int>(static_cast<int64_t>(head_part) * c.Hkv / g.heads);
    const int h1 = static_cast<int>(static_cast<int64_t>(head_part + 1) * c.Hkv / g.heads);

    // tokens that see any of these keys: those from the first key's place on; with a window, as far as it reaches from the last one
    const int before = rows.length - rows.n;                  // places of tokens that are not new (negative: rows without a place)
    const int from = max(max(0, -before), j0 - before);
    int to = rows.n;
    if (c.window > 0 && j0 >= c.sinks)
        to = static_cast<int>(min(static_cast<int64_t>(to), static_cast<int64_t>(j0) + S::kKeys - 1 + c.window - before));
    const int first = from * group, count = max(to - from, 0) * group;           // T Hq is at most 2^30
    const int all = (count + S::kRows - 1) / S::kRows;
    const int begin = static_cast<int>(static_cast<int64_t>(all) * part / g.parts), end = static_cast<int>(static_cast<int64_t>(all) * (part + 1) / g.parts);

    const int mine = j0 + wave * S::kOwn + col;               // this lane's keys: this one and, 32 behind it, another
    const int shift = c.seq.page_shift, in_page = (1 << shift) - 1;
    int64_t at[S::kCols];
#pragma unroll
    for (int n = 0; n < S::kCols; ++n) {
        const int j = mine + 32 * n, page = j < rows.length ? page_of(c.seq, b, j) : -1;
        at[n] = page < 0 ? -1 : (static_cast<int64_t>(page) * c.Hkv * (in_page + 1) + (j & in_page)) * c.Dh;
    }
    const float scale = c.scale == 0.0f ? 1.0f : fabsf(c.scale) * 1.44269504088896340736f;
    const unsigned flip = c.scale < 0.0f ? (S::kSize == 4 ? 0x80000000u : 0x80008000u) : 0u;
    const bool whole_pieces = reinterpret_cast<uintptr_t>(c.q) % 16 == 0 && c.q_stride % S::kPerPiece == 0;
    const int Dq = c.scale == 0.0f ? 0 : kWhole ? DP : c.Dh;  // scale 0: scores of 0 at scale 1

    float sum[S::kCols] = {};
    for (int h = h0; h < h1 && begin < end; ++h) {
        float of_head[S::kCols] = {};                         // sums of sums: a rounding step is one of the few that there are at each level
        v4i k[S::kCols][S::kSteps];
#pragma unroll
        for (int n = 0; n < S::kCols; ++n)
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                const int d = (2 * s + half) * S::kPerPiece;
                k[n][s] = v4i{0, 0, 0, 0};                    // behind the head, behind the sequence, or on no page
                if (at[n] >= 0 && (kWhole || d < c.Dh))
                    k[n][s] = *reinterpret_cast<const v4i *>(static_cast<const V *>(c.k_pool) + at[n] +
                                                             static_cast<int64_t>(h) * (in_page + 1) * c.Dh + d);
            }
        v4i q_next[S::kLoads];
        float base_next = 0.0f, inverse_next = 0.0f;
        int place_next = -1;
        const auto load = [&](int tile) {
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * 256 + threadIdx.x;
                const unsigned row = first + tile * S::kRows + index / S::kPieces;
                q_next[n] = v4i{0, 0, 0, 0};
                if (index < S::kRows * S::kPieces && row < static_cast<unsigned>(first + count)) {
                    const unsigned token = row / static_cast<unsigned>(group), g = row - token * group;
                    const V *x = static_cast<const V *>(c.q) + (rows.start + token) * c.q_stride + (h * group + g) * static_cast<int64_t>(c.Dh);
                    q_next[n] = query_piece<E>(x, index % S::kPieces * S::kPerPiece, Dq, whole_pieces, flip);
                }
            }
            if (threadIdx.x < S::kRows) {
                const unsigned row = first + tile * S::kRows + threadIdx.x;
                place_next = -1;
                base_next = inverse_next = 0.0f;
                if (row < static_cast<unsigned>(first + count)) {
                    const unsigned token = row / static_cast<unsigned>(group);
                    const float *x = c.stats + 2 * ((rows.start + token) * c.Hq + h * group + row - token * group);
                    base_next = x[0];
                    inverse_next = x[1];
                    place_next = rows.place(token);
                }
            }
        };
        const auto put = [&](int buffer) {
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * 256 + threadIdx.x;
                if (index < S::kRows * S::kPieces)
                    *reinterpret_cast<v4i *>(tiles[buffer] + piece_at<S::kStride>(index / S::kPieces, index % S::kPieces)) = q_next[n];
            }
            if (threadIdx.x < S::kRows) {
                infos[buffer].base[threadIdx.x] = base_next;
                infos[buffer].inverse[threadIdx.x] = inverse_next;
                infos[buffer].place[threadIdx.x] = place_next;
            }
        };
        load(begin);
        put(0);
        __syncthreads();
        for (int tile = begin; tile < end; ++tile) {
            const int now = (tile - begin) & 1;
            if (tile + 1 < end) load(tile + 1);
            const char *const qt = tiles[now];
            const MassRows &info = infos[now];
#pragma unroll 1
            for (int r0 = 0; r0 < S::kRows; r0 += 32) {       // 32 of its rows
            v16f s[S::kCols];
#pragma unroll
            for (int n = 0; n < S::kCols; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[n][e] = 0.0f;
#pragma unroll
            for (int p = 0; p < S::kSteps; ++p) {
                const v4i x = *reinterpret_cast<const v4i *>(qt + piece_at<S::kStride>(r0 + col, 2 * p + half));
#pragma unroll
                for (int n = 0; n < S::kCols; ++n) s[n] = multiply<E>(x, k[n][p], s[n]);
            }
            const int p0 = info.place[r0], p1 = info.place[r0 + 31];             // -1 where rows end within them
            const int j = j0 + wave * S::kOwn;
            if (p0 < j && p1 >= 0 && p1 < j) continue;        // none sees a key of this wave's
            float of_tile[S::kCols] = {};
            const bool whole = j + S::kOwn - 1 <= p0 && p1 >= 0 && (c.window == 0 || j > p1 - c.window || j + S::kOwn <= c.sinks);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int r = r0 + 2 * e + 4 * half;          // rows r .. r + 3
                const v4f base = *reinterpret_cast<const v4f *>(info.base + r), inverse = *reinterpret_cast<const v4f *>(info.inverse + r);
                const v4i place = *reinterpret_cast<const v4i *>(info.place + r);
#pragma unroll
                for (int n = 0; n < S::kCols; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = __builtin_amdgcn_exp2f(fmaf(s[n][e + i], scale, -base[i]));
                        if (whole) {
                            of_tile[n] = fmaf(w, inverse[i], of_tile[n]);
                        } else {
                            const int key = mine + 32 * n;
                            const bool sees = key <= place[i] && (c.window == 0 || key > place[i] - c.window || key < c.sinks);
                            of_tile[n] += sees ? w * inverse[i] : 0.0f;
                        }
                    }
            }
#pragma unroll
            for (int n = 0; n < S::kCols; ++n) of_head[n] += of_tile[n];
            }
            if (tile + 1 < end) put(now ^ 1);
            __syncthreads();
        }
#pragma unroll
        for (int n = 0; n < S::kCols; ++n) sum[n] += of_head[n];
    }
#pragma unroll
    for (int n = 0; n < S::kCols; ++n) {
        const float x = half_sum(sum[n]);
        const int j = mine + 32 * n;
        if (half != 0 || j >= rows.length) continue;
        if (slices == 1) mass[b * mass_stride + j] += x;
        else sums[(static_cast<int64_t>(slice) * c.seq.B + b) * g.stride + j] = x;
    }
}

template <class E, int DP, bool kWhole>
__global__ __launch_bounds__(256, (MassShape<E, DP>::kSteps > 16 ? 1 : 2)) void attend_mass_kernel(AttendCall c, MassGrid g, float *mass,
                                                                                                  int64_t mass_stride, float *sums) {
    typedef MassShape<E, DP> S;
    __shared__ __align__(16) char tiles[2][S::kTile];
    __shared__ __align__(16) MassRows infos[2];
    const int64_t work = g.blocks * (kMassKeys / S::kKeys) * c.seq.B * g.slices();
    for (int64_t index = blockIdx.x; index < work; index += gridDim.x)
        mass_block<E, DP, kWhole>(c, g, mass, mass_stride, sums, index, tiles, infos);
}

template <class E, int DP, bool kWhole>
hipError_t launch_mass(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream) {
    typedef MassShape<E, DP> S;
    static_assert(S::kKeys == kMassKeys || S::kKeys == kMassKeys / 2, "keys of a block");
    const int64_t blocks = g.blocks * (kMassKeys / S::kKeys) * c.seq.B * g.slices();
    return launch_kernel(attend_mass_kernel<E, DP, kWhole>, dim3(static_cast<unsigned>(blocks < kMassBlocks ? blocks : kMassBlocks)), dim3(256),
                         0, stream, c, g, mass, mass_stride, sums);
}

template <class E>
hipError_t launch_mass_of(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream) {
    if (c.Dh == 64) return launch_mass<E, 64, true>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh == 128) return launch_mass<E, 128, true>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh == 256) return launch_mass<E, 256, true>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh < 64) return launch_mass<E, 64, false>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh <= 96) return launch_mass<E, 96, false>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh < 128) return launch_mass<E, 128, false>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh <= 192) return launch_mass<E, 192, false>(c, g, mass, mass_stride, sums, stream);
    return launch_mass<E, 256, false>(c, g, mass, mass_stride, sums, stream);
}

// ---- few rows: from the scores that attention has kept
template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (DP > 128 ? 1 : 2)) void attend_scores_kernel(AttendCall c, TokenGrid g, float *workspace) {
    attend_tokens<E, DP, kWhole, kSmall, false, true>(c, g, workspace, SharedCall{});
}
template <class E, int DP, bool kWhole, bool kSmall>
hipError_t launch_scores(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    return launch_kernel(attend_scores_kernel<E, DP, kWhole, kSmall>, dim3(static_cast<unsigned>(token_blocks(c, g))), dim3(256), 0, stream, c, g,
                         workspace);
}
template <class E, bool kSmall>
hipError_t launch_scores_of(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    if (c.Dh == 64) return launch_scores<E, 64, true, kSmall>(c, g, workspace, stream);
    if (c.Dh == 128) return launch_scores<E, 128, true, kSmall>(c, g, workspace, stream);
    if (c.Dh == 256) return launch_scores<E, 256, true, kSmall>(c, g, workspace, stream);
    if (c.Dh < 64) return launch_scores<E, 64, false, kSmall>(c, g, workspace, stream);
    if (c.Dh <= 96) return launch_scores<E, 96, false, kSmall>(c, g, workspace, stream);
    if (c.Dh < 128) return launch_scores<E, 128, false, kSmall>(c, g, workspace, stream);
    if (c.Dh <= 192) return launch_scores<E, 192, false, kSmall>(c, g, workspace, stream);
    return launch_scores<E, 256, false, kSmall>(c, g, workspace, stream);
}
template <class E>
hipError_t launch_scores_of(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    return c.seq.page_shift >= 4 ? launch_scores_of<E, false>(c, g, workspace, stream) : launch_scores_of<E, true>(c, g, workspace, stream);
}

hipError_t launch_scores_f32(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_scores_f16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_scores_bf16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_mass_f32(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream);
hipError_t launch_mass_f16(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream);
hipError_t launch_mass_bf16(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream);

}  // namespace approxifer
