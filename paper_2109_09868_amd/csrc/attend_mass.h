// The weights that attention gave, added up per key: mass[j] += sum over rows and heads of exp2(c S - base) / total.
//
// A row's weights need its total, so this comes behind attention, which leaves every row's maximum and total.  For few rows it leaves the
// scores, too: 4 bytes for a key and head next to the 4 Dh and more that the key and its value are, and not read from memory
// again.  For many rows they are formed again, the other way round than there: a wave holds 32 keys as operands in
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
    static constexpr int kWaves = 4;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kOwn = 32;                                      // keys of a wave
    static constexpr int kKeys = kOwn * kWaves;
    static constexpr int kRows = kStride <= 16 ? 64 : 32;               // of a tile
    static constexpr int kLoads = (kRows * kPieces + kThreads - 1) / kThreads;       // pieces of a tile of rows that a thread brings
    static constexpr int kTile = kRows * kStride * 16;
    static constexpr int kAhead = kSteps % 4 == 0 ? 4 : 2;               // operands that are read at a time
};

// blocks: blocks of keys of the longest sequence; heads: workgroups to a block's heads of the cache; parts: at most as many to the tiles of
// each of them, `chunk` to one.
struct MassGrid {
    int64_t blocks;
    int heads, parts, chunk;
    int keys, rows;                                           // of a block, and tokens of a tile
    int64_t stride;                                           // of a sequence's sums in the workspace
    __host__ __device__ __forceinline__ int slices() const { return heads * parts; }
};
// The new tokens of a sequence that see a key of the block at j0, from..to - 1: those from the first key's place on; with a window, as far
// as it reaches from the last one.
struct MassTokens {
    int from, to;
    __device__ __forceinline__ MassTokens(const AttendCall &c, const MassGrid &g, const Rows &rows, int j0) {
        const int before = rows.length - rows.n;              // places of tokens that are not new (negative: rows without a place)
        from = max(max(0, -before), j0 - before);
        to = rows.n;
        if (c.window > 0 && j0 >= c.sinks)
            to = static_cast<int>(min(static_cast<int64_t>(to), static_cast<int64_t>(j0) + g.keys - 1 + c.window - before));
    }
    // tiles of one head; of all heads of a group, one head's after the other's, and the parts that they make
    __device__ __forceinline__ int tiles(const MassGrid &g) const { return to > from ? (to - from + g.rows - 1) / g.rows : 0; }
    __device__ __forceinline__ int parts(const AttendCall &c, const MassGrid &g) const {
        return max((tiles(g) * (c.Hq / c.Hkv) + g.chunk - 1) / g.chunk, 1);
    }
};
constexpr int kMassBlocks = 4096;                             // of sequences and of keys in a launch: more are taken in turn

// What a tile's rows need besides themselves.
struct MassRows {
    float base[128], inverse[128];
    int place[128];
};

// One block of keys of a sequence, for one range of heads and part of the rows.  kAligned: queries are at multiples of 16 bytes, a
// tile's rows within 2^31 elements, and the scale is above 0; rows of whole heads then go straight from memory into LDS.
template <class E, int DP, bool kWhole, bool kAligned>
__device__ __forceinline__ void mass_block(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, int slice, int b, int j0) {
    typedef typename E::Value V;
    typedef MassShape<E, DP> S;
    // two objects, not one of two parts: reads of one do not wait for what is on its way into the other
    __shared__ __align__(16) char tile0[S::kTile], tile1[S::kTile];
    __shared__ __align__(16) MassRows info0, info1;
    constexpr bool kDirect = kWhole && kAligned && S::kStride == S::kPieces && S::kRows * S::kPieces % S::kThreads == 0;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), half = lane >> 5, col = lane & 31;
    const Rows rows = rows_of(c.seq, b);
    if (!rows.ok || rows.n == 0 || rows.n > c.max_rows || rows.length > c.max_len || j0 >= rows.length) return;
    const MassTokens tokens(c, g, rows, j0);
    // heads next to each other: a head keeps its XCD where there are 8 of them, and the parts that there are come before the others
    const int group = c.Hq / c.Hkv, head_part = slice % g.heads, part = slice / g.heads;
    if (part > 0 && part >= tokens.parts(c, g)) return;
    const int h0 = head_part * c.Hkv / g.heads, h1 = (head_part + 1) * c.Hkv / g.heads;
    const int tiles = tokens.tiles(g), begin = part * g.chunk, end = min(begin + g.chunk, tiles * group);

    const int mine = j0 + wave * S::kOwn + col;               // this lane's key
    const int shift = c.seq.page_shift, in_page = (1 << shift) - 1;
    const int page = mine < rows.length ? page_of(c.seq, b, mine) : -1;
    const int64_t at = page < 0 ? 0 : (static_cast<int64_t>(page) * c.Hkv * (in_page + 1) + (mine & in_page)) * c.Dh;
    const float scale = c.scale == 0.0f ? 1.0f : fabsf(c.scale) * 1.44269504088896340736f;
    const unsigned flip = c.scale < 0.0f ? (S::kSize == 4 ? 0x80000000u : 0x80008000u) : 0u;
    const bool whole_pieces = reinterpret_cast<uintptr_t>(c.q) % 16 == 0 && c.q_stride % S::kPerPiece == 0;
    const int Dq = c.scale == 0.0f ? 0 : kWhole ? DP : c.Dh;  // scale 0: scores of 0 at scale 1

    // A thread's pieces of a tile.  LDS takes what goes straight there one lane's 16 bytes behind the other's: each lane asks for the piece
    // that the row's permutation has there.
    const int piece0 = kDirect ? wave * S::kLoads * kWave + lane : static_cast<int>(threadIdx.x);
    constexpr int kPieceStep = kDirect ? kWave : S::kThreads;
    const auto row_of = [&](int n) { return (piece0 + n * kPieceStep) / S::kPieces; };
    const auto column_of = [&](int n) {
        const int piece = (piece0 + n * kPieceStep) % S::kPieces;
        return (kDirect ? piece ^ permuted<S::kStride>(row_of(n)) : piece) * S::kPerPiece;
    };
    float sum = 0.0f;
    for (int h = h0; h < h1 && begin < end; ++h) {
        float of_head = 0.0f;                                 // sums of sums: a rounding step is one of the few that there are at each level
        const V *const keys = static_cast<const V *>(c.k_pool) + at + static_cast<int64_t>(h) * (in_page + 1) * c.Dh;
        v4i k[S::kSteps];
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {
            const int d = (2 * s + half) * S::kPerPiece;
            const bool there = kWhole || d < c.Dh;            // behind the head: zeros
            // (a key behind the sequence, or on no page, is whatever there is: its sum is not kept, or no number)
            k[s] = *reinterpret_cast<const v4i *>(keys + (there ? d : 0));
            if (!kWhole && !there) k[s] = v4i{0, 0, 0, 0};
        }
        v4i q_next[S::kLoads];
        v2f stats_next = {0.0f, 0.0f};                        // not looked at before all else of the tile is on its way
        int place_next = -1;
        const V *const queries = static_cast<const V *>(c.q) + (rows.start + tokens.from) * c.q_stride + static_cast<int64_t>(h) * group * c.Dh;
        int next_head = begin / max(tiles, 1), next_tile = begin - next_head * tiles;      // of what load() brings next
        const auto load = [&](auto second) {
            char *const to = second ? tile1 : tile0;
            const V *const x = queries + next_tile * (S::kRows * c.q_stride) + next_head * c.Dh;
            const int last = tokens.to - tokens.from - 1 - next_tile * S::kRows;           // rows behind it stand where it stands
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                if constexpr (kDirect) {
                    const int at = min(row_of(n), last) * static_cast<int>(c.q_stride) + column_of(n);
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(x + at),
                                                     (__attribute__((address_space(3))) void *)(to + (wave * S::kLoads + n) * kWave * 16), 16, 0, 0);
                } else {
                    q_next[n] = v4i{0, 0, 0, 0};
                    if (row_of(n) < S::kRows && row_of(n) <= last)
                        q_next[n] = query_piece<E>(x + row_of(n) * c.q_stride, column_of(n), Dq, whole_pieces, flip);
                }
            }
            if (threadIdx.x < S::kRows) {
                const int token = tokens.from + next_tile * S::kRows + min(static_cast<int>(threadIdx.x), last);
                stats_next = *reinterpret_cast<const v2f *>(c.stats + 2 * ((h * group + next_head) * c.seq.T + rows.start + token));
                place_next = static_cast<int>(threadIdx.x) <= last ? rows.place(token) : -1;
            }
            if (++next_tile == tiles) {
                next_tile = 0;
                ++next_head;
            }
        };
        const auto put = [&](auto second) {
            char *const to = second ? tile1 : tile0;
            MassRows &info = second ? info1 : info0;
            if constexpr (!kDirect) {
#pragma unroll
                for (int n = 0; n < S::kLoads; ++n) {
                    if (row_of(n) < S::kRows)
                        *reinterpret_cast<v4i *>(to + piece_at<S::kStride>(row_of(n), column_of(n) / S::kPerPiece)) = q_next[n];
                }
            }
            if (threadIdx.x < S::kRows) {
                info.base[threadIdx.x] = stats_next[0];
                info.inverse[threadIdx.x] = stats_next[1];
                info.place[threadIdx.x] = place_next;
            }
            if constexpr (kDirect) __builtin_amdgcn_s_waitcnt(kNoVmem);
        };
        load(std::false_type{});
        put(std::false_type{});
        __syncthreads();
        const auto step = [&](int tile, auto second) {
            typedef std::integral_constant<bool, !decltype(second)::value> Other;
            if (tile + 1 < end) load(Other{});
            const char *const qt = second ? tile1 : tile0;
            const MassRows &info = second ? info1 : info0;
            const int j = j0 + wave * S::kOwn;
#pragma unroll 1
            for (int r0 = 0; r0 < S::kRows; r0 += 32) {       // 32 of its rows
                const int p0 = info.place[r0], p1 = info.place[r0 + 31];         // -1 where rows end within them
                if (p0 < 0 || (p1 >= 0 && p1 < j)) continue;  // there are none, or none sees a key of this wave's
                v16f s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.0f;
                // operands of the next products are on their way while these are formed: left alone, each product waits for its own
                v4i x[2][S::kAhead];
                const auto read = [&](int p0) {
#pragma unroll
                    for (int p = 0; p < S::kAhead; ++p)
                        x[p0 / S::kAhead & 1][p] = *reinterpret_cast<const v4i *>(qt + piece_at<S::kStride>(r0 + col, 2 * (p0 + p) + half));
                };
                read(0);
#pragma unroll
                for (int p0 = 0; p0 < S::kSteps; p0 += S::kAhead) {
                    if (p0 + S::kAhead < S::kSteps) read(p0 + S::kAhead);
#pragma unroll
                    for (int p = 0; p < S::kAhead; ++p) s = multiply<E>(x[p0 / S::kAhead & 1][p], k[p0 + p], s);
                }
                float of_rows = 0.0f;
                const bool whole = j + S::kOwn - 1 <= p0 && p1 >= 0 && (c.window == 0 || j > p1 - c.window || j + S::kOwn <= c.sinks);
                const auto add = [&](auto masked) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const int r = r0 + 2 * e + 4 * half;  // rows r .. r + 3
                        const v4f base = *reinterpret_cast<const v4f *>(info.base + r), inverse = *reinterpret_cast<const v4f *>(info.inverse + r);
                        v4i place = {0, 0, 0, 0};
                        if constexpr (masked) place = *reinterpret_cast<const v4i *>(info.place + r);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float score = s[e + i], share = inverse[i];
                            if constexpr (masked) {           // a row that is no number must not reach what it does not see either
                                const bool sees = mine <= place[i] && (c.window == 0 || mine > place[i] - c.window || mine < c.sinks);
                                score = sees ? score : -INFINITY;
                                share = sees ? share : 0.0f;
                            }
                            of_rows = fmaf(__builtin_amdgcn_exp2f(fmaf(score, scale, -base[i])), share, of_rows);
                        }
                    }
                };
                if (whole) add(std::false_type{});
                else add(std::true_type{});
                of_head += of_rows;
            }
            if (tile + 1 < end) put(Other{});
            __syncthreads();
        };
        for (int tile = begin; tile < end; tile += 2) {
            step(tile, std::false_type{});
            if (tile + 1 < end) step(tile + 1, std::true_type{});
        }
        sum += of_head;
    }
    sum = half_sum(sum);
    if (half != 0 || mine >= rows.length) return;
    if (g.slices() == 1) mass[b * mass_stride + mine] += sum;
    else sums[(static_cast<int64_t>(slice) * c.seq.B + b) * g.stride + mine] = sum;
}

// Waits for the matrix cores and for the vector units by turns: a score takes one product and then a shift, a power and a sum.  Two prompts of
// up to 4001 tokens (32 heads of 128 on 8, bf16) 177 to 189 us by card, 555 to 520 TFLOP/s of the scores that are seen, of the call's 383; matrix
// cores busy 27 %, vector units 52 %.  Registers for three workgroups a CU; two take as long (185).  A wave with 64 keys and
// rows of all heads of a group in a tile took 223.
template <class E, int DP, bool kWhole, bool kAligned>
__global__ __launch_bounds__(256, (MassShape<E, DP>::kSteps > 16 ? 1 : MassShape<E, DP>::kSteps > 8 ? 2 : 3)) void attend_mass_kernel(
    AttendCall c, MassGrid g, float *mass, int64_t mass_stride, float *sums) {
    typedef MassShape<E, DP> S;
    for (int64_t block = blockIdx.z; block < g.blocks; block += gridDim.z)
        for (int b = blockIdx.y; b < c.seq.B; b += gridDim.y)
            mass_block<E, DP, kWhole, kAligned>(c, g, mass, mass_stride, sums, blockIdx.x, b, static_cast<int>(block * S::kKeys));
}

template <class E, int DP, bool kWhole, bool kAligned>
hipError_t launch_mass(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream) {
    typedef MassShape<E, DP> S;
    if (g.keys != S::kKeys || g.rows != S::kRows) return hipErrorInvalidValue;   // mass_grid() says otherwise than MassShape
    const dim3 grid(g.slices(), c.seq.B < kMassBlocks ? c.seq.B : kMassBlocks,
                    static_cast<unsigned>(g.blocks < kMassBlocks ? g.blocks : kMassBlocks));
    return launch_kernel(attend_mass_kernel<E, DP, kWhole, kAligned>, grid, dim3(S::kThreads), 0, stream, c, g, mass, mass_stride, sums);
}

template <class E>
hipError_t launch_mass_of(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream) {
    const bool aligned = reinterpret_cast<uintptr_t>(c.q) % 16 == 0 && c.q_stride % (16 / sizeof(typename E::Value)) == 0 &&
                         c.q_stride < 1 << 24 && c.scale > 0.0f;
    if (c.Dh == 64 && aligned) return launch_mass<E, 64, true, true>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh == 128 && aligned) return launch_mass<E, 128, true, true>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh == 256 && aligned) return launch_mass<E, 256, true, true>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh <= 64) return launch_mass<E, 64, false, false>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh <= 96) return launch_mass<E, 96, false, false>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh <= 128) return launch_mass<E, 128, false, false>(c, g, mass, mass_stride, sums, stream);
    if (c.Dh <= 192) return launch_mass<E, 192, false, false>(c, g, mass, mass_stride, sums, stream);
    return launch_mass<E, 256, false, false>(c, g, mass, mass_stride, sums, stream);
}

// ---- few rows: from the scores that attention has kept
// attend()'s kernel of few rows, which keeps its scores: 16 sequences of up to 32768 keys (8 heads of 128, bf16) 306 us, of which 255 are the
// keys and values at a copy's rate.
template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (DP > 128 ? 1 : 2)) void attend_scores_kernel(AttendCall c, TokenGrid g, float *workspace) {
    __shared__ __align__(16) char lds[TokenShape<E, DP>::kLds];
    attend_tokens<E, DP, kWhole, kSmall, false, true>(c, g, workspace, SharedCall{}, 0, lds);
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
