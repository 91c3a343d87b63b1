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

#include "attend_join.h"

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
    static_assert(kPieces % 4 == 0 && kKeys * kPieces % kWave == 0, "whole pieces per lane");
};

// parts: workgroups that share a block of rows, each with `chunk` tiles, or as many more as it takes; blocks: blocks of 16 rows of the longest sequence; rows: of those
// 16, as many as there can be.
struct TokenGrid {
    int pairs, blocks, parts, chunk, rows;
    __device__ __forceinline__ int chunk_of(int steps) const { return parts == 1 ? 0x7fffffff : max(chunk, (steps + parts - 1) / parts); }
};

// kWhole: Dh is DP.  kSmall: pages of fewer than 16 tokens.
template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (DP > 128 ? 1 : 2)) void attend_tokens_kernel(AttendCall c, TokenGrid g, float *workspace) {
    typedef typename E::Value V;
    typedef TokenShape<E, DP> S;
    constexpr int kKeys = S::kKeys, kOut = DP / 16;
    __shared__ __align__(16) char lds[S::kWaves * S::kBytes];
    __shared__ float tops[S::kWaves][16], totals[S::kWaves][16];
    __shared__ int dirty;
    const int lane = lane_id(), wave = wave_id(), quarter = lane >> 4, row16 = lane & 15;
    const int64_t units = static_cast<int64_t>(g.pairs) * g.parts, work = units * g.blocks;
    if (blockIdx.x >= work) {                                 // the last workgroups: statuses, a wave for each
        const int64_t b = (blockIdx.x - work) * S::kWaves + wave;
        if (b >= c.seq.B) return;
        const int st = attend_status(c, static_cast<int>(b));
        if (lane == 0) c.status[b] = st;
        return;
    }
    const int unit = static_cast<int>(blockIdx.x % units), block = static_cast<int>(blockIdx.x / units);
    const int pair = unit % g.pairs, part = unit / g.pairs;
    const int h = pair % c.Hkv, group = c.Hq / c.Hkv;
    const Rows rows = rows_of(c.seq, pair / c.Hkv);
    const int64_t row_count = static_cast<int64_t>(rows.n) * group, first = static_cast<int64_t>(block) * S::kRows;
    if (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || first >= row_count) return;

    const int64_t row = min(first + row16, row_count - 1);
    const int token = static_cast<int>(row / group), head = h * group + static_cast<int>(row % group);
    const int place = rows.place(token);
    const int p0 = __builtin_amdgcn_readfirstlane(place), p1 = __builtin_amdgcn_readlane(place, 15);
    const KeyTiles<kKeys> keys(c.window, c.sinks, p0, p1);
    const int chunk = g.chunk_of(keys.steps), begin = part * chunk, end = min(keys.steps, begin + chunk);
    if (begin >= end && part > 0) return;                     // the parts that there are end before this one
    if (threadIdx.x == 0) dirty = 0;

    v4i q[S::kSteps];
    {
        const V *x = static_cast<const V *>(c.q) + (rows.start + token) * c.q_stride + static_cast<int64_t>(head) * c.Dh;
        const bool whole = reinterpret_cast<uintptr_t>(c.q) % 16 == 0 && c.q_stride % S::kPerPiece == 0;
        const unsigned flip = c.scale < 0.0f ? (S::kSize == 4 ? 0x80000000u : 0x80008000u) : 0u;
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) q[s] = query_piece<E>(x, (4 * s + quarter) * S::kPerPiece, c.Dh, whole, flip);
    }
    const float scale = fabsf(c.scale) * 1.44269504088896340736f;
    const int32_t *table = c.seq.table + static_cast<int64_t>(rows.b) * c.seq.M;
    const int shift = c.seq.page_shift, slots = (1 << shift) - 1;
    const V *const k_pool = static_cast<const V *>(c.k_pool), *const v_pool = static_cast<const V *>(c.v_pool);
    char *const vt = lds + wave * S::kBytes;

    const int Dh = kWhole ? DP : c.Dh;
    v4i k_next[S::kBlocks][S::kSteps], v_next[S::kLoads];
    const auto page_at = [&](int it) { return table[keys.seen(keys.begin_of(min(it, end - 1)) + (lane & (kKeys - 1))) >> shift]; };
    int page_next = begin < end ? page_at(begin + wave) : 0, page = 0;
    unsigned long long bad_next = 0;
    // Element `at` of a key of the tile at j0.  Blocks of 16 keys lie in one page unless pages are small: the address is then the wave's
    // plus an offset of the lane's that never changes.  What nobody sees is not used, but it may be read.
    const auto address = [&](const V *pool, int j0, int block, int key, int at) {
        if constexpr (kSmall) {
            const int p = __shfl(page, block * 16 + key);
            return pool + ((static_cast<int64_t>(p) * c.Hkv + h) * (slots + 1) + (keys.seen(j0 + block * 16 + key) & slots)) * Dh + at;
        } else {
            const int p = __builtin_amdgcn_readlane(page, block * 16);
            return pool + ((static_cast<int64_t>(p) * c.Hkv + h) * (slots + 1) + ((j0 + block * 16) & slots)) * Dh + (key * Dh + at);
        }
    };
    // Loads return in order: a tile's pages are asked for before the keys of the tile before it, and its keys before that tile's values are
    // waited for, so that half a tile at least is on its way at any time.
    const auto load_keys = [&](int it) {
        const bool off = page_next < 0 || page_next >= c.seq.P;
        bad_next = __ballot(off);
        page = off ? 0 : page_next;
        page_next = page_at(it + S::kWaves);
        const int j0 = keys.begin_of(it);
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) {
                const int d = (4 * s + quarter) * S::kPerPiece;
                k_next[b][s] = *reinterpret_cast<const v4i *>(address(k_pool, j0, b, row16, kWhole || d < Dh ? d : 0));
            }
    };
    const auto load_values = [&](int it) {
        const int j0 = keys.begin_of(it);
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            const int index = n * kWave + lane, d = index % S::kPieces * S::kPerPiece;
            v_next[n] = *reinterpret_cast<const v4i *>(
                address(v_pool, j0, n * 4 / S::kPieces, index / S::kPieces % 16, kWhole || d < Dh ? d : 0));
        }
    };

    v4f out[kOut];
#pragma unroll
    for (int n = 0; n < kOut; ++n) out[n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float top = -INFINITY, total = 0.0f;
    bool odd = false;
    if (begin + wave < end) {
        load_keys(begin + wave);
        load_values(begin + wave);
    }
    const auto step = [&](int it, auto more) {
        const int j0 = keys.begin_of(it);
        const unsigned long long bad = bad_next;
        const bool whole = j0 + kKeys - 1 <= p0 && (c.window == 0 || j0 > p1 - c.window || j0 + kKeys <= c.sinks);
        v4f s[S::kBlocks];
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b) {
            s[b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int n = 0; n < S::kSteps; ++n) {
                if (!kWhole && (4 * n + quarter) * S::kPerPiece >= Dh) k_next[b][n] = v4i{0, 0, 0, 0};  // behind the head
                s[b] = multiply16<E>(k_next[b][n], q[n], s[b]);
            }
        }
        if constexpr (more) load_keys(it + S::kWaves);
        if (!kSmall && !whole) {                              // seen by nobody: whatever the page holds there
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int j = j0 + (n * kWave + lane) / S::kPieces;
                if (keys.seen(j) != j) v_next[n] = v4i{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            const int index = n * kWave + lane;
            *reinterpret_cast<v4i *>(vt + piece_at<S::kStride>(index / S::kPieces, index % S::kPieces)) = v_next[n];
        }
        if (!whole && p0 != p1) {                             // rows of one place see all that is read
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) odd |= not_finite<E>(v_next[n]);
        }
        if constexpr (more) load_values(it + S::kWaves);
        const bool masked = !whole || bad != 0;
        if (masked) {
            const int reach = place - j0 - 4 * quarter, start = c.sinks - j0 - 4 * quarter;
            const unsigned long long off = bad >> (4 * quarter);
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int key = b * 16 + k;
                    const bool sees = key <= reach && (c.window == 0 || key > reach - c.window || key < start);
                    if (off >> key & 1) s[b][k] = NAN;
                    s[b][k] = sees ? s[b][k] : -INFINITY;
                }
        }
        float most = s[0][0];
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) most = fmaxf(most, s[b][k]);
        most = fmaxf(quarters_max(most), top);
        if (__any((most - top) * scale > 8.0f || (top == -INFINITY && most > -INFINITY))) {
            const float f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((top - most) * scale);
            total *= f;
#pragma unroll
            for (int n = 0; n < kOut; ++n)
#pragma unroll
                for (int k = 0; k < 4; ++k) out[n][k] *= f;
            top = most;
        }
        const float base = top == -INFINITY ? 0.0f : top * scale - kLift<E>;
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float was = s[b][k];
                float w = __builtin_amdgcn_exp2f(fmaf(was, scale, -base));
                if (masked) w = was == -INFINITY ? 0.0f : w;
                s[b][k] = w;
                total += w;
            }
        if constexpr (S::kSize == 2) {
            const float w[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};
            // weights in two 16-bit pieces, what the first leaves in the second: the products wait for memory anyway, and the result is
            // as exact as its own rounding.  (0, or a negative rest, times an infinity is wrong: see below.)
            typedef V V8 __attribute__((ext_vector_type(8)));
            const v4i p = rounded8<E>(w);
            float rest[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) rest[k] = w[k] - E::load(__builtin_bit_cast(V8, p)[k]);
            const v4i p2 = rounded8<E>(rest);
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                v4s x[2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    x[u] = load_transposed(vt + piece_at<S::kStride>(16 * u + 4 * quarter + (row16 >> 2), 2 * o + (row16 >> 1 & 1)) +
                                           (row16 & 1) * 8);
                const v8s y = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
                out[o] = multiply16<E>(__builtin_bit_cast(v4i, y), p, out[o]);
                out[o] = multiply16<E>(__builtin_bit_cast(v4i, y), p2, out[o]);
            }
        } else {
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int o = 0; o < kOut; ++o) {
                        const float x = *reinterpret_cast<const float *>(
                            vt + piece_at<S::kStride>(b * 16 + 4 * quarter + k, 4 * o + (row16 >> 2)) + (row16 & 3) * 4);
                        out[o] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[b][k], out[o], 0, 0, 0);
                    }
        }
    };
    // the last tile on its own: a load that may or may not be on its way would have to be waited for as if it were not
    int it = begin + wave;
    for (; it + S::kWaves < end; it += S::kWaves) step(it, std::true_type{});
    if (it < end) step(it, std::false_type{});

    // infinities among the values: element by element.  (A hidden key's place in the product is taken by one that is seen, with weight 0.)
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int k = 0; k < 4; ++k) odd |= !(fabsf(out[o][k]) <= 3.402823466e38f);

    // the waves meet: one maximum per row, sums relative to it
    total = quarters_sum(total);
    if (quarter == 0) {
        tops[wave][row16] = top;
        totals[wave][row16] = total;
    }
    __syncthreads();
    if (__any(odd) && lane == 0) dirty = 1;
    float all = tops[0][row16];
#pragma unroll
    for (int w = 1; w < S::kWaves; ++w) all = fmaxf(all, tops[w][row16]);
    {
        const float f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((top - all) * scale);
        float *const sums = reinterpret_cast<float *>(vt);
#pragma unroll
        for (int o = 0; o < kOut; ++o)
            *reinterpret_cast<v4f *>(sums + row16 * DP + ((16 * o + 4 * quarter) ^ (row16 & 7) * 4)) =
                v4f{out[o][0] * f, out[o][1] * f, out[o][2] * f, out[o][3] * f};
    }
    __syncthreads();
    const bool alone = keys.steps <= chunk;
    const int64_t slot = (static_cast<int64_t>(pair) * g.blocks + block) * g.parts + part;
    float *const partial = workspace + slot * part_floats(S::kRows, c.Dh);
    if (dirty != 0) {                                         // rows that must not see what the product cannot hide
        __syncthreads();
        float *const scratch = reinterpret_cast<float *>(vt);
        for (int n = wave; n < S::kRows; n += S::kWaves)
            if (first + n < row_count)
                attend_part<E>(c, rows, first + n, h, scratch, keys, begin, end, alone, partial, S::kRows, n);
        return;
    }
    constexpr int kQuads = DP / 4;
    for (int n = threadIdx.x; n < S::kRows * kQuads; n += 256) {
        const int r = n / kQuads, d = n % kQuads * 4;
        if (first + r >= row_count || (DP != c.Dh && d >= c.Dh)) continue;
        float m = tops[0][r];
#pragma unroll
        for (int w = 1; w < S::kWaves; ++w) m = fmaxf(m, tops[w][r]);
        v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
        float l = 0.0f;
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) {
            const v4f x = *reinterpret_cast<const v4f *>(reinterpret_cast<const float *>(lds + w * S::kBytes) + r * DP + (d ^ (r & 7) * 4));
            sum += x;
            l += tops[w][r] == -INFINITY ? totals[w][r] : totals[w][r] * __builtin_amdgcn_exp2f((tops[w][r] - m) * scale);
        }
        if (alone) {
            const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
            const int64_t at = first + r, t = at / group;
            V *const y = static_cast<V *>(c.out) + ((rows.start + t) * c.Hq + h * group + at % group) * c.Dh + d;
            store4<E>(y, sum[0] * inverse, sum[1] * inverse, sum[2] * inverse, sum[3] * inverse);
        } else {
            *reinterpret_cast<v4f *>(partial + r * c.Dh + d) = sum;
            if (d == 0) {
                partial[16 * c.Dh + r] = m == -INFINITY ? m : m * scale - kLift<E>;
                partial[16 * c.Dh + 16 + r] = l;
            }
        }
    }
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

template <class E, int DP, bool kWhole, bool kSmall>
hipError_t launch_tokens(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    typedef TokenShape<E, DP> S;
    const int64_t work = static_cast<int64_t>(g.pairs) * g.parts * g.blocks;
    const int64_t blocks = work + (c.status != nullptr ? (c.seq.B + S::kWaves - 1) / S::kWaves : 0);
    if (blocks == 0) return hipSuccess;                       // max_rows is 0: nothing but statuses is written
    hipError_t e = launch_kernel(attend_tokens_kernel<E, DP, kWhole, kSmall>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, c, g, workspace);
    if (e == hipSuccess && g.parts > 1) {
        const int64_t all = static_cast<int64_t>(g.pairs) * g.blocks * g.rows;
        const bool many = g.parts > 8;
        e = launch_kernel(many ? attend_join_kernel<E, DP, 4> : attend_join_kernel<E, DP, 1>,
                          dim3(static_cast<unsigned>(many ? all : (all + 3) / 4)), dim3(256), 0, stream, c, g,
                          static_cast<const float *>(workspace));
    }
    return e;
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

hipError_t launch_tokens_f32(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_tokens_f16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);
hipError_t launch_tokens_bf16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream);

}  // namespace approxifer
