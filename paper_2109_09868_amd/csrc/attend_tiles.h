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
// always meet in the workspace.  lds: TileShape::kLds bytes.
template <class E, int DP, bool kWhole, bool kSmall, bool kShared>
__device__ __forceinline__ void attend_tiles(const AttendCall &c, const TileGrid &g, float *workspace, const SharedCall &shared, int64_t group_index,
                                             char *lds) {
    typedef typename E::Value V;
    typedef TileShape<E, DP> S;
    constexpr bool kDirect = kWhole && !kSmall && S::kStride == S::kPieces;
    constexpr int kKeys = S::kKeys, kBlocks = kKeys / 32, kSteps = S::kPieces / 2, kOut = DP / 32;
    constexpr int kVec = S::kSize == 2 ? 1 : kOut % 4 == 0 ? 4 : kOut % 2 == 0 ? 2 : 1;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), half = lane >> 5, row32 = lane & 31;
    const int group = c.Hq / c.Hkv;
    int part, index = 0, h, b;
    int64_t tile = 0;
    SharedUnit unit;
    if constexpr (kShared) {
        unit = shared_unit(c, shared, group_index, S::kRows);
        if (unit.rows == 0) return;
        part = unit.part;
        h = unit.h;
        b = unit.b;
        tile = unit.block;
    } else {
        const int64_t heads = g.slots * c.Hkv, work = heads * g.parts;
        if (blockIdx.x >= work) {                             // the last workgroups: statuses, a wave for each
            const int64_t b = (blockIdx.x - work) * S::kWaves + wave;
            if (b >= c.seq.B) return;
            const int st = attend_status(c, static_cast<int>(b));
            if (lane == 0) c.status[b] = st;
            return;
        }
        part = static_cast<int>(blockIdx.x / heads);
        index = static_cast<int>(blockIdx.x % heads);
        h = index % c.Hkv;
        const int64_t slot = g.slots - 1 - index / c.Hkv;
        b = g.single ? static_cast<int>(slot) : slot_owner(c.seq, slot, group, S::kRows, &tile);
    }
    Rows rows;
    if constexpr (!kShared) rows = rows_of(c.seq, b);
    const int64_t row_count = kShared ? unit.rows : static_cast<int64_t>(rows.n) * group, first = tile * S::kRows;
    if (!kShared && (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || tile < 0 || first >= row_count)) return;

    // this lane's row; lanes behind the last row repeat it
    const int64_t row = min(first + wave * 32 + row32, row_count - 1);
    const int token = static_cast<int>(row / group), head = h * group + static_cast<int>(row % group);
    const int64_t start = kShared ? unit.start : rows.start;
    int place, p0, p1, w0, w1;                                // places: this row's, and the least and largest of the tile and of the wave
    if constexpr (kShared) {
        place = shared_place(c, unit, start + token);
        unit.find_leader(c);
        b = unit.b;
        unit.places_of(place, S::kWaves, reinterpret_cast<int *>(lds), &p0, &p1, &w0, &w1);
    } else {
        place = rows.place(token);
        p0 = rows.place(static_cast<int>(first / group));
        p1 = rows.place(static_cast<int>(min(first + S::kRows - 1, row_count - 1) / group));
        w0 = __builtin_amdgcn_readfirstlane(place);
        w1 = __builtin_amdgcn_readlane(place, 31);
    }
    const int end = kShared ? unit.end : 0x7fffffff, low = kShared ? unit.low : 0;         // of the keys that there are here
    const int near = kShared ? min(place, end - 1) : place;   // the last that this row sees of them

    v4i q[kSteps];
    {
        const V *x = static_cast<const V *>(c.q) + (start + token) * c.q_stride + static_cast<int64_t>(head) * c.Dh;
        const bool whole = reinterpret_cast<uintptr_t>(c.q) % 16 == 0 && c.q_stride % S::kPerPiece == 0;
        const unsigned flip = c.scale < 0.0f ? (S::kSize == 4 ? 0x80000000u : 0x80008000u) : 0u;
        const int Dh = c.scale == 0.0f ? 0 : kWhole ? DP : c.Dh;  // scale 0: scores of 0 at scale 1
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = query_piece<E>(x, (2 * s + half) * S::kPerPiece, Dh, whole, flip);
    }
    const float scale = c.scale == 0.0f ? 1.0f : fabsf(c.scale) * 1.44269504088896340736f;

    const KeyTiles<kKeys, kShared> keys(c.window, c.sinks, p0, p1, low, end);
    const int chunk = kShared ? unit.chunk_of<kKeys>(keys.steps) : g.chunk_of<kKeys>(keys.steps);
    const int begin = part * chunk, steps = min(keys.steps, begin + chunk);       // this part's tiles: begin .. steps - 1
    if (!kShared && begin >= steps && part > 0) return;
    const bool alone = !kShared && keys.steps <= chunk;
    const auto begin_of = [&](int it) { return keys.begin_of(it); };
    const int32_t *table = c.seq.table + static_cast<int64_t>(b) * c.seq.M;
    const int shift = c.seq.page_shift, in_page = (1 << shift) - 1;
    const auto page_at = [&](int it) {                        // of key `lane` of the tile
        return table[keys.seen(begin_of(min(it, steps - 1)) + (lane & (kKeys - 1))) >> shift];
    };
    const V *const k_pool = static_cast<const V *>(c.k_pool), *const v_pool = static_cast<const V *>(c.v_pool);

    v4i k_next[S::kLoads], v_next[S::kLoads];
    unsigned long long bad_next = 0, bad = 0;
    int page_next = begin < steps ? page_at(begin) : 0;
    const int Dh = kWhole ? DP : c.Dh;
    const auto load = [&](int it) {                           // this wave's keys of tile `it` into registers
        const bool off = page_next < 0 || page_next >= c.seq.P;
        bad_next = __ballot(off);
        const int page = off ? 0 : page_next, j0 = begin_of(it) + wave * S::kOwn;
        const auto piece = [&](const V *x, int at) {
            v4i y = *reinterpret_cast<const v4i *>(x + (kWhole || at < Dh ? at : 0));
            if (!kWhole && at >= Dh) y = v4i{0, 0, 0, 0};     // values behind the head
            return y;
        };
        if constexpr (!kSmall) {                         // one page: the address is the wave's, plus a constant of the lane's
            const int p = __builtin_amdgcn_readlane(page, wave * S::kOwn);
            const int64_t base = ((static_cast<int64_t>(p) * c.Hkv + h) * (in_page + 1) + (j0 & in_page)) * Dh;
            const V *const k = k_pool + base, *const v = v_pool + base;
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * kWave + lane, key = index / S::kPieces, at = index % S::kPieces * S::kPerPiece;
                k_next[n] = piece(k + key * Dh, at);
                v_next[n] = piece(v + key * Dh, at);
            }
        } else {
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * kWave + lane, key = index / S::kPieces, at = index % S::kPieces * S::kPerPiece;
                const int p = __shfl(page, wave * S::kOwn + key);
                const int64_t base = ((static_cast<int64_t>(p) * c.Hkv + h) * (in_page + 1) + ((j0 + key) & in_page)) * Dh;
                k_next[n] = piece(k_pool + base, at);
                v_next[n] = piece(v_pool + base, at);
            }
        }
        page_next = page_at(it + 1);
    };
    // The same straight into LDS, without a register: LDS takes the lanes' 16 bytes one behind the other, so each lane asks for the piece that
    // the row's permutation has there.
    const auto fetch = [&](int it) {
        char *const kt = lds + (it & 1) * 2 * S::kBytes, *const vt = kt + S::kBytes;
        const bool off = page_next < 0 || page_next >= c.seq.P;
        bad_next = __ballot(off);
        const int page = off ? 0 : page_next, j0 = begin_of(it) + wave * S::kOwn;
        const int p = __builtin_amdgcn_readlane(page, wave * S::kOwn);
        const int64_t base = ((static_cast<int64_t>(p) * c.Hkv + h) * (in_page + 1) + (j0 & in_page)) * Dh;
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            const int index = n * kWave + lane, key = index / S::kStride;
            const int at = key * Dh + ((index % S::kStride) ^ permuted<S::kStride>(wave * S::kOwn + key)) * S::kPerPiece;
            const int to = wave * S::kOwn * S::kStride * 16 + n * kWave * 16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(k_pool + base + at),
                                             (__attribute__((address_space(3))) void *)(kt + to), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(v_pool + base + at),
                                             (__attribute__((address_space(3))) void *)(vt + to), 16, 0, 0);
        }
        page_next = page_at(it + 1);
    };
    const auto whole_tile = [&](int j0, int a, int b) {       // every row from place a to place b sees every key
        if (kShared && (j0 < low || j0 + kKeys > end)) return false;
        return j0 + kKeys - 1 <= a && (c.window == 0 || j0 > b - c.window || j0 + kKeys <= c.sinks);
    };
    const auto put = [&](int it) {                            // from the registers into LDS
        char *const kt = lds + (it & 1) * 2 * S::kBytes, *const vt = kt + S::kBytes;
        if (!whole_tile(begin_of(it), p0, p1)) {              // seen by nobody: whatever the page holds there
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int j = begin_of(it) + wave * S::kOwn + (n * kWave + lane) / S::kPieces;
                if (keys.seen(j) != j) v_next[n] = v4i{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int n = 0; n < S::kLoads; ++n) {
            const int index = n * kWave + lane, key = wave * S::kOwn + index / S::kPieces, piece = index % S::kPieces;
            *reinterpret_cast<v4i *>(kt + S::at(key, piece)) = k_next[n];
            *reinterpret_cast<v4i *>(vt + S::at(key, piece)) = v_next[n];
        }
        bad = bad_next;
    };
    const auto settle = [&](int it) {                         // what fetch() brings is there, and cleared as put() does
        __builtin_amdgcn_s_waitcnt(kNoVmem);
        if (!whole_tile(begin_of(it), p0, p1)) {
            char *const vt = lds + (it & 1) * 2 * S::kBytes + S::kBytes + wave * S::kOwn * S::kStride * 16;
#pragma unroll
            for (int n = 0; n < S::kLoads; ++n) {
                const int index = n * kWave + lane, j = begin_of(it) + wave * S::kOwn + index / S::kStride;
                v4i *const at = reinterpret_cast<v4i *>(vt + index * 16);
                if (keys.seen(j) != j) *at = v4i{0, 0, 0, 0};
            }
        }
        bad = bad_next;
    };

    v16f out[kOut];
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int k = 0; k < 16; ++k) out[n][k] = 0.0f;
    float top = -INFINITY, total = 0.0f;

    if (begin < steps) {
        if constexpr (kDirect) {
            fetch(begin);
            settle(begin);
        } else {
            load(begin);
            put(begin);
        }
    }
    __syncthreads();
    for (int it = begin; it < steps; ++it) {
        const int j0 = begin_of(it);
        const unsigned long long bad_now = bad;
        if (it + 1 < steps) {
            if constexpr (kDirect) fetch(it + 1);
            else load(it + 1);
        }
        const char *const kt = lds + (it & 1) * 2 * S::kBytes, *const vt = kt + S::kBytes;
        const bool none = j0 > (kShared ? min(w1, end - 1) : w1) || (c.window > 0 && j0 + kKeys - 1 <= w0 - c.window && j0 >= c.sinks);
        if (!none) {
            v16f s[kBlocks];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
                for (int k = 0; k < 16; ++k) s[b][k] = 0.0f;
#pragma unroll
                for (int n = 0; n < kSteps; ++n)
                    s[b] = multiply<E>(*reinterpret_cast<const v4i *>(kt + S::at(b * 32 + row32, 2 * n + half)), q[n], s[b]);
            }
            // the products one behind the other with kAhead operands on their way: left alone, each waits for its own read
            __builtin_amdgcn_sched_group_barrier(kDsRead, S::kAhead, 0);
#pragma unroll
            for (int n = 0; n < kBlocks * kSteps - S::kAhead; ++n) {
                __builtin_amdgcn_sched_group_barrier(kMfma, S::kSize == 4 ? 4 : 1, 0);
                __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kMfma, S::kAhead * (S::kSize == 4 ? 4 : 1), 0);
            // what is hidden from a row: keys behind it, keys before its window; and keys of bad pages are no numbers.  Few tiles need any
            // of it, and hardly one needs all.
            const int reach = near - j0 - 4 * half;
            if (bad_now != 0) {
                const unsigned long long off = bad_now >> (4 * half);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (off >> (b * 32 + 8 * (k / 4) + k % 4) & 1) s[b][k] = NAN;
            }
            if (kShared && j0 < low) {
                const int ahead = low - j0 - 4 * half;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) s[b][k] = b * 32 + 8 * (k / 4) + k % 4 >= ahead ? s[b][k] : -INFINITY;
            }
            if (j0 + kKeys - 1 > (kShared ? min(w0, end - 1) : w0)) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) s[b][k] = b * 32 + 8 * (k / 4) + k % 4 <= reach ? s[b][k] : -INFINITY;
            }
            if (c.window != 0 && j0 <= w1 - c.window && j0 + kKeys > c.sinks) {
                const int start = c.sinks - j0 - 4 * half, back = (kShared ? place - j0 - 4 * half : reach) - c.window;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int key = b * 32 + 8 * (k / 4) + k % 4;
                        s[b][k] = key > back || key < start ? s[b][k] : -INFINITY;
                    }
            }
            float most = s[0][0];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 16; ++k) most = fmaxf(most, s[b][k]);
            most = fmaxf(half_max(most), top);
            // the maximum moves only where it has grown by a factor of 256 in the weights: they stay below that, and within their types
            if (__any((most - top) * scale > 8.0f)) {
                const float f = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((top - most) * scale);
                total *= f;
#pragma unroll
                for (int n = 0; n < kOut; ++n)
#pragma unroll
                    for (int k = 0; k < 16; ++k) out[n][k] *= f;
                top = most;
            }
            const float base = top == -INFINITY ? 0.0f : top * scale - kLift<E>;
            float sum = 0.0f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    s[b][k] = __builtin_amdgcn_exp2f(fmaf(s[b][k], scale, -base));
                    sum += s[b][k];
                }
            total += sum;
            if constexpr (S::kSize == 2) {
                // weights in one piece of their type, at 2.1e-3 (bf16) and 2.7e-4 (fp16) of the outputs' norm from 64 bits; in two pieces, as the
                // few-rows kernel has them, 1.6e-3 and 2.0e-4, as the result's own rounding, but the two prompts of bf16 take 884 us
                // instead of 671 and the window of fp16 265 instead of 198
                const int i = lane & 15, quad = lane >> 4 & 1;
#pragma unroll
                for (int n = 0; n < kKeys / 16; ++n) {
                    float w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = s[n / 2][8 * (n % 2) + k];
                    const v4i p = rounded8<E>(w);
#pragma unroll
                    for (int o = 0; o < kOut; ++o) {
                        v4s x[2];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int key = 16 * n + 8 * u + 4 * half + (i >> 2);
                            const char *a = vt + S::at(key, 4 * o + 2 * quad + (i >> 1 & 1)) + (i & 1) * 8;
                            x[u] = load_transposed(a);
                        }
                        const v8s y = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
                        out[o] = multiply<E>(__builtin_bit_cast(v4i, y), p, out[o]);
                    }
                }
                // as above, with the weights of the next 16 keys between the products of these
                __builtin_amdgcn_sched_group_barrier(kDsRead, 6, 0);
#pragma unroll
                for (int n = 0; n < kKeys / 16 * kOut; ++n) {
                    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
                }
            } else {
                // a lane reads kVec neighbouring values of a key at once: they are its operands of kVec products, whose rows are every
                // kVec-th dimension
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int key = b * 32 + 8 * (k / 4) + 4 * half + k % 4;
#pragma unroll
                        for (int o = 0; o < kOut; o += kVec) {
                            typedef float VV __attribute__((ext_vector_type(kVec)));
                            const int at = 32 * o + kVec * row32;
                            const VV x = *reinterpret_cast<const VV *>(vt + S::at(key, at >> 2) + (at & 3) * 4);
#pragma unroll
                            for (int e = 0; e < kVec; ++e)
                                out[o + e] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], s[b][k], out[o + e], 0, 0, 0);
                        }
                    }
            }
        }
        if (it + 1 < steps) {
            if constexpr (kDirect) settle(it + 1);
            else put(it + 1);
        }
        __syncthreads();
    }

    float *const partial = kShared ? nullptr : workspace + (index * static_cast<int64_t>(g.parts) + part) * part_floats(S::kRows, c.Dh);
    total = half_sum(total);
    if (!kShared && c.stats != nullptr && alone && half == 0 && first + wave * 32 + row32 < row_count)
        RowStats(top == -INFINITY ? top : top * scale - kLift<E>, total).store(c, start + token, head);
    // A weight of 0 (hidden, or rounded to it) times an infinity is NaN, and so is all that a hidden NaN touches: the product cannot hide it.
    // Rows with such sums are computed again, element by element; those whose weights are no numbers are NaN as they have to be.  (A prompt of 2048
    // tokens, 8 heads of 128 on 2, bf16: 0.08 to 0.1 ms, with an infinity that all rows see too; with a NaN in their place, where all rows are
    // computed again, 8.6 ms.)
    bool odd = false;
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int k = 0; k < 16; ++k) odd |= out[o][k] != out[o][k];
    const unsigned long long odd_lanes = __ballot(odd && total == total);
    const unsigned odd_rows = static_cast<unsigned>(odd_lanes | odd_lanes >> 32);
    if (first + wave * 32 + row32 < row_count && (odd_rows >> row32 & 1) == 0) {
        const float inverse = !alone ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
        const int n = wave * 32 + row32;
        const int64_t at = (start + token) * c.Hq + head;
        float *sums = kShared ? shared.sums(c, unit.sum_part, at) : partial + n * c.Dh;
        if (!alone && half == 0) {
            const float most = top == -INFINITY ? top : top * scale - kLift<E>;
            if constexpr (kShared) {
                shared.settle(c, unit.sum_part, at, most, total);
            } else {
                partial[S::kRows * c.Dh + n] = most;
                partial[S::kRows * c.Dh + S::kRows + n] = total;
            }
        }
        V *y = static_cast<V *>(c.out) + at * c.Dh;
#pragma unroll
        for (int o = 0; o < kOut; o += kVec)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < kVec; ++j) {              // values 4 j ..+3 of the 4 kVec that lie next to each other
                    const int d = 32 * o + kVec * (8 * k + 4 * half) + 4 * j;
                    const auto value = [&](int n) { return out[o + (4 * j + n) % kVec][4 * k + (4 * j + n) / kVec] * inverse; };
                    if (!kWhole && d >= c.Dh) continue;
                    if (alone) store4<E>(y + d, value(0), value(1), value(2), value(3));
                    else *reinterpret_cast<v4f *>(sums + d) = v4f{value(0), value(1), value(2), value(3)};
                }
    }
    float *const scratch = reinterpret_cast<float *>(lds) + wave * APPROXIFER_MAX_HEAD_DIM;      // the tiles are done with
    for (unsigned left = odd_rows; left != 0; left &= left - 1) {
        const int n = wave * 32 + __builtin_ctz(left);
        if (first + n >= row_count) continue;
        if constexpr (kShared) shared_part<E>(c, shared, unit, first + n, scratch, keys, begin, steps);
        else attend_part<E>(c, rows, first + n, h, scratch, keys, begin, steps, alone, partial, S::kRows, n);
    }
}

template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (TileShape<E, DP>::kGroups)) void attend_tiles_kernel(AttendCall c, TileGrid g, float *workspace) {
    __shared__ __align__(16) char lds[TileShape<E, DP>::kLds];
    attend_tiles<E, DP, kWhole, kSmall, false>(c, g, workspace, SharedCall{}, 0, lds);
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
