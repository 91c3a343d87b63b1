// Sequences that begin alike: their rows meet the keys that they have in common once, all of them together, and their own keys each for
// itself; what either says of a row meets in the workspace.
//
// For a row with maxima m and totals l of the two (and of the parts that either is cut into), out = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p.
// The tokens of a group's sequences are neighbours in the queries, so that a group's rows are packed as one sequence's are, token by token
// and head by head; only their places have to be looked up.  A part's sums lie as the output does, [part][T][Hq][Dh], and so do its
// maxima and totals: who joins a row need not know which workgroup had it.
#pragma once

#include "attend_join.h"

namespace approxifer {

// C groups: sequences groups[c] .. groups[c + 1] - 1 have the first shared[c] places in common.
// A launch's workgroups: for `common_slots` blocks of the groups' rows, each head of the cache and each of `common_parts` parts of the keys;
// then for `own_slots` blocks of the sequences' rows (single: one of each sequence).  Chunks are keys, at least, of a part.
struct SharedCall {
    const int32_t *groups, *shared;
    int C, max_shared;
    int64_t common_slots, own_slots;
    int common_parts, common_chunk, own_parts, own_chunk;
    bool single;
    float *outs, *tops;                                       // of the parts: common ones first; tops: maximum and total

    __device__ __forceinline__ float *sums(const AttendCall &c, int part, int64_t row) const {
        return outs + (part * (c.seq.T * c.Hq) + row) * c.Dh;
    }
    __device__ __forceinline__ void settle(const AttendCall &c, int part, int64_t row, float top, float total) const {
        *reinterpret_cast<v2f *>(tops + 2 * (part * (c.seq.T * c.Hq) + row)) = v2f{top, total};
    }
};

// Whether there is an instance of the kernel of tiles.  float32 heads of more than 64 floats and up to 128 have none: at 1024 rows it takes 245 us
// for 233.
inline bool shared_tiles(int Dh, int dtype) { return dtype != APPROXIFER_F32 || Dh <= 64 || Dh > 128; }
// Whether there is an instance of both kernels in one: of heads for which two of its workgroups share a CU.
inline bool shared_both(int Dh, int dtype, int page_shift) { return (Dh == 64 || (Dh == 128 && dtype != APPROXIFER_F32)) && page_shift >= 4; }

// The last k of 0..n-1 with at(k) <= x, where at() rises and at(0) <= x; 64 at a time, by the whole wave.
template <class F>
__device__ __forceinline__ int last_at_most(int n, int64_t x, F at) {
    int lo = 0, span = n;
    while (span > 1) {
        const int step = (span + kWave - 1) / kWave, k = lane_id() * step;
        const unsigned long long before = __ballot(k < span && at(lo + k) <= x);
        const int last = before != 0 ? (63 - __clzll(before)) * step : 0;
        span = min(step, span - last);
        lo += last;
    }
    return lo;
}

// A group as the device holds it.  ok: its sequences are some, and their shared length is one that the call allows.
struct SharedGroup {
    int g0, g1, length;
    bool ok;
    __device__ __forceinline__ SharedGroup(const Sequences &s, const SharedCall &shared, int c)
        : SharedGroup(s, shared, shared.groups[c], shared.groups[c + 1], shared.shared[c]) {}
    __device__ __forceinline__ SharedGroup(const Sequences &s, const SharedCall &shared, int a, int b, int l) : g0(a), g1(b), length(l) {
        ok = g0 >= 0 && g0 <= g1 && g1 <= s.B && length >= 0 && length <= shared.max_shared;
    }
};

// The first 64 groups, one to a lane: asked for early, so that a search waits for no load of its own.
struct GroupLanes {
    int g0, g1, length;
    __device__ __forceinline__ explicit GroupLanes(const SharedCall &shared) {
        const int k = min(lane_id(), shared.C - 1);
        g0 = shared.groups[k];
        g1 = shared.groups[k + 1];
        length = shared.shared[k];
    }
};

// How many of sequence b's first places are its group's: 0 without a group that can be used.
__device__ __forceinline__ int shared_length(const Sequences &s, const SharedCall &shared, const GroupLanes &lanes, int b, int *group = nullptr) {
    if (shared.C <= kWave) {
        const unsigned long long in = __ballot(lane_id() < shared.C && lanes.g0 <= b && b < lanes.g1);
        if (in == 0) return 0;
        const int k = __ffsll(in) - 1, length = __builtin_amdgcn_readlane(lanes.length, k);
        if (group != nullptr) *group = k;
        return __builtin_amdgcn_readlane(lanes.g0, k) >= 0 && __builtin_amdgcn_readlane(lanes.g1, k) <= s.B && length >= 0 && length <= shared.max_shared
                   ? length
                   : 0;
    }
    const int c = last_at_most(shared.C, b, [&](int k) { return static_cast<int64_t>(shared.groups[k]); });
    const SharedGroup g(s, shared, c);
    if (group != nullptr) *group = c;
    return b >= g.g0 && b < g.g1 && g.ok ? g.length : 0;
}

// The sequence of a group that its common places are read from, the first that holds them all, or the longest; and how many it holds.
// lens: those of the group's first 64 sequences, one to a lane.
__device__ __forceinline__ int shared_leader(const AttendCall &c, int g0, int g1, int shared_length, int lens, int *length) {
    const int64_t room = static_cast<int64_t>(c.seq.M) << c.seq.page_shift;
    int best = -1, leader = g0;
    for (int i0 = g0; i0 < g1; i0 += kWave) {
        const int i = i0 + lane_id();
        int l = i >= g1 ? -1 : i0 == g0 ? lens : c.seq.lens[i];
        if (l > room || l > c.max_len) l = -1;
        l = min(l, shared_length);
        int most = l;
        for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o));
        if (most > best) {
            best = most;
            leader = i0 + __ffsll(__ballot(l == most)) - 1;
        }
        if (best == shared_length) break;
    }
    *length = max(best, 0);
    return leader;
}
__device__ __forceinline__ int shared_lens(const AttendCall &c, int g0, int g1) { return c.seq.lens[min(g0 + lane_id(), g1 - 1)]; }

// What a workgroup does: rows (tokens times heads) from token `start` on, of which it has block `block`, and keys low..end-1 of sequence b.
struct SharedUnit {
    int64_t start, rows, block;
    int h, b, low, end, part, parts, chunk, sum_part;
    int g0, g1, before;                                       // common: the group's sequences; own: g0 = g1, and the place of the first token
    int64_t tokens;                                           // common: of the group
    int length, lens;                                         // common: the shared length, and lengths of its first sequences by lane

    template <int kKeys>
    __device__ __forceinline__ int chunk_of(int steps) const {
        return parts == 1 ? 0x7fffffff : max(chunk / kKeys, (steps + parts - 1) / parts);
    }
    // of common places: whose pages they are read from, and how many there are.  (Last: places are looked up meanwhile.)
    __device__ __forceinline__ void find_leader(const AttendCall &c) {
        if (g0 != g1) {
            b = __builtin_amdgcn_readfirstlane(shared_leader(c, g0, g1, length, lens, &end));
            end = __builtin_amdgcn_readfirstlane(end);
        }
    }
    // the least and largest place of a wave's 16 rows
    __device__ __forceinline__ void places_of(int place, int *p0, int *p1) const {
        int a = place, b = place;
        for (int o = 8; o > 0; o >>= 1) {
            a = min(a, __shfl_xor(a, o));
            b = max(b, __shfl_xor(b, o));
        }
        *p0 = __builtin_amdgcn_readfirstlane(a);
        *p1 = __builtin_amdgcn_readfirstlane(b);
    }
    // of a workgroup's rows, 32 a wave, and of this wave's; scratch: two numbers of LDS for each wave
    __device__ __forceinline__ void places_of(int place, int waves, int *scratch, int *p0, int *p1, int *w0, int *w1) const {
        int a = place, b = place;
        for (int o = 16; o > 0; o >>= 1) {
            a = min(a, __shfl_xor(a, o));
            b = max(b, __shfl_xor(b, o));
        }
        *w0 = __builtin_amdgcn_readfirstlane(a);
        *w1 = __builtin_amdgcn_readfirstlane(b);
        if (lane_id() == 0) {
            scratch[2 * wave_id()] = a;
            scratch[2 * wave_id() + 1] = b;
        }
        __syncthreads();
        a = scratch[0];
        b = scratch[1];
        for (int w = 1; w < waves; ++w) {
            a = min(a, scratch[2 * w]);
            b = max(b, scratch[2 * w + 1]);
        }
        *p0 = __builtin_amdgcn_readfirstlane(a);
        *p1 = __builtin_amdgcn_readfirstlane(b);
        __syncthreads();
    }
};

__device__ __forceinline__ SharedUnit shared_unit_of(const AttendCall &c, const SharedCall &shared, int64_t x, int R) {
    SharedUnit u{};
    const int group = c.Hq / c.Hkv;
    const GroupLanes lanes(shared);
    const int64_t heads = shared.common_slots * c.Hkv, common = heads * shared.common_parts;
    if (x < common) {
        u.part = u.sum_part = static_cast<int>(x / heads);
        u.parts = shared.common_parts;
        u.chunk = shared.common_chunk;
        const int64_t index = x % heads, slot = index / c.Hkv;
        u.h = static_cast<int>(index % c.Hkv);
        // rows of sequences that are bad may lie anywhere
        const auto row_of = [&](int b) { return min(max(static_cast<int64_t>(c.seq.starts[min(max(b, 0), c.seq.B)]), int64_t{0}), c.seq.T); };
        int g0, g1, length;
        int64_t r0, r1, first;                                // its rows, and the number of its first block
        if (shared.C <= kWave) {
            const int64_t rows0 = row_of(lanes.g0), rows1 = row_of(lanes.g1), begin = rows0 * group / R + min(lane_id(), shared.C - 1);
            const unsigned long long before = __ballot(lane_id() < shared.C && begin <= slot);
            const int k = before != 0 ? 63 - __clzll(before) : 0;
            g0 = __builtin_amdgcn_readlane(lanes.g0, k);
            g1 = __builtin_amdgcn_readlane(lanes.g1, k);
            length = __builtin_amdgcn_readlane(lanes.length, k);
            r0 = __builtin_amdgcn_readlane(static_cast<int>(rows0), k);       // T is at most 2^24
            r1 = __builtin_amdgcn_readlane(static_cast<int>(rows1), k);
            first = r0 * group / R + k;
        } else {
            const auto begin_of = [&](int k) { return row_of(shared.groups[k]) * group / R + k; };
            const int k = last_at_most(shared.C, slot, begin_of);
            g0 = shared.groups[k];
            g1 = shared.groups[k + 1];
            length = shared.shared[k];
            r0 = row_of(g0);
            r1 = row_of(g1);
            first = begin_of(k);
        }
        const SharedGroup g(c.seq, shared, g0, g1, length);
        if (!g.ok || length == 0 || g0 == g1) return u;
        u.block = slot - first;
        if (u.block < 0 || u.block * R >= (r1 - r0) * group) return u;
        u.lens = shared_lens(c, g0, g1);
        u.length = length;
        u.start = r0;
        u.low = 0;
        u.g0 = g0;
        u.g1 = g1;
        u.tokens = r1 - r0;
        u.rows = u.tokens * group;
        return u;
    }
    x -= common;
    const int64_t own = shared.own_slots * c.Hkv, index = x % own, slot = index / c.Hkv;
    u.part = static_cast<int>(x / own);
    u.sum_part = shared.common_parts + u.part;
    u.parts = shared.own_parts;
    u.chunk = shared.own_chunk;
    u.h = static_cast<int>(index % c.Hkv);
    u.block = 0;
    u.b = static_cast<int>(slot);
    if (!shared.single) {
        const auto begin_of = [&](int b) { return static_cast<int64_t>(c.seq.starts[b]) * group / R + b; };
        u.b = last_at_most(c.seq.B, slot, begin_of);
        u.block = slot - begin_of(u.b);
    }
    const Rows rows = rows_of(c.seq, u.b);
    if (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || u.block < 0 || u.block * R >= static_cast<int64_t>(rows.n) * group) return u;
    u.low = shared_length(c.seq, shared, lanes, u.b);
    u.start = rows.start;
    u.end = rows.length;
    u.g0 = u.g1 = u.b;
    u.before = rows.length - rows.n;
    u.rows = static_cast<int64_t>(rows.n) * group;
    return u;
}

// The unit of workgroup x, R rows a block; rows = 0: none.  All of it is the workgroup's, which the compiler cannot know: loops and addresses
// that depend on what is not known to be are kept by lanes, and their loads wait one for the other.
__device__ __forceinline__ SharedUnit shared_unit(const AttendCall &c, const SharedCall &shared, int64_t x, int R) {
    SharedUnit u = shared_unit_of(c, shared, x, R);
    const auto same = [](auto &v) { v = __builtin_amdgcn_readfirstlane(static_cast<int>(v)); };       // T is at most 2^24, T Hq 2^30
    same(u.rows);
    if (u.rows == 0) return u;
    same(u.start);
    same(u.block);
    same(u.h);
    same(u.b);
    same(u.low);
    same(u.end);
    same(u.part);
    same(u.sum_part);
    same(u.g0);
    same(u.g1);
    same(u.before);
    same(u.tokens);
    same(u.length);
    return u;
}

// The place of token t of a unit in its sequence; negative where there is none.
__device__ __forceinline__ int shared_place(const AttendCall &c, const SharedUnit &u, int64_t t) {
    if (u.g0 == u.g1) return u.before + static_cast<int>(t - u.start);
    const int32_t *const starts = c.seq.starts, *const lens = c.seq.lens;
    // where all have as many rows, this is it
    const int64_t tokens = u.tokens;
    int b = u.g0 + static_cast<int>((t - u.start) * (u.g1 - u.g0) / (tokens > 0 ? tokens : 1));
    b = min(max(b, u.g0), u.g1 - 1);
    int r0 = starts[b], r1 = starts[b + 1], length = lens[b];
    if (r0 > t || r1 <= t) {
        int lo = u.g0, hi = u.g1;
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (starts[mid] <= t) lo = mid;
            else hi = mid;
        }
        r0 = starts[lo];
        r1 = starts[lo + 1];
        length = lens[lo];
    }
    // as rows_of() has it
    const bool ok = r0 >= 0 && r0 <= r1 && r1 <= c.seq.T && length >= 0 && length <= (static_cast<int64_t>(c.seq.M) << c.seq.page_shift) &&
                    r1 - r0 <= c.max_rows && length <= c.max_len && t >= r0 && t < r1;
    return ok ? length - (r1 - r0) + static_cast<int>(t - r0) : -1;
}

// One wave: a row of a unit over tiles begin..end-1, element by element.  scratch: 256 floats of LDS.
template <class E, class Keys, int kKeys>
__device__ void shared_row(const AttendCall &c, const SharedCall &shared, const SharedUnit &u, int64_t row, float *scratch, const Keys &keys,
                           int begin, int end) {
    const int group = c.Hq / c.Hkv, head = u.h * group + static_cast<int>(row % group), lane = lane_id();
    const int64_t t = u.start + row / group;
    const int place = shared_place(c, u, t), sinks = min(end, keys.sink_tiles), main_from = max(begin, keys.sink_tiles);
    const auto clip = [&](int j) { return min(max(j, u.low), u.end); };
    const Rows one{u.b, t, 1, place + 1, true};
    const RowSum y = attend_row<E>(c, one, 0, head, scratch, begin < sinks ? clip(keys.begin_of(begin)) : 0,
                                   begin < sinks ? clip(keys.begin_of(sinks - 1) + kKeys) : 0,
                                   main_from < end ? clip(keys.begin_of(main_from)) : 0,
                                   main_from < end ? clip(keys.begin_of(end - 1) + kKeys) : 0);
    float *const sums = shared.sums(c, u.sum_part, t * c.Hq + head);
    for (int k = 0; k < APPROXIFER_MAX_HEAD_DIM / kWave; ++k)
        if (lane + k * kWave < c.Dh) sums[lane + k * kWave] = y.out[k];
    if (lane == 0) shared.settle(c, u.sum_part, t * c.Hq + head, y.top * 1.44269504088896340736f, y.total);
}
template <class E, int kKeys>
__device__ __forceinline__ void shared_part(const AttendCall &c, const SharedCall &shared, const SharedUnit &u, int64_t row, float *scratch,
                                            const KeyTiles<kKeys, true> &keys, int begin, int end) {
    shared_row<E, KeyTiles<kKeys, true>, kKeys>(c, shared, u, row, scratch, keys, begin, end);
}

// One wave: the status of sequence b.
__device__ __forceinline__ int shared_status(const AttendCall &c, const SharedCall &shared, int b) {
    int k = 0;
    const GroupLanes lanes(shared);
    const int length = shared_length(c.seq, shared, lanes, b, &k), st = attend_status(c, b);
    if (st != APPROXIFER_GROUP_OK || length == 0) return st;
    const Rows r = rows_of(c.seq, b);
    if (r.n == 0) return APPROXIFER_GROUP_OK;
    // the pages that are read for it: those of its group's places that its rows see
    int there = 0;
    const int g0 = shared.groups[k], g1 = shared.groups[k + 1];
    const int leader = shared_leader(c, g0, g1, length, shared_lens(c, g0, g1), &there);
    const int upto = min(there, r.length);
    const Visible first(c.window, c.sinks, max(r.place(0), 0));
    return pages_status(c.seq, leader, 0, min(min(c.sinks, upto), first.from), min(first.from, upto), upto);
}

// 4 us for 24 rows of 12 heads in 5 parts, 13 for 192 of 32 heads of 128 in 10.  A wave joins a row: its parts' sums in their order, eight of them on
// their way at a time.  The last workgroups: statuses, a wave for each.
template <class E, int DP>
__global__ __launch_bounds__(256) void attend_shared_join_kernel(AttendCall c, SharedCall shared) {
    typedef typename E::Value V;
    constexpr int kPerLane = (DP + kWave - 1) / kWave, kAhead = 8;
    const int lane = lane_id();
    const int64_t all = c.seq.T * c.Hq, work = (all + 3) / 4;
    if (blockIdx.x >= work) {
        const int64_t b = (blockIdx.x - work) * 4 + wave_id();
        if (b >= c.seq.B) return;
        const int st = shared_status(c, shared, static_cast<int>(b));
        if (lane == 0) c.status[b] = st;
        return;
    }
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + wave_id(), t = at / c.Hq;
    if (at >= all) return;
    const GroupLanes lanes(shared);
    const int b = last_at_most(c.seq.B, t, [&](int k) { return static_cast<int64_t>(c.seq.starts[k]); });
    const Rows rows = rows_of(c.seq, b);
    if (!rows.ok || rows.n > c.max_rows || rows.length > c.max_len || t < rows.start || t >= rows.start + rows.n) return;
    const int first = shared_length(c.seq, shared, lanes, b) > 0 ? 0 : shared.common_parts, parts = shared.common_parts + shared.own_parts;
    float top = -INFINITY, total = 0.0f, out[kPerLane] = {};
    for (int from = first; from < parts; from += kWave) {
        const int p = from + lane;
        const v2f x = p < parts ? *reinterpret_cast<const v2f *>(shared.tops + 2 * (p * all + at)) : v2f{-INFINITY, 0.0f};
        float most = fmaxf(x[0], top);
        for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float shrink = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - most);
        const float f = x[0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x[0] - most);
        // a part that saw nothing but what is no number has no maximum, and a total that says so
        total = total * shrink + (x[0] == -INFINITY ? x[1] : f * x[1]);
        top = most;
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) out[k] *= shrink;
        // (a part without keys has left neither, nor sums)
        const unsigned long long there = __ballot(!(x[0] == -INFINITY && x[1] == 0.0f));
        const int count = there == 0 ? 0 : 64 - __clzll(there);
        for (int i = 0; i < count; i += kAhead) {
            float y[kAhead][kPerLane], w[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int j = min(i + a, count - 1);
                w[a] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), j));
                const float *const sums = shared.sums(c, from + j, at);
#pragma unroll
                for (int k = 0; k < kPerLane; ++k) y[a][k] = lane + k * kWave < c.Dh ? sums[lane + k * kWave] : 0.0f;
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
#pragma unroll
                for (int k = 0; k < kPerLane; ++k) out[k] += there >> (i + a) & 1 ? w[a] * y[a][k] : 0.0f;
        }
    }
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
    V *const y = static_cast<V *>(c.out) + at * c.Dh;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k)
        if (lane + k * kWave < c.Dh) y[lane + k * kWave] = E::store(out[k] * inverse);
}

}  // namespace approxifer
