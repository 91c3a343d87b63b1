// Attention of sequences that begin alike: when their common places are read once for all, by which kernels, and how keys are cut.
#include <cmath>

#include "attend_shared.h"

namespace approxifer {

hipError_t launch_shared_tiles_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_tiles_f16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_tiles_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_tokens_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_tokens_f16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_tokens_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_both_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_both_f16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_both_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_join_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_join_f16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);
hipError_t launch_shared_join_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream);

namespace {

struct SharedPlan {
    SharedCall call;
    bool common_tiles, own_tiles;                             // which kernel has which rows
    int joined;                                               // parts of a row of a group
    int64_t bytes;                                            // of workspace; 0: not worth it for rows as many as these, or not possible
};

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

// Whether what is common is long enough.  attend() reads it at about 4.5 bytes a ps for each sequence; to read it once costs the second launch and
// the lookups, as many microseconds as `fixed`, and several times the traffic of the parts, which is written by many and read by few.  Fitted to 2600
// random shapes of 1 to 20 groups of 2 to 100 sequences behind 48 to 20000 places (heads of 64 to 256, 1 to 8 for one of the cache): taken always,
// time against attend()'s is 0.98 by geometric mean (16-bit) and 0.80 (float32); by this rule 0.82 and 0.75; by who knew it 0.81 and 0.74; 42 of the
// 980 that it takes are longer by more than 2 %.  8 heads of 128, bf16: 8 groups of 8 behind 512 18.5 -> 21.6, 32 of 8 58.5 -> 51.5, one of 4 behind
// 4000 15.8 -> 17.2; 8 of 35, two tokens of 32 heads on 8 of 96, behind 336 49 -> 80; 9 of 9 behind 1904 (4 heads of 128) 41 -> 23.
bool shared_pays(const SharedPlan &p, int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_len, int64_t max_shared,
                 int64_t window, int64_t sinks, int page_shift) {
    const bool wide = dtype == APPROXIFER_F32, two = p.common_tiles != p.own_tiles && !(p.common_tiles && shared_both(Dh, dtype, page_shift));
    // windows reach what is common over what is their own
    const int64_t own = max_len - max_shared, seen = window > 0 ? least(max_shared, (window > own ? window - own : 0) + sinks) : max_shared;
    const double saved = static_cast<double>(B - C) * seen * Hkv * Dh * (wide ? 8 : 4) / 4.5e6;
    const double join = static_cast<double>(T) * Hq * Dh * 8 * p.joined / 4.5e6;
    if (wide) return saved > 8 + (p.common_tiles ? 10 : 20) * join;
    if (p.common_tiles && p.own_tiles) return saved > 4 + 2.5 * join;
    return saved > (two ? 50 + 8 * join : (p.common_tiles ? 15 : 26) + 12 * join);
}

SharedPlan shared_plan(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                       int64_t max_shared, int64_t window, int64_t sinks, size_t workspace_bytes) {
    SharedPlan p{};
    const int64_t group = Hq / Hkv, rows = max_rows * group;
    const bool wide = dtype == APPROXIFER_F32;
    // Whether it pays.  What is saved is keys that come from a cache where the sequences are read side by side, and rows that are empty in every
    // sequence's own tiles; what it costs is that two parts of every row at least are written and joined.  Microseconds, attend() -> here, 8
    // heads of the cache of 128, new tokens times heads of a group = rows:
    //   bf16, 64 sequences behind 8000 places: rows 32 263 -> 114, 48 270 -> 157, 64 272 -> 246, 128 290 -> 344; behind 2000: 74 -> 52,
    //   75 -> 67, 77 -> 88, 83 -> 139.
    //   float32, which waits for products: 64 behind 2000: rows 8 103 -> 71, 12 101 -> 112, 16 101 -> 125, 20 192 -> 167, 24 192 -> 182, 32
    //   193 -> 237; four groups of them behind 4000: 701 -> 434, 703 -> 622, 706 -> 810, 1386 -> 1046, 1390 -> 1233, 1392 -> 1614.  A quarter of
    //   the rows of attend()'s tiles of 16 has to be empty.
    //   bf16, rows 4, 32 groups behind 4000: of 2 sequences 105 -> 115, of 3 151 -> 132, of 4 173 -> 122, of 8 311 -> 154; with heads that are
    //   no group (12 of 64) of 2 119 -> 78, of 8 254 -> 105.
    if (C < 1 || B < (group > 1 ? 3 : 2) * C || max_shared < 1 || rows < 1 || max_len < 1) return p;
    if (rows > (wide ? 12 * ((rows + 15) / 16) : 48)) return p;
    // Which kernel has a group's common places: tiles of 128 rows wait less for keys, tiles of 16 split finer.  Rows of a group, tokens -> tiles,
    // behind 4000 places: bf16, 8 groups, heads of 128: 16 37 -> 45, 32 46 -> 41, 64 83 -> 55, 256 208 -> 114; 16 groups, 12 heads of 64: 16
    // 63 -> 62, 24 83 -> 76, 32 93 -> 87, 64 166 -> 132 (one group: 32 15.7 -> 15.9).  float32 behind 2000: 4 groups, 128 rows of 64 147 -> 150,
    // 512 99 -> 90 (4 heads of the cache), 384 of 96 104 -> 118, 512 of 256 247 -> 211; of 128, behind 4000, 460 -> 652.
    p.common_tiles = shared_tiles(Dh, dtype) && T * group >= (wide ? 257 : 32) * C;
    // and its sequences' own ones: bf16, 4 groups of 16, 1024 places: 16 rows 58 -> 70, 32 91 -> 81, 64 144 -> 101; float32 64 341 -> 412
    p.own_tiles = !wide && rows > 16;
    SharedCall &s = p.call;
    s.C = static_cast<int>(C);
    s.max_shared = static_cast<int>(max_shared);
    const int64_t R = p.common_tiles ? 128 : 16, r = p.own_tiles ? 128 : 16;
    s.single = rows <= r;
    s.common_slots = T * group / R + C;
    s.own_slots = s.single ? B : T * group / r + B;
    // parts: as many as fill the GPU once, of a tile a wave or two of a workgroup's at least, as far as writing and joining them costs less than it gives
    const auto cut = [&](bool tiles, int64_t units, int64_t keys, int *chunk) {
        const int64_t places = !tiles ? 512 : Dh > 128 || (wide && Dh > 64) ? 256 : wide ? 768 : 512;
        int64_t parts = least(places / (units > 0 ? units : 1), (keys + 127) / 128);
        if (tiles) {
            const double tile_us = Dh * (!wide ? 0.0086 : Dh > 64 ? 0.0625 : 0.053), part_us = static_cast<double>(T) * Hq * Dh * 8.0 / 4.5e6;
            parts = least(parts, static_cast<int64_t>(std::sqrt(keys / 64.0 * tile_us / part_us) + 0.5));
        }
        if (parts < 1) parts = 1;
        *chunk = static_cast<int>(((keys + parts - 1) / parts + 127) / 128 * 128);
        return static_cast<int>((keys + *chunk - 1) / *chunk);
    };
    const int64_t own_keys = max_len > max_shared ? max_len - max_shared : 1, seen = window > 0 ? window + sinks + 64 : max_len;
    const int64_t own_units = (s.single ? B : T * group / r + (B + 1) / 2) * Hkv;
    s.common_parts = cut(p.common_tiles, (T * group / R + (C + 1) / 2) * Hkv, window > 0 ? least(max_shared, window + 64) : max_shared, &s.common_chunk);
    s.own_parts = cut(p.own_tiles, own_units, least(own_keys, seen), &s.own_chunk);
    p.joined = s.common_parts + s.own_parts;
    // Sequences in no group, or in one with less in common, have more of their own: up to two rounds of parts, of 768 keys at least, that others
    // leave empty.  24 sequences behind 4000 places and one of 8000 places of its own (12 heads of 64, float32) 134
    // us -> 82; 192 behind 8003 (8 of 128, bf16), where nobody needs them, 117.9 -> 119.2.
    if (!p.own_tiles) {
        const int64_t more = least(1024 / own_units, least(max_len, seen) / 768);
        if (more > s.own_parts) s.own_parts = static_cast<int>(more);
    }
    const int64_t each = T * Hq * (Dh + 2) * 4;
    const int64_t room = static_cast<int64_t>(workspace_bytes / static_cast<size_t>(each));
    if (room < 2) return p;
    if (s.common_parts + s.own_parts > room) {
        s.own_parts = static_cast<int>(least(s.own_parts, room / 2));
        s.common_parts = static_cast<int>(least(s.common_parts, room - s.own_parts));
    }
    // a launch's threads
    if ((s.common_slots * s.common_parts + s.own_slots * s.own_parts) * Hkv >= 1 << 24 || T * Hq / 4 + B / 4 >= (1 << 24) - 2) return p;
    p.bytes = each * (s.common_parts + s.own_parts);
    return p;
}

}  // namespace

size_t attend_shared_workspace_bytes(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                                     int64_t max_shared, int64_t window, int64_t sinks) {
    const SharedPlan p = shared_plan(T, B, C, Hq, Hkv, Dh, dtype, least(max_rows, T), max_len, max_shared, window, sinks, static_cast<size_t>(1) << 60);
    return p.bytes > 0 ? static_cast<size_t>(p.bytes) : attend_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks);
}

bool attend_shared_pays(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                        int64_t max_shared, int64_t window, int64_t sinks, int page_shift) {
    const SharedPlan p = shared_plan(T, B, C, Hq, Hkv, Dh, dtype, least(max_rows, T), max_len, max_shared, window, sinks, static_cast<size_t>(1) << 60);
    return p.bytes > 0 && shared_pays(p, T, B, C, Hq, Hkv, Dh, dtype, max_len, max_shared, window, sinks, page_shift);
}

int launch_attend_shared(const AttendCall &c, const int32_t *groups, const int32_t *shared, int64_t C, int64_t max_shared, void *workspace,
                         size_t workspace_bytes, hipStream_t stream) {
    SharedPlan p{};
    if (c.seq.T > 0)
        p = shared_plan(c.seq.T, c.seq.B, C, c.Hq, c.Hkv, c.Dh, c.dtype, c.max_rows, c.max_len, max_shared, c.window, c.sinks, workspace_bytes);
    if (p.bytes == 0) return launch_attend(c, workspace, workspace_bytes, stream);
    SharedCall s = p.call;
    s.groups = groups;
    s.shared = shared;
    s.outs = static_cast<float *>(workspace);
    s.tops = s.outs + static_cast<int64_t>(s.common_parts + s.own_parts) * c.seq.T * c.Hq * c.Dh;
    const auto run = [&](bool tiles, const SharedCall &call) {
        if (c.dtype == APPROXIFER_F32) return tiles ? launch_shared_tiles_f32(c, call, stream) : launch_shared_tokens_f32(c, call, stream);
        if (c.dtype == APPROXIFER_F16) return tiles ? launch_shared_tiles_f16(c, call, stream) : launch_shared_tokens_f16(c, call, stream);
        return tiles ? launch_shared_tiles_bf16(c, call, stream) : launch_shared_tokens_bf16(c, call, stream);
    };
    hipError_t e = hipSuccess;
    if (p.common_tiles == p.own_tiles) {
        e = run(p.own_tiles, s);
    } else if (p.common_tiles && shared_both(c.Dh, c.dtype, c.seq.page_shift)) {
        e = c.dtype == APPROXIFER_F32   ? launch_shared_both_f32(c, s, stream)
            : c.dtype == APPROXIFER_F16 ? launch_shared_both_f16(c, s, stream)
                                        : launch_shared_both_bf16(c, s, stream);
    } else {
        SharedCall only = s;
        only.own_slots = 0;
        e = run(p.common_tiles, only);
        only = s;
        only.common_slots = 0;
        if (e == hipSuccess) e = run(p.own_tiles, only);
    }
    if (e == hipSuccess)
        e = c.dtype == APPROXIFER_F32   ? launch_shared_join_f32(c, s, stream)
            : c.dtype == APPROXIFER_F16 ? launch_shared_join_f16(c, s, stream)
                                        : launch_shared_join_bf16(c, s, stream);
    return launch_status(e);
}

}  // namespace approxifer
