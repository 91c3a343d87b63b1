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
    int64_t bytes;                                            // of workspace; 0: not worth it, or not possible
};

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

SharedPlan shared_plan(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                       int64_t max_shared, int64_t window, size_t workspace_bytes) {
    SharedPlan p{};
    const int64_t group = Hq / Hkv, rows = max_rows * group;
    const bool wide = dtype == APPROXIFER_F32;
    if (C < 1 || B < 2 * C || max_shared < 1 || rows > 64 || rows < 1 || max_len < 1) return p;
    p.common_tiles = T * group > (wide ? 64 : 32) * C;
    p.own_tiles = rows > (wide ? 64 : 16);
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
    const int64_t own_keys = max_len > max_shared ? max_len - max_shared : 1;
    s.common_parts = cut(p.common_tiles, (T * group / R + (C + 1) / 2) * Hkv, window > 0 ? least(max_shared, window + 64) : max_shared, &s.common_chunk);
    s.own_parts = cut(p.own_tiles, (s.single ? B : T * group / r + (B + 1) / 2) * Hkv, own_keys, &s.own_chunk);
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
    const SharedPlan p = shared_plan(T, B, C, Hq, Hkv, Dh, dtype, least(max_rows, T), max_len, max_shared, window, static_cast<size_t>(1) << 60);
    return p.bytes > 0 ? static_cast<size_t>(p.bytes) : attend_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks);
}

int launch_attend_shared(const AttendCall &c, const int32_t *groups, const int32_t *shared, int64_t C, int64_t max_shared, void *workspace,
                         size_t workspace_bytes, hipStream_t stream) {
    SharedPlan p{};
    if (c.seq.T > 0)
        p = shared_plan(c.seq.T, c.seq.B, C, c.Hq, c.Hkv, c.Dh, c.dtype, c.max_rows, c.max_len, max_shared, c.window, workspace_bytes);
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
