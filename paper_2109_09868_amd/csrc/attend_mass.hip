// Attention that adds up the weights it gives: attention itself, then the weights per key.
#include "attend_mass.h"

namespace approxifer {

namespace {

int64_t stats_bytes(int64_t T, int Hq) { return (T * Hq * 8 + 255) / 256 * 256; }

// Workgroups to a block of keys: its heads first, then its rows, until there are four for every CU or a part has no more than four tiles.
MassGrid mass_grid(int64_t B, int Hq, int Hkv, int64_t max_rows, int64_t max_len, size_t room) {
    MassGrid g;
    g.blocks = (max_len + kMassKeys - 1) / kMassKeys;
    g.stride = g.blocks * kMassKeys;
    const int64_t blocks = g.blocks * B, want = (1024 + blocks - 1) / (blocks > 0 ? blocks : 1);
    const int64_t tiles = (max_rows * (Hq / Hkv) + 31) / 32;
    const int64_t most = static_cast<int64_t>(room / (static_cast<size_t>(B > 0 ? B : 1) * (g.stride > 0 ? g.stride : 1) * 4));
    const int64_t slices = want < most ? want : most;
    g.heads = static_cast<int>(slices < 1 ? 1 : slices < Hkv ? slices : Hkv);
    int64_t parts = slices / Hkv < (tiles + 3) / 4 ? slices / Hkv : (tiles + 3) / 4;
    g.parts = static_cast<int>(parts < 1 ? 1 : parts);
    return g;
}

constexpr int64_t kAddBlocks = 1 << 20;

// A thread for every key: the slices' sums in their order.
__global__ __launch_bounds__(256) void add_slices_kernel(AttendCall c, MassGrid g, float *mass, int64_t mass_stride, const float *sums) {
    const int64_t work = g.blocks * c.seq.B;
    static_assert(kMassKeys == 256, "a thread for every key of a block");
    for (int64_t index = blockIdx.x; index < work; index += gridDim.x) {
        const int b = static_cast<int>(index % c.seq.B), j = static_cast<int>(index / c.seq.B) * 256 + threadIdx.x;
        const Rows rows = rows_of(c.seq, b);
        if (!rows.ok || rows.n == 0 || rows.n > c.max_rows || rows.length > c.max_len || j >= rows.length) continue;
        float x = 0.0f;
        for (int s = 0; s < g.slices(); ++s) x += sums[(static_cast<int64_t>(s) * c.seq.B + b) * g.stride + j];
        mass[b * mass_stride + j] += x;
    }
}

}  // namespace

size_t attend_mass_least_bytes(int64_t T, int Hq) { return static_cast<size_t>(stats_bytes(T, Hq)); }

size_t attend_mass_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                                   int64_t window, int64_t sinks) {
    const size_t parts = attend_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks);
    const MassGrid g = mass_grid(B, Hq, Hkv, max_rows < T ? max_rows : T, max_len, static_cast<size_t>(1) << 60);
    const size_t sums = g.slices() < 2 ? 0 : static_cast<size_t>(g.slices()) * B * g.stride * 4;
    return static_cast<size_t>(stats_bytes(T, Hq)) + (parts > sums ? parts : sums);
}

int launch_attend_mass(AttendCall c, float *mass, int64_t mass_stride, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (c.seq.T == 0) return launch_attend(c, nullptr, 0, stream);
    // the rows' statistics, then room that attention's parts and afterwards the slices' sums use
    const size_t stats = static_cast<size_t>(stats_bytes(c.seq.T, c.Hq)), room = workspace_bytes > stats ? workspace_bytes - stats : 0;
    c.stats = static_cast<float *>(workspace);
    float *const sums = c.stats + stats / 4;
    const int rc = launch_attend(c, sums, room, stream);
    if (rc != APPROXIFER_OK || c.max_rows == 0 || c.max_len == 0) return rc;
    const MassGrid g = mass_grid(c.seq.B, c.Hq, c.Hkv, c.max_rows, c.max_len, room);
    hipError_t e = c.dtype == APPROXIFER_F32   ? launch_mass_f32(c, g, mass, mass_stride, sums, stream)
                   : c.dtype == APPROXIFER_F16 ? launch_mass_f16(c, g, mass, mass_stride, sums, stream)
                                               : launch_mass_bf16(c, g, mass, mass_stride, sums, stream);
    if (e == hipSuccess && g.slices() > 1) {
        const int64_t work = g.blocks * c.seq.B;
        e = launch_kernel(add_slices_kernel, dim3(static_cast<unsigned>(work < kAddBlocks ? work : kAddBlocks)), dim3(256), 0, stream, c, g,
                          mass, mass_stride, static_cast<const float *>(sums));
    }
    return launch_status(e);
}

}  // namespace approxifer
