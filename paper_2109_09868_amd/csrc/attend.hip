// Attention over a cache in pages.
#include "attend_tiles.h"

namespace approxifer {

namespace {

// One wave per row and head; behind the T rows a wave per sequence for the status.
template <class E>
__global__ __launch_bounds__(kWave) void attend_rows_kernel(AttendCall c) {
    __shared__ float q[APPROXIFER_MAX_HEAD_DIM], p[kWave];
    const int64_t t = blockIdx.x;
    if (t >= c.seq.T) {
        const int64_t b = (t - c.seq.T) * c.Hq + blockIdx.y;
        if (c.status == nullptr || b >= c.seq.B) return;
        const int st = attend_status(c, static_cast<int>(b));
        if (lane_id() == 0) c.status[b] = st;
        return;
    }
    const Rows r = rows_of(c.seq, sequence_of(c.seq, t));
    if (!r.ok || t < r.start || t >= r.start + r.n || r.n > c.max_rows || r.length > c.max_len) return;
    attend_row<E>(c, r, static_cast<int>(t - r.start), blockIdx.y, q, p);
}

}  // namespace

size_t attend_workspace_bytes(int64_t, int64_t, int, int, int, int, int64_t, int64_t, int64_t, int64_t) { return 0; }

int launch_attend(const AttendCall &c, void *, size_t, hipStream_t stream) {
    if (static_cast<int64_t>(c.max_rows) * (c.Hq / c.Hkv) >= 32)
        return launch_status(c.dtype == APPROXIFER_F32   ? launch_tiles_f32(c, stream)
                             : c.dtype == APPROXIFER_F16 ? launch_tiles_f16(c, stream)
                                                         : launch_tiles_bf16(c, stream));
    const int64_t blocks = c.seq.T + (c.status != nullptr ? (c.seq.B + c.Hq - 1) / c.Hq : 0);
    const dim3 grid(static_cast<unsigned>(blocks), c.Hq), block(kWave);
    const auto kernel = c.dtype == APPROXIFER_F32   ? attend_rows_kernel<F32>
                        : c.dtype == APPROXIFER_F16 ? attend_rows_kernel<F16>
                                                    : attend_rows_kernel<BF16>;
    return launch_status(launch_kernel(kernel, grid, block, 0, stream, c));
}

}  // namespace approxifer
