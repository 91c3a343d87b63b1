// Appending new tokens to a cache in pages: per-head norm, rotary position, and the write into the pages, in one pass.
#include "sequences.h"

namespace approxifer {

namespace {

// Rotation of the head: frequencies in turns per position (so that an angle is reduced by dropping whole turns, exactly, in
// float64), and the axis that each pair's position is read from.
struct Rotation {
    double turns[APPROXIFER_MAX_HEAD_DIM / 2];
    uint8_t axis[APPROXIFER_MAX_HEAD_DIM / 2];
};

struct AppendCall {
    Sequences seq;
    int Hq, Hkv, Dh, pairs, axes;
    bool interleaved;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    void *q_out, *k_pool, *v_pool;
    const void *q_weight, *k_weight;
    float eps;
    const int32_t *positions;
    int32_t *status;
};

__device__ __forceinline__ void angle_of(const Rotation &rot, int i, int position, float *c, float *s) {
    const double t = position * rot.turns[i];
    sincospif(2.0f * static_cast<float>(t - rint(t)), s, c);
}

// One wave per head of a token: queries, keys, then values; behind the T tokens a wave per sequence for the status.
template <class E>
__global__ __launch_bounds__(kWave) void append_kernel(AppendCall c, Rotation rot) {
    typedef typename E::Value V;
    const int heads = c.Hq + 2 * c.Hkv, lane = lane_id();
    const int64_t t = blockIdx.x;
    int h = blockIdx.y;
    if (t >= c.seq.T) {                                       // the last blocks: statuses
        const int64_t b = (t - c.seq.T) * heads + h;
        if (c.status == nullptr || b >= c.seq.B) return;
        const Rows r = rows_of(c.seq, static_cast<int>(b));
        int st = APPROXIFER_SEQUENCE_BAD;
        if (r.ok) st = pages_status(c.seq, r.b, max(r.place(0), 0), r.n > 0 ? r.length : 0, 0, 0);
        if (lane == 0) c.status[b] = st;
        return;
    }
    const int b = sequence_of(c.seq, t);
    const Rows r = rows_of(c.seq, b);
    if (!r.ok || t < r.start || t >= r.start + r.n) return;
    const int place = r.place(static_cast<int>(t - r.start));
    const bool is_q = h < c.Hq, is_v = h >= c.Hq + c.Hkv;
    const V *x, *w = nullptr;
    V *y;
    if (is_q) {
        x = static_cast<const V *>(c.q) + t * c.q_stride + static_cast<int64_t>(h) * c.Dh;
        y = static_cast<V *>(c.q_out) + (t * c.Hq + h) * c.Dh;
        w = static_cast<const V *>(c.q_weight);
    } else {
        h -= is_v ? c.Hq + c.Hkv : c.Hq;
        x = static_cast<const V *>(is_v ? c.v : c.k) + t * (is_v ? c.v_stride : c.k_stride) + static_cast<int64_t>(h) * c.Dh;
        w = is_v ? nullptr : static_cast<const V *>(c.k_weight);
        const int page = place >= 0 ? page_of(c.seq, b, place) : -1;
        if (page < 0) return;
        const int size = 1 << c.seq.page_shift;
        y = static_cast<V *>(is_v ? c.v_pool : c.k_pool) +
            ((static_cast<int64_t>(page) * c.Hkv + h) * size + (place & (size - 1))) * c.Dh;
    }
    // each lane has elements lane, lane + 64, ..; all are read before any is written (q_out may be q)
    constexpr int kPerLane = APPROXIFER_MAX_HEAD_DIM / kWave;
    const bool turned = !is_v && c.pairs > 0;
    float out[kPerLane];
    float scale = 1.0f;
    if (w != nullptr) {
        float sum = 0.0f;
        for (int d = lane; d < c.Dh; d += kWave) {
            const float f = E::load(x[d]);
            sum += f * f;
        }
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        scale = 1.0f / sqrtf(sum / c.Dh + c.eps);
    }
    for (int k = 0; k < kPerLane; ++k) {
        const int d = lane + k * kWave;
        if (d >= c.Dh) break;
        const float f = E::load(x[d]) * scale * (w != nullptr ? E::load(w[d]) : 1.0f);
        out[k] = f;
        if (turned && d < 2 * c.pairs) {
            const int i = c.interleaved ? d >> 1 : d < c.pairs ? d : d - c.pairs;
            const bool second = c.interleaved ? d & 1 : d >= c.pairs;
            const int o = c.interleaved ? d ^ 1 : second ? d - c.pairs : d + c.pairs;
            const float g = E::load(x[o]) * scale * (w != nullptr ? E::load(w[o]) : 1.0f);
            const int position = c.positions != nullptr ? c.positions[t * c.axes + rot.axis[i]] : place;
            float cs, sn;
            angle_of(rot, i, position, &cs, &sn);
            out[k] = second ? g * sn + f * cs : f * cs - g * sn;
        }
    }
    for (int k = 0; k < kPerLane; ++k) {
        const int d = lane + k * kWave;
        if (d < c.Dh) y[d] = E::store(out[k]);
    }
}

}  // namespace

int launch_append(const Sequences &s, int Hq, int Hkv, int Dh, int dtype, const void *q, int64_t q_stride, const void *k,
                  int64_t k_stride, const void *v, int64_t v_stride, void *q_out, void *k_pool, void *v_pool,
                  const void *q_weight, const void *k_weight, double eps, const int32_t *positions, int axes,
                  const double *h_freq, const int32_t *h_axis, int pairs, bool interleaved, int32_t *status, hipStream_t stream) {
    Rotation rot{};
    for (int i = 0; i < pairs; ++i) {
        rot.turns[i] = h_freq[i] / 6.28318530717958647692528676655900577;
        rot.axis[i] = static_cast<uint8_t>(h_axis != nullptr ? h_axis[i] : 0);
    }
    const AppendCall c{s, Hq, Hkv, Dh, pairs, axes, interleaved, q, k, v, q_stride, k_stride, v_stride, q_out, k_pool, v_pool,
                       q_weight, k_weight, static_cast<float>(eps), positions, status};
    const int heads = Hq + 2 * Hkv;
    const int64_t blocks = s.T + (status != nullptr ? (s.B + heads - 1) / heads : 0);
    const dim3 grid(static_cast<unsigned>(blocks), heads), block(kWave);
    const auto kernel = dtype == APPROXIFER_F32 ? append_kernel<F32> : dtype == APPROXIFER_F16 ? append_kernel<F16> : append_kernel<BF16>;
    return launch_status(launch_kernel(kernel, grid, block, 0, stream, c, rot));
}

}  // namespace approxifer
