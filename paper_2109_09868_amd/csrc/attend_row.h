// Attention of one row to what its sequence holds, straight from the definition: one wave, float32, a key per lane for the
// scores and a dimension per lane for the sum.  The tiled kernels fall back on it where a tile cannot be computed as a
// product: a value that is not finite and that some of the tile's rows must not see.
#pragma once

#include "sequences.h"

namespace approxifer {

// The places a row at `place` sees: [0, sinks_end) and [from, place].
struct Visible {
    int sinks_end, from, place;
    __device__ __forceinline__ Visible(int window, int sinks, int t) : place(t) {
        from = window > 0 ? max(t - window + 1, 0) : 0;
        sinks_end = min(sinks, from);
    }
    __device__ __forceinline__ bool sees(int j) const { return j <= place && (j >= from || j < sinks_end); }
};

// q: [256] and p: [64] floats of LDS of this wave.
template <class E>
__device__ void attend_row(const AttendCall &c, const Rows &r, int i, int head, float *q, float *p) {
    typedef typename E::Value V;
    constexpr int kPerLane = APPROXIFER_MAX_HEAD_DIM / kWave;
    const int lane = lane_id(), h = head / (c.Hq / c.Hkv), size = 1 << c.seq.page_shift;
    const int64_t t = r.start + i;
    const V *x = static_cast<const V *>(c.q) + t * c.q_stride + static_cast<int64_t>(head) * c.Dh;
    for (int d = lane; d < c.Dh; d += kWave) q[d] = E::load(x[d]) * c.scale;
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    const Visible see(c.window, c.sinks, r.place(i));
    float out[kPerLane] = {}, top = -INFINITY, total = 0.0f;
    for (int part = 0; part < 2; ++part) {
        const int from = part ? see.from : 0, to = part ? see.place + 1 : see.sinks_end;
        for (int j0 = from; j0 < to; j0 += kWave) {
            const int j = j0 + lane, count = min(to - j0, kWave);
            float s = -INFINITY;
            if (j < to) {
                const int page = page_of(c.seq, r.b, j);
                if (page < 0) {
                    s = NAN;
                } else {
                    const V *k = static_cast<const V *>(c.k_pool) +
                                 ((static_cast<int64_t>(page) * c.Hkv + h) * size + (j & (size - 1))) * c.Dh;
                    s = 0.0f;
                    for (int d = 0; d < c.Dh; ++d) s += q[d] * E::load(k[d]);
                }
            }
            float m = s;
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            const float next = fmaxf(top, m), safe = next == -INFINITY ? 0.0f : next;
            const float w = j < to ? expf(s - safe) : 0.0f, shrink = expf(top - safe);
            float sum = w;
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            total = total * shrink + sum;
            top = next;
            p[lane] = w;
            __builtin_amdgcn_wave_barrier();
            __threadfence_block();
            for (int k = 0; k < kPerLane; ++k) out[k] *= shrink;
            for (int n = 0; n < count; ++n) {
                const int page = page_of(c.seq, r.b, j0 + n);
                if (page < 0) continue;
                const V *v = static_cast<const V *>(c.v_pool) +
                             ((static_cast<int64_t>(page) * c.Hkv + h) * size + ((j0 + n) & (size - 1))) * c.Dh;
                for (int k = 0; k < kPerLane; ++k)
                    if (lane + k * kWave < c.Dh) out[k] += p[n] * E::load(v[lane + k * kWave]);
            }
            __builtin_amdgcn_wave_barrier();
            __threadfence_block();
        }
    }
    V *y = static_cast<V *>(c.out) + (t * c.Hq + head) * c.Dh;
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
    for (int k = 0; k < kPerLane; ++k)
        if (lane + k * kWave < c.Dh) y[lane + k * kWave] = E::store(out[k] * inverse);
}

// One wave: the status of sequence b.
__device__ __forceinline__ int attend_status(const AttendCall &c, int b) {
    const Rows r = rows_of(c.seq, b);
    if (!r.ok || r.n > c.max_rows || r.length > c.max_len) return APPROXIFER_SEQUENCE_BAD;
    if (r.n == 0) return APPROXIFER_GROUP_OK;
    const Visible first(c.window, c.sinks, max(r.place(0), 0));
    return pages_status(c.seq, b, 0, min(min(c.sinks, r.length), first.from), first.from, r.length);
}

}  // namespace approxifer
