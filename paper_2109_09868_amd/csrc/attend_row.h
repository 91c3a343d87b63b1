// Attention of one row to what its sequence holds, straight from the definition: one wave, float32, a key per lane for the
// scores and a dimension per lane for the sum.  The tiled kernels fall back on it where a row cannot be computed as a
// product: a value that is not finite times a weight of 0.
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

// The keys that rows at places p0..p1 see, in tiles of kKeys: those of the first tokens, then those of the window.
template <int kKeys>
struct KeyTiles {
    int last, from, sinks_end, sink_tiles, main_tile, steps;
    __device__ __forceinline__ KeyTiles(int window, int sinks, int p0, int p1) : last(p1) {
        from = window > 0 ? max(p0 - window + 1, 0) : 0;
        sinks_end = min(sinks, from);
        sink_tiles = (sinks_end + kKeys - 1) / kKeys;
        main_tile = max(from / kKeys, sink_tiles);
        steps = p1 < 0 ? 0 : sink_tiles + max(p1 / kKeys + 1 - main_tile, 0);
    }
    __device__ __forceinline__ int begin_of(int it) const { return (it < sink_tiles ? it : main_tile + it - sink_tiles) * kKeys; }
    // the key itself, or one that some row sees where none sees this one: what nobody sees is not read
    __device__ __forceinline__ int seen(int j) const { return j > last ? last : j < from && j >= sinks_end ? from : j; }
};

// One row over the places [a0, a1) and [b0, b1), as far as it sees them.  q: [256] floats of LDS of this wave.  Lane l has
// dimensions l, l + 64, .. of `out`, not yet divided by `total`; both relative to exp(top).  Every key's value row takes a load of its
// own, kAhead of them on their way.
struct RowSum {
    float out[APPROXIFER_MAX_HEAD_DIM / kWave], top, total;
};
template <class E>
__device__ RowSum attend_row(const AttendCall &c, const Rows &r, int i, int head, float *q, int a0, int a1, int b0, int b1) {
    typedef typename E::Value V;
    typedef V VP __attribute__((ext_vector_type(16 / sizeof(V))));
    constexpr int kPerLane = APPROXIFER_MAX_HEAD_DIM / kWave, kPiece = 16 / sizeof(V), kAhead = 4;
    const int lane = lane_id(), h = head / (c.Hq / c.Hkv), size = 1 << c.seq.page_shift;
    const int64_t t = r.start + i;
    const V *x = static_cast<const V *>(c.q) + t * c.q_stride + static_cast<int64_t>(head) * c.Dh;
    for (int d = lane; d < c.Dh; d += kWave) q[d] = E::load(x[d]) * c.scale;
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    const Visible see(c.window, c.sinks, r.place(i));
    RowSum y{};
    y.top = -INFINITY;
    for (int part = 0; part < 2; ++part) {
        const int from = part ? b0 : a0, to = min(part ? b1 : a1, see.place + 1);
        for (int j0 = from; j0 < to; j0 += kWave) {
            const int j = j0 + lane;
            const bool mine = j < to && see.sees(j);
            float s = -INFINITY;
            int page = -1;
            if (mine) {
                page = page_of(c.seq, r.b, j);
                if (page < 0) {
                    s = NAN;
                } else {
                    const V *k = static_cast<const V *>(c.k_pool) +
                                 ((static_cast<int64_t>(page) * c.Hkv + h) * size + (j & (size - 1))) * c.Dh;
                    s = 0.0f;
                    for (int d = 0; d < c.Dh; d += kPiece) {
                        const VP x = *reinterpret_cast<const VP *>(k + d);
#pragma unroll
                        for (int e = 0; e < kPiece; ++e) s += q[d + e] * E::load(x[e]);
                    }
                }
            }
            float m = s;
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            const float next = fmaxf(y.top, m), safe = next == -INFINITY ? 0.0f : next;
            const float w = mine ? expf(s - safe) : 0.0f, shrink = expf(y.top - safe);
            float sum = w;
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            y.total = y.total * shrink + sum;
            y.top = next;
            for (int k = 0; k < kPerLane; ++k) y.out[k] *= shrink;
            for (unsigned long long left = __ballot(page >= 0); left != 0;) {
                const int count = min(__popcll(left), kAhead);
                float weight[kAhead], x[kAhead][kPerLane];
#pragma unroll
                for (int a = 0; a < kAhead; ++a) {
                    const int n = __ffsll(left) - 1;          // behind the last one: that again, not used
                    if (a + 1 < count) left &= left - 1;
                    weight[a] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), n));
                    const V *v = static_cast<const V *>(c.v_pool) +
                                 ((static_cast<int64_t>(__builtin_amdgcn_readlane(page, n)) * c.Hkv + h) * size + ((j0 + n) & (size - 1))) * c.Dh;
#pragma unroll
                    for (int k = 0; k < kPerLane; ++k) x[a][k] = lane + k * kWave < c.Dh ? E::load(v[lane + k * kWave]) : 0.0f;
                }
                left &= left - 1;
#pragma unroll
                for (int a = 0; a < kAhead; ++a)
#pragma unroll
                    for (int k = 0; k < kPerLane; ++k) y.out[k] += a < count ? weight[a] * x[a][k] : 0.0f;
            }
        }
    }
    return y;
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
