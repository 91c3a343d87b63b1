// Rows whose keys were cut into parts: a part's sums in the workspace, and their join.
#pragma once

#include "attend_pieces.h"

namespace approxifer {

// A part's sums of R rows: R x Dh floats, not yet divided, then R maxima (of c S, base 2) and R totals.
__device__ __host__ __forceinline__ int64_t part_floats(int R, int Dh) { return static_cast<int64_t>(R) * Dh + 2 * R; }

// The parts of a row joined, always in the same order, eight parts' sums on their way at a time.  kWaves of a workgroup share a row, every
// kWaves-th part to each: 4 for many parts (one wave and one part after the other took 38 us for 43 parts, a seventh of the call), 1 for a
// few, where rows are many.  base: the block's first part; n: the row there, `row` in its sequence.
template <class E, int DP, int kWaves>
__device__ __forceinline__ void join_row(const AttendCall &c, const Rows &rows, int64_t row, int h, const float *base, int R, int n,
                                         int parts) {
    typedef typename E::Value V;
    constexpr int kPerLane = (DP + kWave - 1) / kWave, kAhead = 8;
    __shared__ float outs[kWaves][kPerLane * kWave], tops[kWaves], totals[kWaves];
    const int lane = lane_id(), group = c.Hq / c.Hkv;
    const int wave = kWaves == 1 ? 0 : __builtin_amdgcn_readfirstlane(wave_id());
    const int64_t stride = part_floats(R, c.Dh);
    float top = -INFINITY, out[kPerLane] = {}, total = 0.0f;
    for (int from = wave; from < parts; from += kWaves * kWave) {
        const int p = from + kWaves * lane, count = min((parts - from + kWaves - 1) / kWaves, kWave);
        const float m = p < parts ? base[p * stride + R * c.Dh + n] : -INFINITY;
        const float l = p < parts ? base[p * stride + R * c.Dh + R + n] : 0.0f;
        float most = fmaxf(m, top);
        for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float shrink = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - most);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - most);
        // a part that saw nothing but what is no number has no maximum, and a total that says so
        total = total * shrink + (m == -INFINITY ? l : f * l);
        top = most;
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) out[k] *= shrink;
        for (int i = 0; i < count; i += kAhead) {
            float x[kAhead][kPerLane], w[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int j = min(i + a, count - 1);
                w[a] = i + a < count ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), j)) : 0.0f;
#pragma unroll
                for (int k = 0; k < kPerLane; ++k)
                    x[a][k] = lane + k * kWave < c.Dh ? base[(from + kWaves * j) * stride + n * c.Dh + lane + k * kWave] : 0.0f;
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
#pragma unroll
                for (int k = 0; k < kPerLane; ++k) out[k] += i + a < count ? w[a] * x[a][k] : 0.0f;
        }
    }
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    const int64_t t = rows.start + row / group;
    V *const y = static_cast<V *>(c.out) + (t * c.Hq + h * group + row % group) * c.Dh;
    if constexpr (kWaves == 1) {
        const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
        for (int k = 0; k < kPerLane; ++k)
            if (lane + k * kWave < c.Dh) y[lane + k * kWave] = E::store(out[k] * inverse);
        if (c.stats != nullptr && lane == 0) RowStats(top, total).store(c, t, h * group + static_cast<int>(row % group));
        return;
    }
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) outs[wave][lane + k * kWave] = out[k];
    if (lane == 0) {
        tops[wave] = top;
        totals[wave] = total;
    }
    __syncthreads();
    float all = tops[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) all = fmaxf(all, tops[w]);
    float sum = 0.0f, f[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        f[w] = tops[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(tops[w] - all);
        sum += tops[w] == -INFINITY ? totals[w] : f[w] * totals[w];
    }
    const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (c.stats != nullptr && threadIdx.x == 0) RowStats(all, sum).store(c, t, h * group + static_cast<int>(row % group));
    for (int d = threadIdx.x; d < c.Dh; d += 256) {
        float x = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += f[w] * outs[w][d];
        y[d] = E::store(x * inverse);
    }
}

// One wave: `row` of a sequence and cache head h over tiles begin..end-1, element by element, as a part of R rows of which it is the n-th, or
// the result where there is but one part.  scratch: 256 floats of LDS.
template <class E, int kKeys>
__device__ void attend_part(const AttendCall &c, const Rows &rows, int64_t row, int h, float *scratch, const KeyTiles<kKeys> &keys, int begin,
                            int end, bool alone, float *partial, int R, int n) {
    typedef typename E::Value V;
    const int group = c.Hq / c.Hkv, i = static_cast<int>(row / group), head = h * group + static_cast<int>(row % group);
    const int main_from = max(begin, keys.sink_tiles), lane = lane_id();
    const RowSum y = attend_row<E>(c, rows, i, head, scratch, begin * kKeys, min(end, keys.sink_tiles) * kKeys,
                                   main_from < end ? keys.begin_of(main_from) : 0,
                                   main_from < end ? keys.begin_of(end - 1) + kKeys : 0);
    V *const out = static_cast<V *>(c.out) + ((rows.start + i) * c.Hq + head) * c.Dh;
    const float inverse = y.total == 0.0f ? 0.0f : 1.0f / y.total;
    for (int k = 0; k < APPROXIFER_MAX_HEAD_DIM / kWave; ++k) {
        const int d = lane + k * kWave;
        if (d >= c.Dh) break;
        if (alone) out[d] = E::store(y.out[k] * inverse);
        else partial[n * c.Dh + d] = y.out[k];
    }
    if (!alone && lane == 0) {
        partial[R * c.Dh + n] = y.top * 1.44269504088896340736f;
        partial[R * c.Dh + R + n] = y.total;
    }
}

}  // namespace approxifer
