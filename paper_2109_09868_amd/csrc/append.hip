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

// Sum over each aligned group of L lanes, in every lane of it.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
    if (L >= 2) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kDppQuadXor1, 0xF, 0xF, true));
    if (L >= 4) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kDppQuadXor2, 0xF, 0xF, true));
    if (L >= 8) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kDppRowHalfMirror, 0xF, 0xF, true));
    if (L >= 16) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kDppRowMirror, 0xF, 0xF, true));
    if (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
        v = __int_as_float(r[0]) + __int_as_float(r[1]);
    }
    return v;
}

// The same for groups of any length: every lane adds the others of its group.
__device__ __forceinline__ float group_sum(float v, int begin, int at, int L) {
    float sum = v;
    for (int o = 1; o < L; ++o) sum += __shfl(v, begin + (at + o < L ? at + o : at + o - L));
    return sum;
}

// The sequence of the wave's token t: 64 starts are compared at once, so that the common cases take one load where bisection takes one
// for every doubling of B.
__device__ __forceinline__ int wave_sequence_of(const Sequences &s, int64_t t) {
    int lo = 0, span = s.B;
    while (span > 1) {
        const int step = (span + kWave - 1) / kWave, k = lane_id() * step;
        const unsigned long long before = __ballot(k < span && s.starts[lo + k] <= t);
        const int last = before != 0 ? (63 - __clzll(before)) * step : 0;
        span = min(step, span - last);
        lo += last;
    }
    return lo;
}

__device__ __forceinline__ void append_status(const AppendCall &c, int b) {
    const Rows r = rows_of(c.seq, b);
    int st = APPROXIFER_SEQUENCE_BAD;
    if (r.ok) st = pages_status(c.seq, b, max(r.place(0), 0), r.n > 0 ? r.length : 0, 0, 0);
    if (lane_id() == 0) c.status[b] = st;
}

typedef int v4i __attribute__((ext_vector_type(4)));

// Heads in pieces of 16 bytes, HBM-bound: every value is read once and written once.
// A wave has one token and `per` of its heads.  `lanes` lanes (kLanes, or any number where that is 0) share a head, two pieces each: those
// whose values are rotated with each other, piece u and the one `pairs` further (neighbours are rotated: pieces 2 u and 2 u + 1), so that a
// rotation stays in the lane.  Heads that lie next to each other are read and written together, and all of kSteps rounds' loads are on
// their way while cosines and sines (float64 reduction, about 80 instructions each) are computed, once for the token, a pair per lane.
// 21288 tokens of 48 heads of 128 (bf16, 523 MB read and written) take 101 us, 5.2 TB/s; 9909 of 48 of 80 (fp16, three axes) 40 us, 3.8 TB/s;
// 24 tokens 4.8 us, which is the host's time for a call.  Stores that do not stay in the caches make the first 97 us, but attention
// that reads the keys next is slower by more than that (8 prompts of 2000 tokens, append and attend together: 416 us, 407 without).
template <class E, int kLanes>
__global__ __launch_bounds__(256) void append_pieces_kernel(AppendCall c, Rotation rot, int lanes, int per, int slices) {
    typedef typename E::Value V;
    constexpr int kPer = 16 / sizeof(V), kSteps = 2;
    typedef V VP __attribute__((ext_vector_type(16 / sizeof(V))));
    __shared__ __align__(16) float turns[4][2][APPROXIFER_MAX_HEAD_DIM / 2];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + wave, work = c.seq.T * slices;
    if (unit >= work) {                                       // the last waves: statuses
        const int64_t b = unit - work;
        if (c.status != nullptr && b < c.seq.B) append_status(c, static_cast<int>(b));
        return;
    }
    const int L = kLanes > 0 ? kLanes : lanes, groups = kWave / L, group = lane / L, u = lane - group * L;
    const int64_t t = unit / slices;
    const int h0 = static_cast<int>(unit % slices) * per, h1 = min(h0 + per, c.Hq + 2 * c.Hkv);

    // this lane's two pieces
    const int pieces = c.Dh / kPer, apart = c.interleaved ? 0 : c.pairs / kPer;
    int a, b;
    if (u < apart) {
        a = u;
        b = u + apart;
    } else {
        a = 2 * apart + 2 * (u - apart);
        b = a + 1;
    }
    const bool has_a = a < pieces && group < groups, has_b = b < pieces && group < groups;
    const int at_a = (has_a ? a : 0) * kPer, at_b = (has_b ? b : 0) * kPer;

    VP xa[kSteps], xb[kSteps];
    const auto load = [&](int h) {
#pragma unroll
        for (int n = 0; n < kSteps; ++n) {
            const int head = min(h + n * groups + group, h1 - 1);
            const V *x = head < c.Hq           ? static_cast<const V *>(c.q) + t * c.q_stride + static_cast<int64_t>(head) * c.Dh
                         : head < c.Hq + c.Hkv ? static_cast<const V *>(c.k) + t * c.k_stride + static_cast<int64_t>(head - c.Hq) * c.Dh
                                               : static_cast<const V *>(c.v) + t * c.v_stride + static_cast<int64_t>(head - c.Hq - c.Hkv) * c.Dh;
            xa[n] = *reinterpret_cast<const VP *>(x + at_a);
            xb[n] = *reinterpret_cast<const VP *>(x + at_b);
        }
    };
    load(h0);

    const int seq = wave_sequence_of(c.seq, t);
    const Rows r = rows_of(c.seq, seq);
    if (!r.ok || t < r.start || t >= r.start + r.n) return;
    const int place = r.place(static_cast<int>(t - r.start));
    const int page = place >= 0 && h1 > c.Hq ? page_of(c.seq, seq, place) : -1;
    const int size = 1 << c.seq.page_shift;
    const int64_t slot = static_cast<int64_t>(page) * c.Hkv * size + (place & (size - 1));

    float cs[kPer], sn[kPer];
    if (h0 < c.Hq + c.Hkv && c.pairs > 0) {
        for (int i = lane; i < c.pairs; i += kWave) {
            const int position = c.positions != nullptr ? c.positions[t * c.axes + rot.axis[i]] : place;
            angle_of(rot, i, position, &turns[wave][0][i], &turns[wave][1][i]);
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = min(u * kPer + k, c.pairs - 1);
            cs[k] = turns[wave][0][i];
            sn[k] = turns[wave][1][i];
        }
    }
    float wq[2][kPer], wk[2][kPer];
    if (c.q_weight != nullptr) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            wq[0][k] = E::load(static_cast<const V *>(c.q_weight)[at_a + k]);
            wq[1][k] = E::load(static_cast<const V *>(c.q_weight)[at_b + k]);
        }
    }
    if (c.k_weight != nullptr) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            wk[0][k] = E::load(static_cast<const V *>(c.k_weight)[at_a + k]);
            wk[1][k] = E::load(static_cast<const V *>(c.k_weight)[at_b + k]);
        }
    }

    for (int h = h0; h < h1; h += kSteps * groups) {
        VP ya[kSteps], yb[kSteps];
#pragma unroll
        for (int n = 0; n < kSteps; ++n) {
            ya[n] = xa[n];
            yb[n] = xb[n];
        }
        if (h + kSteps * groups < h1) load(h + kSteps * groups);
#pragma unroll
        for (int n = 0; n < kSteps; ++n) {
            if (h + n * groups >= h1) break;
            const int head = h + n * groups + group;
            const bool is_q = head < c.Hq, is_v = head >= c.Hq + c.Hkv;
            VP za = ya[n], zb = yb[n];
            if (h + n * groups < c.Hq + c.Hkv) {              // not values only
                float p[kPer], q[kPer];
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    p[k] = E::load(za[k]);
                    q[k] = E::load(zb[k]);
                }
                if (c.q_weight != nullptr || c.k_weight != nullptr) {
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < kPer; ++k) sum += has_a ? p[k] * p[k] : 0.0f;
#pragma unroll
                    for (int k = 0; k < kPer; ++k) sum += has_b ? q[k] * q[k] : 0.0f;
                    const float all = kLanes > 0 ? lanes_sum<kLanes>(sum) : group_sum(sum, group * L, u, L);
                    if ((is_q ? c.q_weight : c.k_weight) != nullptr) {
                        const float scale = 1.0f / sqrtf(all / c.Dh + c.eps);
#pragma unroll
                        for (int k = 0; k < kPer; ++k) {
                            p[k] *= scale * (is_q ? wq[0][k] : wk[0][k]);
                            q[k] *= scale * (is_q ? wq[1][k] : wk[1][k]);
                        }
                    }
                }
                if (c.interleaved) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {          // pair u kPer + k: in the first piece, then in the second
                        float &f = k < kPer / 2 ? p[2 * k] : q[2 * k - kPer], &g = k < kPer / 2 ? p[2 * k + 1] : q[2 * k - kPer + 1];
                        const float x = f, y = g;
                        const bool turned = u * kPer + k < c.pairs;
                        f = turned ? x * cs[k] - y * sn[k] : x;
                        g = turned ? x * sn[k] + y * cs[k] : y;
                    }
                } else if (u < apart) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {
                        const float x = p[k], y = q[k];
                        p[k] = x * cs[k] - y * sn[k];
                        q[k] = x * sn[k] + y * cs[k];
                    }
                }
                if (!is_v) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {
                        za[k] = E::store(p[k]);
                        zb[k] = E::store(q[k]);
                    }
                }
            }
            if (head >= h1) continue;
            V *y = nullptr;
            if (is_q) {
                y = static_cast<V *>(c.q_out) + (t * c.Hq + head) * c.Dh;
            } else if (page >= 0) {
                const int kv = head - (is_v ? c.Hq + c.Hkv : c.Hq);
                y = static_cast<V *>(is_v ? c.v_pool : c.k_pool) + (slot + static_cast<int64_t>(kv) * size) * c.Dh;
            }
            if (y == nullptr) continue;
            if (has_a) *reinterpret_cast<VP *>(y + at_a) = za;
            if (has_b) *reinterpret_cast<VP *>(y + at_b) = zb;
        }
    }
}

template <class E, int kLanes>
hipError_t launch_pieces(const AppendCall &c, const Rotation &rot, int lanes, hipStream_t stream) {
    const int heads = c.Hq + 2 * c.Hkv, groups = kWave / lanes;
    // enough waves to fill the GPU, `groups` heads each at the least; beyond that whole tokens
    int64_t slices = (8192 + c.seq.T - 1) / (c.seq.T > 0 ? c.seq.T : 1);
    const int most = (heads + groups - 1) / groups;
    slices = slices < most ? slices : most;
    const int per = static_cast<int>(((heads + slices - 1) / slices + groups - 1) / groups * groups);
    slices = (heads + per - 1) / per;
    const int64_t units = c.seq.T * slices + (c.status != nullptr ? c.seq.B : 0);
    return launch_kernel(append_pieces_kernel<E, kLanes>, dim3(static_cast<unsigned>((units + 3) / 4)), dim3(256), 0, stream, c, rot, lanes,
                         per, static_cast<int>(slices));
}
template <class E>
hipError_t launch_pieces_of(const AppendCall &c, const Rotation &rot, hipStream_t stream) {
    constexpr int kPer = 16 / sizeof(typename E::Value);
    const int pieces = c.Dh / kPer, apart = c.interleaved ? 0 : c.pairs / kPer, lanes = apart + (pieces - 2 * apart + 1) / 2;
    switch (lanes) {
        case 4: return launch_pieces<E, 4>(c, rot, lanes, stream);
        case 8: return launch_pieces<E, 8>(c, rot, lanes, stream);
        case 16: return launch_pieces<E, 16>(c, rot, lanes, stream);
        case 32: return launch_pieces<E, 32>(c, rot, lanes, stream);
        default: return launch_pieces<E, 0>(c, rot, lanes, stream);
    }
}

// Heads element by element, for rows that do not begin at 16 bytes and halves that are no whole pieces.  One wave per head of a token: queries,
// keys, then values; behind the T tokens a wave per sequence for the status.
template <class E>
__global__ __launch_bounds__(kWave) void append_kernel(AppendCall c, Rotation rot) {
    typedef typename E::Value V;
    const int heads = c.Hq + 2 * c.Hkv, lane = lane_id();
    const int64_t t = blockIdx.x;
    int h = blockIdx.y;
    if (t >= c.seq.T) {                                       // the last blocks: statuses
        const int64_t b = (t - c.seq.T) * heads + h;
        if (c.status == nullptr || b >= c.seq.B) return;
        append_status(c, static_cast<int>(b));
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
    const int per = dtype == APPROXIFER_F32 ? 4 : 8;
    const auto whole = [&](const void *p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % per == 0; };
    if (s.T > 0 && whole(q, q_stride) && whole(k, k_stride) && whole(v, v_stride) && (interleaved || pairs % per == 0))
        return launch_status(dtype == APPROXIFER_F32   ? launch_pieces_of<F32>(c, rot, stream)
                             : dtype == APPROXIFER_F16 ? launch_pieces_of<F16>(c, rot, stream)
                                                       : launch_pieces_of<BF16>(c, rot, stream));
    const int heads = Hq + 2 * Hkv;
    const int64_t blocks = s.T + (status != nullptr ? (s.B + heads - 1) / heads : 0);
    const dim3 grid(static_cast<unsigned>(blocks), heads), block(kWave);
    const auto kernel = dtype == APPROXIFER_F32 ? append_kernel<F32> : dtype == APPROXIFER_F16 ? append_kernel<F16> : append_kernel<BF16>;
    return launch_status(launch_kernel(kernel, grid, block, 0, stream, c, rot));
}

}  // namespace approxifer
