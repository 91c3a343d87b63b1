// Sequences kept in pages: what the append, attention and page kernels share.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "common.h"

namespace approxifer {

// The caller's descriptor as kernels take it; sizes are below 2^31 (checked on the host).
struct Sequences {
    const int32_t *table, *lens, *starts;
    int64_t T;
    int B, M, P;
    int page_shift;                                           // tokens per page = 1 << page_shift
};

// One element of each type, to and from float32: to the nearest, ties to even.
struct F32 {
    typedef float Value;
    static __device__ __forceinline__ float load(Value v) { return v; }
    static __device__ __forceinline__ Value store(float v) { return v; }
};
struct F16 {
    typedef _Float16 Value;
    static __device__ __forceinline__ float load(Value v) { return static_cast<float>(v); }
    static __device__ __forceinline__ Value store(float v) { return static_cast<Value>(v); }
};
struct BF16 {
    typedef __bf16 Value;
    static __device__ __forceinline__ float load(Value v) { return static_cast<float>(v); }
    static __device__ __forceinline__ Value store(float v) { return static_cast<Value>(v); }
};

// The new tokens of one sequence.
struct Rows {
    int b;
    int64_t start;                                            // row of the first of them
    int n, length;                                            // how many, and the sequence's length with them
    bool ok;                                                  // rows inside 0..T, length inside 0..M page
    __device__ __forceinline__ int place(int i) const { return length - n + i; }
};

__device__ __forceinline__ Rows rows_of(const Sequences &s, int b) {
    const int64_t r0 = s.starts[b], r1 = s.starts[b + 1];
    const int length = s.lens[b];
    Rows r;
    r.b = b;
    r.start = r0;
    r.length = length;
    r.ok = r0 >= 0 && r0 <= r1 && r1 <= s.T && length >= 0 && length <= (static_cast<int64_t>(s.M) << s.page_shift);
    r.n = r.ok ? static_cast<int>(r1 - r0) : 0;
    return r;
}

// The sequence that row t belongs to: the last whose rows begin at t or before.  Whatever starts holds, the search ends at one
// of the B sequences; rows_of() says whether it holds the row.
__device__ __forceinline__ int sequence_of(const Sequences &s, int64_t t) {
    int lo = 0, hi = s.B;                                     // starts[lo] <= t is assumed, starts[hi] > t
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (s.starts[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The page of a place, or -1.
__device__ __forceinline__ int page_of(const Sequences &s, int b, int place) {
    const int p = s.table[static_cast<int64_t>(b) * s.M + (place >> s.page_shift)];
    return p >= 0 && p < s.P ? p : -1;
}

// One wave: the status of sequence b for a call that needs the pages of places [a0, a1) and [b0, b1).
__device__ __forceinline__ int pages_status(const Sequences &s, int b, int a0, int a1, int b0, int b1) {
    bool bad = false;
    const int32_t *row = s.table + static_cast<int64_t>(b) * s.M;
    for (int part = 0; part < 2; ++part) {
        const int from = part ? b0 : a0, to = part ? b1 : a1;
        if (from >= to) continue;
        const int last = (to - 1) >> s.page_shift;
        for (int j = (from >> s.page_shift) + lane_id(); j <= last; j += kWave) bad |= row[j] < 0 || row[j] >= s.P;
    }
    return __any(bad) ? APPROXIFER_SEQUENCE_BAD_PAGE : APPROXIFER_GROUP_OK;
}

int launch_append(const Sequences &s, int Hq, int Hkv, int Dh, int dtype, const void *q, int64_t q_stride, const void *k,
                  int64_t k_stride, const void *v, int64_t v_stride, void *q_out, void *k_pool, void *v_pool,
                  const void *q_weight, const void *k_weight, double eps, const int32_t *positions, int axes,
                  const double *h_freq, const int32_t *h_axis, int pairs, bool interleaved, int32_t *status, hipStream_t stream);

struct AttendCall {
    Sequences seq;
    int Hq, Hkv, Dh, dtype;
    const void *q;
    int64_t q_stride;
    const void *k_pool, *v_pool;
    void *out;
    int32_t *status;
    int max_rows, max_len, window, sinks;                     // window: 0 no limit
    float scale;
    float *stats = nullptr;                                   // [Hq][T][2], or null: of every row what RowStats says
    float *scores = nullptr;                                  // [T][Hq][score_stride]: q . k of every key that is looked at, if they are kept
    int64_t score_stride = 0;
};
// Of a row that attention has settled: what its weights are relative to (of c S, base 2), and the inverse of their sum.
struct RowStats {
    float base, inverse;
    __device__ __forceinline__ RowStats(float top, float total)
        : base(top == -INFINITY ? 0.0f : top), inverse(total == 0.0f ? 0.0f : 1.0f / total) {}
    __device__ __forceinline__ void store(const AttendCall &c, int64_t t, int head) const {
        float *const at = c.stats + 2 * (head * c.seq.T + t);
        at[0] = base;
        at[1] = inverse;
    }
};
int launch_attend(const AttendCall &c, void *workspace, size_t workspace_bytes, hipStream_t stream);
int launch_attend_shared(const AttendCall &c, const int32_t *groups, const int32_t *shared, int64_t C, int64_t max_shared, void *workspace,
                         size_t workspace_bytes, hipStream_t stream);
size_t attend_shared_workspace_bytes(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                                     int64_t max_shared, int64_t window, int64_t sinks);
bool attend_shared_pays(int64_t T, int64_t B, int64_t C, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                        int64_t max_shared, int64_t window, int64_t sinks, int page_shift);
int launch_attend_mass(AttendCall c, float *mass, int64_t mass_stride, void *workspace, size_t workspace_bytes, hipStream_t stream);
size_t attend_mass_least_bytes(int64_t T, int Hq);
size_t attend_mass_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                                   int64_t window, int64_t sinks);
size_t attend_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                              int64_t window, int64_t sinks);

int launch_cache_reserve(int32_t *table, int32_t *lens, int32_t *refs, const int32_t *add, int32_t *status, int B, int M, int P,
                         int page_shift, hipStream_t stream);
int launch_cache_fork(const int32_t *table, const int32_t *lens, const int32_t *refs, const int32_t *parents,
                      const int32_t *keep, int32_t *table_out, int32_t *lens_out, int32_t *refs_out, int32_t *status,
                      void *pools, int64_t planes, int64_t page_bytes, int B, int B_out, int M, int P, int page_shift,
                      void *workspace, hipStream_t stream);
int launch_cache_compact(int32_t *table, const int32_t *lens, int32_t *refs, int32_t *moved, int32_t *live, void *pools,
                         int64_t planes, int64_t page_bytes, int B, int M, int P, int page_shift, void *workspace,
                         hipStream_t stream);
size_t cache_workspace_bytes(int64_t B, int64_t B_out, int64_t P);
int launch_cache_evict(int32_t *table, int32_t *lens, int32_t *refs, float *mass, int64_t mass_stride, int32_t *kept, int32_t *status,
                       void *pools, int64_t planes, int64_t heads, int64_t row_bytes, int B, int M, int P, int page_shift, int budget,
                       int first, int recent, void *workspace, hipStream_t stream);
size_t evict_workspace_bytes(int64_t B, int64_t budget, int64_t P, int page_shift);

}  // namespace approxifer
