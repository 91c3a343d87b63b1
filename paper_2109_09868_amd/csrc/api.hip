// C ABI of the ApproxIFER coding layer: argument validation on the host, then one kernel
// launch on the caller's stream.  See include/approxifer.h for the contract.
#include <cmath>

#include "sequences.h"

using approxifer::Nodes;

namespace {

constexpr double kPi = 3.14159265358979323846264338327950288;

int check_nodes(const double *h, int n) {
    bool rising = true, falling = true;
    for (int i = 0; i < n; ++i) {
        if (!std::isfinite(h[i])) return APPROXIFER_ERR_BAD_NODES;
        if (i > 0) {
            rising = rising && h[i] > h[i - 1];
            falling = falling && h[i] < h[i - 1];
        }
    }
    if (rising || falling) return APPROXIFER_OK;          // as node generators list them: distinct without comparing pairs
    for (int i = 0; i < n; ++i)
        for (int k = 0; k < i; ++k)
            if (h[k] == h[i]) return APPROXIFER_ERR_BAD_NODES;
    return APPROXIFER_OK;
}

int check_common(int K, int N, const double *h_alpha, const double *h_beta, Nodes *nodes) {
    if (h_alpha == nullptr || h_beta == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    if (K < 1 || N < 2) return APPROXIFER_ERR_BAD_SHAPE;
    if (K > APPROXIFER_MAX_K || N > APPROXIFER_MAX_N) return APPROXIFER_ERR_LIMIT;
    int rc = check_nodes(h_alpha, K);
    if (rc != APPROXIFER_OK) return rc;
    rc = check_nodes(h_beta, N);
    if (rc != APPROXIFER_OK) return rc;
    for (int j = 0; j < APPROXIFER_MAX_K; ++j) nodes->alpha[j] = j < K ? h_alpha[j] : 0.0;
    for (int i = 0; i < APPROXIFER_MAX_N; ++i) nodes->beta[i] = i < N ? h_beta[i] : 0.0;
    return APPROXIFER_OK;
}

// Sizes of a cache; *shift: log2 of the page.
int check_cache(int64_t B, int64_t M, int64_t P, int page, int *shift) {
    if (B < 0 || M < 1 || P < 1 || page < 1 || (page & (page - 1)) != 0) return APPROXIFER_ERR_BAD_CACHE;
    if (page > APPROXIFER_MAX_PAGE || B > APPROXIFER_MAX_SEQUENCES || P > APPROXIFER_MAX_PAGES || M > APPROXIFER_MAX_TOKENS / page)
        return APPROXIFER_ERR_LIMIT;
    *shift = __builtin_ctz(static_cast<unsigned>(page));
    return APPROXIFER_OK;
}

bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_sequences(const approxifer_sequences *h, int Hq, int Hkv, int Dh, int dtype, approxifer::Sequences *s) {
    if (h == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    if (h->T < 0 || Hkv < 1 || Hq < 1 || Hq % Hkv != 0 || Dh < 1 || Dh % 8 != 0) return APPROXIFER_ERR_BAD_CACHE;
    if (dtype != APPROXIFER_F32 && dtype != APPROXIFER_F16 && dtype != APPROXIFER_BF16) return APPROXIFER_ERR_BAD_DTYPE;
    int shift = 0;
    const int rc = check_cache(h->B, h->M, h->P, h->page, &shift);
    if (rc != APPROXIFER_OK) return rc;
    if (h->T > APPROXIFER_MAX_ROWS || Hq > APPROXIFER_MAX_HEADS || Dh > APPROXIFER_MAX_HEAD_DIM) return APPROXIFER_ERR_LIMIT;
    if (h->T * Hq > (1LL << 30) || h->B * Hkv > (1LL << 22)) return APPROXIFER_ERR_LIMIT;    // workgroups of one launch
    *s = approxifer::Sequences{h->d_table, h->d_lens, h->d_starts, h->T, static_cast<int>(h->B), static_cast<int>(h->M),
                               static_cast<int>(h->P), shift};
    return APPROXIFER_OK;
}

// Rows of `values` elements, `stride` elements apart: whether they can be read element by element.
int check_rows(const void *p, int64_t stride, int64_t values, int dtype) {
    if (stride < values || stride > (1LL << 31)) return APPROXIFER_ERR_BAD_SHAPE;
    return aligned(p, dtype == APPROXIFER_F32 ? 4 : 2) ? APPROXIFER_OK : APPROXIFER_ERR_ALIGNMENT;
}

int check_pools(const void *d_pools, int64_t planes, int64_t page_bytes, int64_t P) {
    if (planes < 0 || page_bytes < 0) return APPROXIFER_ERR_BAD_SHAPE;
    if (planes == 0 || page_bytes == 0) return APPROXIFER_OK;
    if (planes > (1 << 20) || page_bytes > (1LL << 31) || P * page_bytes > (1LL << 48) / planes) return APPROXIFER_ERR_LIMIT;
    if (d_pools == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return aligned(d_pools, 16) && page_bytes % 16 == 0 ? APPROXIFER_OK : APPROXIFER_ERR_ALIGNMENT;
}

}  // namespace

extern "C" {

int approxifer_version(void) { return 400; }   // 0.4.0: sequences in pages

const char *approxifer_strerror(int code) {
    switch (code) {
        case APPROXIFER_OK: return "ok";
        case APPROXIFER_ERR_NULL_POINTER: return "a required pointer is NULL";
        case APPROXIFER_ERR_BAD_SHAPE: return "bad shape: need G,D,C >= 0, K >= 1, N >= 2, -1 <= S < N, A >= 1";
        case APPROXIFER_ERR_LIMIT: return "size above the compiled limits (K <= 64, N <= 128, N-S <= 64 for the Byzantine decoder)";
        case APPROXIFER_ERR_BAD_NODES: return "nodes must be finite and pairwise distinct within each set";
        case APPROXIFER_ERR_TOO_FEW_WORKERS: return "the Byzantine decoder needs N - S >= 2 (K + A) available workers";
        case APPROXIFER_ERR_BAD_SIGN_MODE: return "sign_mode must be 0 (worker index) or 1 (survivor rank)";
        case APPROXIFER_ERR_LAUNCH: return "the HIP runtime refused the kernel launch";
        case APPROXIFER_ERR_WORKSPACE_LIMIT:
            return "the shape needs more scratch memory than the built-in workspace holds (APPROXIFER_STATIC_WORKSPACE_BYTES); "
                   "use approxifer_decode_byzantine with a workspace of approxifer_workspace_bytes()";
        case APPROXIFER_ERR_BAD_DTYPE: return "dtype must be APPROXIFER_F32, APPROXIFER_F16 or APPROXIFER_BF16";
        case APPROXIFER_ERR_ALIGNMENT: return "pools, outputs and workspaces must be 16-byte aligned, rows aligned to their type";
        case APPROXIFER_ERR_BAD_CACHE:
            return "bad cache: need T, B >= 0, M, P >= 1, a page that is a power of two, Dh a positive multiple of 8, Hq a positive "
                   "multiple of Hkv";
        case APPROXIFER_ERR_WORKSPACE: return "the call needs a workspace of approxifer_cache_workspace_bytes()";
        default: return "unknown approxifer error code";
    }
}

int approxifer_chebyshev_nodes(int K, int N, double *h_alpha, double *h_beta) {
    if (h_alpha == nullptr || h_beta == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    if (K < 1 || N < 2) return APPROXIFER_ERR_BAD_SHAPE;
    for (int j = 0; j < K; ++j) h_alpha[j] = std::cos((2.0 * j + 1.0) * kPi / (2.0 * K));
    for (int i = 0; i < N; ++i) h_beta[i] = std::cos(i * kPi / (N - 1.0));
    return APPROXIFER_OK;
}

int approxifer_encode(const float *d_queries, float *d_coded, int64_t G, int K, int N, int64_t D,
                      const double *h_alpha, const double *h_beta, void *stream) {
    if (G < 0 || D < 0) return APPROXIFER_ERR_BAD_SHAPE;
    Nodes nodes;
    const int rc = check_common(K, N, h_alpha, h_beta, &nodes);
    if (rc != APPROXIFER_OK) return rc;
    if (G == 0 || D == 0) return APPROXIFER_OK;
    if (d_queries == nullptr || d_coded == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_encode(d_queries, d_coded, G, K, N, D, nodes, static_cast<hipStream_t>(stream));
}

int64_t approxifer_group_count(int64_t Q, int K) {
    if (Q < 0 || K < 1) return -1;
    return (Q + K - 1) / K;
}

int approxifer_pad_last_group(float *d_queries, int64_t Q, int K, int64_t D, void *stream) {
    if (Q < 0 || D < 0 || K < 1) return APPROXIFER_ERR_BAD_SHAPE;
    if (K > APPROXIFER_MAX_K) return APPROXIFER_ERR_LIMIT;
    if (Q == 0 || D == 0 || Q % K == 0) return APPROXIFER_OK;
    if (d_queries == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_pad_last_group(d_queries, Q, K, D, static_cast<hipStream_t>(stream));
}

int approxifer_decode(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_status, int64_t G, int K,
                      int N, int S, int64_t C, const double *h_alpha, const double *h_beta, int sign_mode,
                      void *stream) {
    if (G < 0 || C < 0) return APPROXIFER_ERR_BAD_SHAPE;
    Nodes nodes;
    const int rc = check_common(K, N, h_alpha, h_beta, &nodes);
    if (rc != APPROXIFER_OK) return rc;
    if (S < APPROXIFER_S_FROM_MASK || S >= N) return APPROXIFER_ERR_BAD_SHAPE;
    if (sign_mode != APPROXIFER_SIGN_WORKER_INDEX && sign_mode != APPROXIFER_SIGN_SURVIVOR_RANK)
        return APPROXIFER_ERR_BAD_SIGN_MODE;
    if (G == 0 || C == 0) return APPROXIFER_OK;
    if (d_mask == nullptr || d_preds == nullptr || d_out == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_decode(d_preds, d_mask, d_out, d_status, G, K, N, S, C, nodes, sign_mode,
                                     static_cast<hipStream_t>(stream));
}

int approxifer_decode_top1(const float *d_preds, const uint8_t *d_mask, int32_t *d_top1, float *d_score,
                           int32_t *d_status, int64_t G, int K, int N, int S, int64_t C, const double *h_alpha,
                           const double *h_beta, int sign_mode, void *stream) {
    if (G < 0 || C < 0) return APPROXIFER_ERR_BAD_SHAPE;
    Nodes nodes;
    const int rc = check_common(K, N, h_alpha, h_beta, &nodes);
    if (rc != APPROXIFER_OK) return rc;
    if (S < APPROXIFER_S_FROM_MASK || S >= N) return APPROXIFER_ERR_BAD_SHAPE;
    if (sign_mode != APPROXIFER_SIGN_WORKER_INDEX && sign_mode != APPROXIFER_SIGN_SURVIVOR_RANK)
        return APPROXIFER_ERR_BAD_SIGN_MODE;
    if (C > 0x7fffffffLL) return APPROXIFER_ERR_LIMIT;   // class indices are int32
    if (G == 0 || C == 0) return APPROXIFER_OK;
    if (d_mask == nullptr || d_preds == nullptr || d_top1 == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_decode_top1(d_preds, d_mask, d_top1, d_score, d_status, G, K, N, S, C, nodes,
                                          sign_mode, static_cast<hipStream_t>(stream));
}

static int decode_byzantine_checked(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_adv,
                                    int32_t *d_status, int64_t G, int K, int N, int S, int A, int64_t C,
                                    const double *h_alpha, const double *h_beta, int sign_mode, bool homogeneous,
                                    void *d_workspace, size_t workspace_bytes, void *stream) {
    if (G < 0 || C < 0) return APPROXIFER_ERR_BAD_SHAPE;
    Nodes nodes;
    const int rc = check_common(K, N, h_alpha, h_beta, &nodes);
    if (rc != APPROXIFER_OK) return rc;
    if (S < APPROXIFER_S_FROM_MASK || S >= N || A < 1) return APPROXIFER_ERR_BAD_SHAPE;
    if (sign_mode != APPROXIFER_SIGN_WORKER_INDEX && sign_mode != APPROXIFER_SIGN_SURVIVOR_RANK)
        return APPROXIFER_ERR_BAD_SIGN_MODE;
    const int most_available = S < 0 ? N : N - S;
    if (most_available < 2 * (K + A)) return APPROXIFER_ERR_TOO_FEW_WORKERS;
    if (S >= 0 && N - S > APPROXIFER_MAX_AVAIL_BYZ) return APPROXIFER_ERR_LIMIT;
    if (G == 0 || C == 0) return APPROXIFER_OK;
    if (d_mask == nullptr || d_adv == nullptr || d_preds == nullptr || d_out == nullptr)
        return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_decode_byzantine(d_preds, d_mask, d_out, d_adv, d_status, G, K, N, S, A, C, nodes,
                                               sign_mode, homogeneous, d_workspace, workspace_bytes,
                                               static_cast<hipStream_t>(stream));
}

int approxifer_decode_byzantine(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_adv,
                                int32_t *d_status, int64_t G, int K, int N, int S, int A, int64_t C,
                                const double *h_alpha, const double *h_beta, int sign_mode, void *d_workspace,
                                size_t workspace_bytes, void *stream) {
    return decode_byzantine_checked(d_preds, d_mask, d_out, d_adv, d_status, G, K, N, S, A, C, h_alpha, h_beta,
                                    sign_mode, false, d_workspace, workspace_bytes, stream);
}

int approxifer_decode_byzantine_homogeneous(const float *d_preds, const uint8_t *d_mask, float *d_out,
                                            int32_t *d_adv, int32_t *d_status, int64_t G, int K, int N, int S,
                                            int A, int64_t C, const double *h_alpha, const double *h_beta,
                                            int sign_mode, void *d_workspace, size_t workspace_bytes, void *stream) {
    return decode_byzantine_checked(d_preds, d_mask, d_out, d_adv, d_status, G, K, N, S, A, C, h_alpha, h_beta,
                                    sign_mode, true, d_workspace, workspace_bytes, stream);
}

int approxifer_decode_rational(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_status, int64_t G,
                               int K, int N, int S, int A, int64_t C, const double *h_alpha, const double *h_beta,
                               void *stream) {
    if (G < 0 || C < 0) return APPROXIFER_ERR_BAD_SHAPE;
    Nodes nodes;
    const int rc = check_common(K, N, h_alpha, h_beta, &nodes);
    if (rc != APPROXIFER_OK) return rc;
    if (S < APPROXIFER_S_FROM_MASK || S >= N || A < 1) return APPROXIFER_ERR_BAD_SHAPE;
    const int most_available = S < 0 ? N : N - S;
    if (most_available < 2 * (K + A)) return APPROXIFER_ERR_TOO_FEW_WORKERS;
    if (S >= 0 && N - S > APPROXIFER_MAX_AVAIL_BYZ) return APPROXIFER_ERR_LIMIT;
    if (G == 0 || C == 0) return APPROXIFER_OK;
    if (d_mask == nullptr || d_preds == nullptr || d_out == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_decode_rational(d_preds, d_mask, d_out, d_status, G, K, N, S, A, C, nodes,
                                              static_cast<hipStream_t>(stream));
}

static size_t workspace_bytes_of(int64_t G, int K, int N, int S, int A, int64_t C, bool pairs) {
    // the shapes the Byzantine decoders accept; anything else needs no workspace because the call is refused
    if (G <= 0 || C <= 0 || K < 1 || K > APPROXIFER_MAX_K || N < 2 || N > APPROXIFER_MAX_N) return 0;
    if (S < APPROXIFER_S_FROM_MASK || S >= N || A < 1) return 0;
    const int most_available = S < 0 ? N : N - S;
    if (most_available < 2 * (K + A) || (S >= 0 && N - S > APPROXIFER_MAX_AVAIL_BYZ)) return 0;
    return approxifer::byzantine_workspace_bytes(G, K, N, S, A, C, pairs);
}

int approxifer_decode_byzantine_static(const float *d_preds, const uint8_t *d_mask, float *d_out, int32_t *d_adv,
                                       int32_t *d_status, int64_t G, int K, int N, int S, int A, int64_t C,
                                       const double *h_alpha, const double *h_beta, int sign_mode, void *stream) {
    // shapes the decoder refuses are refused by the checked call below with their own codes (need is 0 for them)
    size_t need = workspace_bytes_of(G, K, N, S, A, C, true);
    if (need > APPROXIFER_STATIC_WORKSPACE_BYTES) need = workspace_bytes_of(G, K, N, S, A, C, false);
    if (need > APPROXIFER_STATIC_WORKSPACE_BYTES) return APPROXIFER_ERR_WORKSPACE_LIMIT;
    void *d_scratch = nullptr;
    if (need > 0) {
        const int rc = approxifer::static_workspace(&d_scratch);
        if (rc != APPROXIFER_OK) return rc;
    }
    return decode_byzantine_checked(d_preds, d_mask, d_out, d_adv, d_status, G, K, N, S, A, C, h_alpha, h_beta,
                                    sign_mode, false, d_scratch, need, stream);
}

size_t approxifer_workspace_bytes(int64_t G, int K, int N, int S, int A, int64_t C) {
    return workspace_bytes_of(G, K, N, S, A, C, true);
}

int approxifer_top1(const float *d_values, int32_t *d_top1, float *d_score, int64_t rows, int64_t C, void *stream) {
    if (rows < 0 || C < 0) return APPROXIFER_ERR_BAD_SHAPE;
    if (C > 0x7fffffffLL) return APPROXIFER_ERR_LIMIT;   // class indices are int32
    if (rows == 0 || C == 0) return APPROXIFER_OK;
    if (d_values == nullptr || d_top1 == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_argmax_rows(d_values, d_top1, d_score, rows, C, static_cast<hipStream_t>(stream));
}

int approxifer_wait_mask(const float *d_arrival, uint8_t *d_mask, int32_t *d_count, int64_t G, int N, int wait_for,
                         void *stream) {
    if (G < 0 || N < 1 || wait_for < 1 || wait_for > N) return APPROXIFER_ERR_BAD_SHAPE;
    if (N > APPROXIFER_MAX_N) return APPROXIFER_ERR_LIMIT;
    if (G == 0) return APPROXIFER_OK;
    if (d_arrival == nullptr || d_mask == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_wait_mask(d_arrival, d_mask, d_count, G, N, wait_for, static_cast<hipStream_t>(stream));
}

int approxifer_rotary_frequencies(int pairs, double base, double *h_freq) {
    if (h_freq == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    if (pairs < 1 || !std::isfinite(base) || base <= 0.0) return APPROXIFER_ERR_BAD_SHAPE;
    for (int i = 0; i < pairs; ++i) h_freq[i] = std::pow(base, -static_cast<double>(i) / pairs);
    return APPROXIFER_OK;
}

int approxifer_append(const approxifer_sequences *h_seq, int Hq, int Hkv, int Dh, int dtype, const void *d_q, int64_t q_stride,
                      const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride, void *d_q_out, void *d_k_pool,
                      void *d_v_pool, const void *d_q_weight, const void *d_k_weight, double eps, const int32_t *d_positions,
                      int axes, const double *h_freq, const int32_t *h_axis, int pairs, int interleaved, int32_t *d_status,
                      void *stream) {
    approxifer::Sequences s;
    int rc = check_sequences(h_seq, Hq, Hkv, Dh, dtype, &s);
    if (rc != APPROXIFER_OK) return rc;
    if (pairs < 0 || 2 * static_cast<int64_t>(pairs) > Dh || axes < 1 || (d_positions == nullptr && axes != 1) || !std::isfinite(eps) ||
        eps < 0.0)
        return APPROXIFER_ERR_BAD_SHAPE;
    if (axes > APPROXIFER_MAX_AXES) return APPROXIFER_ERR_LIMIT;
    if (pairs > 0 && h_freq == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    for (int i = 0; i < pairs; ++i) {
        if (!std::isfinite(h_freq[i])) return APPROXIFER_ERR_BAD_NODES;
        if (h_axis != nullptr && (h_axis[i] < 0 || h_axis[i] >= axes)) return APPROXIFER_ERR_BAD_SHAPE;
    }
    if (s.B == 0 && s.T > 0) return APPROXIFER_ERR_BAD_CACHE;
    if (s.B == 0) return APPROXIFER_OK;
    if (s.table == nullptr || s.lens == nullptr || s.starts == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    if (s.T == 0 && d_status == nullptr) return APPROXIFER_OK;
    if (s.T > 0) {
        if (d_q == nullptr || d_k == nullptr || d_v == nullptr || d_q_out == nullptr || d_k_pool == nullptr || d_v_pool == nullptr)
            return APPROXIFER_ERR_NULL_POINTER;
        if ((rc = check_rows(d_q, q_stride, static_cast<int64_t>(Hq) * Dh, dtype)) != APPROXIFER_OK ||
            (rc = check_rows(d_k, k_stride, static_cast<int64_t>(Hkv) * Dh, dtype)) != APPROXIFER_OK ||
            (rc = check_rows(d_v, v_stride, static_cast<int64_t>(Hkv) * Dh, dtype)) != APPROXIFER_OK)
            return rc;
        if (!aligned(d_q_out, 16) || !aligned(d_k_pool, 16) || !aligned(d_v_pool, 16) || !aligned(d_q_weight, dtype == APPROXIFER_F32 ? 4 : 2) ||
            !aligned(d_k_weight, dtype == APPROXIFER_F32 ? 4 : 2))
            return APPROXIFER_ERR_ALIGNMENT;
    }
    return approxifer::launch_append(s, Hq, Hkv, Dh, dtype, d_q, q_stride, d_k, k_stride, d_v, v_stride, d_q_out, d_k_pool, d_v_pool,
                                     d_q_weight, d_k_weight, eps, d_positions, axes, h_freq, h_axis, pairs, interleaved != 0, d_status,
                                     static_cast<hipStream_t>(stream));
}

int approxifer_attend(const approxifer_sequences *h_seq, int Hq, int Hkv, int Dh, int dtype, const void *d_q, int64_t q_stride,
                      const void *d_k_pool, const void *d_v_pool, void *d_out, int64_t max_rows, int64_t max_len, int64_t window,
                      int64_t sinks, double scale, int32_t *d_status, void *d_workspace, size_t workspace_bytes, void *stream) {
    approxifer::AttendCall c;
    int rc = check_sequences(h_seq, Hq, Hkv, Dh, dtype, &c.seq);
    if (rc != APPROXIFER_OK) return rc;
    if (max_rows < 0 || max_len < 0 || window < 0 || sinks < 0 || !(std::fabs(scale) <= 0x1p126)) return APPROXIFER_ERR_BAD_SHAPE;
    if (c.seq.B == 0 && c.seq.T > 0) return APPROXIFER_ERR_BAD_CACHE;
    if (c.seq.B == 0) return APPROXIFER_OK;
    if (c.seq.table == nullptr || c.seq.lens == nullptr || c.seq.starts == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    if (c.seq.T == 0 && d_status == nullptr) return APPROXIFER_OK;
    if (c.seq.T > 0) {
        if (d_q == nullptr || d_k_pool == nullptr || d_v_pool == nullptr || d_out == nullptr) return APPROXIFER_ERR_NULL_POINTER;
        if ((rc = check_rows(d_q, q_stride, static_cast<int64_t>(Hq) * Dh, dtype)) != APPROXIFER_OK) return rc;
        if (!aligned(d_out, 16) || !aligned(d_k_pool, 16) || !aligned(d_v_pool, 16)) return APPROXIFER_ERR_ALIGNMENT;
        if (d_workspace != nullptr && !aligned(d_workspace, 16)) return APPROXIFER_ERR_ALIGNMENT;
    }
    const int64_t most = h_seq->M * h_seq->page;              // no sequence is longer, no window reaches further
    c.Hq = Hq;
    c.Hkv = Hkv;
    c.Dh = Dh;
    c.dtype = dtype;
    c.q = d_q;
    c.q_stride = q_stride;
    c.k_pool = d_k_pool;
    c.v_pool = d_v_pool;
    c.out = d_out;
    c.status = d_status;
    c.max_rows = static_cast<int>(max_rows < c.seq.T ? max_rows : c.seq.T);
    c.max_len = static_cast<int>(max_len < most ? max_len : most);
    c.window = static_cast<int>(window < most ? window : 0);
    c.sinks = c.window == 0 ? 0 : static_cast<int>(sinks < most ? sinks : most);
    c.scale = static_cast<float>(scale);
    return approxifer::launch_attend(c, d_workspace, d_workspace != nullptr ? workspace_bytes : 0, static_cast<hipStream_t>(stream));
}

size_t approxifer_attend_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                                         int64_t window, int64_t sinks) {
    if (T < 1 || T > APPROXIFER_MAX_ROWS || B < 1 || B > APPROXIFER_MAX_SEQUENCES || Hkv < 1 || Hq < 1 || Hq % Hkv != 0 ||
        Hq > APPROXIFER_MAX_HEADS || Dh < 1 || Dh % 8 != 0 || Dh > APPROXIFER_MAX_HEAD_DIM || dtype < APPROXIFER_F32 ||
        dtype > APPROXIFER_BF16 || max_rows < 1 || max_len < 1 || window < 0 || sinks < 0 || T * Hq > (1LL << 30) ||
        B * Hkv > (1LL << 22))
        return 0;
    const int64_t most = APPROXIFER_MAX_TOKENS;               // no sequence is longer
    return approxifer::attend_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len < most ? max_len : most, window < most ? window : 0,
                                              sinks < most ? sinks : most);
}

int approxifer_cache_reserve(int32_t *d_table, int32_t *d_lens, int32_t *d_refs, const int32_t *d_add, int32_t *d_status, int64_t B,
                             int64_t M, int64_t P, int page, void *stream) {
    int shift = 0;
    const int rc = check_cache(B, M, P, page, &shift);
    if (rc != APPROXIFER_OK) return rc;
    if (B == 0) return APPROXIFER_OK;
    if (d_table == nullptr || d_lens == nullptr || d_refs == nullptr || d_add == nullptr) return APPROXIFER_ERR_NULL_POINTER;
    return approxifer::launch_cache_reserve(d_table, d_lens, d_refs, d_add, d_status, static_cast<int>(B), static_cast<int>(M),
                                            static_cast<int>(P), shift, static_cast<hipStream_t>(stream));
}

int approxifer_cache_fork(const int32_t *d_table, const int32_t *d_lens, const int32_t *d_refs, const int32_t *d_parents,
                          const int32_t *d_keep, int32_t *d_table_out, int32_t *d_lens_out, int32_t *d_refs_out,
                          int32_t *d_status, void *d_pools, int64_t planes, int64_t page_bytes, int64_t B, int64_t B_out, int64_t M,
                          int64_t P, int page, void *d_workspace, size_t workspace_bytes, void *stream) {
    int shift = 0;
    int rc = check_cache(B, M, P, page, &shift);
    if (rc == APPROXIFER_OK) rc = check_cache(B_out, M, P, page, &shift);
    if (rc == APPROXIFER_OK) rc = check_pools(d_pools, planes, page_bytes, P);
    if (rc != APPROXIFER_OK) return rc;
    if (d_refs == nullptr || d_refs_out == nullptr || (B > 0 && (d_table == nullptr || d_lens == nullptr)) ||
        (B_out > 0 && (d_parents == nullptr || d_table_out == nullptr || d_lens_out == nullptr)))
        return APPROXIFER_ERR_NULL_POINTER;
    if (d_workspace == nullptr || workspace_bytes < approxifer_cache_workspace_bytes(B, B_out, P)) return APPROXIFER_ERR_WORKSPACE;
    if (!aligned(d_workspace, 16)) return APPROXIFER_ERR_ALIGNMENT;
    return approxifer::launch_cache_fork(d_table, d_lens, d_refs, d_parents, d_keep, d_table_out, d_lens_out, d_refs_out, d_status,
                                         d_pools, planes, page_bytes, static_cast<int>(B), static_cast<int>(B_out),
                                         static_cast<int>(M), static_cast<int>(P), shift, d_workspace,
                                         static_cast<hipStream_t>(stream));
}

int approxifer_cache_compact(int32_t *d_table, const int32_t *d_lens, int32_t *d_refs, int32_t *d_moved, int32_t *d_live, void *d_pools,
                             int64_t planes, int64_t page_bytes, int64_t B, int64_t M, int64_t P, int page, void *d_workspace,
                             size_t workspace_bytes, void *stream) {
    int shift = 0;
    int rc = check_cache(B, M, P, page, &shift);
    if (rc == APPROXIFER_OK) rc = check_pools(d_pools, planes, page_bytes, P);
    if (rc != APPROXIFER_OK) return rc;
    if (d_refs == nullptr || d_moved == nullptr || d_live == nullptr || (B > 0 && (d_table == nullptr || d_lens == nullptr)))
        return APPROXIFER_ERR_NULL_POINTER;
    if (d_workspace == nullptr || workspace_bytes < approxifer_cache_workspace_bytes(B, B, P)) return APPROXIFER_ERR_WORKSPACE;
    if (!aligned(d_workspace, 16)) return APPROXIFER_ERR_ALIGNMENT;
    return approxifer::launch_cache_compact(d_table, d_lens, d_refs, d_moved, d_live, d_pools, planes, page_bytes, static_cast<int>(B),
                                            static_cast<int>(M), static_cast<int>(P), shift, d_workspace,
                                            static_cast<hipStream_t>(stream));
}

size_t approxifer_cache_workspace_bytes(int64_t B, int64_t B_out, int64_t P) {
    if (B < 0 || B_out < 0 || P < 1 || B > APPROXIFER_MAX_SEQUENCES || B_out > APPROXIFER_MAX_SEQUENCES || P > APPROXIFER_MAX_PAGES) return 0;
    return approxifer::cache_workspace_bytes(B, B_out, P);
}

}  // extern "C"
