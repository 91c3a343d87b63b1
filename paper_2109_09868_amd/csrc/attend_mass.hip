// Attention that adds up the weights it gives: attention itself, then the weights per key.
#include "attend_mass.h"

namespace approxifer {

namespace {

// Workgroups that a launch is cut into where there are the tiles for it.  Two prompts of up to 4001 tokens (32 heads of 128 on 8, bf16):
// 4096 214 us, 8192 208; three workgroups a CU are 768, and the causal ones differ in what they see.
constexpr int64_t kMassGroups = 8192;
int64_t stats_bytes(int64_t T, int Hq) { return (T * Hq * 8 + 255) / 256 * 256; }

// First a block's heads are dealt out, which reads each key once, then the tiles of all rows of a head of the cache, the same number to each
// workgroup (keys that come first are seen by more rows), four at least: their keys are loaded and their sums written once.
MassGrid mass_grid(int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len, size_t room) {
    const int bytes = (Dh <= 64 ? 64 : Dh <= 96 ? 96 : Dh <= 128 ? 128 : Dh <= 192 ? 192 : 256) * (dtype == APPROXIFER_F32 ? 4 : 2);
    MassGrid g;
    g.keys = 128;                                             // as MassShape has it
    g.rows = bytes <= 256 ? 64 : 32;
    g.blocks = (max_len + g.keys - 1) / g.keys;
    g.stride = g.blocks * g.keys;
    const int64_t blocks = g.blocks * B, tiles = (max_rows + g.rows - 1) / g.rows * (Hq / Hkv);
    const int64_t most = static_cast<int64_t>(room / (static_cast<size_t>(B > 0 ? B : 1) * (g.stride > 0 ? g.stride : 1) * 4));
    int64_t heads = (kMassGroups + blocks - 1) / (blocks > 0 ? blocks : 1);
    heads = heads < Hkv ? heads : Hkv;
    g.heads = static_cast<int>(heads < 1 || most < heads ? 1 : heads);
    int64_t chunk = blocks * Hkv * tiles / kMassGroups;
    chunk = chunk > 4 ? chunk : 4;
    const int64_t parts = most / g.heads;
    if (g.heads * parts < 2) chunk = tiles;
    else if ((tiles + chunk - 1) / chunk > parts) chunk = (tiles + parts - 1) / parts;
    g.chunk = static_cast<int>(chunk < tiles ? chunk : tiles > 0 ? tiles : 1);
    g.parts = static_cast<int>(tiles > 0 ? (tiles + g.chunk - 1) / g.chunk : 1);
    return g;
}

constexpr int64_t kAddBlocks = 1 << 20;
// One CU is slow to bring the scores of many rows, so that short sequences are dealt out to more of them: with fewer blocks of 256
// keys than this and more rows than 64 a block is of 64 keys.  12 heads of 64, float32, prompts of 34 tokens 28.7 -> 15.7 us the call, of 64
// 44 -> 18.6, twelve of them 52 -> 26; one token of 48 sequences behind 2000 127 -> 130.
// Eight waves a block there; of 256 keys and few rows they took 18 for four's 15 us (16 sequences of up to 32768 keys, 32 heads).
constexpr int64_t kFewScoreBlocks = 512;
constexpr int kRowsAhead = 4;                                 // of scores that a lane has on their way

// Scores of few rows are kept where they fit into this many bytes; more is formed again.  16 sequences of up to 32768 keys, 32 heads (67 MB of
// scores): 327 us, formed again 583; 24 of up to 129 17 and 30.
constexpr int64_t kMostScores = int64_t{1} << 31;
// Whether that is what is done: for the rows for which attention has its kernel of few rows, and of float32, whose products are dear, for up to
// 256 rows of a sequence and head of the cache, heads of more than 64.  Attention's kernel reads keys again for every 16 rows, and
// heads of more than 192 leave it one workgroup a CU: there while that is all there are, else up to 16 of them a CU.  Kept against formed again, by
// geometric mean of 500 random shapes: up to 64 rows 0.63, 65 to 192 0.57, 193 to 256 0.70, 257 to 700 0.89, more 1.16; by this rule 0.66, 2 of the 500
// longer by more than 2 %.  Microseconds, formed again -> kept: 8 heads of 96, two prompts of 88 40 -> 22; 8 heads of 128 on 2, 12
// prompts of 34 37 -> 16; 4 heads of 256, 48 prompts of 34 55 -> 45; 16 heads on 4 of 256, 39 prompts of 192 404 -> 649; 96 heads on 12 of 96, one of 172
// behind 120 78 -> 211; 12 heads of 64, 12 prompts of 88 27 -> 32.  bf16, 32 heads of 128 on 8, 12 prompts of 34 24 -> 31, of 64 26 -> 48.
bool keeps_scores(int64_t B, int Hq, int Hkv, int Dh, int64_t max_rows, int dtype) {
    const int64_t rows = max_rows * (Hq / Hkv), blocks = B * Hkv * ((rows + 15) / 16);
    return few_rows(B, Hq, Hkv, max_rows, dtype) || (dtype == APPROXIFER_F32 && Dh > 64 && rows <= 256 && blocks <= (Dh > 192 ? 256 : 4096));
}
int64_t score_stride(int64_t max_len) { return (max_len + 255) / 256 * 256; }
int64_t score_bytes(int64_t T, int Hq, int64_t max_len) { return T * Hq * score_stride(max_len) * 4; }
size_t parts_bytes(const TokenGrid &g, int Dh) {
    return g.parts < 2 ? 0 : static_cast<size_t>(g.pairs) * g.blocks * g.parts * part_floats(16, Dh) * 4;
}

// 5 us of two prompts' 383.  A block of keys: four threads to each, with a quarter of the slices' sums, and those in their order.
__global__ __launch_bounds__(512) void add_slices_kernel(AttendCall c, MassGrid g, float *mass, int64_t mass_stride, const float *sums) {
    __shared__ float quarters[4][128];
    const int64_t work = g.blocks * c.seq.B;
    const int quarter = threadIdx.x >> 7, key = threadIdx.x & 127;
    for (int64_t index = blockIdx.x; index < work; index += gridDim.x) {
        const int b = static_cast<int>(index % c.seq.B), j0 = static_cast<int>(index / c.seq.B) * g.keys, j = j0 + key;
        const Rows rows = rows_of(c.seq, b);
        if (!rows.ok || rows.n == 0 || rows.n > c.max_rows || rows.length > c.max_len || j0 >= rows.length) continue;
        const int64_t step = c.seq.B * g.stride;
        const int parts = MassTokens(c, g, rows, j0).parts(c, g), all = g.heads * parts;
        const int begin = all * quarter / 4, end = all * (quarter + 1) / 4;
        float x = 0.0f;
        for (int n0 = begin; n0 < end; n0 += 8) {             // eight of them on their way at a time
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int n = min(n0 + k, end - 1);
                y[k] = sums[n * step + b * g.stride + j];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x += n0 + k < end ? y[k] : 0.0f;
        }
        quarters[quarter][key] = x;
        __syncthreads();
        if (quarter == 0 && j < rows.length)
            mass[b * mass_stride + j] += ((x + quarters[1][key]) + quarters[2][key]) + quarters[3][key];
        __syncthreads();
    }
}

// Waits for the scores, which attention has just left: 16 sequences of up to 32768 keys and 32 heads 15 us, 24 of up to 129 and 12 heads 4.
// 4 kLanes keys of a sequence, 4 to a lane; the groups of kLanes lanes of kWaves waves have its rows' heads in turn, and add their sums in order.
template <int kLanes, int kWaves>
__global__ __launch_bounds__(kWave * kWaves) void mass_of_scores_kernel(AttendCall c, float *mass, int64_t mass_stride, int64_t blocks) {
    __shared__ v4f sums[kWaves * kWave / kLanes][kLanes];
    const float scale = fabsf(c.scale) * 1.44269504088896340736f;
    constexpr int kSets = kWave / kLanes, kAll = kWaves * kSets;
    const int lane = lane_id() % kLanes, set = kSets == 1 ? __builtin_amdgcn_readfirstlane(wave_id()) : wave_id() * kSets + lane_id() / kLanes;
    const int64_t work = blocks * c.seq.B;
    for (int64_t index = blockIdx.x; index < work; index += gridDim.x) {
        const int b = static_cast<int>(index % c.seq.B), j0 = static_cast<int>(index / c.seq.B) * (4 * kLanes), j = j0 + 4 * lane;
        const Rows rows = rows_of(c.seq, b);
        if (!rows.ok || rows.n == 0 || rows.n > c.max_rows || rows.length > c.max_len || j0 >= rows.length) continue;
        const float *const scores = c.scores + rows.start * c.Hq * c.score_stride + j, *const stats = c.stats + 2 * rows.start;
        v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
        // from the first token that sees one of them to the last; what a row does not see has no scores, but there is memory
        const int before = rows.length - rows.n, from = max(0, j0 - before) * c.Hq;
        int to = rows.n;
        if (c.window > 0 && j0 >= c.sinks)
            to = static_cast<int>(min(static_cast<int64_t>(to), static_cast<int64_t>(j0) + 4 * kLanes - 1 + c.window - before));
        const int all = to * c.Hq;
        for (int r0 = from + set; r0 < all; r0 += kAll * kRowsAhead) {
            v4f s[kRowsAhead];
            v2f of_row[kRowsAhead];
            int tokens[kRowsAhead];
#pragma unroll
            for (int a = 0; a < kRowsAhead; ++a) {
                const int row = min(r0 + kAll * a, all - 1), i = rows.n == 1 ? 0 : row / c.Hq, h = row - i * c.Hq;
                tokens[a] = i;
                of_row[a] = *reinterpret_cast<const v2f *>(stats + 2 * (h * c.seq.T + i));
                s[a] = *reinterpret_cast<const v4f *>(scores + row * c.score_stride);
            }
#pragma unroll
            for (int a = 0; a < kRowsAhead; ++a) {
                const Visible see(c.window, c.sinks, rows.place(tokens[a]));
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(s[a][k], scale, -of_row[a][0])) * of_row[a][1];
                    sum[k] += see.sees(j + k) && r0 + kAll * a < all ? w : 0.0f;
                }
            }
        }
        sums[set][lane] = sum;
        __syncthreads();
        if (set == 0) {
            for (int w = 1; w < kAll; ++w) sum += sums[w][lane];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < rows.length) mass[b * mass_stride + j + k] += sum[k];
        }
        __syncthreads();
    }
}

}  // namespace

size_t attend_mass_least_bytes(int64_t T, int Hq) { return static_cast<size_t>(stats_bytes(T, Hq)); }

size_t attend_mass_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                                   int64_t window, int64_t sinks) {
    constexpr size_t kAll = static_cast<size_t>(1) << 60;
    max_rows = max_rows < T ? max_rows : T;
    if (keeps_scores(B, Hq, Hkv, Dh, max_rows, dtype) && score_bytes(T, Hq, max_len) <= kMostScores)
        return static_cast<size_t>(stats_bytes(T, Hq) + score_bytes(T, Hq, max_len)) +
               parts_bytes(token_grid(B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks, kAll, true), Dh);
    const size_t parts = attend_workspace_bytes(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks);
    const MassGrid g = mass_grid(B, Hq, Hkv, Dh, dtype, max_rows, max_len, kAll);
    const size_t sums = g.slices() < 2 ? 0 : static_cast<size_t>(g.slices()) * B * g.stride * 4;
    return static_cast<size_t>(stats_bytes(T, Hq)) + (parts > sums ? parts : sums);
}

int launch_attend_mass(AttendCall c, float *mass, int64_t mass_stride, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (c.seq.T == 0) return launch_attend(c, nullptr, 0, stream);
    // the rows' statistics, then room that attention's parts and afterwards the slices' sums use
    const size_t stats = static_cast<size_t>(stats_bytes(c.seq.T, c.Hq)), room = workspace_bytes > stats ? workspace_bytes - stats : 0;
    c.stats = static_cast<float *>(workspace);
    float *const sums = c.stats + stats / 4;
    const int64_t scores = score_bytes(c.seq.T, c.Hq, c.max_len);
    if (keeps_scores(c.seq.B, c.Hq, c.Hkv, c.Dh, c.max_rows, c.dtype) && c.max_rows > 0 && c.max_len > 0 && scores <= kMostScores &&
        static_cast<size_t>(scores) <= room) {
        c.scores = sums;
        c.score_stride = score_stride(c.max_len);
        float *const parts = sums + scores / 4;
        const TokenGrid g = token_grid(c.seq.B, c.Hq, c.Hkv, c.Dh, c.dtype, c.max_rows, c.max_len, c.window, c.sinks, room - scores, true);
        hipError_t e = c.dtype == APPROXIFER_F32   ? launch_scores_f32(c, g, parts, stream)
                       : c.dtype == APPROXIFER_F16 ? launch_scores_f16(c, g, parts, stream)
                                                   : launch_scores_bf16(c, g, parts, stream);
        if (e == hipSuccess)
            e = c.dtype == APPROXIFER_F32   ? join_tokens_f32(c, g, parts, stream)
                : c.dtype == APPROXIFER_F16 ? join_tokens_f16(c, g, parts, stream)
                                            : join_tokens_bf16(c, g, parts, stream);
        const bool few = (c.max_len + 255) / 256 * c.seq.B < kFewScoreBlocks && c.max_rows * c.Hq > 64;
        const int64_t blocks = few ? (c.max_len + 63) / 64 : (c.max_len + 255) / 256, work = blocks * c.seq.B;
        const dim3 grid(static_cast<unsigned>(work < kAddBlocks ? work : kAddBlocks));
        if (e == hipSuccess)
            e = few ? launch_kernel(mass_of_scores_kernel<16, 8>, grid, dim3(512), 0, stream, c, mass, mass_stride, blocks)
                    : launch_kernel(mass_of_scores_kernel<64, 4>, grid, dim3(256), 0, stream, c, mass, mass_stride, blocks);
        return launch_status(e);
    }
    const int rc = launch_attend(c, sums, room, stream);
    if (rc != APPROXIFER_OK || c.max_rows == 0 || c.max_len == 0) return rc;
    const MassGrid g = mass_grid(c.seq.B, c.Hq, c.Hkv, c.Dh, c.dtype, c.max_rows, c.max_len, room);
    hipError_t e = c.dtype == APPROXIFER_F32   ? launch_mass_f32(c, g, mass, mass_stride, sums, stream)
                   : c.dtype == APPROXIFER_F16 ? launch_mass_f16(c, g, mass, mass_stride, sums, stream)
                                               : launch_mass_bf16(c, g, mass, mass_stride, sums, stream);
    if (e == hipSuccess && g.slices() > 1) {
        const int64_t work = g.blocks * c.seq.B;
        e = launch_kernel(add_slices_kernel, dim3(static_cast<unsigned>(work < kAddBlocks ? work : kAddBlocks)), dim3(512), 0, stream, c, g,
                          mass, mass_stride, static_cast<const float *>(sums));
    }
    return launch_status(e);
}

}  // namespace approxifer
