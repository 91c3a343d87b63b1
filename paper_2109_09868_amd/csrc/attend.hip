// Attention over a cache in pages: which kernel a call takes, and how its keys are cut.
#include "attend_tiles.h"
#include "attend_tokens.h"

namespace approxifer {

namespace {

constexpr int kTokenRows = 32;                                // most rows of a sequence and head that the tokens kernel takes
// Workgroups that it is given if keys are cut: two on every CU, in one round.  With 256 / 512 / 768 / 1024 / 2048 three sequences of up to
// 131072 keys take 258 / 244 / 257 / 257 / 255 us.
constexpr int64_t kTokenGroups = 512;

// How the tokens kernel cuts the keys of a call into parts, given what workspace there is.
TokenGrid token_grid(int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks,
                     size_t workspace_bytes) {
    const int64_t group = Hq / Hkv, pairs = B * Hkv, blocks = (max_rows * group + 15) / 16;
    const int64_t keys = dtype != APPROXIFER_F32 || Dh <= 64 ? 32 : 16;
    int64_t tiles = (max_len + keys - 1) / keys;
    if (window > 0) {                                         // no block of 16 rows sees more
        const int64_t most = (sinks + keys - 1) / keys + (window + 16) / keys + 2;
        tiles = tiles < most ? tiles : most;
    }
    int64_t parts = kTokenGroups / (pairs * blocks > 0 ? pairs * blocks : 1);
    parts = parts < (tiles + 7) / 8 ? parts : (tiles + 7) / 8;           // two tiles a wave at least
    const int64_t room = static_cast<int64_t>(workspace_bytes) / (pairs * blocks * part_floats(Dh) * 4 + 1);
    parts = parts < room ? parts : room;
    TokenGrid g;
    g.pairs = static_cast<int>(pairs);
    g.blocks = static_cast<int>(blocks);
    g.rows = static_cast<int>(max_rows * group < 16 ? max_rows * group : 16);
    if (parts < 2) {
        g.parts = 1;
        g.chunk = 0x7fffffff;
        return g;
    }
    g.chunk = static_cast<int>(((tiles + parts - 1) / parts + 3) / 4 * 4);
    g.parts = static_cast<int>((tiles + g.chunk - 1) / g.chunk);
    return g;
}

}  // namespace

size_t attend_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                              int64_t window, int64_t sinks) {
    max_rows = max_rows < T ? max_rows : T;
    if (max_rows * (Hq / Hkv) > kTokenRows) return 0;
    const TokenGrid g = token_grid(B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks, static_cast<size_t>(1) << 60);
    return g.parts < 2 ? 0 : static_cast<size_t>(g.pairs) * g.blocks * g.parts * part_floats(Dh) * 4;
}

int launch_attend(const AttendCall &c, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const int dtype = c.dtype;
    if (static_cast<int64_t>(c.max_rows) * (c.Hq / c.Hkv) > kTokenRows)
        return launch_status(dtype == APPROXIFER_F32   ? launch_tiles_f32(c, stream)
                             : dtype == APPROXIFER_F16 ? launch_tiles_f16(c, stream)
                                                       : launch_tiles_bf16(c, stream));
    const TokenGrid g = token_grid(c.seq.B, c.Hq, c.Hkv, c.Dh, dtype, c.max_rows, c.max_len, c.window, c.sinks, workspace_bytes);
    float *const w = static_cast<float *>(workspace);
    return launch_status(dtype == APPROXIFER_F32   ? launch_tokens_f32(c, g, w, stream)
                         : dtype == APPROXIFER_F16 ? launch_tokens_f16(c, g, w, stream)
                                                   : launch_tokens_bf16(c, g, w, stream));
}

}  // namespace approxifer
