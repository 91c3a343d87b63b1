// Attention over a cache in pages: which kernel a call takes, and how its keys are cut.
#include <cmath>

#include "attend_tiles.h"
#include "attend_tokens.h"

namespace approxifer {

// Most rows of a sequence and cache head that the tokens kernel takes: more are read again for every 16, and the tiles kernel's products are
// the better ones for them.  8 tokens by 4 heads (32 rows) of 8 sequences of up to 40000 keys: 284 us here, 186 there; 32-bit products cost
// more than memory does, whichever kernel forms them, and the tiles kernel's 128 rows are mostly empty: 16 tokens (64 rows) of up to 6000
// keys 108 us here, 121 there.
// Neither kernel's calls reach 2^32 threads, which a launch cannot have: the tiles kernel's because T Hq / 128 + B Hkv workgroups are enough,
// and calls that would take more than 2^24 blocks of 16 rows go there.
bool few_rows(int64_t B, int Hq, int Hkv, int64_t max_rows, int dtype) {
    const int64_t rows = max_rows * (Hq / Hkv), blocks = (rows + 15) / 16;
    return rows <= (dtype == APPROXIFER_F32 ? 64 : 16) && B * Hkv * blocks + (B + 3) / 4 < 1 << 24;
}
namespace {

// Workgroups that it is given if keys are cut: two on every CU, in one round.  With 256 / 512 / 768 / 1024 / 2048 three sequences of up to
// 131072 keys take 258 / 244 / 257 / 257 / 255 us.  Of heads of more than 128 a CU has room for one: one sequence of 40000 keys (2 heads of
// 256, bf16) 30 us in 256 workgroups, 41 in 314; 12 of 8000 42 in 240, 47 in 504; one of 10000 (8 of 256) 26 and 36 in 320.
int64_t token_groups(int Dh) { return Dh > 128 ? 256 : 512; }
// Parts of a row that are worth their writing and joining.  Whole / two: 32 sequences of 4000 keys (8 heads of 128, bf16) 92 / 96 us, 16 of
// 1000 (12 of 64, 32 bits) 21 / 27, 96 of 2000 (8 of 128, bf16) 134 / 142, one of 512 10 / 12; heads of 256 leave CUs empty: one of 512 keys
// 20 / 18, of 270 16 / 18.
bool worth_two(int Dh, int64_t units, int64_t tiles) { return Dh > 128 && 2 * units <= token_groups(Dh) && tiles > 12; }
// Where that leaves more than a seventh of the places empty, as many as make three rounds, if each still has 24 tiles: 264 heads of sequences
// of 4000 keys (bf16, 128) 108 us in six parts each and 136 in one, 288 (32 bits, 64) 116 and 144; with 1000 keys 40 us either way, and
// 384 windows of 1024 keys 44 us whole, 53 in two parts.
constexpr int64_t kTokenRounds = 3, kTokenChunk = 24;
// If they have not, and some CUs would have two workgroups and some one, one each: one sequence of 17230 keys (32 heads on 4 of 64, fp16) 12.5 us
// in 180 workgroups, 13.6 in 272; 11 of 1574 (4 of 128, fp16) 14.2 in 220, 15.8 in 308; 12 of 1000 (12 of 64, 32 bits) 20 in 144, 23 in 432.
constexpr int64_t kCUs = 256;

}  // namespace

// How the tokens kernel cuts the keys of a call into parts, given what workspace there is.
TokenGrid token_grid(int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks,
                     size_t workspace_bytes, bool ragged) {
    const int64_t group = Hq / Hkv, pairs = B * Hkv, blocks = (max_rows * group + 15) / 16;
    const int64_t keys = dtype != APPROXIFER_F32 || Dh <= 64 ? 32 : 16;
    int64_t tiles = (max_len + keys - 1) / keys;
    if (window > 0) {                                         // no block of 16 rows sees more
        const int64_t most = (sinks + keys - 1) / keys + (window + 16) / keys + 2;
        tiles = tiles < most ? tiles : most;
    }
    const int64_t units = pairs * blocks > 0 ? pairs * blocks : 1, round = ragged ? 512 : token_groups(Dh);
    int64_t parts = round / units;
    parts = parts < (tiles + 7) / 8 ? parts : (tiles + 7) / 8;           // two tiles a wave at least
    const int64_t groups = units * (parts > 1 ? parts : 1), places = (groups + round - 1) / round * round;
    if (ragged || groups * 7 < places * 6) {
        int64_t more = (kTokenRounds * round + units - 1) / units;
        more = more < tiles / kTokenChunk ? more : tiles / kTokenChunk;
        if (!ragged && more <= parts && Dh <= 128 && groups > kCUs) parts = kCUs / units;
        parts = parts > more ? parts : more;
    }
    if (parts == 2 && !ragged && !worth_two(Dh, units, tiles)) parts = 1;
    const int64_t room = static_cast<int64_t>(workspace_bytes / (static_cast<size_t>(units) * part_floats(16, Dh) * 4));
    parts = parts < room ? parts : room;
    TokenGrid g;
    g.pairs = static_cast<int>(pairs);
    g.blocks = static_cast<int>(blocks);
    g.rows = static_cast<int>(max_rows * group < 16 ? max_rows * group : 16);
    if (parts < 2 || blocks == 0) {
        g.parts = 1;
        g.chunk = 0x7fffffff;
        return g;
    }
    g.chunk = static_cast<int>(((tiles + parts - 1) / parts + 3) / 4 * 4);
    g.parts = static_cast<int>((tiles + g.chunk - 1) / g.chunk);
    return g;
}

namespace {

// Into how many parts the tiles kernel cuts the keys of `heads` tiles of rows and cache heads.  A part takes `tile_us` a tile of 64 keys, all of
// them at once as long as the GPU has room; the parts of a row are written and read again at 4.5 bytes a ps, and joined by a launch of
// about 6 us more.  So sqrt(tiles tile_us / us a part) of them are the least time, if that is less than without any.  Whole / two or three / more
// parts: 1000 tokens of 32 heads on 8 (bf16, 128) 30 us / 46 in two, 16 tokens of 4 sequences of up to 40000 keys 932 / 106 in sixteen; in 32 bits four
// prompts of 500 (8 heads of 128) 80 / 60 / 71, one of 1000 (4 heads on one) 49 in four, 35 in eight.  Where every CU has a tile already, 32-bit
// products gain nothing from a second one: four prompts of 1000 (12 heads of 64) 117 us whole, 138 in two.
int64_t tile_parts(int64_t rows, int64_t heads, int64_t tiles, int Dh, int dtype) {
    const bool wide = dtype == APPROXIFER_F32;
    const int64_t places = Dh > 128 || (wide && Dh > 64) ? 256 : wide ? 768 : 512;       // workgroups at a time
    int64_t most = places / (heads > 0 ? heads : 1);
    most = most < tiles / 2 ? most : tiles / 2;
    if (most < 2 || (wide && heads > kCUs)) return 1;
    const double tile_us = Dh * (!wide ? 0.0086 : Dh > 64 ? 0.0625 : 0.053);
    const double part_us = static_cast<double>(rows) * Dh * 8.0 / 4.5e6;
    int64_t parts = static_cast<int64_t>(std::sqrt(tiles * tile_us / part_us) + 0.5);
    parts = parts < most ? parts : most;
    return parts < 2 || tiles * tile_us / parts + parts * part_us + 6.0 > tiles * tile_us ? 1 : parts;
}

TileGrid tile_grid(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len, int64_t window, int64_t sinks,
                   size_t workspace_bytes) {
    const int64_t group = Hq / Hkv;
    TileGrid g;
    g.single = max_rows * group <= kTileRows;                 // a tile for each sequence
    g.slots = g.single ? B : T * group / kTileRows + B;
    int64_t tiles = (max_len + 63) / 64;
    if (window > 0) {                                         // no tile of rows sees more
        const int64_t most = (sinks + 63) / 64 + (window + kTileRows) / 64 + 2;
        tiles = tiles < most ? tiles : most;
    }
    // as many as there are where all sequences have max_rows tokens; half of the tiles that only make up a sequence's number can be empty
    const int64_t heads = (T == B * max_rows ? B * ((max_rows * group + kTileRows - 1) / kTileRows) : g.single ? B : T * group / kTileRows + (B + 1) / 2) * Hkv;
    int64_t parts = tile_parts(T * Hq, heads, tiles, Dh, dtype);
    const int64_t room = static_cast<int64_t>(workspace_bytes / (static_cast<size_t>(g.slots) * Hkv * part_floats(kTileRows, Dh) * 4));
    parts = parts < room ? parts : room;
    g.parts = static_cast<int>(parts < 2 ? 1 : parts);
    g.chunk = static_cast<int>((tiles + g.parts - 1) / g.parts);
    return g;
}

}  // namespace

size_t attend_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int Dh, int dtype, int64_t max_rows, int64_t max_len,
                              int64_t window, int64_t sinks) {
    constexpr size_t kAll = static_cast<size_t>(1) << 60;
    max_rows = max_rows < T ? max_rows : T;
    if (!few_rows(B, Hq, Hkv, max_rows, dtype)) {
        const TileGrid g = tile_grid(T, B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks, kAll);
        return g.parts < 2 ? 0 : static_cast<size_t>(g.slots) * Hkv * g.parts * part_floats(kTileRows, Dh) * 4;
    }
    const TokenGrid g = token_grid(B, Hq, Hkv, Dh, dtype, max_rows, max_len, window, sinks, kAll);
    return g.parts < 2 ? 0 : static_cast<size_t>(g.pairs) * g.blocks * g.parts * part_floats(16, Dh) * 4;
}

int launch_attend(const AttendCall &c, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const int dtype = c.dtype;
    float *const w = static_cast<float *>(workspace);
    if (!few_rows(c.seq.B, c.Hq, c.Hkv, c.max_rows, dtype)) {
        const TileGrid g = tile_grid(c.seq.T, c.seq.B, c.Hq, c.Hkv, c.Dh, dtype, c.max_rows, c.max_len, c.window, c.sinks,
                                     workspace_bytes);
        return launch_status(dtype == APPROXIFER_F32   ? launch_tiles_f32(c, g, w, stream)
                             : dtype == APPROXIFER_F16 ? launch_tiles_f16(c, g, w, stream)
                                                       : launch_tiles_bf16(c, g, w, stream));
    }
    const TokenGrid g = token_grid(c.seq.B, c.Hq, c.Hkv, c.Dh, dtype, c.max_rows, c.max_len, c.window, c.sinks, workspace_bytes);
    return launch_status(dtype == APPROXIFER_F32   ? launch_tokens_f32(c, g, w, stream)
                         : dtype == APPROXIFER_F16 ? launch_tokens_f16(c, g, w, stream)
                                                   : launch_tokens_bf16(c, g, w, stream));
}

}  // namespace approxifer
