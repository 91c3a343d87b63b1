// The attention kernels for groups of sequences that begin alike, and their launches.
#pragma once

#include "attend_tiles.h"
#include "attend_tokens.h"

namespace approxifer {

// Common places by tiles: 8 x 6 blocks of 128 rows on 8003 places take 48 us (192 sequences, 32 heads of 128 on 8, bf16), 524 TFLOP/s: each
// workgroup has a few tiles of keys, of which one is on its way while another is used, and waits for them.
template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (TileShape<E, DP>::kGroups)) void attend_shared_tiles_kernel(AttendCall c, SharedCall shared) {
    __shared__ __align__(16) char lds[TileShape<E, DP>::kLds];
    attend_tiles_shared<E, DP, kWhole, kSmall>(c, shared, blockIdx.x, lds);
}

// Own places, and common ones of few rows.  192 sequences' 33 to 512 own places (8 heads of 128, bf16) 50 us, 4.3 TB/s.  24 sequences behind
// 500 places (12 heads of 64, float32) 15 us, 6 to 7.5 of which it takes for a single key.
template <class E, int DP, bool kWhole, bool kSmall>
__global__ __launch_bounds__(256, (DP > 128 ? 1 : 2)) void attend_shared_tokens_kernel(AttendCall c, SharedCall shared) {
    __shared__ __align__(16) char lds[TokenShape<E, DP>::kLds];
    attend_tokens<E, DP, kWhole, kSmall, true, false>(c, TokenGrid{}, nullptr, shared, blockIdx.x, lds);
}

// Common places by tiles and own ones by tokens in one launch, the tiles first: they are fewer and take longer, and the others go where they
// leave room.  192 sequences behind 8003 tokens (8 heads of 128, bf16) 94 us, in two launches 48 and 51, and 156 with tiles dealt out among
// the others; 200 behind 16 prompts (2 heads of 128, fp16) 32 us, in two launches 28 and 17.
template <class E, int DP>
__global__ __launch_bounds__(256, 2) void attend_shared_both_kernel(AttendCall c, SharedCall shared, int tiles) {
    constexpr int kTiles = TileShape<E, DP>::kLds, kTokens = TokenShape<E, DP>::kLds;
    __shared__ __align__(16) char lds[kTiles > kTokens ? kTiles : kTokens];
    const int x = blockIdx.x;
    if (x < tiles) {
        shared.own_slots = 0;
        attend_tiles_shared<E, DP, true, false>(c, shared, x, lds);
    } else {
        shared.common_slots = 0;
        attend_tokens<E, DP, true, false, true, false>(c, TokenGrid{}, nullptr, shared, x - tiles, lds);
    }
}

// F<E, DP, kWhole, kSmall>::run() for a call's head: as many instances as the kernels for single sequences have.
template <template <class, int, bool, bool> class F, class E, bool kSmall>
hipError_t shared_instance(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    if (c.Dh == 64) return F<E, 64, true, kSmall>::run(c, shared, stream);
    if (c.Dh == 128) return F<E, 128, true, kSmall>::run(c, shared, stream);
    if (c.Dh == 256) return F<E, 256, true, kSmall>::run(c, shared, stream);
    if (c.Dh < 64) return F<E, 64, false, kSmall>::run(c, shared, stream);
    if (c.Dh <= 96) return F<E, 96, false, kSmall>::run(c, shared, stream);
    if (c.Dh < 128) return F<E, 128, false, kSmall>::run(c, shared, stream);
    if (c.Dh <= 192) return F<E, 192, false, kSmall>::run(c, shared, stream);
    return F<E, 256, false, kSmall>::run(c, shared, stream);
}

inline unsigned shared_blocks(const AttendCall &c, const SharedCall &shared) {
    return static_cast<unsigned>((shared.common_slots * shared.common_parts + shared.own_slots * shared.own_parts) * c.Hkv);
}
template <class E, int DP, bool kWhole, bool kSmall>
struct SharedTiles {
    static hipError_t run(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
        if constexpr (sizeof(typename E::Value) == 4 && DP > 64 && DP <= 128) return hipErrorInvalidValue;   // as shared_tiles() says
        else return launch_kernel(attend_shared_tiles_kernel<E, DP, kWhole, kSmall>, dim3(shared_blocks(c, shared)), dim3(256), 0, stream, c, shared);
    }
};
template <class E, int DP, bool kWhole, bool kSmall>
struct SharedTokens {
    static hipError_t run(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
        return launch_kernel(attend_shared_tokens_kernel<E, DP, kWhole, kSmall>, dim3(shared_blocks(c, shared)), dim3(256), 0, stream, c, shared);
    }
};

template <class E>
hipError_t launch_shared_tiles_of(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return c.seq.page_shift >= 4 ? shared_instance<SharedTiles, E, false>(c, shared, stream) : shared_instance<SharedTiles, E, true>(c, shared, stream);
}
template <class E>
hipError_t launch_shared_tokens_of(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return c.seq.page_shift >= 4 ? shared_instance<SharedTokens, E, false>(c, shared, stream)
                                 : shared_instance<SharedTokens, E, true>(c, shared, stream);
}
template <class E, int DP>
hipError_t launch_shared_both(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_kernel(attend_shared_both_kernel<E, DP>, dim3(shared_blocks(c, shared)), dim3(256), 0, stream, c, shared,
                         static_cast<int>(shared.common_slots * shared.common_parts * c.Hkv));
}
template <class E>
hipError_t launch_shared_both_of(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    if constexpr (sizeof(typename E::Value) == 2)
        if (c.Dh == 128) return launch_shared_both<E, 128>(c, shared, stream);
    return launch_shared_both<E, 64>(c, shared, stream);
}
template <class E>
hipError_t launch_shared_join_of(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    const int64_t blocks = (c.seq.T * c.Hq + 3) / 4 + (c.status != nullptr ? (c.seq.B + 3) / 4 : 0);
    const dim3 grid(static_cast<unsigned>(blocks));
    if (c.Dh <= 64) return launch_kernel(attend_shared_join_kernel<E, 64>, grid, dim3(256), 0, stream, c, shared);
    if (c.Dh <= 128) return launch_kernel(attend_shared_join_kernel<E, 128>, grid, dim3(256), 0, stream, c, shared);
    return launch_kernel(attend_shared_join_kernel<E, 256>, grid, dim3(256), 0, stream, c, shared);
}

}  // namespace approxifer
