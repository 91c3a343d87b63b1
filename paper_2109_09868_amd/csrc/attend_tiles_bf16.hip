#include "attend_tiles.h"

namespace approxifer {

hipError_t launch_tiles_bf16(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream) {
    return launch_tiles_of<BF16>(c, g, workspace, stream);
}

}  // namespace approxifer
