#include "attend_tiles.h"

namespace approxifer {

hipError_t launch_tiles_f16(const AttendCall &c, const TileGrid &g, float *workspace, hipStream_t stream) {
    return launch_tiles_of<F16>(c, g, workspace, stream);
}

}  // namespace approxifer
