#include "attend_tiles.h"

namespace approxifer {

hipError_t launch_tiles_f16(const AttendCall &c, hipStream_t stream) { return launch_tiles_of<F16>(c, stream); }

}  // namespace approxifer
