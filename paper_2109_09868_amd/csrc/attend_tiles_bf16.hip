#include "attend_tiles.h"

namespace approxifer {

hipError_t launch_tiles_bf16(const AttendCall &c, hipStream_t stream) { return launch_tiles_of<BF16>(c, stream); }

}  // namespace approxifer
