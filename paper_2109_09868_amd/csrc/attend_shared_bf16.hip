#include "attend_shared_kernels.h"

namespace approxifer {

hipError_t launch_shared_tiles_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_tiles_of<BF16>(c, shared, stream);
}
hipError_t launch_shared_tokens_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_tokens_of<BF16>(c, shared, stream);
}
hipError_t launch_shared_both_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_both_of<BF16>(c, shared, stream);
}
hipError_t launch_shared_join_bf16(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_join_of<BF16>(c, shared, stream);
}

}  // namespace approxifer
