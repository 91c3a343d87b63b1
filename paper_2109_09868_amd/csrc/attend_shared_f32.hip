#include "attend_shared_kernels.h"

namespace approxifer {

hipError_t launch_shared_tiles_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_tiles_of<F32>(c, shared, stream);
}
hipError_t launch_shared_tokens_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_tokens_of<F32>(c, shared, stream);
}
hipError_t launch_shared_both_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_both_of<F32>(c, shared, stream);
}
hipError_t launch_shared_join_f32(const AttendCall &c, const SharedCall &shared, hipStream_t stream) {
    return launch_shared_join_of<F32>(c, shared, stream);
}

}  // namespace approxifer
