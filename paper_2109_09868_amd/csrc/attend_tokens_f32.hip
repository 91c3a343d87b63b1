#include "attend_tokens.h"

namespace approxifer {

hipError_t launch_tokens_f32(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    return launch_tokens_of<F32>(c, g, workspace, stream);
}

}  // namespace approxifer
