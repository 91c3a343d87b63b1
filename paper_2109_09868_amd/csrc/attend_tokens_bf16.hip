#include "attend_tokens.h"

namespace approxifer {

hipError_t launch_tokens_bf16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    return launch_tokens_of<BF16>(c, g, workspace, stream);
}

hipError_t join_tokens_bf16(const AttendCall &c, const TokenGrid &g, const float *workspace, hipStream_t stream) {
    return join_tokens_of<BF16>(c, g, workspace, stream);
}

}  // namespace approxifer
