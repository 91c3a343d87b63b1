#include "attend_mass.h"

namespace approxifer {

hipError_t launch_mass_bf16(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream) {
    return launch_mass_of<BF16>(c, g, mass, mass_stride, sums, stream);
}

hipError_t launch_scores_bf16(const AttendCall &c, const TokenGrid &g, float *workspace, hipStream_t stream) {
    return launch_scores_of<BF16>(c, g, workspace, stream);
}

}  // namespace approxifer
