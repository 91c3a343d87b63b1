#include "attend_mass.h"

namespace approxifer {

hipError_t launch_mass_f16(const AttendCall &c, const MassGrid &g, float *mass, int64_t mass_stride, float *sums, hipStream_t stream) {
    return launch_mass_of<F16>(c, g, mass, mass_stride, sums, stream);
}

}  // namespace approxifer
