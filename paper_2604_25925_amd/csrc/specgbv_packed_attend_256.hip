// Attention over a cache held in 4 bits: heads of 129 to 256 entries.
#include "specgbv_packed_attend.hpp"

namespace specgbv {

hipError_t launch_packed_attend_256(const PackedProblem &p, int dtype, hipStream_t stream)
{
    return dtype == 1 ? launch_typed<uint16_t, 256>(p, stream) : launch_typed<float, 256>(p, stream);
}

}  // namespace specgbv
