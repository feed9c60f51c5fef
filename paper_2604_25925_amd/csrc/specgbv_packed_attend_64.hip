// Attention over a cache held in 4 bits: heads of up to 64 entries.
#include "specgbv_packed_attend.hpp"

namespace specgbv {

hipError_t launch_packed_attend_64(const PackedProblem &p, int dtype, hipStream_t stream)
{
    return dtype == 1 ? launch_typed<uint16_t, 64>(p, stream) : launch_typed<float, 64>(p, stream);
}

}  // namespace specgbv
