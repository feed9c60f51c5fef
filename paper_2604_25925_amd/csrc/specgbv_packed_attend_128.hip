// Attention over a cache held in 4 bits: heads of 65 to 128 entries.
#include "specgbv_packed_attend.hpp"

namespace specgbv {

hipError_t launch_packed_attend_128(const PackedProblem &p, int dtype, hipStream_t stream)
{
    return dtype == 1 ? launch_typed<uint16_t, 128>(p, stream) : launch_typed<float, 128>(p, stream);
}

}  // namespace specgbv
