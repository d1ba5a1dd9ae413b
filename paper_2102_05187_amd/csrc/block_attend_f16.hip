// Attention over chosen blocks, f16.
#include "block_attend.hpp"

namespace comet {
hipError_t attend_f16(const AttendArgs &a, int wide, int mt, hipStream_t st) { return attend_type<COMET_F16>(a, wide, mt, st); }
}  // namespace comet
