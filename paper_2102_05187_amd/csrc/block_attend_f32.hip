// Attention over chosen blocks, f32.
#include "block_attend.hpp"

namespace comet {
hipError_t attend_f32(const AttendArgs &a, int wide, int mt, hipStream_t st) { return attend_type<COMET_F32>(a, wide, mt, st); }
}  // namespace comet
