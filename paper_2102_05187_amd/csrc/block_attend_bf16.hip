// Attention over chosen blocks, bf16.
#include "block_attend.hpp"

namespace comet {
hipError_t attend_bf16(const AttendArgs &a, int wide, int mt, hipStream_t st) { return attend_type<COMET_BF16>(a, wide, mt, st); }
}  // namespace comet
