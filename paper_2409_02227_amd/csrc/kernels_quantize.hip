// Rows to 8-bit integers.
#include "quantize.h"
template <int DT, bool WHOLE> static const void* held_kernel(int held) {
  using namespace gdy;
  return held == 1 ? reinterpret_cast<const void*>(&quantize_rows<DT, 1, WHOLE>)
         : held == 2 ? reinterpret_cast<const void*>(&quantize_rows<DT, 2, WHOLE>)
                     : reinterpret_cast<const void*>(&quantize_rows<DT, kQuantMost, WHOLE>);
}
const void* gdy::quantize_kernel(int dt, int held, bool whole) {
  switch (dt) {
    case DT_BF16: return whole ? held_kernel<DT_BF16, true>(held) : held_kernel<DT_BF16, false>(held);
    case DT_F16: return whole ? held_kernel<DT_F16, true>(held) : held_kernel<DT_F16, false>(held);
    case DT_F32: return whole ? held_kernel<DT_F32, true>(held) : held_kernel<DT_F32, false>(held);
    default: return nullptr;
  }
}
