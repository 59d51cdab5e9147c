// Rows to 8-bit integers.
#include "quantize.h"
const void* gdy::quantize_kernel(int dt) {
  switch (dt) {
    case DT_BF16: return reinterpret_cast<const void*>(&quantize_rows<DT_BF16>);
    case DT_F16: return reinterpret_cast<const void*>(&quantize_rows<DT_F16>);
    case DT_F32: return reinterpret_cast<const void*>(&quantize_rows<DT_F32>);
    default: return nullptr;
  }
}
