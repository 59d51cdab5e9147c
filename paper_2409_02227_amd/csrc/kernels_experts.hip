// Rows of experts: their order, and tokens' rows to them and back.
#include "experts.h"
const void* gdy::scatter_kernel(int dt, int mode) {
#define GDY_SCATTER(DT, MODE) reinterpret_cast<const void*>(&scatter_rows<DT, MODE>)
  switch (dt * 3 + mode) {
    case DT_FP8 * 3: return GDY_SCATTER(DT_FP8, 0);
    case DT_F16 * 3:  // a copy of the same size
    case DT_BF16 * 3: return GDY_SCATTER(DT_BF16, 0);
    case DT_F32 * 3: return GDY_SCATTER(DT_F32, 0);
    case DT_BF16 * 3 + 1: return GDY_SCATTER(DT_BF16, 1);
    case DT_F16 * 3 + 1: return GDY_SCATTER(DT_F16, 1);
    case DT_F32 * 3 + 1: return GDY_SCATTER(DT_F32, 1);
    case DT_BF16 * 3 + 2: return GDY_SCATTER(DT_BF16, 2);
    case DT_F16 * 3 + 2: return GDY_SCATTER(DT_F16, 2);
    case DT_F32 * 3 + 2: return GDY_SCATTER(DT_F32, 2);
    default: return nullptr;
  }
#undef GDY_SCATTER
}
const void* gdy::combine_kernel(int dt) {
  switch (dt) {
    case DT_BF16: return reinterpret_cast<const void*>(&combine_rows<DT_BF16>);
    case DT_F16: return reinterpret_cast<const void*>(&combine_rows<DT_F16>);
    case DT_F32: return reinterpret_cast<const void*>(&combine_rows<DT_F32>);
    default: return nullptr;
  }
}
const void* gdy::route_count_kernel(bool few) {
  return few ? reinterpret_cast<const void*>(&route_count<kRouteFew>) : reinterpret_cast<const void*>(&route_count<kMaxExperts>);
}
const void* gdy::route_sums_kernel() { return reinterpret_cast<const void*>(&route_sums); }
const void* gdy::route_slots_kernel(bool few, int waves) {
#define GDY_SLOTS(EXPERTS, WAVES) reinterpret_cast<const void*>(&route_slots<EXPERTS, WAVES>)
  if (waves == kRouteSmall) return few ? GDY_SLOTS(kRouteFew, kRouteSmall) : nullptr;
  return few ? GDY_SLOTS(kRouteFew, kRoutePart / 64) : GDY_SLOTS(kMaxExperts, kRoutePart / 64);
#undef GDY_SLOTS
}
