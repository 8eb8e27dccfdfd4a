// The float32 kernels of rm_paged_attention (rm_paged.h).
#include "rm_paged.h"

namespace rm_serve {

void paged_shape_f32(int D, int G, PagedPlan *p) { shape_of<false>(D, G, *p); }
hipError_t launch_paged_f32(const PagedPlan &p, const PagedArgs &a, hipStream_t st) { return by_width<false>(p, a, st); }

}  // namespace rm_serve
