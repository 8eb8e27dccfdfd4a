// The bf16 kernels of rm_paged_attention (rm_paged.h).
#include "rm_paged.h"

namespace rm_serve {

void paged_shape_bf16(int D, int G, PagedPlan *p) { shape_of<true>(D, G, *p); }
hipError_t launch_paged_bf16(const PagedPlan &p, const PagedArgs &a, hipStream_t st) { return by_width<true>(p, a, st); }

}  // namespace rm_serve
