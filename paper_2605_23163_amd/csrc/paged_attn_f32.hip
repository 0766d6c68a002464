// Attention over a paged cache (paged_attn.h): fp32.
#include "paged_attn.h"

namespace fdd {
namespace paged_attn {

hipError_t launch_f32(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl, const Args& a)
{
    return c.D == 128 ? launch<float, 128, 4>(c, p, pl, a) : launch<float, 64, 4>(c, p, pl, a);
}

}  // namespace paged_attn
}  // namespace fdd
