// gsd_verify_attn_paged, tcgen05 back end: the instances for a cache in pages (no plans from tables).
#include "gsd_attn_tc.cuh"

namespace gsd {

template <bool LONG_MASK>
static int launch_plan(const AttnArgs& a) {
    switch (a.plan.dev.balanced == 3 ? PLAN_WAVE : a.plan.dev.longest_first ? PLAN_ORDERED : PLAN_FIXED) {
        case PLAN_WAVE: return a.D == 128 ? launch_tc<128, PLAN_WAVE, LONG_MASK, true>(a) : launch_tc<64, PLAN_WAVE, LONG_MASK, true>(a);
        case PLAN_ORDERED: return a.D == 128 ? launch_tc<128, PLAN_ORDERED, LONG_MASK, true>(a) : launch_tc<64, PLAN_ORDERED, LONG_MASK, true>(a);
        default: return a.D == 128 ? launch_tc<128, PLAN_FIXED, LONG_MASK, true>(a) : launch_tc<64, PLAN_FIXED, LONG_MASK, true>(a);
    }
}

int launch_attn_tcgen05_paged(const AttnArgs& a, bool long_mask) { return long_mask ? launch_plan<true>(a) : launch_plan<false>(a); }

}  // namespace gsd
