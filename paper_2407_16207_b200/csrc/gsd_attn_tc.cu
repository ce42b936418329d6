// gsd_verify_attn, tcgen05 back end: its instances for a cache of padded ranges, and the choice among them.
#include "gsd_attn_tc.cuh"

namespace gsd {

unsigned long long g_wait_limit_ns = kWaitLimitNs;
int g_withhold_first_k = 0;

int attn_tcgen05_rows(int G) { return G <= BM ? BM / G * G : BM; }

bool attn_tcgen05_supports(int D, int G) { return (D == 128 || D == 64) && G >= 1 && G <= BM; }

template <bool LONG_MASK>
static int launch_plan(const AttnArgs& a) {
    switch (a.plan.dev.balanced == 3 ? PLAN_WAVE : a.plan.dev.balanced ? PLAN_TABLE : a.plan.dev.longest_first ? PLAN_ORDERED : PLAN_FIXED) {
        case PLAN_WAVE: return a.D == 128 ? launch_tc<128, PLAN_WAVE, LONG_MASK, false>(a) : launch_tc<64, PLAN_WAVE, LONG_MASK, false>(a);
        case PLAN_ORDERED: return a.D == 128 ? launch_tc<128, PLAN_ORDERED, LONG_MASK, false>(a) : launch_tc<64, PLAN_ORDERED, LONG_MASK, false>(a);
        case PLAN_TABLE: return launch_tc<128, PLAN_TABLE, LONG_MASK, false>(a);     // (D = 128 only)
        default: return a.D == 128 ? launch_tc<128, PLAN_FIXED, LONG_MASK, false>(a) : launch_tc<64, PLAN_FIXED, LONG_MASK, false>(a);
    }
}

// The mask words of a unit are more than a warp fetches in one round of 16-byte loads (one head a group: N above
// 170, two: above 256, three: above 384, four and more: never).  A kernel of its own: the code for slices in the
// others' prologue cost calls of a few tiles up to 4%; with up to 1024 words it is a wash (D 64, 4 x 32/8 heads, N 428,
// L 20322, 896 words: 586 us, 592 so).
static bool long_mask(const AttnArgs& a) {
    const int nodes = 2 * (BM / a.G);
    return (nodes < a.N ? nodes : a.N) * a.W > 8 * 32 * 4;
}

int launch_attn_tcgen05(const AttnArgs& a) {
    if (!attn_tcgen05_supports(a.D, a.G)) {
        set_error_text("tcgen05 back end needs a head dimension of 64 or 128 and a group size of at most 128");
        return GSD_ERR_UNSUPPORTED;
    }
    if (a.pages.table) return launch_attn_tcgen05_paged(a, long_mask(a));
    return long_mask(a) ? launch_plan<true>(a) : launch_plan<false>(a);
}

void debug_attn_wait(unsigned long long limit_ns, int withhold_first_k) {
    g_wait_limit_ns = limit_ns ? limit_ns : kWaitLimitNs;
    g_withhold_first_k = withhold_first_k;
}

}  // namespace gsd
