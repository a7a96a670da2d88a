// C entry points to the plans of the cache operators (cache_plan.h), compiled
// for the CPU by tests/test_cache_plans_cpu.py.
#include "cache_plan.h"

extern "C" {

// out: total, ml, then kc, chunks, slot0 and first of the four kinds
void prefix_plan(const logo_problem *p, const logo_prefix *x, int share, size_t room,
                 long long out[18]) {
    const logo::PrefixPlan d = logo::prefix_plan(p, x, share, room);
    out[0] = (long long)d.total;
    out[1] = (long long)d.ml;
    for (int i = 0; i < 4; i++) {
        out[2 + i] = d.kc[i];
        out[6 + i] = d.chunks[i];
        out[10 + i] = d.slot0[i];
        out[14 + i] = d.first[i + 1] - d.first[i];
    }
}

// out: total, kc, chunks
void score_plan(const logo_problem *p, int cap, size_t room, long long out[3]) {
    const logo::ScorePlan d = logo::score_plan(p, cap, room);
    out[0] = (long long)d.total;
    out[1] = d.lse_kc;
    out[2] = d.lse_chunks;
}

void step_plan(const logo_problem *p, size_t room, long long out[3]) {
    const logo::StepScorePlan d = logo::step_score_plan(p, room);
    out[0] = (long long)d.total;
    out[1] = d.kc;
    out[2] = d.chunks;
}

int score_key_waves(const logo_problem *p, int cap) {
    return logo::score_plan(p, cap, SIZE_MAX).key_waves;
}

int step_head_copies(const logo_problem *p) {
    return logo::step_score_plan(p, SIZE_MAX).head_copies;
}

long long evict_total(const logo_problem *p) { return (long long)logo::evict_plan(p).total; }

}  // extern "C"
