// Optional per-kernel timing with HIP events on the caller's stream, shared by the entry points' units: which families of
// kernels there are, and the macro that every launch goes through.
#pragma once
#include <hip/hip_runtime.h>

#define TFLA_TRY(expr)                         \
    do {                                       \
        hipError_t e_ = (expr);                \
        if (e_ != hipSuccess) return (int)e_;  \
    } while (0)

namespace tfla {

enum { K_GATES = 0, K_BWD_PREP, K_REC_FWD, K_REC_BWD, K_TILE_H, K_TILE_DV, K_TILE_DQ, K_TILE_DK, K_GATE_GRADS,
       K_STATE_DOT, K_STEP, K_NORM_FWD, K_NORM_BWD, K_GAIN, K_TILE_GRADS, K_ROWNORM_FWD, K_ROWNORM_BWD,
       K_GEMM, K_ACT_BWD, K_COUNT };
const char* const kKernelNames[K_COUNT] = {"gates", "gate_bwd_prep", "recurrent_fwd", "recurrent_bwd", "tile_H",
                                           "tile_dV", "tile_dQ", "tile_dK", "gate_grads", "state_dot",
                                           "recurrent_step", "norm_gate_fwd", "norm_gate_bwd", "transfer_gain", "tile_grads",
                                           "rownorm_fwd", "rownorm_bwd", "gemm", "act_bwd"};
struct Profiler {
    bool on = false;
    int cap = 0, used = 0;
    hipEvent_t* beg = nullptr;
    hipEvent_t* end = nullptr;
    int* slot = nullptr;
    double total_ms[K_COUNT] = {};
    long launches[K_COUNT] = {};
};
extern Profiler g_prof;

struct ProfScope {
    int idx;
    hipStream_t s;
    ProfScope(int slot, hipStream_t st) : idx(-1), s(st) {
        if (g_prof.on && g_prof.used < g_prof.cap) {
            idx = g_prof.used++;
            g_prof.slot[idx] = slot;
            (void)hipEventRecord(g_prof.beg[idx], s);
        }
    }
    ~ProfScope() {
        if (idx >= 0) (void)hipEventRecord(g_prof.end[idx], s);
    }
};

}  // namespace tfla

#define TFLA_LAUNCH(slot, expr)     \
    do {                            \
        ProfScope ps_((slot), s);   \
        TFLA_TRY(expr);             \
    } while (0)
