// The gated block in front of the layer: x = act(e V_gate^T) * (e V_up^T), both projections and what follows them in one kernel (k_dense_forward.h).
#include "k_dense_forward.h"

using namespace dense;

usl_status usl_launch_gated(usl_ctx* c, const void* e, const void* V_gate, const void* V_up, int32_t w, int32_t act, void* x, void* gate, void* up, int32_t b) {
    Forward a = {};
    a.V[0] = V_gate; a.V[1] = V_up; a.e = e;
    a.x = x; a.gate = gate; a.up = up;
    a.d = c->d; a.b = b;
    if (c->storage == USL_F32) {
        a.row_bytes = w * 4;
        return act == USL_SILU ? launch_forward<float, float, 2, 0>(c, a, "gated_block") : launch_forward<float, float, 2, 1>(c, a, "gated_block");
    }
    a.row_bytes = w * 2;
    return act == USL_SILU ? launch_forward<bf16, bf16, 2, 0>(c, a, "gated_block") : launch_forward<bf16, bf16, 2, 1>(c, a, "gated_block");
}
