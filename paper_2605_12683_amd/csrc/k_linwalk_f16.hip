// The walk of linear attention (linwalk.h) for f16 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_f16(const LinArgs &a, const LinRole *roles, int n, bool states, bool fine, hipStream_t st) {
    if (states) return launch_walk_parts<F16, 2, false>(a, roles, n, st);
    return fine ? launch_walk_parts<F16, 3, true>(a, roles, n, st) : launch_walk_parts<F16, 2, true>(a, roles, n, st);
}

}  // namespace deer
