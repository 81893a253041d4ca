// The walk of linear attention (linwalk.h) for f32 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_f32(const LinArgs &a, const LinRole *roles, int n, bool states, bool fine, hipStream_t st) {
    return states ? launch_walk_parts<F32, 3, false>(a, roles, n, st) : launch_walk_parts<F32, 3, true>(a, roles, n, st);
}

}  // namespace deer
