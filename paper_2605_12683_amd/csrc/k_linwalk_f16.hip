// The walk of linear attention (linwalk.h) for f16 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_f16(const LinArgs &a, const LinRole *roles, int n, bool states, bool dots, hipStream_t st) {
    if (states) return launch_walk_parts<F16, 2, kStates>(a, roles, n, st);
    return dots ? launch_walk_parts<F16, 3, kOutDots>(a, roles, n, st) : launch_walk_parts<F16, 2, kOut>(a, roles, n, st);
}

}  // namespace deer
