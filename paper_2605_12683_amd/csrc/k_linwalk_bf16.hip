// The walk of linear attention (linwalk.h) for bf16 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_bf16(const LinArgs &a, const LinRole *roles, int n, bool states, bool dots, hipStream_t st) {
    if (states) return launch_walk_parts<Bf16, 2, kStates>(a, roles, n, st);
    return dots ? launch_walk_parts<Bf16, 3, kOutDots>(a, roles, n, st) : launch_walk_parts<Bf16, 2, kOut>(a, roles, n, st);
}

}  // namespace deer
