// The walk of linear attention (linwalk.h) for f32 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_f32(const LinArgs &a, const LinRole *roles, int n, bool states, bool dots, hipStream_t st) {
    return launch_walk_type<F32>(a, roles, n, states, dots, st);
}

}  // namespace deer
