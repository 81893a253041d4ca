// The walk of linear attention (linwalk.h) for f16 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_f16(const LinArgs &a, const LinRole *roles, int n, bool states, bool dots, hipStream_t st) {
    return launch_walk_type<F16>(a, roles, n, states, dots, st);
}

}  // namespace deer
