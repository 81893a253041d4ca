// The walk of linear attention (linwalk.h) for bf16 operands.
#include "linwalk.h"

namespace deer {

int launch_lin_walk_bf16(const LinArgs &a, const LinRole *roles, int n, bool states, bool dots, hipStream_t st) {
    return launch_walk_type<Bf16>(a, roles, n, states, dots, st);
}

}  // namespace deer
