// Host-side geometry of the operators of a decoding tenant that both their launchers and the executor need.
#pragma once
#include <stddef.h>
#include "kernels.h"

namespace gacer {

// Floats of workspace that the unsplit operator needs.
inline size_t token_ws_floats(const TokenArgs &a)
{
    (void)a;
    return 0;
}

}  // namespace gacer
