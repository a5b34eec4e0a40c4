// Geometry-only launcher of the operators of a decoding tenant, beside stub_kernels.cpp: the executor's own code runs, kernels do not.
#include "../../paper_2304_11745_amd/csrc/kernels.h"
#include "../../paper_2304_11745_amd/csrc/tokens_geom.h"
#include "token_kernels.h"

namespace gacer {
TokenLaunches token_launches;
int current_device = 0;
LaunchInfo launch_tokens(const TokenArgs &a, hipStream_t, bool dry, int phase)
{
    LaunchInfo li;
    li.workgroups = (a.b_hi - a.b_lo) * (a.op == TK_SAMPLE ? a.S : 1);
    li.threads = 256; li.lds_bytes = 0; li.wg_per_cu = 8; li.kernel = phase == 2 ? "token_join" : "token";
    li.phases = a.op == TK_CACHE_ATTENTION && attend_geom(a).splits > 1 ? 2 : 1;
    if (a.op == TK_QKNORM_ROPE && a.R == 0 && (a.positions || a.axes || a.table)) ++token_launches.stray_positions;
    if (!dry) {
        ++token_launches.all;
        token_launches.device = current_device;
        if (a.op == TK_QKNORM_ROPE && a.x == a.y) ++token_launches.in_place_at[a.x];
        if (token_ws_floats(a)) a.ws[token_ws_floats(a) - 1] = 1.f;      // the last float of the workspace is there
    }
    return li;
}
}  // namespace gacer

// two devices (linked with --wrap)
extern "C" hipError_t __wrap_hipGetDevice(int *d) { *d = gacer::current_device; return hipSuccess; }
extern "C" hipError_t __wrap_hipSetDevice(int d) { gacer::current_device = d; return d < 2 ? hipSuccess : hipErrorInvalidDevice; }
