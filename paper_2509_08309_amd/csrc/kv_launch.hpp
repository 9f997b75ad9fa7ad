// Launches of the cache calls, with the events of hetis_kv_profile_events (defined in hetis_kv.hip).
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include "../../include/hetis_attn.h"

namespace hetis {

// Optional events attached to the kernel's dispatch (measurement hook, per host thread):
// start is stamped when the kernel begins to execute, stop when it has finished.
extern thread_local hipEvent_t t_kv_begin, t_kv_end;

// `first` / `last`: of the launches of one call.
template <class Kernel, class Params>
int launch_kv(Kernel kernel, dim3 grid, hipStream_t st, const Params &p, bool first = true, bool last = true,
              unsigned threads = 256)
{
    if (t_kv_begin)
        hipExtLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, first ? t_kv_begin : nullptr,
                              last ? t_kv_end : nullptr, 0, p);
    else
        kernel<<<grid, threads, 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? HETIS_OK : HETIS_ERR_LAUNCH;
}

}  // namespace hetis
