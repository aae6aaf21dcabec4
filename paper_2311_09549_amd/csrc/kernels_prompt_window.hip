// Prompt attention through a window (prompt_launch.h has the kernels).
#include "prompt_launch.h"

namespace sck {

hipError_t launch_prompt_window(const AttendArgs &a, sc_dtype dtype, bool paged, hipStream_t stream)
{
    launch_all<kWindow>(a, dtype, paged, stream);
    return hipGetLastError();
}

}  // namespace sck
