// Trees of many rows: prompt attention whose rows see what is before their tree, their ancestors and themselves (prompt_launch.h has the kernels).
#include "prompt_launch.h"

namespace sck {

hipError_t launch_prompt_tree(const AttendArgs &a, sc_dtype dtype, hipStream_t stream)
{
    if (dtype == SC_BF16) launch_typed<Bf16, true, kTree>(a, stream);
    else launch_typed<F16, true, kTree>(a, stream);
    return hipGetLastError();
}

}  // namespace sck
