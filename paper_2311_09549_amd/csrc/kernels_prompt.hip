// Prompt attention: every key before a row (prompt_launch.h has the kernels).
#include "prompt_launch.h"

namespace sck {

int prompt_shares(int n_cu) { return n_cu; }   // the registers of a workgroup are a compute unit's

size_t prompt_workspace(sc_dtype dtype, int head_dim, int n_cu)
{
    if (dtype == SC_F32) return 0;
    const int dp = padded_dim(head_dim), n = prompt_shares(n_cu);
    const size_t piece = dp == 64 ? kPromptWaves<64> * kPromptPiece<64> : dp == 128 ? kPromptWaves<128> * kPromptPiece<128> : kPromptWaves<256> * kPromptPiece<256>;
    return 2 * n * (piece * sizeof(float) + sizeof(int32_t));
}

hipError_t launch_prompt(const AttendArgs &a, sc_dtype dtype, bool paged, hipStream_t stream)
{
    if (a.window) return launch_prompt_window(a, dtype, paged, stream);
    launch_all<kEverything>(a, dtype, paged, stream);
    return hipGetLastError();
}

}  // namespace sck
