// Attention of several new tokens over e4m3 caches.
#include "prompt_kernel.h"

namespace apc {

hipError_t launch_prompt_e4m3(int dt, const apc_kv& c, const PromptArgs& a, const PromptPlan& p, hipStream_t s)
{
    return dt == APC_F16 ? launch_prompt<APC_F16, APC_E4M3>(c, a, p, s) : launch_prompt<APC_BF16, APC_E4M3>(c, a, p, s);
}

}  // namespace apc
