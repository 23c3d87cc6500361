// Attention of several new tokens over f16 caches.
#include "prompt_kernel.h"

namespace apc {

hipError_t launch_prompt_f16(const apc_kv& c, const PromptArgs& a, const PromptPlan& p, hipStream_t s)
{
    return launch_prompt<APC_F16, APC_F16>(c, a, p, s);
}

}  // namespace apc
