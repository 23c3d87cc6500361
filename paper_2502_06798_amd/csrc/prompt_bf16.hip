// Attention of several new tokens over bf16 caches.
#include "prompt_kernel.h"

namespace apc {

hipError_t launch_prompt_bf16(const apc_kv& c, const PromptArgs& a, const PromptPlan& p, hipStream_t s)
{
    return launch_prompt<APC_BF16, APC_BF16>(c, a, p, s);
}

}  // namespace apc
