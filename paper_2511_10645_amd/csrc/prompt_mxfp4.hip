// The prompts' attention over MXFP4 caches.
#include "prompt_kernel.h"

hipError_t paro::launch_prompt_mxfp4(int head_dim, bool scored, PromptArgs &a, hipStream_t s) { return launch_prompt<kMxfp4>(head_dim, scored, a, s); }
