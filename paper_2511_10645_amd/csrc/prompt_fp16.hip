// The prompts' attention over fp16 caches.
#include "prompt_kernel.h"

hipError_t paro::launch_prompt_fp16(int head_dim, bool scored, PromptArgs &a, hipStream_t s) { return launch_prompt<kFp16>(head_dim, scored, a, s); }
