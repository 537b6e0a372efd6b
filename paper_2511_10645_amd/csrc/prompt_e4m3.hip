// The prompts' attention over E4M3 caches.
#include "prompt_kernel.h"

hipError_t paro::launch_prompt_e4m3(int head_dim, bool scored, PromptArgs &a, hipStream_t s) { return launch_prompt<kE4m3>(head_dim, scored, a, s); }
