// Launches of packed rows over the bf16 cache that kv_prompt.hip hands to kv_prompt_wide.hip.
#pragma once

#include "kv_internal.h"

namespace mdi {

struct PromptGeo { int n_blocks, sets, g_sh, from; };            // bound of the blocks of all samples; sets of 2^g_sh query heads; of the launch's first workgroup
bool kv_wide_allow_lds();
void launch_kv_wide(hipStream_t s, const KvCache& c, const KvRows& r, const KvAttn& a, const PromptGeo& g, int wgs, bool many);

}  // namespace mdi
