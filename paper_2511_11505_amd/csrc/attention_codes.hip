// Attention over an 8-bit cache, bf16 queries: the kernels of each width and row count.

#include "attention_kernel.hpp"

namespace fs {

template hipError_t run_attention<CACHE_CODES_BF16, 64, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 1, PAGES_GROUPS_SHORT, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 1, PAGES_GROUPS_SHORT, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 2, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 2, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 2, PAGES_GROUPS_SHORT, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 64, 2, PAGES_GROUPS_SHORT, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 1, PAGES_GROUPS_SHORT, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 1, PAGES_GROUPS_SHORT, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 2, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 2, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 2, PAGES_GROUPS_SHORT, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 128, 2, PAGES_GROUPS_SHORT, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_GROUPS_SHORT, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_GROUPS_SHORT, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 1, PAGES_GROUPS_SHORT, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_BF16, 256, 2, PAGES_GROUPS_SHORT, NEW_SOME>(const AttnPlan&, hipStream_t);

}  // namespace fs
