// Attention over a bf16 cache: the kernels of each width and row count.

#include "attention_kernel.hpp"

namespace fs {

template hipError_t run_attention<CACHE_BF16, 64, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 2, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 2, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 4, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 2, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 2, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 4, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);

}  // namespace fs
