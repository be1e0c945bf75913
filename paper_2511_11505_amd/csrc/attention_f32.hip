// Attention over an fp32 cache: the kernels of each width and row count.

#include "attention_kernel.hpp"

namespace fs {

template hipError_t run_attention<CACHE_F32, 64, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 1, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 1, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 64, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 1, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 1, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 2, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 128, 2, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 256, 1, PAGES_ANY, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 256, 1, PAGES_ANY, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 256, 1, PAGES_ANY, NEW_PROMPT>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 256, 1, PAGES_GROUPS, NEW_ONE>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 256, 1, PAGES_GROUPS, NEW_SOME>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_F32, 256, 1, PAGES_GROUPS, NEW_PROMPT>(const AttnPlan&, hipStream_t);

}  // namespace fs
