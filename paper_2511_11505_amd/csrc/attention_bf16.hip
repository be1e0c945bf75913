// Attention over a bf16 cache: the kernels of each width and row count.

#include "attention_kernel.hpp"

namespace fs {

template hipError_t run_attention<CACHE_BF16, 64, 1, true, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 1, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 1, false, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 1, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 2, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 2, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 4, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 64, 4, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, true, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, false, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 1, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 2, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 2, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 4, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 128, 4, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, true, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, false, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 1, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 2, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_BF16, 256, 2, false, true>(const AttnPlan&, hipStream_t);

}  // namespace fs
