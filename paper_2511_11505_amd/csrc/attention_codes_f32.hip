// Attention over an 8-bit cache, fp32 queries: the kernels of each width and row count.

#include "attention_kernel.hpp"

namespace fs {

template hipError_t run_attention<CACHE_CODES_F32, 64, 1, true, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 64, 1, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 64, 1, false, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 64, 1, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 64, 2, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 64, 2, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 128, 1, true, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 128, 1, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 128, 1, false, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 128, 1, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 128, 2, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 128, 2, false, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 256, 1, true, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 256, 1, true, true>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 256, 1, false, false>(const AttnPlan&, hipStream_t);
template hipError_t run_attention<CACHE_CODES_F32, 256, 1, false, true>(const AttnPlan&, hipStream_t);

}  // namespace fs
