// Attention over a cache held in 4 bits: the kernels for all widths up to 128.
#include "cache_attention_kernels.cuh"

namespace lilicorr {
template lilicorr_status_t ca_launch_rows<32, 0>(const CaArgs&, const CaPlan&, cudaStream_t);
template lilicorr_status_t ca_launch_rows<64, 0>(const CaArgs&, const CaPlan&, cudaStream_t);
template lilicorr_status_t ca_launch_rows<128, 0>(const CaArgs&, const CaPlan&, cudaStream_t);
}  // namespace lilicorr
