#include "tree_attn.hpp"

kvb::TreeKernel kvb::tree_kernel_16_paged(int D, bool bf16, bool f32, int nb) { return tree_kernel_for<KV_FORMAT_16, kTreePaged>(D, bf16, f32, nb); }
