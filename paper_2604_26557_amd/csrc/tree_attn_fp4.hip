#include "tree_attn.hpp"

kvb::TreeKernel kvb::tree_kernel_fp4(int D, bool bf16, bool f32, int nb) { return tree_kernel_for<KV_FORMAT_FP4>(D, bf16, f32, nb); }
