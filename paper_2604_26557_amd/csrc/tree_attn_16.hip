#include "tree_attn.hpp"

kvb::TreeKernel kvb::tree_kernel_16(int D, bool bf16, bool f32, int nb) { return TreeKernelOf<false, false>::choose<KV_FORMAT_16>(D, bf16, f32, nb); }
