#include "tree_attn.hpp"

kvb::TreeKernel kvb::tree_kernel_fp8(int D, bool bf16, bool f32, int nb) { return TreeKernelOf<false, false>::choose<KV_FORMAT_FP8>(D, bf16, f32, nb); }
