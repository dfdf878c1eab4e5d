#include "tree_attn.hpp"

kvb::GroupKernel kvb::group_kernel_fp8(int D, bool bf16, bool f32, int nb, bool mixed)
{
    return mixed ? TreeKernelOf<true, false>::choose_mixed<KV_FORMAT_FP8>(D, bf16, f32) : TreeKernelOf<true, false>::choose<KV_FORMAT_FP8>(D, bf16, f32, nb);
}
