#include "tree_attn.hpp"

kvb::GroupKernel kvb::shaped_kernel_16(int D, bool bf16, bool f32, int nb, bool mixed)
{
    return mixed ? TreeKernelOf<true, true>::choose_mixed<KV_FORMAT_16>(D, bf16, f32) : TreeKernelOf<true, true>::choose<KV_FORMAT_16>(D, bf16, f32, nb);
}
