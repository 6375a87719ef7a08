// The adapters' kernels on bf16 operands (a translation unit of its own: the types
// compile side by side).
#include "polyq_adapters_dev.cuh"

namespace polyq {
namespace lora {
template Kernel shrink_of<__nv_bfloat16>(int bm, int rn, bool trans, bool any);
template Kernel expand_of<__nv_bfloat16>(int bm, int rn, bool trans, bool f32);
template Kernel gradients_of<__nv_bfloat16>(int rn, bool any);
}  // namespace lora
}  // namespace polyq
