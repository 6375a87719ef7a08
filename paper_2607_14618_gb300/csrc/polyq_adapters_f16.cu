// The adapters' kernels on f16 operands (a translation unit of its own: the types
// compile side by side).
#include "polyq_adapters_dev.cuh"

namespace polyq {
namespace lora {
template Kernel shrink_of<__half>(int bm, int rn, bool trans, bool any);
template Kernel expand_of<__half>(int bm, int rn, bool trans, bool f32);
template Kernel gradients_of<__half>(int rn, bool any);
}  // namespace lora
}  // namespace polyq
