// The kernels of the attention over a paged K/V cache whose pools hold int8 codes.
#include "kv_attn_launch.h"

namespace hk {
namespace kvattn {

hipError_t launch_int8(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s)
{
    return launch_format<kvfmt::kInt8>(p, pl, head_dim, dtype, s);
}

}  // namespace kvattn
}  // namespace hk
