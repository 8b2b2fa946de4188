// The launch of the attention over the paged K/V cache in one format.
#pragma once
#include "kv_attn_kernel.h"
#include "kv_attn_rows.h"

namespace hk {
namespace kvattn {

template <int DH, int DT, int FMT>
hipError_t launch_as(const Params &p, const Plan &pl, hipStream_t s)
{
    const dim3 grid((unsigned)pl.groups), block(kThreads);
    if (pl.shared && pl.tiles == 1) hipLaunchKernelGGL((kv_rows_kernel<DH, DT, FMT, 1>), grid, block, 0, s, p);
    else if (pl.shared) hipLaunchKernelGGL((kv_rows_kernel<DH, DT, FMT, 2>), grid, block, 0, s, p);
    else if (pl.tiles == 2) hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 2, true>), grid, block, 0, s, p);
    else if (p.k) hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 1, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((kv_attn_kernel<DH, DT, FMT, 1, false>), grid, block, 0, s, p);
    return hipGetLastError();
}

template <int FMT>
hipError_t launch_format(const Params &p, const Plan &pl, int head_dim, int dtype, hipStream_t s)
{
    if (head_dim == 128) return dtype == 1 ? launch_as<128, 1, FMT>(p, pl, s) : launch_as<128, 0, FMT>(p, pl, s);
    return dtype == 1 ? launch_as<64, 1, FMT>(p, pl, s) : launch_as<64, 0, FMT>(p, pl, s);
}

}  // namespace kvattn
}  // namespace hk
