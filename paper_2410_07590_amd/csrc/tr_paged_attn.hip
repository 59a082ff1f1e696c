// Decode attention over a paged cache in the type of the shape.
#include "tr_paged_decode.h"

namespace {

template <int DTYPE> int launch_decode(const TrPagedDecodeArgs& a, int head_dim, int grid, hipStream_t s)
{
    constexpr int W = TR_PAGED_WORKERS;
    if (a.group <= 16) return head_dim == 128 ? launch_decode<DTYPE, 128, 1, W>(a, grid, s) : launch_decode<DTYPE, 64, 1, W>(a, grid, s);
    return head_dim == 128 ? launch_decode<DTYPE, 128, 2, W>(a, grid, s) : launch_decode<DTYPE, 64, 2, W>(a, grid, s);
}

} // namespace

int tr_launch_paged_decode(const TrPagedDecodeArgs& a, int dtype, int head_dim, int grid, hipStream_t s)
{
    return dtype == TR_BF16 ? launch_decode<FMT_BF16>(a, head_dim, grid, s) : launch_decode<FMT_F32>(a, head_dim, grid, s);
}
