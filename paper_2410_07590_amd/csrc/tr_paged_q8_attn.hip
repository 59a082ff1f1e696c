// Decode attention over a paged cache in 8 bits.
#include "tr_paged_decode.h"

namespace {

template <int FMT, int D> int launch_decode(const TrPagedDecodeArgs& a, int grid, hipStream_t s)
{
    constexpr int W = tr_q8_workers(D);
    return a.group <= 16 ? launch_decode<FMT, D, 1, W>(a, grid, s) : launch_decode<FMT, D, 2, W>(a, grid, s);
}

} // namespace

int tr_launch_paged_decode_q8(const TrPagedDecodeArgs& a, int dtype, int head_dim, int grid, hipStream_t s)
{
    if (dtype == TR_BF16) return head_dim == 128 ? launch_decode<FMT_Q8_BF16, 128>(a, grid, s) : launch_decode<FMT_Q8_BF16, 64>(a, grid, s);
    return head_dim == 128 ? launch_decode<FMT_Q8_F32, 128>(a, grid, s) : launch_decode<FMT_Q8_F32, 64>(a, grid, s);
}
