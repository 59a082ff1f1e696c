// Decode attention over a paged cache in 8 bits.
#include "tr_paged_decode.h"

namespace {

template <int FMT> int launch_decode(const TrPagedDecodeArgs& a, int head_dim, int grid, hipStream_t s)
{
    constexpr int W1 = tr_q8_workers(FMT & 1, 16), W2 = tr_q8_workers(FMT & 1, 32);
    if (a.group <= 16) return head_dim == 128 ? launch_decode<FMT, 128, 1, W1>(a, grid, s) : launch_decode<FMT, 64, 1, W1>(a, grid, s);
    return head_dim == 128 ? launch_decode<FMT, 128, 2, W2>(a, grid, s) : launch_decode<FMT, 64, 2, W2>(a, grid, s);
}

} // namespace

int tr_launch_paged_decode_q8(const TrPagedDecodeArgs& a, int dtype, int head_dim, int grid, hipStream_t s)
{
    return dtype == TR_BF16 ? launch_decode<FMT_Q8_BF16>(a, head_dim, grid, s) : launch_decode<FMT_Q8_F32>(a, head_dim, grid, s);
}
