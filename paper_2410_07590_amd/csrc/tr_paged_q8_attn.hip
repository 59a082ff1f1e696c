// Decode attention over a paged cache in 8 bits: one new token per request, lengths and page ids known on the GPU only.
#include "tr_device.h"
#include "tr_internal.h"
#include "tr_q8.h"

namespace {

// A wave per query head of a request; each lane takes every 64th visible key, and the lanes' sums are joined at the end.
template <int DTYPE, int D>
__global__ __launch_bounds__(64) void decode_q8_kernel(const TrPagedDecodeArgs a)
{
    const int lane = threadIdx.x, head = blockIdx.x % a.n_q_heads, r = blockIdx.x / a.n_q_heads, kvh = head / a.group;
    __shared__ float q[D], sums[D];
    for (int c = lane; c < D; c += 64) {
        const int64_t at = (int64_t)blockIdx.x * D + c;
        q[c] = DTYPE == TR_BF16 ? (float)((const __bf16*)a.q)[at] : ((const float*)a.q)[at];
        sums[c] = 0.0f;
    }
    __syncthreads();
    const int shift = a.pool.page_shift, kv_len = max(a.kv_lens[r], 0);
    const int len = min((int64_t)kv_len, (int64_t)a.max_blocks << shift);
    float o[D], m = -__FLT_MAX__, l = 0.0f;
#pragma unroll
    for (int c = 0; c < D; ++c) o[c] = 0.0f;
    for (int j = lane; j < len; j += 64) {
        if (a.window && j < kv_len - a.window && j >= a.n_sink) continue;
        const int page = a.table[(int64_t)r * a.max_blocks + (j >> shift)], row = j & ((1 << shift) - 1);
        if ((uint32_t)page >= (uint32_t)a.pool.n_pages) continue;
        const int64_t at = (int64_t)page * a.pool.page_stride + (int64_t)row * a.pool.row_stride + (int64_t)kvh * a.pool.head_stride;
        const int64_t block = (((int64_t)page * a.n_kv_heads + kvh) << (shift - 4)) + (row >> 4);
        const float ks = q8_power(a.pool.k_scale[block] - 127), vs = q8_power(a.pool.v_scale[block] - 127);
        float s = 0.0f;
        for (int c = 0; c < D; c += 4) {
            float x[4];
            q8_decode(*(const uint32_t*)(a.pool.k + at + c), x);
            for (int i = 0; i < 4; ++i) s = fmaf(x[i] * ks, q[c + i], s);
        }
        const float to = fmaxf(m, s), alpha = __builtin_amdgcn_exp2f((m - to) * a.scale_log2e), w = __builtin_amdgcn_exp2f((s - to) * a.scale_log2e);
        m = to;
        l = l * alpha + w;
#pragma unroll
        for (int c = 0; c < D; c += 4) {
            float x[4];
            q8_decode(*(const uint32_t*)(a.pool.v + at + c), x);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[c + i] = fmaf(x[i] * vs, w, o[c + i] * alpha);
        }
    }
    float top = m;
    for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float f = __builtin_amdgcn_exp2f((m - top) * a.scale_log2e);
    l *= f;
    for (int i = 32; i; i >>= 1) l += __shfl_xor(l, i);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int c = 0; c < D; ++c) {
        float x = o[c] * f;
        for (int i = 32; i; i >>= 1) x += __shfl_xor(x, i);
        if (lane == 0) sums[c] = x * inv;
    }
    __syncthreads();
    for (int c = lane; c < D; c += 64) {
        const int64_t at = (int64_t)blockIdx.x * D + c;
        if (DTYPE == TR_BF16) ((__bf16*)a.out)[at] = (__bf16)sums[c];
        else ((float*)a.out)[at] = sums[c];
    }
}

} // namespace

int tr_launch_paged_decode_q8(const TrPagedDecodeArgs& a, int dtype, int head_dim, int, hipStream_t s)
{
    const dim3 grid((uint32_t)(a.n_req * a.n_q_heads)), block(64);
    if (dtype == TR_BF16) {
        if (head_dim == 128) decode_q8_kernel<TR_BF16, 128><<<grid, block, 0, s>>>(a);
        else decode_q8_kernel<TR_BF16, 64><<<grid, block, 0, s>>>(a);
    } else {
        if (head_dim == 128) decode_q8_kernel<TR_F32, 128><<<grid, block, 0, s>>>(a);
        else decode_q8_kernel<TR_F32, 64><<<grid, block, 0, s>>>(a);
    }
    TR_HIP(hipGetLastError());
    return TR_OK;
}
