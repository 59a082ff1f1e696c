// Kernels of the paged cache: block tables and slots of a batch, append with head norms and rotation, decode attention.
#include "tr_internal.h"

#include <algorithm>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// ---- block tables, slots, position ids ------------------------------------------------------------------------------------
// One launch and no traffic between workgroups: each works out the prefix sums of the whole batch again (two lengths per
// request, from the caches) and then the slots of its own 1024 tokens, a few pages and, the first, the batch's lengths.
// A token finds its request by bisection of the sums in LDS, a thread does it once for four neighbours.

// Largest r with starts[r] <= x, for starts[0] = 0 <= x < starts[n]: requests without entries are passed over.
__device__ __forceinline__ int owner(const int32_t* starts, int n, int x)
{
    int lo = 0, hi = n; // starts[lo] <= x < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ int32_t cut(int64_t x) { return (int32_t)min(x, (int64_t)INT32_MAX); }

__global__ __launch_bounds__(256) void page_map_kernel(const TrPageMapArgs a)
{
    extern __shared__ int32_t sums[];
    __shared__ int64_t wave_sum[4][2];
    int32_t* const cu = sums;               // [n_req + 1] first token of each request
    int32_t* const pg = sums + a.n_req + 1; // [n_req + 1] first new page
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.n_req + 255) / 256, shift = a.page_shift;
    const int64_t round = (1 << shift) - 1;
    auto pages = [&](int64_t tokens) { return (tokens + round) >> shift; };

    int64_t tok = 0, pag = 0;
    for (int i = 0; i < per; ++i) {
        const int r = tid * per + i;
        if (r >= a.n_req) break;
        const int64_t c = max(a.cached[r], 0), f = max(a.fresh[r], 0);
        tok += f;
        pag += pages(c + f) - pages(c);
    }
    int64_t tok_to = tok, pag_to = pag; // inclusive sums over the wave
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t t = __shfl_up(tok_to, o), p = __shfl_up(pag_to, o);
        if (lane >= o) tok_to += t, pag_to += p;
    }
    if (lane == 63) wave_sum[wave][0] = tok_to, wave_sum[wave][1] = pag_to;
    __syncthreads();
    tok_to -= tok;
    pag_to -= pag;
    int64_t tok_all = 0, pag_all = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) tok_to += wave_sum[w][0], pag_to += wave_sum[w][1];
        tok_all += wave_sum[w][0], pag_all += wave_sum[w][1];
    }
    for (int i = 0; i < per; ++i) {
        const int r = tid * per + i;
        if (r >= a.n_req) break;
        const int64_t c = max(a.cached[r], 0), f = max(a.fresh[r], 0);
        cu[r] = cut(tok_to);
        pg[r] = cut(pag_to);
        if (blockIdx.x == 0) {
            a.cu[r] = cut(tok_to);
            a.kv_lens[r] = cut(c + f);
        }
        tok_to += f;
        pag_to += pages(c + f) - pages(c);
    }
    if (tid == 0) {
        cu[a.n_req] = cut(tok_all);
        pg[a.n_req] = cut(pag_all);
        if (blockIdx.x == 0) {
            a.cu[a.n_req] = cut(tok_all);
            a.counts[0] = cut(tok_all);
            a.counts[1] = cut(pag_all);
        }
    }
    __syncthreads();

    const int n_tok = cu[a.n_req], n_pag = pg[a.n_req];
    auto free_page = [&](int i) { return i < a.n_free ? a.free_pages[i] : -1; };
    for (int64_t p = (int64_t)blockIdx.x * 256 + tid; p < n_pag; p += (int64_t)gridDim.x * 256) {
        const int r = owner(pg, a.n_req, (int)p);
        const int64_t blk = pages(max(a.cached[r], 0)) + p - pg[r];
        if (blk < a.max_blocks) a.table[(int64_t)r * a.max_blocks + blk] = free_page((int)p);
    }

    const int64_t t0 = (int64_t)blockIdx.x * TR_MAP_TOKENS + 4 * tid;
    if (t0 >= a.n_slots) return;
    int32_t slot[4], pos[4];
    int r = t0 < n_tok ? owner(cu, a.n_req, (int)t0) : 0;
    int last = -1, c = 0, first = 0;
    for (int i = 0; i < 4; ++i) {
        const int64_t t = t0 + i;
        slot[i] = -1;
        pos[i] = 0;
        if (t >= n_tok) continue;
        while (cu[r + 1] <= t) ++r;
        if (r != last) {
            last = r;
            c = max(a.cached[r], 0);
            first = a.first_pos ? a.first_pos[r] : c;
        }
        const int64_t at = t - cu[r], row = c + at, blk = row >> shift, have = pages(c);
        pos[i] = (int32_t)((uint32_t)first + (uint32_t)at);
        if (blk >= a.max_blocks) continue;
        const int page = blk < have ? a.table[(int64_t)r * a.max_blocks + blk] : free_page((int)min(pg[r] + blk - have, (int64_t)INT32_MAX));
        const int64_t s = ((int64_t)page << shift) + (row & round);
        slot[i] = page < 0 || s > INT32_MAX ? -1 : (int32_t)s;
    }
    if (t0 + 4 <= a.n_slots) {
        *(i32x4_any*)(a.slots + t0) = i32x4_any{slot[0], slot[1], slot[2], slot[3]};
        *(i32x4_any*)(a.pos + t0) = i32x4_any{pos[0], pos[1], pos[2], pos[3]};
    } else {
        for (int i = 0; i < 4 && t0 + i < a.n_slots; ++i) a.slots[t0 + i] = slot[i], a.pos[t0 + i] = pos[i];
    }
}

// ---- heads: norm, rotation, rows of the pool --------------------------------------------------------------------------------

// A 16-byte unit of a head in fp32: 8 bf16 or 4 fp32 channels.
template <int DTYPE> struct Vec;
template <> struct Vec<TR_BF16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void open(u32x4 u, float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ u32x4 close(const float (&x)[8])
    {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        bf16x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (__bf16)x[i];
        return __builtin_bit_cast(u32x4, y);
    }
};
template <> struct Vec<TR_F32> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void open(u32x4 u, float (&x)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(u[i]);
    }
    static __device__ __forceinline__ u32x4 close(const float (&x)[4])
    {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(x[i]);
        return u;
    }
};

template <int LANES> __device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = LANES / 2; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// A workgroup owns one token; LPH neighbouring lanes own a head, a 16-byte unit each.  The token's angles are worked out once
// (a thread per pair, 64 bits) into LDS for all of its heads.
template <int DTYPE, int D, bool HALF>
__global__ __launch_bounds__(256) void paged_append_kernel(const TrPagedAppendArgs a)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N;
    __shared__ float2 turn[64]; // cosine and sine of each pair, times the amplitude
    const int tid = threadIdx.x, piece = tid % LPH;
    const int pairs = a.rotary_dim / 2;
    const int half_units = pairs / N; // units of half the turned channels
    const bool turns = piece * N < a.rotary_dim, low = piece < half_units;
    const int n_heads = a.n_q_heads + 2 * a.n_kv_heads;
    float qw[N], kw[N];
    if (a.q_norm) V::open(((const u32x4*)a.q_norm)[piece], qw);
    if (a.k_norm) V::open(((const u32x4*)a.k_norm)[piece], kw);
    for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
        __syncthreads();
        if (tid < pairs) {
            double sn, cn;
            tr_sincos((double)a.pos[t] * a.freq[tid], &sn, &cn);
            turn[tid] = make_float2((float)(cn * a.amplitude), (float)(sn * a.amplitude));
        }
        __syncthreads();
        const int slot = a.n_kv_heads ? a.slots[t] : -1;
        const int page = slot >> a.pool.page_shift;
        const bool stored = slot >= 0 && page < a.pool.n_pages;
        const int64_t row = (int64_t)page * a.pool.page_stride + (int64_t)(slot & ((1 << a.pool.page_shift) - 1)) * a.pool.row_stride;
        for (int h = tid / LPH; h < n_heads; h += 256 / LPH) {
            const bool is_q = h < a.n_q_heads, is_v = h >= a.n_q_heads + a.n_kv_heads;
            const int hk = h - a.n_q_heads - (is_v ? a.n_kv_heads : 0);
            const char* src = is_q ? a.q + t * a.q_stride + (int64_t)h * D * sizeof(u32x4) / N
                                   : (is_v ? a.v + t * a.v_stride : a.k + t * a.k_stride) + (int64_t)hk * D * sizeof(u32x4) / N;
            u32x4 u = ((const u32x4*)src)[piece];
            const bool normed = is_q ? a.q_norm != nullptr : a.k_norm != nullptr;
            if (!is_v && (normed || pairs)) {
                float x[N];
                V::open(u, x);
                if (normed) {
                    float ss = 0.0f;
#pragma unroll
                    for (int i = 0; i < N; ++i) ss = fmaf(x[i], x[i], ss);
                    const float r = 1.0f / sqrtf(lanes_sum<LPH>(ss) * (1.0f / D) + a.eps);
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] = x[i] * r * (is_q ? qw[i] : kw[i]);
                }
                if (HALF) {
                    float y[N];
                    const int partner = (tid & 63) + (low ? half_units : -half_units);
#pragma unroll
                    for (int i = 0; i < N; ++i) y[i] = __shfl(x[i], turns ? partner : tid & 63);
                    if (turns) {
                        const int m0 = (low ? piece : piece - half_units) * N;
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const float2 e = turn[m0 + i];
                            x[i] = low ? x[i] * e.x - y[i] * e.y : x[i] * e.x + y[i] * e.y;
                        }
                    }
                } else if (turns) {
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) {
                        const float2 e = turn[piece * (N / 2) + i];
                        const float p = x[2 * i], s = x[2 * i + 1];
                        x[2 * i] = p * e.x - s * e.y;
                        x[2 * i + 1] = s * e.x + p * e.y;
                    }
                }
                if (normed || turns) u = V::close(x);
            }
            if (is_q) ((u32x4*)(a.q_out + (t * a.n_q_heads + h) * (int64_t)(D * sizeof(u32x4) / N)))[piece] = u;
            else if (stored) ((u32x4*)((is_v ? a.pool.v : a.pool.k) + row + hk * a.pool.head_stride))[piece] = u;
        }
    }
}

} // namespace

int tr_launch_page_map(const TrPageMapArgs& a, hipStream_t s)
{
    const int blocks = std::max((int)(((int64_t)a.n_slots + TR_MAP_TOKENS - 1) / TR_MAP_TOKENS), 1);
    page_map_kernel<<<dim3(blocks), dim3(256), 2 * (a.n_req + 1) * sizeof(int32_t), s>>>(a);
    TR_HIP(hipGetLastError());
    return TR_OK;
}

template <int DTYPE, int D> static void launch_append(const TrPagedAppendArgs& a, int layout, hipStream_t s)
{
    const dim3 grid(std::min(a.n_tokens, TR_MAX_BLOCKS_256));
    if (layout == TR_ROPE_HALF) paged_append_kernel<DTYPE, D, true><<<grid, dim3(256), 0, s>>>(a);
    else paged_append_kernel<DTYPE, D, false><<<grid, dim3(256), 0, s>>>(a);
}
int tr_launch_paged_append(const TrPagedAppendArgs& a, int dtype, int head_dim, int layout, hipStream_t s)
{
    if (dtype == TR_BF16) head_dim == 128 ? launch_append<TR_BF16, 128>(a, layout, s) : launch_append<TR_BF16, 64>(a, layout, s);
    else head_dim == 128 ? launch_append<TR_F32, 128>(a, layout, s) : launch_append<TR_F32, 64>(a, layout, s);
    TR_HIP(hipGetLastError());
    return TR_OK;
}
