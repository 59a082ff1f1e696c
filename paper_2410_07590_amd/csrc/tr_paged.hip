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

// Sum over LANES neighbouring lanes, within a row of 16 on the vector unit's cross-lane path.
template <int LANES> __device__ __forceinline__ float lanes_sum(float x)
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32, "");
    auto bits = [&]() { return __builtin_bit_cast(int, x); };
    auto add = [&](int y) { x += __builtin_bit_cast(float, y); };
    add(__builtin_amdgcn_update_dpp(bits(), bits(), 0xB1, 0xf, 0xf, false));                   // quad_perm [1,0,3,2]
    add(__builtin_amdgcn_update_dpp(bits(), bits(), 0x4E, 0xf, 0xf, false));                   // quad_perm [2,3,0,1]
    add(__builtin_amdgcn_update_dpp(bits(), bits(), 0x141, 0xf, 0xf, false));                  // row_half_mirror
    if (LANES >= 16) add(__builtin_amdgcn_update_dpp(bits(), bits(), 0x140, 0xf, 0xf, false)); // row_mirror
    if (LANES == 32) x += __shfl_xor(x, 16);
    return x;
}

// Bound by memory: a head is read once and written once.  A workgroup owns a few tokens; LPH neighbouring lanes own a head, a
// 16-byte unit each, so a norm and a rotation stay within a wave.  The tokens' angles (a thread per pair, 64 bits) are worked out
// once for all of their heads, while the first UNITS loads of every thread are on their way.
constexpr int APPEND_UNITS = 4;
template <int DTYPE, int D, bool HALF>
__global__ __launch_bounds__(256) void paged_append_kernel(const TrPagedAppendArgs a)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = APPEND_UNITS, HEAD = D * 16 / N; // channels of a unit, units and bytes of a head
    __shared__ float2 turn[TR_PAGED_APPEND_TOKENS * 64]; // cosine and sine of each token's pairs, times the amplitude
    const int tid = threadIdx.x, piece = tid % LPH;
    const int pairs = a.rotary_dim / 2, half_units = pairs / N; // units of half the turned channels
    const bool turns = piece * N < a.rotary_dim, low = piece < half_units;
    const int partner = !HALF || !turns ? (tid & 63) : (tid & 63) + (low ? half_units : -half_units);
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2); // first pair of the unit
    const int n_heads = a.n_q_heads + 2 * a.n_kv_heads;
    const int64_t t0 = (int64_t)blockIdx.x * a.tile_tokens;
    const int tokens = (int)min((int64_t)a.tile_tokens, a.n_tokens - t0), heads = tokens * n_heads;

    float qw[N], kw[N];
    if (a.q_norm) V::open(((const u32x4*)a.q_norm)[piece], qw);
    if (a.k_norm) V::open(((const u32x4*)a.k_norm)[piece], kw);
    struct Unit {
        u32x4 x;
        int tok, h; // of the tile; head of the token: queries, keys, values
    };
    auto load = [&](int i) { // the i-th head that this thread has part in
        Unit u;
        const int at = tid / LPH + i * (256 / LPH);
        if (at >= heads) {
            u.h = -1;
            return u;
        }
        u.tok = a.tile_tokens == 1 ? 0 : at / n_heads;
        u.h = at - u.tok * n_heads;
        const int hk = u.h - a.n_q_heads, hv = hk - a.n_kv_heads;
        const int64_t t = t0 + u.tok;
        const char* src = hk < 0 ? a.q + t * a.q_stride + (int64_t)u.h * HEAD : hv < 0 ? a.k + t * a.k_stride + (int64_t)hk * HEAD : a.v + t * a.v_stride + (int64_t)hv * HEAD;
        u.x = __builtin_nontemporal_load((const u32x4*)src + piece);
        return u;
    };
    Unit u[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) u[i] = load(i);
    for (int i = tid; i < tokens * pairs; i += 256) {
        const int tok = i / pairs, m = i - tok * pairs;
        double sn, cn;
        tr_sincos((double)a.pos[t0 + tok] * a.freq[m], &sn, &cn);
        turn[tok * 64 + m] = make_float2((float)(cn * a.amplitude), (float)(sn * a.amplitude));
    }
    __syncthreads();
    for (int i0 = 0;; i0 += UNITS) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            if (u[i].h < 0) continue; // heads are dealt out whole, so the lanes of one are here together
            const int h = u[i].h, hk = h - a.n_q_heads, hv = hk - a.n_kv_heads;
            const int64_t t = t0 + u[i].tok;
            const bool normed = hk < 0 ? a.q_norm != nullptr : a.k_norm != nullptr;
            if (hv < 0 && (normed || pairs)) {
                const float2* const e = turn + u[i].tok * 64 + m0;
                float x[N];
                V::open(u[i].x, x);
                if (normed) {
                    float ss = 0.0f;
#pragma unroll
                    for (int c = 0; c < N; ++c) ss = fmaf(x[c], x[c], ss);
                    const float r = rsqrtf(lanes_sum<LPH>(ss) * (1.0f / D) + a.eps);
#pragma unroll
                    for (int c = 0; c < N; ++c) x[c] = x[c] * r * (hk < 0 ? qw[c] : kw[c]);
                }
                if (HALF) {
                    float y[N];
#pragma unroll
                    for (int c = 0; c < N; ++c) y[c] = __shfl(x[c], partner);
                    if (turns) {
#pragma unroll
                        for (int c = 0; c < N; ++c) x[c] = x[c] * e[c].x + (low ? -y[c] : y[c]) * e[c].y;
                    }
                } else if (turns) {
#pragma unroll
                    for (int c = 0; c < N / 2; ++c) {
                        const float p = x[2 * c], s = x[2 * c + 1];
                        x[2 * c] = p * e[c].x - s * e[c].y;
                        x[2 * c + 1] = s * e[c].x + p * e[c].y;
                    }
                }
                if (normed || turns) u[i].x = V::close(x);
            }
            if (hk < 0) {
                ((u32x4*)(a.q_out + (t * a.n_q_heads + h) * HEAD))[piece] = u[i].x;
            } else {
                const int slot = a.slots[t], page = slot >> a.pool.page_shift;
                const int64_t row = (int64_t)page * a.pool.page_stride + (int64_t)(slot & ((1 << a.pool.page_shift) - 1)) * a.pool.row_stride;
                if (slot >= 0 && page < a.pool.n_pages)
                    ((u32x4*)(hv < 0 ? a.pool.k + row + (int64_t)hk * a.pool.head_stride : a.pool.v + row + (int64_t)hv * a.pool.head_stride))[piece] = u[i].x;
            }
        }
        if ((i0 + UNITS) * (256 / LPH) >= heads) break;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) u[i] = load(i0 + UNITS + i);
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

template <int DTYPE, int D> static void launch_append(const TrPagedAppendArgs& a, int blocks, int layout, hipStream_t s)
{
    if (layout == TR_ROPE_HALF) paged_append_kernel<DTYPE, D, true><<<dim3(blocks), dim3(256), 0, s>>>(a);
    else paged_append_kernel<DTYPE, D, false><<<dim3(blocks), dim3(256), 0, s>>>(a);
}
int tr_launch_paged_append(const TrPagedAppendArgs& args, int dtype, int head_dim, int layout, hipStream_t s)
{
    TrPagedAppendArgs a = args;
    const int tile = a.tile_tokens;
    // a launch has fewer than 2^32 threads
    for (int64_t at = 0; at < args.n_tokens; at += (int64_t)TR_MAX_BLOCKS_256 * tile) {
        a.n_tokens = (int32_t)std::min<int64_t>(args.n_tokens - at, (int64_t)TR_MAX_BLOCKS_256 * tile);
        if (a.q) a.q = args.q + at * a.q_stride, a.q_out = args.q_out + at * a.n_q_heads * head_dim * (dtype == TR_F32 ? 4 : 2);
        if (a.k) a.k = args.k + at * a.k_stride, a.v = args.v + at * a.v_stride, a.slots = args.slots + at;
        if (a.pos) a.pos = args.pos + at;
        const int blocks = (a.n_tokens + tile - 1) / tile;
        if (dtype == TR_BF16) head_dim == 128 ? launch_append<TR_BF16, 128>(a, blocks, layout, s) : launch_append<TR_BF16, 64>(a, blocks, layout, s);
        else head_dim == 128 ? launch_append<TR_F32, 128>(a, blocks, layout, s) : launch_append<TR_F32, 64>(a, blocks, layout, s);
        TR_HIP(hipGetLastError());
    }
    return TR_OK;
}
