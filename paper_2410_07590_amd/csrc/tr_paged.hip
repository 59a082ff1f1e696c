// Kernels of the paged cache: block tables and slots of a batch, append with head norms and rotation.  Times: us of a call, twelve in
// a replayed graph over three sets of buffers in turn.
#include "tr_internal.h"

#include <algorithm>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// ---- block tables, slots, position ids ------------------------------------------------------------------------------------
// A chain of latencies: one launch and no traffic between workgroups.  Each works out the prefix sums of the whole batch again (two
// lengths per request, from the caches) and then the slots of its own 1024 tokens, a few pages and, the first, the batch's
// lengths.  A token finds its request by bisection of the sums in LDS, a thread does it once for four neighbours.
// Sums are cut at 2^32 - 1 by every addition, which leaves addition associative, and at 2^31 - 1 where they are kept.
// us: five requests with a new token each 4.4 (an empty launch 3.4), 256 prompts of 193 thousand tokens 6.5 (sums of 64 bits through
// LDS permutes, two trips to memory for the lengths: 4.9 and 6.9).

__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) // inclusive, on the vector unit's cross-lane path
{
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false)); // row_shr 1, 2, 4, 8
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false)); // last lane of a row to the next row
    return add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false)); // lane 31 to the upper half
}
__device__ __forceinline__ int32_t cut(uint32_t x) { return (int32_t)min(x, (uint32_t)INT32_MAX); }

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

__global__ __launch_bounds__(256) void page_map_kernel(const TrPageMapArgs a)
{
    extern __shared__ int32_t arrays[];
    __shared__ uint32_t wave_sum[4][2];
    int32_t* const cu = arrays;          // [n_req + 1] first token of each request
    int32_t* const pg = cu + a.n_req + 1; // [n_req + 1] first new page
    int32_t* const held = pg + a.n_req + 1; // [n_req] tokens that it holds
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.n_req + 255) / 256, shift = a.page_shift;
    const uint32_t round = (1u << shift) - 1;
    auto pages = [&](uint32_t tokens) { return (tokens >> shift) + ((tokens & round) != 0); }; // tokens < 2^32
    struct Lens {
        uint32_t c, f; // below 2^31 each
    };
    auto lens = [&](int r) { return Lens{(uint32_t)max(a.cached[r], 0), (uint32_t)max(a.fresh[r], 0)}; };

    uint32_t tok = 0, pag = 0;
    Lens mine = {0, 0};
    for (int i = 0; i < per; ++i) {
        const int r = tid * per + i;
        if (r >= a.n_req) break;
        mine = lens(r);
        tok = add(tok, mine.f);
        pag = add(pag, pages(mine.c + mine.f) - pages(mine.c));
    }
    uint32_t tok_to = wave_sums(tok), pag_to = wave_sums(pag);
    if (lane == 63) wave_sum[wave][0] = tok_to, wave_sum[wave][1] = pag_to;
    // sums in front of this lane's requests
    tok_to = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)tok_to, 0x138, 0xf, 0xf, false); // wave_shr 1
    pag_to = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)pag_to, 0x138, 0xf, 0xf, false);
    __syncthreads();
    uint32_t tok_all = 0, pag_all = 0, tok_before = 0, pag_before = 0;
    for (int w = 0; w < 4; ++w) {
        if (w == wave) tok_before = tok_all, pag_before = pag_all;
        tok_all = add(tok_all, wave_sum[w][0]);
        pag_all = add(pag_all, wave_sum[w][1]);
    }
    tok_to = add(tok_to, tok_before);
    pag_to = add(pag_to, pag_before);
    for (int i = 0; i < per; ++i) {
        const int r = tid * per + i;
        if (r >= a.n_req) break;
        if (per > 1) mine = lens(r);
        cu[r] = cut(tok_to);
        pg[r] = cut(pag_to);
        held[r] = (int32_t)mine.c;
        if (blockIdx.x == 0) {
            a.cu[r] = cut(tok_to);
            a.kv_lens[r] = cut(mine.c + mine.f);
        }
        tok_to = add(tok_to, mine.f);
        pag_to = add(pag_to, pages(mine.c + mine.f) - pages(mine.c));
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
    auto free_page = [&](int64_t i) { return i < a.n_free ? a.free_pages[i] : -1; };
    const int64_t t0 = (int64_t)blockIdx.x * TR_MAP_TOKENS + 4 * tid;
    if (t0 < a.n_slots) {
        int32_t slot[4], pos[4];
        int r = t0 < n_tok ? owner(cu, a.n_req, (int)t0) : 0;
        int last = -1, first = 0;
        uint32_t c = 0, have = 0;
        for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + i;
            slot[i] = -1;
            pos[i] = 0;
            if (t >= n_tok) continue;
            while (cu[r + 1] <= t) ++r;
            if (r != last) {
                last = r;
                c = (uint32_t)held[r];
                have = pages(c);
                first = a.first_pos ? a.first_pos[r] : (int)c;
            }
            const uint32_t at = (uint32_t)(t - cu[r]), row = c + at, blk = row >> shift;
            pos[i] = (int32_t)((uint32_t)first + at);
            if (blk >= (uint32_t)a.max_blocks) continue;
            const int page = blk < have ? a.table[(int64_t)r * a.max_blocks + blk] : free_page((int64_t)pg[r] + blk - have);
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
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t p = (int64_t)blockIdx.x * 256 + tid; p < n_pag; p += step) {
        const int r = owner(pg, a.n_req, (int)p);
        const int64_t blk = pages((uint32_t)held[r]) + p - pg[r];
        if (blk < a.max_blocks) a.table[(int64_t)r * a.max_blocks + blk] = free_page(p);
        else p += (pg[r + 1] - 1 - p) / step * step; // nor do the request's other pages have an entry
    }
    if (n_pag != INT32_MAX) return;
    for (int r = 0; r < a.n_req; ++r) { // entries of pages behind the cut sum
        if (pg[r + 1] != INT32_MAX) continue;
        const Lens l = lens(r);
        const int64_t need = min((int64_t)pages(l.c + l.f), (int64_t)a.max_blocks);
        for (int64_t blk = (int64_t)pages(l.c) + (INT32_MAX - pg[r]) + (int64_t)blockIdx.x * 256 + tid; blk < need; blk += step)
            a.table[(int64_t)r * a.max_blocks + blk] = -1;
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

// The value of the lane half a head away, where the whole head turns.
template <int LANES> __device__ __forceinline__ float other_half(float x)
{
    const int b = __builtin_bit_cast(int, x);
    if constexpr (LANES == 16) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, 0x128, 0xf, 0xf, false)); // row_ror 8
    else if constexpr (LANES == 8) { // of eight lanes, and of each four: the mirror of the mirror
        const int m = __builtin_amdgcn_update_dpp(b, b, 0x141, 0xf, 0xf, false);
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(m, m, 0x1B, 0xf, 0xf, false));
    } else return __shfl_xor(x, LANES / 2);
}

// Bound by memory: a head is read once and written once.  A workgroup owns a few tokens; LPH neighbouring lanes own a head, a
// 16-byte unit each, so a norm and a rotation stay within a wave.  A thread has part in heads of one token only, always the same
// unit of them: its cosines and sines, weights and the token's row are looked up once (looked up for each unit, 16001 tokens of 32 / 8 heads
// of 128 took 101 us, 88.6 so: vector instructions were half of the time).  The tokens' angles (a thread per pair, 64 bits) are
// worked out while the first UNITS loads of every thread are on their way.
// us: 16384 tokens (padding included) of 32 / 8 heads of 128, norm, all channels turned, 400 MB: 78.5, 5.1 TB/s (a copy of as many bytes, one
// by one on a stream, 74.4; this 72.6); 24000 rows of 4 KV heads, 98 MB: 23.6; 64 tokens of 28 / 4 heads: 4.5, a launch and one chain of
// position, angle, rotation, store.  The check of the norm's range is 0.1 of that.
// UNITS two / three / four: 16001 tokens of 40 heads and values 78.6 / 79.0 / 78.2, 1000 9.3 / 9.1 / 9.1, 64 of 28 / 4 heads 4.6 / 4.5 / 4.5, one 4.6 /
// 4.4 / 4.4, the documents 22.8 / 23.6 / 23.1.
constexpr int APPEND_UNITS = 3;
template <int DTYPE, int D, bool HALF, bool STREAM>
__global__ __launch_bounds__(256) void paged_append_kernel(const TrPagedAppendArgs a)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = APPEND_UNITS, HEAD = D * 16 / N; // channels of a unit, units and bytes of a head
    constexpr int TURNS = HALF ? N : N / 2;                                       // pairs that a unit has part in
    __shared__ float2 turn[TR_PAGED_APPEND_TOKENS * 64]; // cosine and sine of each token's pairs, times the amplitude
    const int tid = threadIdx.x, piece = tid % LPH;
    const int pairs = a.rotary_dim / 2, half_units = pairs / N; // units of half the turned channels
    const bool turns = piece * N < a.rotary_dim, low = piece < half_units, full = a.rotary_dim == D;
    const int partner = turns ? (tid & 63) + (low ? half_units : -half_units) : (tid & 63);
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2); // first pair of the unit
    const int n_heads = a.n_q_heads + 2 * a.n_kv_heads;
    const int step = 256 / LPH >> a.tile_shift; // heads of a token that are worked on at a time
    const int64_t t0 = (int64_t)blockIdx.x << a.tile_shift;
    const int tokens = (int)min((int64_t)1 << a.tile_shift, a.n_tokens - t0);
    const int tok = tid / LPH / step;
    const bool live = tok < tokens;
    const int64_t t = t0 + (live ? tok : 0);
    int h = tid / LPH % step; // of queries, keys and values in a row
    const char* const q = a.q + t * a.q_stride + piece * 16;
    const char* const k = a.k + t * a.k_stride + piece * 16;
    const char* const v = a.v + t * a.v_stride + piece * 16;

    u32x4 u[UNITS];
    auto load = [&](int head) {
        const int hk = head - a.n_q_heads, hv = hk - a.n_kv_heads;
        if (!live || head >= n_heads) return u32x4{};
        return __builtin_nontemporal_load((const u32x4*)(hk < 0 ? q + (int64_t)head * HEAD : hv < 0 ? k + (int64_t)hk * HEAD : v + (int64_t)hv * HEAD));
    };
#pragma unroll
    for (int i = 0; i < UNITS; ++i) u[i] = load(h + i * step);
    const int slot = a.n_kv_heads ? a.slots[t] : -1;
    u32x4 qw_raw = {}, kw_raw = {};
    if (a.q_norm) qw_raw = ((const u32x4*)a.q_norm)[piece];
    if (a.k_norm) kw_raw = ((const u32x4*)a.k_norm)[piece];
    for (int i = tid; i < tokens * pairs; i += 256) {
        const int at = i / pairs, m = i - at * pairs;
        double sn, cn;
        tr_sincos((double)a.pos[t0 + at] * a.freq[m], &sn, &cn);
        turn[at * 64 + m] = make_float2((float)(cn * a.amplitude), (float)(sn * a.amplitude));
    }
    __syncthreads();
    float2 e[TURNS];
#pragma unroll
    for (int c = 0; c < TURNS; ++c) {
        e[c] = turns && live ? turn[tok * 64 + m0 + c] : make_float2(1.0f, 0.0f); // channels that do not turn
        if (HALF && low) e[c].y = -e[c].y;
    }
    const int page = slot >> a.pool.page_shift;
    const bool stored = slot >= 0 && page < a.pool.n_pages;
    const int64_t row = (int64_t)page * a.pool.page_stride + (int64_t)(slot & ((1 << a.pool.page_shift) - 1)) * a.pool.row_stride + piece * 16;
    char* const qd = a.q_out + t * a.n_q_heads * HEAD + piece * 16;
    char *const kd = a.pool.k + row, *const vd = a.pool.v + row;
    float qw[N], kw[N];
    V::open(qw_raw, qw);
    V::open(kw_raw, kw);
    for (;; h += UNITS * step) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int head = h + i * step, hk = head - a.n_q_heads, hv = hk - a.n_kv_heads;
            if (!live || head >= n_heads) continue; // heads are dealt out whole, so the lanes of one are here together
            const bool normed = hk < 0 ? a.q_norm != nullptr : a.k_norm != nullptr;
            if (hv < 0 && (pairs || normed)) {
                float x[N];
                V::open(u[i], x);
                if (normed) {
                    auto mean_square = [&]() {
                        float ss = 0.0f;
#pragma unroll
                        for (int c = 0; c < N; ++c) ss = fmaf(x[c], x[c], ss);
                        return lanes_sum<LPH>(ss) * (1.0f / D);
                    };
                    float under = mean_square() + a.eps;
                    if (!(under <= __FLT_MAX__)) { // for all lanes of the head: the same of a head 2^70 times smaller
#pragma unroll
                        for (int c = 0; c < N; ++c) x[c] *= 0x1p-70f;
                        under = mean_square() + a.eps * 0x1p-70f * 0x1p-70f;
                    }
                    const float r = rsqrtf(under);
#pragma unroll
                    for (int c = 0; c < N; ++c) x[c] = x[c] * r * (hk < 0 ? qw[c] : kw[c]); // in this order: x r is of size 1
                }
                if (HALF) {
                    float y[N];
                    if (full) {
#pragma unroll
                        for (int c = 0; c < N; ++c) y[c] = other_half<LPH>(x[c]);
                    } else {
#pragma unroll
                        for (int c = 0; c < N; ++c) y[c] = __shfl(x[c], partner);
                    }
#pragma unroll
                    for (int c = 0; c < N; ++c) x[c] = turns ? x[c] * e[c].x + y[c] * e[c].y : x[c];
                } else {
#pragma unroll
                    for (int c = 0; c < N / 2; ++c) {
                        const float one = x[2 * c], two = x[2 * c + 1];
                        x[2 * c] = turns ? one * e[c].x - two * e[c].y : one;
                        x[2 * c + 1] = turns ? two * e[c].x + one * e[c].y : two;
                    }
                }
                if (normed || turns) u[i] = V::close(x);
            }
            char* const to = hk < 0 ? qd + (int64_t)head * HEAD : hv < 0 ? kd + (int64_t)hk * a.pool.head_stride : vd + (int64_t)hv * a.pool.head_stride;
            if (hk >= 0 && !stored) continue;
            if (STREAM) __builtin_nontemporal_store(u[i], (u32x4*)to);
            else *(u32x4*)to = u[i];
        }
        if (h - tid / LPH % step + UNITS * step >= n_heads) break;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) u[i] = load(h + (UNITS + i) * step);
    }
}

} // namespace

int tr_launch_page_map(const TrPageMapArgs& a, hipStream_t s)
{
    const int blocks = std::max((int)(((int64_t)a.n_slots + TR_MAP_TOKENS - 1) / TR_MAP_TOKENS), 1);
    page_map_kernel<<<dim3(blocks), dim3(256), (3 * a.n_req + 2) * sizeof(int32_t), s>>>(a);
    TR_HIP(hipGetLastError());
    return TR_OK;
}

template <int DTYPE, int D, bool HALF> static void launch_append(const TrPagedAppendArgs& a, int blocks, hipStream_t s)
{
    if (a.stream) paged_append_kernel<DTYPE, D, HALF, true><<<dim3(blocks), dim3(256), 0, s>>>(a);
    else paged_append_kernel<DTYPE, D, HALF, false><<<dim3(blocks), dim3(256), 0, s>>>(a);
}
template <int DTYPE, int D> static void launch_append(const TrPagedAppendArgs& a, int blocks, int layout, hipStream_t s)
{
    layout == TR_ROPE_HALF ? launch_append<DTYPE, D, true>(a, blocks, s) : launch_append<DTYPE, D, false>(a, blocks, s);
}
int tr_launch_paged_append(const TrPagedAppendArgs& args, int dtype, int head_dim, int layout, hipStream_t s)
{
    TrPagedAppendArgs a = args;
    const int tile = 1 << a.tile_shift;
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
