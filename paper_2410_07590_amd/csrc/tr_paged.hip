// Kernels of the paged cache: block tables and slots of a batch, append with head norms and rotation.  Times: us of a call, twelve in
// a replayed graph over three sets of buffers in turn.
#include "tr_internal.h"
#include "tr_paged_heads.h"

#include <algorithm>

namespace {

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

template <int DTYPE, int D, bool HALF, bool STREAM>
__global__ __launch_bounds__(256) void paged_append_kernel(const TrPagedAppendArgs a)
{
    __shared__ float2 turn[TR_PAGED_APPEND_TOKENS * 64];
    append_heads<DTYPE, D, HALF, STREAM, 256, false>(a, turn, blockIdx.x);
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
