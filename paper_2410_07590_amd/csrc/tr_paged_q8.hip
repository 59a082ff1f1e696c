// Kernels of the paged cache in 8 bits: append with head norms, rotation and quantisation; rows read back.
#include "tr_internal.h"
#include "tr_paged_heads.h"
#include "tr_q8.h"

#include <algorithm>

namespace {

// Largest of the lanes that share a head.
template <int LANES> __device__ __forceinline__ int lanes_max(int x)
{
    auto with = [&](int y) { x = max(x, y); };
    with(__builtin_amdgcn_update_dpp(x, x, 0xB1, 0xf, 0xf, false));                    // quad_perm [1,0,3,2]
    with(__builtin_amdgcn_update_dpp(x, x, 0x4E, 0xf, 0xf, false));                    // quad_perm [2,3,0,1]
    with(__builtin_amdgcn_update_dpp(x, x, 0x141, 0xf, 0xf, false));                   // row_half_mirror
    if (LANES >= 16) with(__builtin_amdgcn_update_dpp(x, x, 0x140, 0xf, 0xf, false));  // row_mirror
    if (LANES == 32) with(__shfl_xor(x, 16));
    return x;
}

// Threads of a workgroup: 16 rows of a head at least.
constexpr int append_q8_threads(int dtype, int d) { return std::max(256, TR_Q8_ROWS * d * (dtype == TR_F32 ? 4 : 2) / 16); }

// A unit of N channels as codes.
template <int N> __device__ __forceinline__ void put(char* to, const float (&x)[N])
{
    if constexpr (N == 8) *(uint2*)to = make_uint2(q8_encode(x[0], x[1], x[2], x[3]), q8_encode(x[4], x[5], x[6], x[7]));
    else *(uint32_t*)to = q8_encode(x[0], x[1], x[2], x[3]);
}

// Quantised heads.  A workgroup looks at `window` tokens and owns the blocks whose first tokens are among them, of keys or of values: the
// tokens that the call writes to a block of 16 rows stand side by side, from one on whose slot lies in another block than that in front of it.
// A block's heads need two steps, the largest value of all its rows and then the codes; values wait for that in registers, and the
// next heads are on their way.
constexpr int append_q8_units(int dtype) { return dtype == TR_F32 ? 4 : 2; } // heads that a thread has part in at a time, 16 channels
// The largest values of a step's heads, and the exponents that they had; what one step reads the next but one clears.
template <int DTYPE, int D> using Tops = int[append_q8_units(DTYPE) * append_q8_threads(DTYPE, D) * Vec<DTYPE>::N / D];
template <int DTYPE, int D, bool HALF, int THREADS>
__device__ __forceinline__ void append_blocks(const TrPagedAppendArgs& a, float2* turn, Tops<DTYPE, D>* tops, Tops<DTYPE, D>* olds, int64_t t0, int window,
                                              bool keys)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = append_q8_units(DTYPE), HEAD = D * 16 / N, ROWS = THREADS / LPH; // ROWS: heads of tokens at a time
    constexpr int TURNS = HALF ? N : N / 2, TOPS = UNITS * ROWS;
    static_assert(ROWS >= TR_Q8_ROWS, "");
    const int tid = threadIdx.x, lane = tid & 63, piece = tid % LPH, g = tid / LPH, scale_shift = a.pool.page_shift - 4;

    const int64_t mine = t0 - 1 + lane; // lane i + 1: the slot of token t0 + i
    const int slot = lane < window + TR_Q8_ROWS && mine >= 0 && mine < a.n_tokens ? a.slots[mine] : -1;
    const int block = slot >> 4;
    const int before = __shfl_up(block, 1);
    uint64_t owners = __ballot(lane >= 1 && lane <= window && block >= 0 && block != before && block >> scale_shift < a.pool.n_pages);
    if (!owners) return;

    const int n_heads = a.n_kv_heads, pairs = keys ? a.rotary_dim / 2 : 0, half_units = pairs / N;
    const bool normed = keys && a.k_norm, turns = keys && piece * N < a.rotary_dim, low = piece < half_units, full = a.rotary_dim == D;
    const int partner = turns ? lane + (low ? half_units : -half_units) : lane;
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2);
    const char* const from = keys ? a.k : a.v;
    const int64_t stride = keys ? a.k_stride : a.v_stride;
    char* const to_pool = keys ? a.pool.k : a.pool.v;
    uint8_t* const scales = keys ? a.pool.k_scale : a.pool.v_scale;
    u32x4 kw_raw = {};
    if (normed) kw_raw = ((const u32x4*)a.k_norm)[piece];
    float kw[N];
    V::open(kw_raw, kw);

    while (owners) {
        const int at0 = __builtin_ctzll(owners); // lane of the block's first token
        owners &= owners - 1;
        const int own = __builtin_amdgcn_readlane(block, at0), page = own >> scale_shift, in_page = own & ((1 << scale_shift) - 1);
        const int run = min(__builtin_ctzll(~(__ballot(block == own) >> at0)), TR_Q8_ROWS);
        uint32_t written = ROWS > TR_Q8_ROWS ? ~0xffffu : 0u; // rows of the block
        for (int j = 0; j < run; ++j) written |= 1u << (__builtin_amdgcn_readlane(slot, at0 + j) & 15);
        const bool anew = written & 1;
        int wide = 0; // log2 of the tokens that are worked on at a time
        while ((1 << wide) < run) ++wide;
        const int step = ROWS >> wide, tok = g / step, h0 = g % step; // heads at a time
        const bool live = tok < run;
        const int64_t t = t0 + at0 - 1 + (live ? tok : 0);
        const int row = __shfl(slot, at0 + (live ? tok : 0)) & 15;
        const char* const heads = from + t * stride + piece * 16;
        char* const rows = to_pool + (int64_t)page * a.pool.page_stride + (int64_t)(in_page * TR_Q8_ROWS) * a.pool.row_stride + piece * N;
        uint8_t* const scale = scales + (((int64_t)page * n_heads) << scale_shift) + in_page;

        u32x4 raw[UNITS];
        int held[UNITS];
        auto load = [&](int c0) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int head = c0 + h0 + i * step;
                raw[i] = u32x4{};
                held[i] = 0;
                if (!live || head >= n_heads) continue;
                raw[i] = __builtin_nontemporal_load((const u32x4*)(heads + (int64_t)head * HEAD));
                if (!anew) held[i] = scale[(int64_t)head << scale_shift];
            }
        };
        load(0);
        __syncthreads(); // the last block's angles are read
        for (int i = tid; i < run * pairs; i += THREADS) {
            const int at = i / pairs, m = i - at * pairs;
            double sn, cn;
            tr_sincos((double)a.pos[t0 + at0 - 1 + at] * a.freq[m], &sn, &cn);
            turn[at * 64 + m] = make_float2((float)(cn * a.amplitude), (float)(sn * a.amplitude));
        }
        for (int i = tid; i < TOPS; i += THREADS) tops[0][i] = 0;
        __syncthreads();
        float2 e[TURNS];
#pragma unroll
        for (int c = 0; c < TURNS; ++c) {
            e[c] = turns && live ? turn[tok * 64 + m0 + c] : make_float2(1.0f, 0.0f);
            if (HALF && low) e[c].y = -e[c].y;
        }
        int buf = 0;
        for (int c0 = 0; c0 < n_heads; c0 += UNITS * step) {
            float x[UNITS][N];
            int old[UNITS];
            const int next = buf == 2 ? 0 : buf + 1;
            for (int i = tid; i < TOPS; i += THREADS) tops[next][i] = 0; // nobody reads or adds to it until the barrier
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int head = c0 + h0 + i * step;
                old[i] = held[i];
                if (!live || head >= n_heads) continue;
                V::open(raw[i], x[i]);
                if (keys) norm_and_turn<N, LPH, HALF>(x[i], normed, kw, a.eps, e, turns, full, partner);
                int top = 0;
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const int bits = __float_as_int(x[i][c]) & 0x7fffffff;
                    top = max(top, bits < 0x7f800000 ? bits : 0);
                }
                top = lanes_max<LPH>(top);
                if (piece == 0) atomicMax(&tops[buf][h0 + i * step], top);
                if (piece == 0 && tok == 0) olds[buf][h0 + i * step] = (int)old[i] - 127;
            }
            if (c0 + UNITS * step < n_heads) load(c0 + UNITS * step);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int head = c0 + h0 + i * step;
                if (!live || head >= n_heads) continue;
                const int need = q8_exponent(tops[buf][h0 + i * step]), was = anew ? need : old[i] - 127, to = max(need, was);
                const float by = q8_power(-to);
#pragma unroll
                for (int c = 0; c < N; ++c) x[i][c] *= by;
                if (to >= Q8_MOST) // the largest numbers would round to what fp32 has not
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        const float most = 1.875f * q8_power(127 - to);
                        if (fabsf(x[i][c]) > most && fabsf(x[i][c]) < 256.0f) x[i][c] = copysignf(most, x[i][c]);
                    }
                put<N>(rows + (int64_t)head * a.pool.head_stride + (int64_t)row * a.pool.row_stride, x[i]);
                if ((anew || to != was) && tok == 0 && piece == 0) scale[(int64_t)head << scale_shift] = (uint8_t)(to + 127);
            }
            if (!anew) { // where a scale has grown, the block's other rows are written again, a row to the lanes of a head
                const int here = min(UNITS * step, n_heads - c0);
                char* const other = rows + (int64_t)g * a.pool.row_stride;
                for (int i = 0; i < here; ++i) {
                    const int was = olds[buf][i], to = max(q8_exponent(tops[buf][i]), was);
                    if (to == was || (written >> g) & 1) continue;
                    uint32_t* const unit = (uint32_t*)(other + (int64_t)(c0 + i) * a.pool.head_stride);
                    const float by = q8_power(was - to);
                    float y[N];
#pragma unroll
                    for (int c = 0; c < N; c += 4) {
                        float z[4];
                        q8_decode(unit[c / 4], z);
#pragma unroll
                        for (int b = 0; b < 4; ++b) y[c + b] = z[b] * by;
                    }
                    put<N>((char*)unit, y);
                }
            }
            buf = next;
        }
    }
}

// Keys and values by separate workgroups, which have half as much to hold, and in front of the queries', as they take longer.
template <int DTYPE, int D, bool HALF, bool STREAM>
__global__ __launch_bounds__(append_q8_threads(DTYPE, D), DTYPE == TR_BF16 ? 4 : 2) void append_q8_kernel(const TrPagedAppendArgs a, int64_t first, int window, int n_blocks)
{
    constexpr int THREADS = append_q8_threads(DTYPE, D);
    __shared__ float2 turn[TR_Q8_ROWS * 64]; // cosine and sine of each token's pairs, times the amplitude
    __shared__ Tops<DTYPE, D> tops[3], olds[3];
    const int block = blockIdx.x;
    if (block < n_blocks) append_blocks<DTYPE, D, HALF, THREADS>(a, turn, tops, olds, first + (int64_t)(block >> 1) * window, window, !(block & 1));
    else append_heads<DTYPE, D, HALF, STREAM, THREADS, true>(a, turn, (first >> a.tile_shift) + block - n_blocks);
}

// Rows of the requests, 16 to a workgroup: a thread looks up where a row is, then each takes 16 codes at a time.
constexpr int READ_ROWS = 16;
template <int DTYPE, int D>
__global__ __launch_bounds__(256) void read_q8_kernel(const TrPagedReadArgs a, int64_t first)
{
    __shared__ int64_t from[READ_ROWS], scale_from[READ_ROWS]; // bytes; -1: no page, -2: no such row
    const int tid = threadIdx.x, shift = a.pool.page_shift;
    const int64_t t0 = first + (int64_t)blockIdx.x * READ_ROWS;
    if (tid < READ_ROWS) {
        const int64_t t = t0 + tid;
        int lo = 0, hi = a.n_req; // the last request that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.row_start[mid] <= t) lo = mid; else hi = mid;
        }
        const int64_t j = t - a.row_start[lo];
        int64_t f = -2, s = 0;
        if (t < a.n_rows && j >= 0 && j < a.kv_lens[lo] && t < a.row_start[lo + 1] && j < (int64_t)a.max_blocks << shift) {
            const int page = a.table[(int64_t)lo * a.max_blocks + (j >> shift)], row = (int)j & ((1 << shift) - 1);
            f = -1;
            if ((uint32_t)page < (uint32_t)a.pool.n_pages) {
                f = (int64_t)page * a.pool.page_stride + (int64_t)row * a.pool.row_stride;
                s = (((int64_t)page * a.n_kv_heads) << (shift - 4)) + (row >> 4);
            }
        }
        from[tid] = f;
        scale_from[tid] = s;
    }
    __syncthreads();
    const int per_row = a.n_kv_heads * (D / 16);
    constexpr int OUT = DTYPE == TR_BF16 ? 2 : 4; // 16-byte units of 16 results
    for (int64_t i = tid; i < (int64_t)READ_ROWS * per_row; i += 256) {
        const int r = (int)(i / per_row), u = (int)(i - (int64_t)r * per_row), head = u / (D / 16), piece = u % (D / 16);
        const int64_t f = from[r];
        if (f == -2) continue;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            u32x4 w = {0, 0, 0, 0};
            int s = 127;
            if (f >= 0) {
                w = *(const u32x4*)((side ? a.pool.v : a.pool.k) + f + (int64_t)head * a.pool.head_stride + piece * 16);
                s = (side ? a.pool.v_scale : a.pool.k_scale)[scale_from[r] + ((int64_t)head << (shift - 4))];
            }
            const float by = q8_power(s - 127);
            u32x4* const to = (u32x4*)((side ? a.out_v : a.out_k) + ((t0 + r) * per_row + u) * (OUT * 16));
            float x[16];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float y[4];
                q8_decode(w[c], y);
#pragma unroll
                for (int b = 0; b < 4; ++b) x[4 * c + b] = y[b] * by;
            }
            constexpr int N = Vec<DTYPE>::N;
#pragma unroll
            for (int c = 0; c < OUT; ++c) {
                float y[N];
#pragma unroll
                for (int b = 0; b < N; ++b) y[b] = x[N * c + b];
                to[c] = Vec<DTYPE>::close(y);
            }
        }
    }
}

} // namespace

// A launch takes a part of the tokens, as it has fewer than 2^32 threads.
template <int DTYPE, int D> static int launch_append(const TrPagedAppendArgs& a, int layout, hipStream_t s)
{
    constexpr int THREADS = append_q8_threads(DTYPE, D);
    const int window = a.n_tokens <= TR_Q8_FEW ? 1 : TR_Q8_ROWS, tile = 1 << a.tile_shift;
    const int64_t most = TR_MAX_BLOCKS_256 / 4; // tokens, a multiple of the window and of the tile; at most that many workgroups of either side
    for (int64_t at = 0; at < a.n_tokens; at += most) {
        const int64_t rest = std::min<int64_t>(a.n_tokens - at, most);
        const int n_blocks = a.k ? 2 * (int)((rest + window - 1) / window) : 0, n_queries = a.q ? (int)((rest + tile - 1) / tile) : 0;
        const dim3 grid(n_blocks + n_queries), block(THREADS);
        const bool half = layout == TR_ROPE_HALF;
        if (half && a.stream) append_q8_kernel<DTYPE, D, true, true><<<grid, block, 0, s>>>(a, at, window, n_blocks);
        else if (half) append_q8_kernel<DTYPE, D, true, false><<<grid, block, 0, s>>>(a, at, window, n_blocks);
        else if (a.stream) append_q8_kernel<DTYPE, D, false, true><<<grid, block, 0, s>>>(a, at, window, n_blocks);
        else append_q8_kernel<DTYPE, D, false, false><<<grid, block, 0, s>>>(a, at, window, n_blocks);
        TR_HIP(hipGetLastError());
    }
    return TR_OK;
}
int tr_launch_paged_append_q8(const TrPagedAppendArgs& a, int dtype, int head_dim, int layout, hipStream_t s)
{
    if (dtype == TR_BF16) return head_dim == 128 ? launch_append<TR_BF16, 128>(a, layout, s) : launch_append<TR_BF16, 64>(a, layout, s);
    return head_dim == 128 ? launch_append<TR_F32, 128>(a, layout, s) : launch_append<TR_F32, 64>(a, layout, s);
}

template <int DTYPE, int D> static int launch_read(const TrPagedReadArgs& a, hipStream_t s)
{
    const int64_t most = (int64_t)TR_MAX_BLOCKS_256 * READ_ROWS;
    for (int64_t at = 0; at < a.n_rows; at += most) {
        const dim3 blocks((uint32_t)((std::min<int64_t>(a.n_rows - at, most) + READ_ROWS - 1) / READ_ROWS));
        read_q8_kernel<DTYPE, D><<<blocks, dim3(256), 0, s>>>(a, at);
        TR_HIP(hipGetLastError());
    }
    return TR_OK;
}
int tr_launch_paged_read_q8(const TrPagedReadArgs& a, int dtype, int head_dim, hipStream_t s)
{
    if (dtype == TR_BF16) return head_dim == 128 ? launch_read<TR_BF16, 128>(a, s) : launch_read<TR_BF16, 64>(a, s);
    return head_dim == 128 ? launch_read<TR_F32, 128>(a, s) : launch_read<TR_F32, 64>(a, s);
}
