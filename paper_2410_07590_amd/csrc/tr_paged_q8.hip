// Kernels of the paged cache in 8 bits: append with head norms, rotation and quantisation; rows read back.
#include "tr_internal.h"
#include "tr_paged_heads.h"
#include "tr_q8.h"

#include <algorithm>

namespace {

// Largest of the lanes that share a head.
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t x)
{
    auto with = [&](int y) { x = max(x, (uint32_t)y); };
    with(__builtin_amdgcn_update_dpp((int)x, (int)x, 0xB1, 0xf, 0xf, false));                    // quad_perm [1,0,3,2]
    with(__builtin_amdgcn_update_dpp((int)x, (int)x, 0x4E, 0xf, 0xf, false));                    // quad_perm [2,3,0,1]
    with(__builtin_amdgcn_update_dpp((int)x, (int)x, 0x141, 0xf, 0xf, false));                   // row_half_mirror
    if (LANES >= 16) with(__builtin_amdgcn_update_dpp((int)x, (int)x, 0x140, 0xf, 0xf, false));  // row_mirror
    if (LANES == 32) with(__shfl_xor((int)x, 16));
    return x;
}

// A workgroup owns the tokens that the call writes to one block of 16 rows: those from its own index on whose slots lie in the block,
// if the token in front does not.  Their heads need two steps, the largest value of the block's and then the codes; values wait for
// that in registers.
constexpr int Q8_UNITS = 4;
template <int DTYPE, int D, bool HALF>
__global__ __launch_bounds__(TR_Q8_ROWS * D / Vec<DTYPE>::N) void append_q8_kernel(const TrPagedAppendArgs a, int64_t first)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = Q8_UNITS, HEAD = D * 16 / N, THREADS = TR_Q8_ROWS * LPH;
    constexpr int TURNS = HALF ? N : N / 2;
    __shared__ float2 turn[TR_Q8_ROWS * 64]; // cosine and sine of each token's pairs, times the amplitude
    __shared__ uint32_t tops[3][UNITS * TR_Q8_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, piece = tid % LPH, g = tid / LPH;
    const int64_t t0 = first + blockIdx.x;

    // lane i + 1: the slot of token t0 + i
    const int64_t mine = t0 - 1 + lane;
    const int slot = lane <= TR_Q8_ROWS && mine >= 0 && mine < a.n_tokens ? a.slots[mine] : -1;
    const int block = slot >> 4;
    const int own = __builtin_amdgcn_readlane(block, 1);
    const int page = own >> (a.pool.page_shift - 4);
    if (own < 0 || page >= a.pool.n_pages || __builtin_amdgcn_readlane(block, 0) == own) return;
    const uint64_t member = __ballot(block == own) >> 1;
    const int run = min(__builtin_ctzll(~member), TR_Q8_ROWS);
    const bool in_run = lane >= 1 && lane <= run;
    const bool anew = __ballot(in_run && (slot & 15) == 0) != 0;
    const int in_page = own & ((1 << (a.pool.page_shift - 4)) - 1);

    int wide = 0; // log2 of the tokens that are worked on at a time
    while ((1 << wide) < run) ++wide;
    const int step = TR_Q8_ROWS >> wide, tok = g / step, h0 = g % step; // heads at a time
    const bool live = tok < run;
    const int64_t t = t0 + (live ? tok : 0);
    const int n_heads = 2 * a.n_kv_heads, pairs = a.rotary_dim / 2, half_units = pairs / N;
    const bool turns = piece * N < a.rotary_dim, low = piece < half_units, full = a.rotary_dim == D;
    const int partner = turns ? lane + (low ? half_units : -half_units) : lane;
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2);
    const char* const k = a.k + t * a.k_stride + piece * 16;
    const char* const v = a.v + t * a.v_stride + piece * 16;
    const int row = __shfl(slot, tok + 1) & 15;
    const int64_t block_at = (int64_t)page * a.pool.page_stride + (int64_t)(in_page * TR_Q8_ROWS) * a.pool.row_stride + piece * N;
    const int scale_shift = a.pool.page_shift - 4;

    u32x4 kw_raw = {};
    if (a.k_norm) kw_raw = ((const u32x4*)a.k_norm)[piece];
    float kw[N];
    V::open(kw_raw, kw);
    for (int i = tid; i < run * pairs; i += THREADS) {
        const int at = i / pairs, m = i - at * pairs;
        double sn, cn;
        tr_sincos((double)a.pos[t0 + at] * a.freq[m], &sn, &cn);
        turn[at * 64 + m] = make_float2((float)(cn * a.amplitude), (float)(sn * a.amplitude));
    }
    for (int i = tid; i < UNITS * TR_Q8_ROWS; i += THREADS) tops[0][i] = 0;
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
        const int next = buf == 2 ? 0 : buf + 1;
        for (int i = tid; i < UNITS * TR_Q8_ROWS; i += THREADS) tops[next][i] = 0; // nobody reads or adds to it until the barrier
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int head = c0 + h0 + i * step, hv = head - a.n_kv_heads;
            if (!live || head >= n_heads) continue;
            V::open(*(const u32x4*)(hv < 0 ? k + (int64_t)head * HEAD : v + (int64_t)hv * HEAD), x[i]);
            if (hv < 0) norm_and_turn<N, LPH, HALF>(x[i], a.k_norm != nullptr, kw, a.eps, e, turns, full, partner);
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const uint32_t bits = __float_as_uint(x[i][c]) & 0x7fffffffu;
                top = max(top, bits < 0x7f800000u ? bits : 0u);
            }
            top = lanes_max<LPH>(top);
            if (piece == 0) atomicMax(&tops[buf][h0 + i * step], top);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int head = c0 + h0 + i * step, hv = head - a.n_kv_heads;
            if (!live || head >= n_heads) continue;
            const int hk = hv < 0 ? head : hv;
            uint8_t* const scale = (hv < 0 ? a.pool.k_scale : a.pool.v_scale) + ((((int64_t)page * a.n_kv_heads + hk) << scale_shift) + in_page);
            char* const rows = (hv < 0 ? a.pool.k : a.pool.v) + block_at + (int64_t)hk * a.pool.head_stride;
            const int need = q8_exponent(tops[buf][h0 + i * step]), old = anew ? need : (int)*scale - 127, to = max(need, old);
            const float by = q8_power(-to);
#pragma unroll
            for (int c = 0; c < N; ++c) x[i][c] *= by;
            if (to >= Q8_MOST) // the largest numbers would round to what fp32 has not
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    const float most = 1.875f * q8_power(127 - to);
                    if (fabsf(x[i][c]) > most && fabsf(x[i][c]) < 256.0f) x[i][c] = copysignf(most, x[i][c]);
                }
            uint32_t w[N / 4];
#pragma unroll
            for (int c = 0; c < N; c += 4) w[c / 4] = q8_encode(x[i][c], x[i][c + 1], x[i][c + 2], x[i][c + 3]);
            uint32_t* const at = (uint32_t*)(rows + (int64_t)row * a.pool.row_stride);
#pragma unroll
            for (int c = 0; c < N / 4; ++c) at[c] = w[c];
            if (tok != 0 || to == old) { // a block that starts anew has old = need
                if (tok == 0 && piece == 0 && anew) *scale = (uint8_t)(to + 127);
                continue;
            }
            // a larger scale: the block's other rows are written again
            uint32_t written = 0;
            for (int j = 0; j < run; ++j) written |= 1u << (__builtin_amdgcn_readlane(slot, j + 1) & 15);
            const float factor = q8_power(old - to);
            for (int j = 0; j < TR_Q8_ROWS; ++j) {
                if (written & (1u << j)) continue;
                uint32_t* const held = (uint32_t*)(rows + (int64_t)j * a.pool.row_stride);
#pragma unroll
                for (int c = 0; c < N / 4; ++c) {
                    float y[4];
                    q8_decode(held[c], y);
                    held[c] = q8_encode(y[0] * factor, y[1] * factor, y[2] * factor, y[3] * factor);
                }
            }
            if (piece == 0) *scale = (uint8_t)(to + 127);
        }
        buf = next;
    }
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

template <int DTYPE, int D> static int launch_append(const TrPagedAppendArgs& a, int layout, hipStream_t s)
{
    constexpr int THREADS = TR_Q8_ROWS * D / Vec<DTYPE>::N;
    const int64_t most = ((int64_t)1 << 31) / THREADS; // a launch has fewer than 2^32 threads
    for (int64_t at = 0; at < a.n_tokens; at += most) {
        const dim3 blocks((uint32_t)std::min<int64_t>(a.n_tokens - at, most));
        if (layout == TR_ROPE_HALF) append_q8_kernel<DTYPE, D, true><<<blocks, dim3(THREADS), 0, s>>>(a, at);
        else append_q8_kernel<DTYPE, D, false><<<blocks, dim3(THREADS), 0, s>>>(a, at);
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
