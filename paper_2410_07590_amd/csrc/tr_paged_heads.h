// What the append kernels of the paged cache share: 16-byte units of heads in fp32, sums over the lanes of a head, norm and rotation,
// and the pass over the heads of tokens that neither needs to know more of than themselves.
#pragma once
#include "tr_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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

// A lane's unit x of a head that LPH neighbouring lanes hold: normalised with the unit's weights w, turned by the cosines and sines e of
// the pairs that it has part in (HALF: sines of the lower half negated).  turns: the unit's channels do; full: the whole head's; partner: the
// lane with the other channels of its pairs.
template <int N, int LPH, bool HALF, int TURNS>
__device__ __forceinline__ void norm_and_turn(float (&x)[N], bool normed, const float (&w)[N], float eps, const float2 (&e)[TURNS], bool turns, bool full, int partner)
{
    static_assert(TURNS == (HALF ? N : N / 2), "");
    if (normed) {
        auto mean_square = [&]() {
            float ss = 0.0f;
#pragma unroll
            for (int c = 0; c < N; ++c) ss = fmaf(x[c], x[c], ss);
            return lanes_sum<LPH>(ss) * (1.0f / (N * LPH));
        };
        float under = mean_square() + eps;
        if (!(under <= __FLT_MAX__)) { // for all lanes of the head: the same of a head 2^70 times smaller
#pragma unroll
            for (int c = 0; c < N; ++c) x[c] *= 0x1p-70f;
            under = mean_square() + eps * 0x1p-70f * 0x1p-70f;
        }
        const float r = rsqrtf(under);
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = x[c] * r * w[c]; // in this order: x r is of size 1
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
// turn: room for the cosine and sine of each token's pairs, times the amplitude.  QUERIES: nothing is done with keys and values.
constexpr int APPEND_UNITS = 3;
template <int DTYPE, int D, bool HALF, bool STREAM, int THREADS, bool QUERIES>
__device__ __forceinline__ void append_heads(const TrPagedAppendArgs& a, float2* turn, int64_t block)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = APPEND_UNITS, HEAD = D * 16 / N; // channels of a unit, units and bytes of a head
    constexpr int TURNS = HALF ? N : N / 2;                                       // pairs that a unit has part in
    const int tid = threadIdx.x, piece = tid % LPH;
    const int pairs = a.rotary_dim / 2, half_units = pairs / N; // units of half the turned channels
    const bool turns = piece * N < a.rotary_dim, low = piece < half_units, full = a.rotary_dim == D;
    const int partner = turns ? (tid & 63) + (low ? half_units : -half_units) : (tid & 63);
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2); // first pair of the unit
    const int n_kv = QUERIES ? 0 : a.n_kv_heads, n_heads = a.n_q_heads + 2 * n_kv;
    const int step = THREADS / LPH >> a.tile_shift; // heads of a token that are worked on at a time
    const int64_t t0 = block << a.tile_shift;
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
        const int hk = head - a.n_q_heads, hv = hk - n_kv;
        if (!live || head >= n_heads) return u32x4{};
        return __builtin_nontemporal_load((const u32x4*)(hk < 0 ? q + (int64_t)head * HEAD : hv < 0 ? k + (int64_t)hk * HEAD : v + (int64_t)hv * HEAD));
    };
#pragma unroll
    for (int i = 0; i < UNITS; ++i) u[i] = load(h + i * step);
    const int slot = n_kv ? a.slots[t] : -1;
    u32x4 qw_raw = {}, kw_raw = {};
    if (a.q_norm) qw_raw = ((const u32x4*)a.q_norm)[piece];
    if (a.k_norm) kw_raw = ((const u32x4*)a.k_norm)[piece];
    for (int i = tid; i < tokens * pairs; i += THREADS) {
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
            const int head = h + i * step, hk = head - a.n_q_heads, hv = hk - n_kv;
            if (!live || head >= n_heads) continue; // heads are dealt out whole, so the lanes of one are here together
            const bool normed = hk < 0 ? a.q_norm != nullptr : a.k_norm != nullptr;
            if (hv < 0 && (pairs || normed)) {
                float x[N];
                V::open(u[i], x);
                norm_and_turn<N, LPH, HALF>(x, normed, hk < 0 ? qw : kw, a.eps, e, turns, full, partner);
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
