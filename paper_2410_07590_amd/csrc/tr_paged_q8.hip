// Kernels of the paged cache in 8 bits: append with head norms, rotation and quantisation; rows read back.  Times: us of a call over three
// sets of buffers in turn, on a stream.
#include "tr_internal.h"
#include "tr_paged_heads.h"
#include "tr_q8.h"

#include <algorithm>

namespace {

// The value of another lane of the row of 16, in a form that the instruction that takes it can contain.
template <int CTRL> __device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
template <int CTRL> __device__ __forceinline__ float from_lane(float x) { return __int_as_float(from_lane<CTRL>(__float_as_int(x))); }
constexpr int PAIRS = 0xB1, FOURS = 0x4E, EIGHTS = 0x141, ROW = 0x140, HALF_ROW = 0x128; // quad_perm [1,0,3,2], [2,3,0,1], mirrors, row_ror 8

// Over the lanes that share a head: the largest, the sum.
template <int LANES> __device__ __forceinline__ int most(int x)
{
    x = max(x, from_lane<PAIRS>(x));
    x = max(x, from_lane<FOURS>(x));
    x = max(x, from_lane<EIGHTS>(x));
    if (LANES >= 16) x = max(x, from_lane<ROW>(x));
    if (LANES == 32) x = max(x, __shfl_xor(x, 16));
    return x;
}
template <int LANES> __device__ __forceinline__ float sum(float x)
{
    x += from_lane<PAIRS>(x);
    x += from_lane<FOURS>(x);
    x += from_lane<EIGHTS>(x);
    if (LANES >= 16) x += from_lane<ROW>(x);
    if (LANES == 32) x += __shfl_xor(x, 16);
    return x;
}

// A lane's unit x of a head that LPH neighbouring lanes hold: normalised with the unit's weights w, turned by the cosines and sines e of
// the pairs that it has part in (HALF: sines of the lower half negated).  turns: the unit's channels do; full: the whole head's; partner: the
// lane with the other channels of its pairs.  The steps of paged_append_kernel, which has them in its own loop: 16001 tokens of 32 / 8 heads take it
// 80.5 us so, 82.2 with a function like this one.
template <int N, int LPH, bool HALF, int TURNS>
__device__ __forceinline__ void norm_and_turn(float (&x)[N], bool normed, const float (&w)[N], float eps, const float2 (&e)[TURNS], bool turns, bool full, int partner)
{
    static_assert(TURNS == (HALF ? N : N / 2), "");
    if (normed) {
        auto mean_square = [&]() {
            float ss = 0.0f;
#pragma unroll
            for (int c = 0; c < N; ++c) ss = fmaf(x[c], x[c], ss);
            return sum<LPH>(ss) * (1.0f / (N * LPH));
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
    if (HALF && full) {
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = x[c] * e[c].x + (LPH == 16 ? from_lane<HALF_ROW>(x[c]) : other_half<LPH>(x[c])) * e[c].y;
    } else if (HALF) {
        float y[N];
#pragma unroll
        for (int c = 0; c < N; ++c) y[c] = __shfl(x[c], partner);
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = turns ? x[c] * e[c].x + y[c] * e[c].y : x[c];
    } else if (full) {
#pragma unroll
        for (int c = 0; c < N / 2; ++c) {
            const float one = x[2 * c], two = x[2 * c + 1];
            x[2 * c] = one * e[c].x - two * e[c].y;
            x[2 * c + 1] = two * e[c].x + one * e[c].y;
        }
    } else {
#pragma unroll
        for (int c = 0; c < N / 2; ++c) {
            const float one = x[2 * c], two = x[2 * c + 1];
            x[2 * c] = turns ? one * e[c].x - two * e[c].y : one;
            x[2 * c + 1] = turns ? two * e[c].x + one * e[c].y : two;
        }
    }
}

// Threads of a workgroup: 16 rows of a head at least.
constexpr int append_q8_threads(int dtype, int d) { return std::max(256, TR_Q8_ROWS * d * (dtype == TR_F32 ? 4 : 2) / 16); }

// A unit of N channels as codes.
template <int N> __device__ __forceinline__ void put(char* to, const float (&x)[N])
{
    if constexpr (N == 8) *(uint2*)to = make_uint2(q8_encode(x[0], x[1], x[2], x[3]), q8_encode(x[4], x[5], x[6], x[7]));
    else *(uint32_t*)to = q8_encode(x[0], x[1], x[2], x[3]);
}

// The rows `which` of a block, a unit of N channels each, at another scale.
template <int N> __device__ __forceinline__ void rescale(char* unit, uint32_t row_stride, uint32_t which, float by)
{
    constexpr int AT_ONCE = 32 / N; // as many as fill eight registers
#pragma unroll 1
    for (int j0 = 0; j0 < TR_Q8_ROWS; j0 += AT_ONCE) {
        uint32_t w[AT_ONCE][N / 4] = {};
        char* const at = unit + (int64_t)j0 * row_stride;
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
            for (int c = 0; c < N / 4; ++c)
                if (which >> (j0 + j) & 1) w[j][c] = ((const uint32_t*)(at + (int64_t)j * row_stride))[c];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            float y[N];
#pragma unroll
            for (int c = 0; c < N; c += 4) {
                float z[4];
                q8_decode(w[j][c / 4], z);
#pragma unroll
                for (int b = 0; b < 4; ++b) y[c + b] = z[b] * by;
            }
            if (which >> (j0 + j) & 1) put<N>(at + (int64_t)j * row_stride, y);
        }
    }
}

// Quantised heads.  The scale of a block is 2^e with the smallest e that holds its largest value, so a head takes two steps: the largest
// value of all rows of the block, then the codes.  A power of two costs no precision, as codes are floating-point numbers, and lets rows
// that a block holds already go over to a larger scale without a second rounding unless they are small.
//
// Work.  The tokens that the call writes to a block stand side by side, as a run, from one on whose slot lies in another block than that in
// front of it.  A workgroup looks at `window` tokens, at most 16, and owns the runs that begin with one of them, for some of the heads of keys or
// of values.  It works on as many runs at a time as have 16 tokens together, a row of lanes to a token, so that a prompt's blocks and
// single tokens of many requests fill it alike: nobody has to know which they are.  (Runs one after another: 1024 requests of a
// token, 8 heads of 128, 41 us, 10.4 so; a workgroup for each token: 13.8, and 58 for four prompts of 1024, 22.9 so.)
//
// Bound by memory where tokens are many: 16000 of 32 / 8 heads (384 of padding), 367 MB, 74.9, 4.9 TB/s, a copy of as many bytes 73; queries alone 51, keys and
// values alone 31, which is half vector instructions and half the chain of slots, heads, barrier, codes, hidden only by other workgroups.  So
// registers count: values wait as they come and keys in fp32, two heads at a time (154 registers, three workgroups to a compute unit; four
// heads at a time took 104.5), and only the next two are on their way.  64 tokens of 28 / 4 heads 4.5, one token 4.5, of which a launch is 3.3.
// Heads that a thread has part in at a time: 16 channels of keys, which it holds in fp32, 32 of values, which it holds as they come.
constexpr int append_q8_units(int dtype, bool keys) { return (dtype == TR_F32 ? 4 : 2) * (keys ? 1 : 2); }
// The largest values of a step's runs and heads; what one step reads the next but one clears.
template <int DTYPE, int D> using Tops = int[append_q8_units(DTYPE, false) * append_q8_threads(DTYPE, D) * Vec<DTYPE>::N / D];
template <int DTYPE, int D, bool HALF, int THREADS, bool KEYS>
__device__ __forceinline__ void append_blocks(const TrPagedAppendArgs& a, float2* turn, Tops<DTYPE, D>* tops, int* slots, int64_t t0, int window, int first_head, int end_head)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = append_q8_units(DTYPE, KEYS), HEAD = D * 16 / N, ROWS = THREADS / LPH; // ROWS: heads of tokens at a time
    constexpr int TURNS = HALF ? N : N / 2, TOPS = UNITS * ROWS, LOOK = 2 * TR_Q8_ROWS;                                 // lanes that hold a token's slot
    static_assert(ROWS >= TR_Q8_ROWS, "");
    const int tid = threadIdx.x, lane = tid & 63, piece = tid % LPH, g = tid / LPH, scale_shift = a.pool.page_shift - 4;

    const int64_t mine = t0 - 1 + lane; // lane i + 1: the slot of token t0 + i
    const int slot = lane < LOOK && mine >= 0 && mine < a.n_tokens ? a.slots[mine] : -1;
    const int block = slot >> 4;
    const int before = __shfl_up(block, 1);
    const uint64_t valid = __ballot(block >= 0 && block >> scale_shift < a.pool.n_pages), changes = __ballot(lane == 0 || block != before);
    uint64_t owned = changes & valid & (((1ull << window) - 1) << 1); // lanes of the first tokens of runs
    if (!owned) return;
    const uint64_t firsts = __ballot(slot >= 0 && (slot & 15) == 0);
    auto end_of = [&](int at) { return min(at + 1 + __builtin_ctzll(changes >> (at + 1) | 1ull << 62), at + TR_Q8_ROWS); }; // of the run that begins there
    if (tid < LOOK) slots[tid] = slot;

    const int pairs = KEYS ? a.rotary_dim / 2 : 0, half_units = pairs / N;
    const bool normed = KEYS && a.k_norm, turns = KEYS && piece * N < a.rotary_dim, low = piece < half_units, full = a.rotary_dim == D;
    const int partner = turns ? lane + (low ? half_units : -half_units) : lane;
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2);
    const char* const from = KEYS ? a.k : a.v;
    const int64_t stride = KEYS ? a.k_stride : a.v_stride;
    const double freq = lane < pairs ? a.freq[lane] : 0.0;
    u32x4 kw_raw = {};
    if (normed) kw_raw = ((const u32x4*)a.k_norm)[piece];
    float kw[N];
    V::open(kw_raw, kw);

    while (owned) {
        const int at0 = __builtin_ctzll(owned);
        int end = end_of(at0);
        owned &= owned - 1;
        while (owned && end_of(__builtin_ctzll(owned)) - at0 <= TR_Q8_ROWS) {
            end = end_of(__builtin_ctzll(owned));
            owned &= owned - 1;
        }
        const int tokens = end - at0;
        int wide = 0; // log2 of the tokens that are worked on at a time
        while ((1 << wide) < tokens) ++wide;
        const int step = ROWS >> wide, tok = g / step, h0 = g % step; // heads at a time
        const int at = min(at0 + tok, end - 1);                       // the token's lane
        const bool live = tok < tokens && (valid >> at & 1);
        const int begin = 63 - __builtin_clzll(changes & ((2ull << at) - 1)); // lane of its run's first token
        const bool anew = (firsts >> begin & ((1ull << (end_of(begin) - begin)) - 1)) != 0, leads = at == begin;
        __syncthreads(); // the slots are there, and the last runs' angles are read
        const int own = slots[at];
        const int64_t page = own >> a.pool.page_shift;
        const int row = own & 15, in_page = (own >> 4) & ((1 << scale_shift) - 1);
        const char* const heads = from + (t0 + at - 1) * stride + piece * 16;
        char* const rows = (KEYS ? a.pool.k : a.pool.v) + page * a.pool.page_stride + (int64_t)(in_page * TR_Q8_ROWS) * a.pool.row_stride + piece * N;
        uint8_t* const scale = (KEYS ? a.pool.k_scale : a.pool.v_scale) + ((page * a.n_kv_heads) << scale_shift) + in_page;

        u32x4 raw[UNITS];
        int held[UNITS];
        auto load = [&](int c0) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int head = c0 + h0 + i * step;
                raw[i] = u32x4{};
                held[i] = 0;
                if (!live || head >= end_head) continue;
                raw[i] = __builtin_nontemporal_load((const u32x4*)(heads + (int64_t)head * HEAD));
                if (!anew) held[i] = scale[(int64_t)head << scale_shift];
            }
        };
        load(first_head);
        if (KEYS) { // a lane has the same pair of every token that its wave takes
            constexpr int WAVES = THREADS / 64, EACH = TR_Q8_ROWS / WAVES;
            const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
            int pos[EACH];
#pragma unroll
            for (int j = 0; j < EACH; ++j) pos[j] = wave + j * WAVES < tokens && pairs ? a.pos[t0 + at0 - 1 + wave + j * WAVES] : 0;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                if (wave + j * WAVES >= tokens || lane >= pairs) continue;
                double sn, cn;
                tr_sincos((double)pos[j] * freq, &sn, &cn);
                turn[(wave + j * WAVES) * 64 + lane] = make_float2((float)(cn * a.amplitude), (float)(sn * a.amplitude));
            }
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
        for (int c0 = first_head; c0 < end_head; c0 += UNITS * step) {
            float x[KEYS ? UNITS : 1][N];
            u32x4 now[UNITS];
            int old[UNITS];
            const int next = buf == 2 ? 0 : buf + 1;
            for (int i = tid; i < TOPS; i += THREADS) tops[next][i] = 0; // nobody reads or adds to it until the barrier
            auto top_of = [&](int i) -> int& { return tops[buf][((h0 + i * step) << wide) + begin - at0]; };
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int head = c0 + h0 + i * step;
                old[i] = held[i];
                if (!live || head >= end_head) continue;
                float (&y)[N] = x[KEYS ? i : 0];
                now[i] = raw[i];
                V::open(raw[i], y);
                if (KEYS) norm_and_turn<N, LPH, HALF>(y, normed, kw, a.eps, e, turns, full, partner);
                int top = 0;
#pragma unroll
                for (int c = 0; c < N; ++c) top = max(top, __float_as_int(y[c]) & 0x7fffffff);
                if (top >= 0x7f800000) { // infinite and NaN channels have no part in it
                    top = 0;
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        const int bits = __float_as_int(y[c]) & 0x7fffffff;
                        top = max(top, bits < 0x7f800000 ? bits : 0);
                    }
                }
                top = most<LPH>(top);
                if (piece == 0) atomicMax(&top_of(i), top);
            }
            if (c0 + UNITS * step < end_head) load(c0 + UNITS * step);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int head = c0 + h0 + i * step;
                if (!live || head >= end_head) continue;
                const int need = q8_exponent(top_of(i)), was = anew ? need : old[i] - 127, to = max(need, was);
                const float by = q8_power(-to);
                float (&y)[N] = x[KEYS ? i : 0];
                if (!KEYS) V::open(now[i], y);
#pragma unroll
                for (int c = 0; c < N; ++c) y[c] *= by;
                if (to >= Q8_MOST) // the largest numbers would round to what fp32 has not
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        const float limit = 1.875f * q8_power(127 - to);
                        if (fabsf(y[c]) > limit && fabsf(y[c]) < 256.0f) y[c] = copysignf(limit, y[c]);
                    }
                char* const block_rows = rows + (int64_t)head * a.pool.head_stride;
                put<N>(block_rows + (int64_t)row * a.pool.row_stride, y);
                if (!leads || !(anew || to != was)) continue;
                if (piece == 0) scale[(int64_t)head << scale_shift] = (uint8_t)(to + 127);
                if (to != was) { // a larger scale: the block's other rows are written again.  A block that starts anew has none
                    uint32_t others = 0xffffu;
                    for (int j = begin; j < end_of(begin); ++j) others &= ~(1u << (slots[j] & 15));
                    rescale<N>(block_rows, a.pool.row_stride, others, q8_power(was - to));
                }
            }
            buf = next;
        }
    }
}

// Query heads: the pass of paged_append_kernel over one side.  A workgroup owns a few tokens, a thread the same unit of several heads of one of
// them.
template <int DTYPE, int D, bool HALF, bool STREAM, int THREADS>
__device__ __forceinline__ void append_queries(const TrPagedAppendArgs& a, float2* turn, int64_t block)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, LPH = D / N, UNITS = 3, HEAD = D * 16 / N, TURNS = HALF ? N : N / 2;
    const int tid = threadIdx.x, piece = tid % LPH;
    const int pairs = a.rotary_dim / 2, half_units = pairs / N, n_heads = a.n_q_heads;
    const bool turns = piece * N < a.rotary_dim, low = piece < half_units, normed = a.q_norm != nullptr;
    const int partner = turns ? (tid & 63) + (low ? half_units : -half_units) : (tid & 63);
    const int m0 = HALF ? (low ? piece : piece - half_units) * N : piece * (N / 2);
    const int step = THREADS / LPH >> a.tile_shift; // heads of a token that are worked on at a time
    const int64_t t0 = block << a.tile_shift;
    const int tokens = (int)min((int64_t)1 << a.tile_shift, a.n_tokens - t0);
    const int tok = tid / LPH / step;
    const bool live = tok < tokens;
    const int64_t t = t0 + (live ? tok : 0);
    int h = tid / LPH % step;
    const char* const q = a.q + t * a.q_stride + piece * 16;
    char* const to = a.q_out + t * n_heads * HEAD + piece * 16;

    u32x4 u[UNITS];
    auto load = [&](int head) { return live && head < n_heads ? __builtin_nontemporal_load((const u32x4*)(q + (int64_t)head * HEAD)) : u32x4{}; };
#pragma unroll
    for (int i = 0; i < UNITS; ++i) u[i] = load(h + i * step);
    u32x4 w_raw = {};
    if (normed) w_raw = ((const u32x4*)a.q_norm)[piece];
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
        e[c] = turns && live ? turn[tok * 64 + m0 + c] : make_float2(1.0f, 0.0f);
        if (HALF && low) e[c].y = -e[c].y;
    }
    float w[N];
    V::open(w_raw, w);
    for (;; h += UNITS * step) {
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int head = h + i * step;
            if (!live || head >= n_heads) continue; // heads are dealt out whole, so the lanes of one are here together
            if (pairs || normed) {
                float x[N];
                V::open(u[i], x);
                norm_and_turn<N, LPH, HALF>(x, normed, w, a.eps, e, turns, a.rotary_dim == D, partner);
                if (normed || turns) u[i] = V::close(x);
            }
            if (STREAM) __builtin_nontemporal_store(u[i], (u32x4*)(to + (int64_t)head * HEAD));
            else *(u32x4*)(to + (int64_t)head * HEAD) = u[i];
        }
        if (h - tid / LPH % step + UNITS * step >= n_heads) break;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) u[i] = load(h + (UNITS + i) * step);
    }
}

// Keys and values by separate workgroups, which have half as much to hold.  They come first, as they take longer than the queries', or, where a
// launch has many rounds of workgroups and most of them are queries', evenly among them, so that the ones' chains overlap with the others' stream.
template <int DTYPE, int D, bool HALF, bool STREAM>
__global__ __launch_bounds__(append_q8_threads(DTYPE, D), DTYPE == TR_BF16 ? 3 : 2) void append_q8_kernel(const TrPagedAppendArgs a, int64_t first, int window, int n_windows, int n_parts, int spread)
{
    constexpr int THREADS = append_q8_threads(DTYPE, D);
    __shared__ float2 turn[TR_Q8_ROWS * 64]; // cosine and sine of each token's pairs, times the amplitude
    __shared__ Tops<DTYPE, D> tops[3];
    __shared__ int slots[2 * TR_Q8_ROWS];
    const int n_blocks = 2 * n_parts * n_windows, at = blockIdx.x;
    auto among = [&](int n) { return spread ? (int)((uint64_t)n * n_blocks / gridDim.x) : min(n, n_blocks); }; // the first n workgroups
    const int block = among(at);
    if (among(at + 1) > block) {
        const int part = block / n_windows; // parts of the heads, of keys and of values in turn
        const int p = part >> 1, per = (a.n_kv_heads + n_parts - 1) / n_parts;
        const int first_head = p * per, end_head = min(first_head + per, a.n_kv_heads);
        if (first_head >= end_head) return; // the heads of a part are rounded up, so the last ones may have none
        const int64_t t0 = first + (int64_t)(block - part * n_windows) * window;
        if (part & 1) append_blocks<DTYPE, D, HALF, THREADS, false>(a, turn, tops, slots, t0, window, first_head, end_head);
        else append_blocks<DTYPE, D, HALF, THREADS, true>(a, turn, tops, slots, t0, window, first_head, end_head);
    } else append_queries<DTYPE, D, HALF, STREAM, THREADS>(a, turn, (first >> a.tile_shift) + at - block);
}

// Largest i of 64 lanes with starts <= x, for ascending starts; -1 if there is none.
__device__ __forceinline__ int lane_not_above(int starts, int x)
{
    int n = 0; // lanes below n are known to be
#pragma unroll
    for (int s = 32; s; s >>= 1)
        if (__shfl(starts, n + s - 1) <= x) n += s;
    if (n == 63 && __shfl(starts, 63) <= x) n = 64;
    return n - 1;
}

__device__ __forceinline__ int64_t lane_of(int64_t x, int lane)
{
    return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}

// Rows of the requests.  Bound by memory, two bytes written for each that is read (bf16), and by a chain of trips to it before the first code is
// asked for: the requests' first rows, a length and a page id, codes and scales.  A wave takes `rows` rows, as many as its lanes have units of, a
// lane looks up one of them, and then each lane makes 16 bytes of keys and of values at a time, so that stores are whole lines.  Many waves with
// little each: with one / two / four such units to a lane at a time 16 requests of 300 to 9000 rows, 8 heads of 128 channels, 478 MB, take 84.0 (5.7 TB/s) /
// 92.9 / 95.8, nine fp32 ones of up to 2500 5.6 / 6.1 / 6.4, one of 700 rows 4.8 / 5.0 / 5.3 (16 codes to a lane and a search by each workgroup: 110.5, 7.6, 4.0).
template <int DTYPE, int D, bool STREAM>
__global__ __launch_bounds__(256) void read_q8_kernel(const TrPagedReadArgs a, int64_t first)
{
    using V = Vec<DTYPE>;
    constexpr int N = V::N, PER_HEAD = D / N;
    const int lane = threadIdx.x & 63, shift = a.pool.page_shift, scale_shift = shift - 4;
    const int64_t t0 = first + ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * a.rows;
    if (t0 >= a.n_rows) return;

    // lane i: the first row of request base + i, none of those in front of which begins behind t0
    int base = 0, n = a.n_req + 1;
    while (n > 64) {
        const int step = (n + 63) >> 6, at = base + min(lane * step, n - 1);
        const uint64_t below = __ballot(a.row_start[at] <= t0);
        const int i = max(__builtin_popcountll(below) - 1, 0); // starts ascend
        base += min(i * step, n - 1);
        n = min(step, n - min(i * step, n - 1));
    }
    n = a.n_req + 1 - base; // the requests behind are of interest, too
    const int start = lane < n ? a.row_start[base + lane] : INT32_MAX;
    int64_t from = -2; // bytes; -1: no page, -2: no such row
    int64_t scale = 0;
    {
        const int64_t t = t0 + lane;
        const int last = (int)min(t0 + a.rows - 1, (int64_t)INT32_MAX - 1);
        int i = __builtin_popcountll(__ballot(start <= (int)t0)) - 1, begin, end;
        if (i == __builtin_popcountll(__ballot(start <= last)) - 1) { // all rows are of one request
            begin = __builtin_amdgcn_readlane(start, max(i, 0));
            end = __builtin_amdgcn_readlane(start, min(i + 1, 63));
        } else {
            i = lane_not_above(start, (int)min(t, (int64_t)last));
            begin = __shfl(start, max(i, 0));
            end = __shfl(start, min(i + 1, 63));
        }
        int r = base + max(i, 0);
        if (i == 63 && lane < a.rows) { // more than 63 requests begin in these rows
            int lo = r, hi = a.n_req;
            while (hi - lo > 1) {
                const int mid = lo + ((hi - lo) >> 1);
                if (a.row_start[mid] <= t) lo = mid; else hi = mid;
            }
            r = min(lo, a.n_req - 1);
            begin = a.row_start[r];
            end = a.row_start[r + 1];
        }
        const int64_t j = t - begin;
        if (lane < a.rows && t < a.n_rows && i >= 0 && r < a.n_req && j >= 0 && t < end && j < (int64_t)a.max_blocks << shift) {
            const int page = a.table[(int64_t)r * a.max_blocks + (j >> shift)], row = (int)j & ((1 << shift) - 1);
            if (j < a.kv_lens[r]) {
                from = -1;
                if ((uint32_t)page < (uint32_t)a.pool.n_pages) {
                    from = (int64_t)page * a.pool.page_stride + (int64_t)row * a.pool.row_stride;
                    scale = (((int64_t)page * a.n_kv_heads) << scale_shift) + (row >> 4);
                }
            }
        }
    }
    const int per_row = a.n_kv_heads * PER_HEAD, units = (int)min((int64_t)a.rows, a.n_rows - t0) * per_row; // below 2^31 as heads are at most 2^20
    const uint64_t unit0 = (uint64_t)t0 * per_row;
    const bool even = per_row % 64 == 0; // then a wave has one row
    const int64_t at0 = lane_of(from, 0), sc0 = lane_of(scale, 0);
    for (int u = lane; u - lane < units; u += 64) {
        int64_t at = at0, sc = sc0;
        int unit = u; // of the row
        if (!even) {
            const int row = (uint32_t)u / (uint32_t)per_row;
            at = __shfl(from, row & 63), sc = __shfl(scale, row & 63);
            unit = u - row * per_row;
        }
        if (u >= units || at == -2) continue;
        const int head = unit / PER_HEAD;
        uint32_t w[2][N / 4] = {};
        int s[2] = {127, 127};
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            if (at < 0) continue;
            const char* const codes = (side ? a.pool.v : a.pool.k) + at + (int64_t)head * a.pool.head_stride + (unit % PER_HEAD) * N;
            if constexpr (N == 8) {
                const uint64_t x = STREAM ? __builtin_nontemporal_load((const uint64_t*)codes) : *(const uint64_t*)codes;
                w[side][0] = (uint32_t)x, w[side][N / 4 - 1] = (uint32_t)(x >> 32);
            } else w[side][0] = STREAM ? __builtin_nontemporal_load((const uint32_t*)codes) : *(const uint32_t*)codes;
            s[side] = (side ? a.pool.v_scale : a.pool.k_scale)[sc + ((int64_t)head << scale_shift)];
        }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const float by = q8_power(s[side] - 127);
            float x[N];
#pragma unroll
            for (int c = 0; c < N; c += 4) {
                float y[4];
                q8_decode(w[side][c / 4], y);
#pragma unroll
                for (int b = 0; b < 4; ++b) x[c + b] = y[b] * by;
            }
            u32x4* const to = (u32x4*)((side ? a.out_v : a.out_k) + (unit0 + u) * 16);
            if (STREAM) __builtin_nontemporal_store(V::close(x), to);
            else *to = V::close(x);
        }
    }
}

} // namespace

// Workgroups of quantised heads that a launch is cut into where tokens are few: first windows of fewer than 16 tokens, then parts of the heads.
// us with windows of 16 always / this: 64 tokens 6.3 / 5.4, a prompt of 512 8.7 / 7.2, six short fp32 prompts 10.1 / 6.3; with 512 / 1024 of them: two
// prompts of 1024 15.5 / 18.4, four 22.9 / 24.6, 4096 requests of a token 22.8 / 25.8, 1024 10.4 / 10.4.
static constexpr int PARTS_WGS = 512;
// Whether they are mixed with the queries'.  us first / mixed, 32 / 8 heads of 128: 4096 single tokens 22.2 / 23.6, 5000 25.8 / 26.4, 8192 39.7 / 39.3,
// 16384 84.2 / 78.6; 1024 requests of 5 25.5 / 28.2; prompts of 1024, four 21.2 / 22.0, eight 38.5 / 37.8, sixteen 77.4 / 75.3.  16384 single tokens of
// other heads of 128: 8 / 8 45.0 / 56.0, 16 / 2 41.3 / 45.0, 20 / 4 50.6 / 50.5, 24 / 4 58.9 / 54.9, 32 / 32 149.0 / 147.1; of 64: 16 / 4 31.6 / 34.8, 32 / 8 45.5 / 46.6,
// 48 / 8 59.6 / 56.8; fp32 of 64: 4 / 4 28.1 / 38.8, 16 / 4 42.5 / 41.5, 32 / 8 81.1 / 73.4; fp32 of 128, in workgroups of 512: 16 / 4 111.9 / 112.8, 32 / 8 185.0 / 189.3.
static constexpr int MIX_TOKENS = 8192, MIX_BYTES = 6144; // MIX_BYTES: of a token's queries
// A launch takes a part of the tokens, as it has fewer than 2^32 threads.
template <int DTYPE, int D> static int launch_append(const TrPagedAppendArgs& a, int layout, hipStream_t s)
{
    constexpr int THREADS = append_q8_threads(DTYPE, D), UNITS = append_q8_units(DTYPE, true);
    const int tile = 1 << a.tile_shift;
    const int64_t most = 1 << 22; // tokens, a multiple of a window and of the tile
    for (int64_t at = 0; at < a.n_tokens; at += most) {
        const int64_t rest = std::min<int64_t>(a.n_tokens - at, most);
        const int all_parts = a.k ? (a.n_kv_heads + UNITS - 1) / UNITS : 0, n_queries = a.q ? (int)((rest + tile - 1) / tile) : 0;
        int window = 1;
        while (window < TR_Q8_ROWS && 2 * all_parts * ((rest + window - 1) / window) > PARTS_WGS) window *= 2;
        const int n_windows = (int)((rest + window - 1) / window), n_parts = std::min(all_parts, std::max(PARTS_WGS / (2 * n_windows), 1));
        const dim3 grid(2 * n_parts * n_windows + n_queries), block(THREADS);
        const bool mixed = THREADS == 256 && rest >= MIX_TOKENS && (int64_t)a.n_q_heads * D * (DTYPE == TR_F32 ? 4 : 2) >= MIX_BYTES;
        const bool half = layout == TR_ROPE_HALF;
        if (half && a.stream) append_q8_kernel<DTYPE, D, true, true><<<grid, block, 0, s>>>(a, at, window, n_windows, n_parts, mixed);
        else if (half) append_q8_kernel<DTYPE, D, true, false><<<grid, block, 0, s>>>(a, at, window, n_windows, n_parts, mixed);
        else if (a.stream) append_q8_kernel<DTYPE, D, false, true><<<grid, block, 0, s>>>(a, at, window, n_windows, n_parts, mixed);
        else append_q8_kernel<DTYPE, D, false, false><<<grid, block, 0, s>>>(a, at, window, n_windows, n_parts, mixed);
        TR_HIP(hipGetLastError());
    }
    return TR_OK;
}
int tr_launch_paged_append_q8(const TrPagedAppendArgs& a, int dtype, int head_dim, int layout, hipStream_t s)
{
    if (dtype == TR_BF16) return head_dim == 128 ? launch_append<TR_BF16, 128>(a, layout, s) : launch_append<TR_BF16, 64>(a, layout, s);
    return head_dim == 128 ? launch_append<TR_F32, 128>(a, layout, s) : launch_append<TR_F32, 64>(a, layout, s);
}

template <int DTYPE, int D> static int launch_read(TrPagedReadArgs a, hipStream_t s)
{
    const int per_row = a.n_kv_heads * (D / Vec<DTYPE>::N);
    a.rows = std::min(std::max(64 / per_row, 1), 64);
    const int64_t most = (int64_t)TR_MAX_BLOCKS_256 * 4 * a.rows;
    // Streamed loads and stores make the call itself faster, and what reads its results, or the pages, next slower where the caches still hold them.  us of
    // the call and a pass over all it wrote, ordinary / streamed, by MB written: 46 MB 47.2 / 50.7, 93 MB 68.4 / 79.2, 187 MB 120.5 / 128.4, 375 MB 234.0 / 230.7.
    const bool stream = 2 * 16ll * per_row * a.n_rows >= 256ll << 20;
    for (int64_t at = 0; at < a.n_rows; at += most) {
        const dim3 blocks((uint32_t)((std::min<int64_t>(a.n_rows - at, most) + 4 * a.rows - 1) / (4 * a.rows)));
        if (stream) read_q8_kernel<DTYPE, D, true><<<blocks, dim3(256), 0, s>>>(a, at);
        else read_q8_kernel<DTYPE, D, false><<<blocks, dim3(256), 0, s>>>(a, at);
        TR_HIP(hipGetLastError());
    }
    return TR_OK;
}
int tr_launch_paged_read_q8(const TrPagedReadArgs& a, int dtype, int head_dim, hipStream_t s)
{
    if (dtype == TR_BF16) return head_dim == 128 ? launch_read<TR_BF16, 128>(a, s) : launch_read<TR_BF16, 64>(a, s);
    return head_dim == 128 ? launch_read<TR_F32, 128>(a, s) : launch_read<TR_F32, 64>(a, s);
}
