// Decode attention over a paged cache, in the type of the shape or in 8 bits: one new token per request, lengths and page ids known
// on the GPU only.
//
// Bound by the stream of keys and values (4 g flops per 4 bytes of bf16 for g query heads to a KV head), so the design is about
// keeping requests for memory on their way on every compute unit, whatever the lengths are.  (The cache is read once for each block of
// at most 32 query heads to a KV head.)
//
// Work.  An item is a (request, KV head, block of at most 16 NT query heads).  Its visible keys are walked in units (32 of bf16,
// 16 of fp32, 64 of codes) by single waves that share nothing.  The host does not know the lengths, so the launch is a fixed number of
// waves, WORKERS: 1024, four per compute unit, twice as many for codes of 64 channels.  Each takes ceil(sum / WORKERS) of the batch's units, in
// order of items (two waves a share, where two heads lie in one line: see the kernel): it works out the sum from kv_lens and finds its
// own range in it.  So no share is longer than that, whatever the mix of lengths; the waves at the end have less or nothing (1744 units
// are 872 shares of two for 1024 waves), which matters where shares are few units long.  At most the first and the last item of a share are cut.  Pieces of cut items go to the workspace and a second, small launch joins them.  (Workgroups of four waves that
// walked an item's keys together and joined them in LDS took 94.3 us for 64 x 4096 rows where single waves took 90.3, 97.5 for one request
// of 131071 rows (90.2), 104 for 200 requests of 50 to 1200 rows (95.1): their waves wait for one another at the end of each item.)
//
// Products.  S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32_bf16 (fp32: 16x16x4), keys and values as the A operands from
// LDS (bf16 V through the transposing read), so that a lane owns one query column: its maximum and denominator are scalars, and
// its share of S^T is, up to the order of the keys, its B operand of the second product.  A bf16 product takes the weights as
// three bf16 parts, which together are the fp32 weight: the matrix unit is idle most of the time (64 x 4096 rows: 89.7 us, 89.4 with two
// parts), and the error against 64 bits is then that of rounding the result, 1.667e-3 of its norm (2.270e-3 with one part), also
// where values cancel.  All parts are positive, so that an infinite value stays one (90.4 us; with signed parts 90.0).
//
// Data movement.  A wave has room for one unit of K and of V (8 KB each at 128 channels) and refills them as soon as their
// operands are read, straight from memory to LDS, counted waits instead of barriers; the first unit of its next item is on its
// way before it is done with the last one of this.  A page id is needed for every 8 rows at the most: a wave keeps the ids of
// its next units in one register, a lane each, and takes them out as scalars.
//
// Times here and below: us of the whole call, twelve in a replayed graph over three pools in turn (called one by one on a stream
// the long ones take 5 % less).  Heads of 128 channels, bf16: 64 requests of 4096 rows, 28 / 4 heads, pages of 64: 91.4 (538 MB: 5.9 TB/s; the
// first kernel alone 83, 6.5 TB/s); one of 131071, 32 / 8 heads, pages of 16: 90.9; 32 of up to 32000 rows through a window of 4000 and
// 4 first tokens: 85.4 (489 MB); five of 300 to 3000 rows: 13.6; one of 700: 8.5, which is two launches and, in the first, four
// dependent trips to memory (lengths, page ids, keys, results).
//
// Codes (e4m3, a power of two to a block of 16 rows and a head) take the same way.  They go to LDS as they are and become bf16 on the way to
// the matrix unit, times their scale and exactly, by one instruction for two of them, so that products, softmax and sums are those of a
// bf16 pool that holds what the codes are worth: the error against 64 bits is the same.  V goes through the transposing read of 8 bits; an fp32 query
// is three bf16 parts.  Scales are asked for with the page ids that name them, a lane each, and come before the keys.  A unit is 64 keys
// (32 and twice the waves: as fast where it is long, 71.3 / 69.8 for 200 requests of 50 to 1200 rows, 12.5 / 10.7 for five of 300 to 3000, 8.5 / 9.2 for one of 700), for
// heads of 64 channels by twice the waves.  64 requests of 8192 rows, 28 / 4 heads: 97.3 (538 MB, 5.5 TB/s; the first kernel alone 85.7, 6.3 TB/s; only
// the stream of it, without products, 96); one of 131071, 32 / 8 heads: 54.7 (270 MB); windows of 4000 over 32 requests: 51.7 (246 MB).  Pools that keep the
// rows of a head together are read 3 % faster.
#pragma once
#include "tr_device.h"
#include "tr_internal.h"

#include <algorithm>
#include <type_traits>

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

#define CONST_AS __attribute__((address_space(4)))

constexpr float NOTHING = -__FLT_MAX__; // reference of a row that has seen no key
// Non-temporal: a key is read once, or once for each block of query heads.  Where a row is half a line and the other half another head's, the
// waves of both heads want the line, and it stays in the L2 for the second.  us, codes of 64 channels, 64 requests of 4000 rows of 16 / 4 heads, non-temporal / not: heads side by
// side 52.7 / 38.6 (114 or 65 thousand KB are fetched), rows side by side 33.5 / 36.5; heads of 128 channels 98.0 / 110.0.
constexpr int DMA_STREAM = 2;
// What a pool holds: a tr_dtype, which is the type of queries and results too, or codes with scales, the latter's type being FMT & 1.
enum { FMT_F32 = TR_F32, FMT_BF16 = TR_BF16, FMT_Q8_F32 = 2 | TR_F32, FMT_Q8_BF16 = 2 | TR_BF16 };
// Loads of 1 KB that a wave has on their way.  us with 5 / 6 / 7 / 8: 64 x 4096 rows 95.5 / 92.6 / 91.7 / 96.2, one request of 131071 95.4 /
// 92.2 / 91.3 / 94.3, windows over 32 requests 89.1 / 86.0 / 85.5 / 90.4, 200 requests of 50 to 1200 99.1 / 96.9 / 96.2 / 98.2.
constexpr int FLIGHT = 7;
// Codes: 64 requests of 8192 rows, 28 / 4 heads, with 7 / 8 / 9 / 10 / 12 / 16: 106.8 / 97.3 / 97.3 / 98.4 / 99.9 / 102.7; one of 131071 59.1 / 55.2 / 56.0 / 55.7 /
// 59.3 / 56.9; windows over 32 requests 58.0 / 52.3 / 53.0 / 53.2 / 52.4 / 53.3.
constexpr int FLIGHT_Q8 = 8;

// A bit for each key of a unit.
template <int UNIT> using Mask = typename std::conditional<UNIT == 64, uint64_t, uint32_t>::type;
template <class M> __device__ __forceinline__ M low_bits(int n) { return n >= 8 * (int)sizeof(M) ? ~(M)0 : n <= 0 ? (M)0 : ((M)1 << n) - 1; }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)uniform((int)x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) { return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x); }

// Inclusive sums over the wave, on the vector unit's cross-lane path: within rows of 16 lanes, then across them.
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false); // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false); // last lane of a row to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false); // lane 31 to the upper half
    return x;
}

// The keys of a request as units: the first `su` hold the sinks, the others run from unit `lu` to the end.
template <int UNIT> struct Walk {
    int len, lo, sink, su, lu, units; // at least one unit, which writes the result
    __device__ __forceinline__ int unit(int i) const { return i < su ? i : i - su + lu; }
    __device__ __forceinline__ Mask<UNIT> seen(int first_key) const // bit b: key first_key + b is visible
    {
        typedef Mask<UNIT> M;
        return low_bits<M>(UNIT) & low_bits<M>(len - first_key) & (low_bits<M>(sink - first_key) | ~low_bits<M>(lo - first_key));
    }
};
template <int UNIT> __device__ __forceinline__ Walk<UNIT> walk_of(const TrPagedDecodeArgs& a, int kv_len)
{
    Walk<UNIT> w;
    w.len = min(max(kv_len, 0), a.max_blocks << a.pool.page_shift);
    w.lo = a.window ? max(max(kv_len, 0) - a.window, 0) : 0; // may lie behind what the table holds
    w.sink = min(a.n_sink, min(w.lo, w.len));
    w.su = (w.sink + UNIT - 1) / UNIT;
    w.lu = max(w.lo / UNIT, w.su);
    w.units = max(w.su + max((w.len + UNIT - 1) / UNIT - w.lu, 0), 1);
    return w;
}

template <bool MAX> __device__ __forceinline__ float column_reduce(float x) // over the four lanes of a query column
{
    auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    u = __float_as_uint(x);
    const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// Two weights as three pairs of bf16 that add up to them, by cutting off 8 bits at a time.  Each rest gets 2^-30 of its weight besides, which no
// sum in fp32 notices, so that no part is zero: infinite values times zero would be NaN.  Codes have no infinity.
struct Split {
    uint32_t pair[3];
};
template <bool INFINITE> __device__ __forceinline__ Split split(float x, float y)
{
    auto upper = [](float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); };
    auto both = [](float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); };
    const float wx = x, wy = y;
    Split s;
    s.pair[0] = both(x, y);
#pragma unroll
    for (int j = 1; j < 3; ++j) {
        x = INFINITE ? fmaf(wx, 0x1p-30f, x - upper(x)) : x - upper(x);
        y = INFINITE ? fmaf(wy, 0x1p-30f, y - upper(y)) : y - upper(y);
        s.pair[j] = both(x, y);
    }
    return s;
}

// A unit is 8 KB of K and 8 KB of V for heads of 128 channels (half of that for 64): 32 rows of bf16 or 16 of fp32; 32 rows of codes are
// half as much, and a unit of them 64.
// Where a wave's loads of it go: load i fills rows RPI i .. of the unit, lane after lane.  K: 16-byte chunk c of row r sits at
// c ^ ksw(r), so that the reads of operands spread over all banks; V: bf16 32-byte group g of row r at g ^ vsw(r), codes 16-byte group
// likewise, for the same reason, fp32 as it comes.
template <int FMT, int D> struct Rows {
    static constexpr bool Q8 = FMT >= 2, BF16 = FMT != FMT_F32; // BF16: what the products take
    static constexpr int IO = FMT & 1, UNIT = Q8 ? TR_Q8_UNIT : tr_paged_unit_keys(FMT), ROW = D * (Q8 ? 1 : BF16 ? 2 : 4);
    static constexpr int CPR = ROW / 16, RPI = 64 / CPR, LPU = UNIT / RPI, BYTES = UNIT * ROW;
    static constexpr int IDS = Q8 ? 768 : 256;                                         // bytes of page ids, and scales
    static constexpr int QROW = D * (IO == TR_BF16 ? 2 : 4), QCPR = QROW / 16, QPI = 64 / QCPR; // a query row, its chunks, rows of a load
    static constexpr int KS = D * (BF16 ? 2 : 4) / 64, QPARTS = FMT == FMT_Q8_F32 ? 3 : 1;      // steps of a product, bf16 parts of a query
    static constexpr bool HALF_LINES = ROW < 128;
    static constexpr int MOST = Q8 ? FLIGHT_Q8 : FLIGHT;
    __device__ static __forceinline__ int ksw(int r) { return CPR >= 16 ? r & 15 : (r / (16 / CPR)) & (CPR - 1); }
    __device__ static __forceinline__ int vsw(int r)
    {
        if (Q8) return ksw(r) ^ ((r >> 4) & 1) * (CPR / 2); // the transposing read takes rows r and r + 16 together
        return CPR >= 16 ? r & 7 : (r / (16 / CPR)) & (CPR / 2 - 1);
    }
    __device__ static __forceinline__ int kchunk(int row, int lane) { return (lane % CPR) ^ ksw(row); }
    __device__ static __forceinline__ int vchunk(int row, int lane)
    {
        if (Q8) return (lane % CPR) ^ vsw(row);
        return BF16 ? (((lane % CPR) >> 1) ^ vsw(row)) * 2 + (lane & 1) : lane % CPR;
    }
};
// What a lane holds of 16 query rows, keys or values as an operand: 16 bytes for every 64 bytes of a row (of bf16 ones, where the pool holds codes).
template <int FMT> struct Operand { typedef bf16x8 T; };
template <> struct Operand<FMT_F32> { typedef f32x4 T; };

// Where scales are, and for how many heads of a page.
struct TrScales {
    const uint8_t *k, *v;
    int heads;
};
// The scale in lane `at` as a factor, and four codes each of two blocks as what they are worth, exactly.
__device__ __forceinline__ float scale_of(int scales, int at) { return __uint_as_float(((uint32_t)__builtin_amdgcn_readlane(scales, at) & 0xffu) << 23); }
__device__ __forceinline__ bf16x8 worth(uint32_t x, float x_by, uint32_t y, float y_by)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, x_by, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, x_by, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, y_by, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, y_by, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One unit of a wave: where its KV head begins, its first key, which of its keys are seen, and where its page ids are among the
// wave's.
template <int UNIT> struct UnitRef {
    uint64_t head;
    int key0, at;
    Mask<UNIT> seen;
};

// A run of units of one item that one wave walks.
template <int UNIT> struct Piece {
    int r, item, u0, n; // item: which of the request's; n == 0: there is none
    int kvh, tile;      // what it is an item of
    Walk<UNIT> w;
    __device__ __forceinline__ bool whole() const { return n == w.units; }
};

// What one wave accumulates: O^T of query column lane % 16 (bf16: element e of block b is channel 16 b + 4 (lane / 16) + e; fp32:
// channel 64 (b / 4) + 16 (lane / 16) + 4 e + b % 4), reference maximum (a score, not yet scaled) and this lane's share of the denominator.
template <int D, int NT> struct Acc {
    f32x4 o[NT][D / 16];
    float m[NT], l[NT];
};

// A wave's loads.
template <int FMT, int D> struct Stream {
    using R = Rows<FMT, D>;
    using P = Piece<R::UNIT>;
    typedef typename Operand<FMT>::T Op;
    static constexpr int LPU = R::LPU, UNIT = R::UNIT, UNIT_SHIFT = UNIT == 64 ? 6 : UNIT == 32 ? 5 : 4;
    typedef UnitRef<UNIT> Ref;
    typedef Mask<UNIT> M;
    static constexpr bool Q8 = R::Q8;
    uint32_t kring, vring, idring, qring, row_bytes, page_bytes;
    int lane, page_shift, sub_shift, per_unit_shift, n_pages; // sub_shift: rows of a unit that have an id (codes: and a scale) of their own
    int32_t max_blocks;
    uint32_t head_stride;
    bool shared; // two heads' rows lie in one line
    uint32_t dk[LPU], dv[LPU]; // what a lane adds to the start of a unit's page for load i

    __device__ __forceinline__ Stream(const TrPagedDecodeArgs& a, uint32_t ring, int lane_) : lane(lane_)
    {
        kring = (uint32_t)uniform((int)ring);
        vring = kring + R::BYTES;
        idring = vring + R::BYTES;
        qring = idring + R::IDS;
        row_bytes = a.pool.row_stride;
        page_bytes = a.pool.page_stride;
        head_stride = a.pool.head_stride;
        shared = a.n_kv_heads > 1 && head_stride < 128;
        page_shift = a.pool.page_shift;
        n_pages = a.pool.n_pages;
        max_blocks = a.max_blocks;
        const int in_page = min(page_shift, UNIT_SHIFT); // rows of a unit that lie in one page
        sub_shift = Q8 ? 4 : in_page;
        per_unit_shift = UNIT_SHIFT - sub_shift;
#pragma unroll
        for (int i = 0; i < LPU; ++i) {
            const int row = i * R::RPI + lane / R::CPR;
            const uint32_t in = (uint32_t)(row & ((1 << in_page) - 1)) * row_bytes;
            dk[i] = in + R::kchunk(row, lane) * 16;
            dv[i] = in + R::vchunk(row, lane) * 16;
        }
    }
    __device__ __forceinline__ int refill() const { return 64 >> per_unit_shift; } // units whose ids a register holds

    // Page ids of a piece's units from its j0-th on, a lane each; -1 where there is none.  They are requested into LDS and taken
    // from there when they are needed: the wait for a register's load would be a wait for all keys and values behind it.
    __device__ __forceinline__ int key_of(const P& p, int j0) const
    {
        return p.w.unit(p.u0 + j0 + (lane >> per_unit_shift)) * UNIT + ((lane & ((1 << per_unit_shift) - 1)) << sub_shift);
    }
    __device__ __forceinline__ int entry(const P& p, int j0) const
    {
        const int key = key_of(p, j0);
        return j0 + (lane >> per_unit_shift) < p.n && key < p.w.len ? key >> page_shift : -1;
    }
    __device__ __forceinline__ void request_ids(const int32_t* __restrict__ table, const P& p, int j0) const
    {
        const int e = entry(p, j0);
        if (e >= 0)
            __builtin_amdgcn_global_load_lds((const GLB_AS void*)(table + (int64_t)p.r * max_blocks + e), (LDS_AS void*)(uintptr_t)idring, 4, 0, 0);
    }
    __device__ __forceinline__ int take_ids(const P& p, int j0) const
    {
        LDS_AS const int* const from = (LDS_AS const int*)(uintptr_t)idring;
        int id = from[lane];
        if (entry(p, j0) < 0 || (uint32_t)id >= (uint32_t)n_pages) id = -1;
        asm volatile("" : "+v"(id) : : "memory"); // read before the next request overwrites it
        return id;
    }
    // The scales of the blocks that ids were taken for, a byte each, likewise; of a block without a page whatever was there before.
    __device__ __forceinline__ void request_scales(const TrScales& sc, const P& p, int j0, int ids) const
    {
        const int64_t block = (((int64_t)ids * sc.heads + p.kvh) << (page_shift - 4)) + ((key_of(p, j0) & ((1 << page_shift) - 1)) >> 4);
        if (ids >= 0) {
            __builtin_amdgcn_global_load_lds((const GLB_AS void*)(sc.k + block), (LDS_AS void*)(uintptr_t)(idring + 256), 1, 0, 0);
            __builtin_amdgcn_global_load_lds((const GLB_AS void*)(sc.v + block), (LDS_AS void*)(uintptr_t)(idring + 512), 1, 0, 0);
        }
    }
    __device__ __forceinline__ void take_scales(int& ks, int& vs) const
    {
        LDS_AS const int* const from = (LDS_AS const int*)(uintptr_t)(idring + 256);
        ks = from[lane];
        vs = from[64 + lane];
        asm volatile("" : "+v"(ks), "+v"(vs) : : "memory"); // read before the next request overwrites them
    }
    // The query rows of an item, likewise; rows past the last one repeat it, and nothing of theirs is looked at.
    template <int NT> __device__ __forceinline__ void request_q(const char* __restrict__ first, int rows) const
    {
#pragma unroll
        for (int i = 0; i < 16 * NT / R::QPI; ++i)
            __builtin_amdgcn_global_load_lds((const GLB_AS void*)(first + min(i * R::QPI + lane / R::QCPR, rows - 1) * R::QROW + lane % R::QCPR * 16),
                                             (LDS_AS void*)(uintptr_t)(qring + i * 1024), 16, 0, 0);
    }
    // Codes: step 2 j + h of a product is channels 64 j + 16 quad + 8 h + 0 .. 7, a lane's share of which is half of a 16-byte unit.  An fp32
    // query is three bf16 parts there, which together are it, so that its products are exact like those of a bf16 one.  bf16 ends at 2^-133, fp32
    // at 2^-149: a query head whose channels are all below 2^-32 is taken 2^24 times as large, which `by`, a factor on its scores, takes
    // back (scores stay below 2^-8 2^128 d).
    template <int NT> __device__ __forceinline__ void take_q(Op (&q)[NT][R::KS][R::QPARTS], float (&by)[NT]) const
    {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t row = qring + (uint32_t)((16 * t + (lane & 15)) * R::QROW);
            by[t] = 1.0f;
            if constexpr (FMT == FMT_Q8_F32) {
                float x[R::KS][8], top = 0.0f;
#pragma unroll
                for (int ks = 0; ks < R::KS; ++ks) {
                    const uint32_t at = row + (64 * (ks >> 1) + 16 * (lane >> 4) + 8 * (ks & 1)) * 4;
                    *(f32x4*)x[ks] = *(LDS_AS const f32x4*)(uintptr_t)at;
                    *(f32x4*)(x[ks] + 4) = *(LDS_AS const f32x4*)(uintptr_t)(at + 16);
                }
#pragma unroll
                for (int ks = 0; ks < R::KS; ++ks)
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[ks][i]));
                if (__any(top < 0x1p-32f)) { // a lane has a quarter of a head's channels
                    const bool small = column_reduce<true>(top) < 0x1p-32f;
                    by[t] = small ? 0x1p-24f : 1.0f;
#pragma unroll
                    for (int ks = 0; ks < R::KS; ++ks)
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[ks][i] *= small ? 0x1p24f : 1.0f;
                }
#pragma unroll
                for (int ks = 0; ks < R::KS; ++ks) {
                    u32x4 part[3];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float a = x[ks][2 * i], b = x[ks][2 * i + 1];
#pragma unroll
                        for (int j = 0; j < 3; ++j) {
                            const uint32_t ua = __float_as_uint(a) & 0xffff0000u, ub = __float_as_uint(b) & 0xffff0000u;
                            part[j][i] = (ua >> 16) | ub;
                            a -= __uint_as_float(ua);
                            b -= __uint_as_float(ub);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 3; ++j) {
                        q[t][ks][j] = __builtin_bit_cast(bf16x8, part[j]);
                        asm volatile("" : "+v"(q[t][ks][j]) : : "memory");
                    }
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < R::KS; ++ks) {
                    const uint32_t at = Q8 ? row + (64 * (ks >> 1) + 16 * (lane >> 4) + 8 * (ks & 1)) * 2 : row + (4 * ks + (lane >> 4)) * 16;
                    q[t][ks][0] = *(LDS_AS const Op*)(uintptr_t)at;
                    asm volatile("" : "+v"(q[t][ks][0]) : : "memory");
                }
            }
        }
    }
    __device__ __forceinline__ Ref ref(const P& p, int j, int ids) const
    {
        Ref u;
        u.head = (uint64_t)(uint32_t)p.kvh * head_stride;
        u.key0 = uniform(p.w.unit(p.u0 + j) * UNIT);
        u.at = (j & (refill() - 1)) << per_unit_shift;
        u.seen = p.w.seen(u.key0);
        uint32_t holes = (uint32_t)(__ballot(ids < 0) >> u.at) & low_bits<uint32_t>(1 << per_unit_shift);
        while (holes) { // pages that are none
            const int s = __builtin_ctz(holes);
            holes &= holes - 1;
            u.seen &= ~(low_bits<M>(1 << sub_shift) << (s << sub_shift));
        }
        u.seen = uniform(u.seen);
        return u;
    }
    // LATER: not the wave's first unit: no more than MOST loads on their way.  The rows of a load lie in one page; where that is
    // none, they are read from page 0, and rows behind the last key from wherever they would be: both exist, and neither is seen.
    template <bool V, bool LATER> __device__ __forceinline__ void issue(const char* __restrict__ base, const Ref& u, int ids) const
    {
        const char* const first_row = base + u.head + (uint64_t)(uint32_t)(u.key0 & ((1 << page_shift) - 1)) * row_bytes;
#pragma unroll
        for (int i = 0; i < LPU; ++i) {
            if (LATER && i + LPU >= R::MOST) wait_vm<R::MOST - 1>();
            const uint32_t id = (uint32_t)max(__builtin_amdgcn_readlane(ids, u.at + ((i * R::RPI) >> sub_shift)), 0);
            const GLB_AS void* const from = (const GLB_AS void*)(first_row + (uint64_t)id * page_bytes + (V ? dv[i] : dk[i]));
            LDS_AS void* const to = (LDS_AS void*)(uintptr_t)((V ? vring : kring) + i * 1024);
            if (R::HALF_LINES && shared) __builtin_amdgcn_global_load_lds(from, to, 16, 0, 0);
            else __builtin_amdgcn_global_load_lds(from, to, 16, 0, DMA_STREAM);
        }
    }
};

// A wave's walk over its units of piece p, the first of which is on its way; at its end the keys of the first unit of piece `then`
// are, whose page ids and queries it leaves in ids and in LDS.  Loads return in order, so the counts below say which of them
// have: a unit's keys once no more than the loads of its values are left, its values once no more than those of the next
// unit's keys are.
// A function of its own with restricted pointers, LDS by whole addresses: the compiler otherwise takes the reads of LDS to
// depend on every load on its way to it.
template <int FMT, int D, int NT>
__device__ __forceinline__ void walk_units(const char* __restrict__ k, const char* __restrict__ v, const int32_t* __restrict__ table,
                                           const Stream<FMT, D>& st, const Piece<Rows<FMT, D>::UNIT>& p, const Piece<Rows<FMT, D>::UNIT>& then,
                                           const char* __restrict__ then_q, int then_rows,
                                           const typename Operand<FMT>::T (&q)[NT][Rows<FMT, D>::KS][Rows<FMT, D>::QPARTS], const TrScales& sc, const float (&scale)[NT], bool first, int& ids, UnitRef<Rows<FMT, D>::UNIT>& cur, Acc<D, NT>& acc)
{
    using R = Rows<FMT, D>;
    typedef typename Operand<FMT>::T Op;
    constexpr bool BF16 = R::BF16, Q8 = R::Q8;
    constexpr int LPU = R::LPU, KB = R::UNIT / 16, KS = R::ROW / 64; // blocks of 16 keys; 64-byte steps of a row
    constexpr Mask<R::UNIT> ALL = R::UNIT == 16 ? 0xffffu : ~(Mask<R::UNIT>)0;
    static_assert(R::MOST <= 2 * LPU, "");
    const int lane = st.lane, c16 = lane & 15, quad = lane >> 4;
    int koff[KS], voff[D / 16]; // V: fp32 four rows of two or one 256-byte groups, bf16 a group of 16 channels each
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = (int)st.kring + c16 * R::ROW + (((4 * ks + quad) ^ R::ksw(c16)) * 16);
    const int vrow = Q8 ? 4 * quad + ((c16 >> 1) & 3) + (c16 >> 3) * 16 : 4 * quad + (c16 >> 2); // codes: rows of both blocks
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb)
        voff[cb] = Q8 ? (int)st.vring + vrow * R::ROW + ((cb ^ R::vsw(vrow)) * 16) + (c16 & 1) * 8 : BF16 ? (int)st.vring + vrow * R::ROW + ((cb ^ R::vsw(vrow)) * 32) + (c16 & 3) * 8 : (int)st.vring + (4 * quad + (cb & 3)) * R::ROW + (cb >> 2) * 256 + c16 * 16;
    LDS_AS const char* lds = (LDS_AS const char*)(uintptr_t)0;

    int ks_of = 0, vs_of = 0; // scales of the blocks that ids are held for, a lane each
    auto request_ids = [&](int j0) { j0 < p.n ? st.request_ids(table, p, j0) : st.request_ids(table, then, 0); };
    for (int t = 0; t < p.n; ++t) {
        UnitRef<R::UNIT> next;
        const bool last = t + 1 == p.n, more = !last || then.n > 0;
        // K(t).  Behind the keys of a piece that is not the first there are, besides its values, the results of the last one: at least
        // D / 16 stores of a lane, none of which touches another and could become one with it.
        if (t == 0 && !first) wait_vm<LPU + D / 16>();
        else wait_vm<LPU>();
        if (t == 0) { // in front of K(1), so that whoever waits for that has them
            request_ids(st.refill());
            if (then.n > 0) st.template request_q<NT>(then_q, then_rows);
            if (last) wait_vm<0>();
        }
        asm volatile("" ::: "memory");
        if constexpr (Q8) {
            if ((t & (st.refill() - 1)) == 0) st.take_scales(ks_of, vs_of); // they came before the keys
        }
        if (!last) {
            if (((t + 1) & (st.refill() - 1)) == 0) {
                ids = st.take_ids(p, t + 1);
                request_ids(t + 1 + st.refill());
                if constexpr (Q8) st.request_scales(sc, p, t + 1, ids);
            }
            next = st.ref(p, t + 1, ids);
        } else {
            ids = st.take_ids(then, 0);
            next = st.ref(then, 0, ids);
            if constexpr (Q8) st.request_scales(sc, then, 0, ids);
        }
        f32x4 s[NT][KB];
        typedef typename std::conditional<Q8, u32x4, Op>::type Raw;
        Raw ka[KB][KS];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) ka[kb][ks] = *(LDS_AS const Raw*)(lds + koff[ks] + kb * 16 * R::ROW);
        wait_lds(); // the unit's keys are read
        if (more) {
            if (t == 0) st.template issue<false, false>(k, next, ids); // not behind the requests and results above
            else st.template issue<false, true>(k, next, ids);
        }
        if constexpr (Q8) {
            float by[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) by[kb] = scale_of(ks_of, cur.at + kb);
#pragma unroll
            for (int ks = 0; ks < 2 * KS; ++ks)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) { // as many chains as there are blocks
                    const bf16x8 a = worth(ka[kb][ks >> 1][2 * (ks & 1)], by[kb], ka[kb][ks >> 1][2 * (ks & 1) + 1], by[kb]);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = R::QPARTS - 1; j >= 0; --j)
                            s[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[n][ks][j], ks == 0 && j == R::QPARTS - 1 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[n][kb], 0, 0, 0);
                }
        } else if constexpr (BF16) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        s[n][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[kb][ks], q[n][ks][0], ks == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[n][kb], 0, 0, 0);
        } else { // which channels make up a product does not matter, as long as both operands agree; two chains, for their length
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f32x4 x[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[0][ks][e], q[n][ks][0][e], x[e & 1], 0, 0, 0);
                s[n][0] = x[0] + x[1];
            }
        }
        // element e of block kb is key 16 kb + 4 quad + e of the unit
        const Mask<R::UNIT> mine = cur.seen >> (4 * quad);
        if (cur.seen != ALL) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!((uint32_t)(mine >> (16 * kb)) & (1u << e))) s[n][kb][e] = -INFINITY;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float top = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3]));
#pragma unroll
            for (int kb = 1; kb < KB; ++kb) top = fmaxf(top, fmaxf(fmaxf(s[n][kb][0], s[n][kb][1]), fmaxf(s[n][kb][2], s[n][kb][3])));
            // A weight is 2^((s - m) scale), the difference first: it is exact or nearly so however large the scores are, where that of
            // two products with the scale would be off by their roundings.  No weight exceeds 1, so that values near the largest do not overflow.
            if (__any(top > acc.m[n])) {
                const float to = fmaxf(acc.m[n], column_reduce<true>(top)), alpha = __builtin_amdgcn_exp2f((acc.m[n] - to) * scale[n]);
                acc.m[n] = to;
                acc.l[n] *= alpha;
#pragma unroll
                for (int cb = 0; cb < D / 16; ++cb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc.o[n][cb][e] *= alpha;
            }
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4 * KB; ++i) {
                const float w = __builtin_amdgcn_exp2f((s[n][i >> 2][i & 3] - acc.m[n]) * scale[n]);
                sum += w;
                s[n][i >> 2][i & 3] = w;
            }
            acc.l[n] += sum;
        }
        if (more) wait_vm<LPU>(); // V(t)
        else wait_vm<0>();
        asm volatile("" ::: "memory");
        if constexpr (Q8) {
            i32x2 raw[KB / 2][D / 16]; // codes of four keys of a block, and of the block behind
#pragma unroll
            for (int g = 0; g < KB / 2; ++g)
#pragma unroll
                for (int cb = 0; cb < D / 16; ++cb) raw[g][cb] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_AS i32x2*)(lds + voff[cb] + g * 32 * R::ROW));
            wait_lds(); // the unit's values are read
            if (!last) st.template issue<true, true>(v, next, ids);
#pragma unroll
            for (int g = 0; g < KB / 2; ++g) {
                const float by[2] = {scale_of(vs_of, cur.at + 2 * g), scale_of(vs_of, cur.at + 2 * g + 1)};
                Op va[D / 16];
#pragma unroll
                for (int cb = 0; cb < D / 16; ++cb) va[cb] = worth((uint32_t)raw[g][cb][0], by[0], (uint32_t)raw[g][cb][1], by[1]);
                if (cur.seen != ALL) { // what is not seen may be anything, and even a weight of zero would make NaN of NaN
                    const uint32_t bits = (uint32_t)(mine >> (32 * g));
                    u32x4 keep;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int bit = 16 * (i >> 1) + 2 * (i & 1);
                        keep[i] = ((bits >> bit) & 1 ? 0xffffu : 0u) | ((bits >> bit) & 2 ? 0xffff0000u : 0u);
                    }
#pragma unroll
                    for (int cb = 0; cb < D / 16; ++cb) va[cb] = __builtin_bit_cast(Op, __builtin_bit_cast(u32x4, va[cb]) & keep);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    u32x4 parts[3];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const auto w = split<false>(s[n][2 * g + (i >> 1)][2 * (i & 1)], s[n][2 * g + (i >> 1)][2 * (i & 1) + 1]);
#pragma unroll
                        for (int j = 0; j < 3; ++j) parts[j][i] = w.pair[j];
                    }
#pragma unroll
                    for (int j = 0; j < 3; ++j)
#pragma unroll
                        for (int cb = 0; cb < D / 16; ++cb)
                            acc.o[n][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[cb], __builtin_bit_cast(bf16x8, parts[j]), acc.o[n][cb], 0, 0, 0);
                }
            }
        } else {
            Op va[D / 16];
#pragma unroll
            for (int cb = 0; cb < D / 16; ++cb) {
                if constexpr (BF16) {
                    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(lds + voff[cb]));
                    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(lds + voff[cb] + 16 * R::ROW));
                    va[cb] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
                } else {
                    va[cb] = *(LDS_AS const f32x4*)(lds + voff[cb]); // key 4 quad + cb % 4, channels 64 (cb / 4) + 4 c16 ..
                }
            }
            wait_lds(); // the unit's values are read
            if (!last) st.template issue<true, true>(v, next, ids);
            u32x4 parts[NT][3]; // of the weights, as bf16; fp32: they stay in s.  Not sooner: the next values are on their way meanwhile
            if constexpr (BF16) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4 * KB; i += 2) {
                        const auto w = split<true>(s[n][i >> 2][i & 3], s[n][i >> 2][(i & 3) + 1]);
#pragma unroll
                        for (int j = 0; j < 3; ++j) parts[n][j][i / 2] = w.pair[j];
                    }
            }
            if (cur.seen != ALL) { // what is not seen may be anything, and even a weight of zero would make NaN of NaN
                u32x4 keep; // bf16: element j of an operand is key 16 (j >> 2) + 4 quad + (j & 3)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int bit = BF16 ? 16 * (i >> 1) + 2 * (i & 1) : i;
                    keep[i] = BF16 ? ((mine >> bit) & 1 ? 0xffffu : 0u) | ((mine >> bit) & 2 ? 0xffff0000u : 0u) : (mine >> bit) & 1 ? 0xffffffffu : 0u;
                }
#pragma unroll
                for (int cb = 0; cb < D / 16; ++cb) {
                    const u32x4 mask = BF16 ? keep : u32x4{keep[cb & 3], keep[cb & 3], keep[cb & 3], keep[cb & 3]};
                    va[cb] = __builtin_bit_cast(Op, __builtin_bit_cast(u32x4, va[cb]) & mask);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int cb = 0; cb < D / 16; ++cb) {
                    if constexpr (BF16) {
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            acc.o[n][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[cb], __builtin_bit_cast(bf16x8, parts[n][j]), acc.o[n][cb], 0, 0, 0);
                    } else { // operand cb holds key cb % 4 of the four; its channel i goes to block 4 (cb / 4) + i
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc.o[n][(cb & ~3) | i] = __builtin_amdgcn_mfma_f32_16x16x4f32(va[cb][i], s[n][0][cb & 3], acc.o[n][(cb & ~3) | i], 0, 0, 0);
                    }
                }
        }
        cur = next;
    }
}

template <int FMT, int D, int NT, int WORKERS>
__global__ __launch_bounds__(64, NT == 1 || WORKERS > 1024 ? 2 : 1) void paged_decode_kernel(const TrPagedDecodeArgs a)
{
    using R = Rows<FMT, D>;
    using P = Piece<R::UNIT>;
    constexpr int ROWS = 16 * NT;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x, c16 = lane & 15, quad = lane >> 4;
    const int tiles = (a.group + ROWS - 1) / ROWS, per_req = a.n_kv_heads * tiles; // items of a request
    // A wave takes the share `turn` of the batch's items.  Where two heads lie in one line they make one item for the shares, and two waves of
    // one die take the same share, a head each, so that the line is fetched once: a wave and the one eight workgroups on.  Waves are counted
    // so that those which have pieces of one head stand side by side.  us with heads shared out by themselves / so, 16 / 4 heads of 64 channels: 91 requests of 3700
    // to 11300 rows 120.4 / 83.8, three of 41000 to 90000 38.7 / 26.4, 64 of 500 to 4000 33.2 / 23.8, 64 of 4000 (where the two were eight apart anyway) 38.9 / 38.9.
    int worker = blockIdx.x, turn = worker, member = 0;
    bool paired = false;
    if constexpr (R::HALF_LINES) {
        paired = a.pool.head_stride < 128 && a.n_kv_heads % 2 == 0 && tiles == 1 && gridDim.x % 2 == 0;
        if (paired) {
            const int half = gridDim.x / 2, full = half & ~7;
            if (worker < 2 * full) {
                turn = (worker >> 4) * 8 + (worker & 7);
                member = (worker >> 3) & 1;
            } else {
                turn = full + ((worker - 2 * full) >> 1);
                member = worker & 1;
            }
            worker = member * half + turn;
        }
    }
    const int share_items = paired ? per_req / 2 : per_req, turns = paired ? WORKERS / 2 : WORKERS;

    // the batch's units, and the request that this wave's share begins in: a lane sums up `per` neighbouring requests
    auto len_of = [&](int r) { return r < a.n_req ? a.kv_lens[r] : 0; };
    auto units_of = [&](int r, int len) { return r < a.n_req ? walk_of<R::UNIT>(a, len).units : 0; };
    const int per = (a.n_req + 63) / 64;
    int lens = len_of(lane * per), own = units_of(lane * per, lens);
    for (int i = 1; i < per; i += 8) {
        int l[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) l[j] = i + j < per ? len_of(lane * per + i + j) : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) own += i + j < per ? units_of(lane * per + i + j, l[j]) : 0;
    }
    int sums = wave_scan(own);
    const int total = __builtin_amdgcn_readlane(sums, 63) * share_items;
    const int share = max((total + turns - 1) / turns, TR_PAGED_MIN_UNITS);
    const int begin = share * turn;
    // who has pieces of the cut items, by the item or by the wave that begins it (a share begins at most one)
    auto record = [&](int64_t at, int x, int pieces) {
        if (lane == 0) *(int2*)(a.ws_items + 2 * at) = make_int2(x, pieces);
    };
    if (begin >= total) {
        if (a.cut == TR_PAGED_JOIN_BY_WAVE) record(worker, 0, 0);
        return;
    }
    const int end = min(begin + share, total);
    int left = end - begin; // behind the pieces described so far
    const int unit = begin / share_items; // in units of all heads together
    int at = __builtin_ctzll(__ballot(sums > unit)), r0 = 0;
    int before = __builtin_amdgcn_readlane(sums, at) - __builtin_amdgcn_readlane(own, at);
    if (per > 1) { // one of that lane's
        r0 = at * per;
        while (true) {
            lens = len_of(r0 + lane), own = units_of(r0 + lane, lens), sums = wave_scan(own);
            const int here = __builtin_amdgcn_readlane(sums, 63);
            if (before + here > unit || r0 + 64 >= a.n_req) break;
            before += here;
            r0 += 64;
        }
        const uint64_t here = __ballot(before + sums > unit);
        at = here ? __builtin_ctzll(here) : 63; // never none, unless the lengths are written meanwhile
        before += __builtin_amdgcn_readlane(sums, at) - __builtin_amdgcn_readlane(own, at);
    }

    P p;
    p.r = min(r0 + at, a.n_req - 1);
    p.w = walk_of<R::UNIT>(a, __builtin_amdgcn_readlane(lens, at));
    const int local = begin - before * share_items;
    p.item = uniform(local / p.w.units);
    p.u0 = local - p.item * p.w.units;
    auto place = [&](P& x) {
        x.kvh = paired ? 2 * x.item + member : tiles == 1 ? x.item : uniform(x.item / tiles);
        x.tile = paired ? 0 : x.item - x.kvh * tiles;
    };
    place(p);
    p.n = min(p.w.units - p.u0, left);
    left -= p.n;
    auto following = [&](const P& from) {
        P x = from;
        x.u0 = x.n = 0;
        if (left == 0) return x;
        if (++x.item == share_items) {
            if (x.r + 1 == a.n_req) { // not reached unless the lengths are written meanwhile
                x.item = left = 0;
                return x;
            }
            x.item = 0;
            ++x.r;
            int len;
            if (x.r < r0 + 64) len = __builtin_amdgcn_readlane(lens, x.r - r0);
            else len = ((const CONST_AS int32_t*)(uintptr_t)a.kv_lens)[x.r]; // through the scalar cache: no wait for what is on its way
            x.w = walk_of<R::UNIT>(a, len);
        }
        place(x);
        x.n = min(x.w.units, left);
        left -= x.n;
        return x;
    };
    auto rows_of = [&](const P& x) { return min(a.group - x.tile * ROWS, ROWS); };
    auto head0_of = [&](const P& x) { return (int64_t)x.r * a.n_q_heads + x.kvh * a.group + x.tile * ROWS; }; // of all heads of the batch
    auto first_q = [&](const P& x) { return (const char*)a.q + head0_of(x) * R::QROW; };

    Stream<FMT, D> st(a, (uint32_t)(uintptr_t)(LDS_AS char*)smem, lane);
    st.request_ids(a.table, p, 0);
    st.template request_q<NT>(first_q(p), rows_of(p));
    wait_vm<16 * NT / R::QPI>(); // the ids
    asm volatile("" ::: "memory");
    int ids = st.take_ids(p, 0);
    UnitRef<R::UNIT> cur = st.ref(p, 0, ids);
    const TrScales sc = {a.pool.k_scale, a.pool.v_scale, a.n_kv_heads};
    if constexpr (R::Q8) st.request_scales(sc, p, 0, ids);
    st.template issue<false, false>(a.pool.k, cur, ids);
    st.template issue<true, false>(a.pool.v, cur, ids);
    wait_vm<2 * R::LPU>(); // the queries
    for (bool first = true;; first = false) {
        const P then = following(p);
        typename Operand<FMT>::T q[NT][R::KS][R::QPARTS];
        asm volatile("" ::: "memory");
        float by[NT], scale[NT];
        st.template take_q<NT>(q, by);
#pragma unroll
        for (int t = 0; t < NT; ++t) scale[t] = by[t] * a.scale_log2e;
        Acc<D, NT> acc;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            acc.m[t] = NOTHING;
            acc.l[t] = 0.0f;
#pragma unroll
            for (int cb = 0; cb < D / 16; ++cb) acc.o[t][cb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        walk_units<FMT, D, NT>(a.pool.k, a.pool.v, a.table, st, p, then, first_q(then), rows_of(then), q, sc, scale, first, ids, cur, acc);
        if (then.n) st.template issue<true, false>(a.pool.v, cur, ids);
        asm volatile("" ::: "memory");

        const int rows = rows_of(p);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float l = column_reduce<false>(acc.l[t]);
            const int row = 16 * t + c16;
            if (row >= rows) continue;
            const bool whole = p.whole();
            const float f = !whole ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l; // a row without any weight is zero
            const int64_t slot = (int64_t)(2 * worker + (p.u0 == 0)) * a.ws_rows + row; // a share cuts at most its first and its last item
            float* const sums = a.ws_o + slot * D;
#pragma unroll
            for (int cb = 0; cb < D / 16; ++cb) {
                const f32x4* const o = acc.o[t];
                if constexpr (R::BF16) {
                    const int ch = 16 * cb + 4 * quad;
                    if constexpr (R::IO == TR_F32) *(f32x4*)((whole ? (float*)a.out + (head0_of(p) + row) * D : sums) + ch) = o[cb] * f;
                    else if (whole) *(bf16x4*)((__bf16*)a.out + (head0_of(p) + row) * D + ch) = __builtin_convertvector(o[cb] * f, bf16x4);
                    else *(f32x4*)(sums + ch) = o[cb];
                } else {
                    const int b = cb & ~3, e = cb & 3;
                    float* const to = whole ? (float*)a.out + (head0_of(p) + row) * D : sums;
                    *(f32x4*)(to + 16 * b + 16 * quad + 4 * e) = f32x4{o[b][e], o[b + 1][e], o[b + 2][e], o[b + 3][e]} * f;
                }
            }
            if (!whole && quad == 0) *(float2*)(a.ws_ml + slot * 2) = make_float2(acc.m[t] == NOTHING ? NOTHING : acc.m[t] * by[t], l);
        }
        const int item = paired ? 2 * p.item + member : p.item; // of the request's
        const int pieces = p.whole() || p.u0 ? 1 : (end - left - then.n - p.n + p.w.units - 1) / share - turn + 1; // of the item that begins here
        if (a.cut == TR_PAGED_JOIN_BY_WAVE) {
            if (then.n == 0) record(worker, p.r * per_req + item, pieces);
        } else if (a.cut && p.u0 == 0) {
            record((int64_t)p.r * per_req + item, worker, pieces);
        }
        if (then.n == 0) break;
        p = then;
    }
}

// Joins the pieces of cut items: out = sum_p f_p O_p / sum_p f_p l_p with f_p = 2^((m_p - max m) scale).  One workgroup per row of the
// result, or per row of the item that a wave of the first launch begins; groups of D / 4 lanes take every GROUPS-th piece and
// are joined through LDS.
template <int DTYPE, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void paged_join_kernel(const TrPagedDecodeArgs a, int rows_per_tile)
{
    constexpr int LPR = D / 4, GROUPS = THREADS / LPR;
    __shared__ f32x4 os[GROUPS][LPR];
    __shared__ float2 mls[GROUPS];
    const int tid = threadIdx.x, grp = tid / LPR, piece = tid % LPR;
    const int tiles = (a.group + rows_per_tile - 1) / rows_per_tile;
    int2 item; // first wave, pieces
    int row, tile, head; // row of the tile, tile of the group, head of the batch
    if (a.cut == TR_PAGED_JOIN_BY_WAVE) {
        const int worker = blockIdx.x / a.ws_rows;
        item = *(const int2*)(a.ws_items + 2 * worker);
        row = blockIdx.x - worker * a.ws_rows;
        const int kvh = item.x / tiles; // of the batch
        tile = item.x - kvh * tiles;
        head = kvh * a.group + tile * rows_per_tile + row;
        item.x = worker;
        if (tile * rows_per_tile + row >= a.group) return;
    } else {
        head = blockIdx.x;
        const int kvh = head / a.group, in = head - kvh * a.group;
        tile = in / rows_per_tile;
        row = in - tile * rows_per_tile;
        item = *(const int2*)(a.ws_items + 2 * ((int64_t)kvh * tiles + tile));
    }
    if (item.y <= 1) return;
    float M = NOTHING, L = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int AHEAD = 1024 / THREADS < 8 ? 1024 / THREADS : 8;
    for (int p0 = grp; p0 < item.y; p0 += GROUPS * AHEAD) {
        f32x4 x[AHEAD];
        float2 ml[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int p = p0 + GROUPS * i;
            const int64_t slot = (int64_t)(2 * (item.x + p) + (p == 0)) * a.ws_rows + row;
            ml[i] = make_float2(NOTHING, 0.0f), x[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (p < item.y) {
                x[i] = *(const f32x4*)(a.ws_o + slot * D + 4 * piece);
                ml[i] = *(const float2*)(a.ws_ml + slot * 2);
            }
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, ml[i].x);
        const float old = __builtin_amdgcn_exp2f((M - top) * a.scale_log2e);
        L *= old;
        o *= old;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float f = __builtin_amdgcn_exp2f((ml[i].x - top) * a.scale_log2e);
            L = fmaf(f, ml[i].y, L);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, x[i][e], o[e]);
        }
        M = top;
    }
    os[grp][piece] = o;
    if (piece == 0) mls[grp] = make_float2(M, L);
    __syncthreads();
    if (grp != 0) return;
    float top = NOTHING, total = 0.0f;
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) top = fmaxf(top, mls[g].x);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const float f = __builtin_amdgcn_exp2f((mls[g].x - top) * a.scale_log2e);
        total = fmaf(f, mls[g].y, total);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmaf(f, os[g][piece][e], y[e]);
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const f32x4 z = y * inv;
    if constexpr (DTYPE == TR_BF16) *(bf16x4*)((__bf16*)a.out + (int64_t)head * D + 4 * piece) = __builtin_convertvector(z, bf16x4);
    else *(f32x4*)((float*)a.out + (int64_t)head * D + 4 * piece) = z;
}

template <int FMT, int D, int NT, int WORKERS> int launch_decode(const TrPagedDecodeArgs& a, int grid, hipStream_t s)
{
    // LDS for as many waves as a compute unit is meant to run: they then spread evenly over the chip
    constexpr int lds = 160 * 1024 / (WORKERS / TrChip::CUS);
    static_assert(lds >= 2 * Rows<FMT, D>::BYTES + Rows<FMT, D>::IDS + 16 * NT * Rows<FMT, D>::QROW && lds <= 64 * 1024, "");
    paged_decode_kernel<FMT, D, NT, WORKERS><<<dim3(grid), dim3(64), lds, s>>>(a);
    TR_HIP(hipGetLastError());
    if (!a.cut) return TR_OK;
    // Items have 1 + (waves / items) pieces on average.  Where there are few items, and many pieces of each, more threads read
    // them sooner; else most of a workgroup has nothing to read, and starting it is what the join costs.  The rule counts KV heads of all
    // requests, which are the items unless a KV head has more than 32 query heads; it was measured where it has not.  us with 256 / 64
    // threads: one request of 5000 rows (8 items) 12.8 / 14.5, five of 300 to 3000 (40) 13.6 / 14.3, 16 of 2000 (64) 19.9 / 20.2, 24 of up to 9000
    // (96) 24.5 / 24.1, 64 of 4096 (256) 92.7 / 92.6, 256 of 20 to 400 (1024) 26.8 / 23.7, 200 of 50 to 1200 (1600) 103.1 / 98.1.
    const dim3 rows(a.cut == TR_PAGED_JOIN_BY_WAVE ? grid * a.ws_rows : a.n_req * a.n_q_heads);
    if ((int64_t)a.n_req * a.n_kv_heads < 96) paged_join_kernel<(FMT & 1), D, 256><<<rows, dim3(256), 0, s>>>(a, 16 * NT);
    else paged_join_kernel<(FMT & 1), D, 64><<<rows, dim3(64), 0, s>>>(a, 16 * NT);
    TR_HIP(hipGetLastError());
    return TR_OK;
}
} // namespace
