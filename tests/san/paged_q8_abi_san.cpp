// Host side of the paged cache in 8 bits under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU.
//
// Built by tests/test_paged_q8_sanitizers.py from csrc/tr_api.hip and csrc/tr_paged_api.hip (host passes instrumented) and this file, which stands in
// for the launchers of the three calls; the others stay unresolved and are never called.  Every entry point is driven with seeded random
// arguments, good and bad; "device" buffers are addresses that nothing dereferences.  The stand-ins check what a kernel relies on without
// checking it itself: shifts and strides that address the pool, counts, and workspace arrays inside the announced workspace.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../include/turborag.h"
#include "../../paper_2410_07590_amd/csrc/tr_internal.h"

namespace {
long g_launches = 0, g_checks = 0;
const char* g_ws = nullptr;
size_t g_ws_bytes = 0;
tr_shape g_shape;
tr_pages_q8 g_pages;
int64_t g_keys = 0;

#define REQUIRE(cond)                                                                         \
    do {                                                                                      \
        ++g_checks;                                                                           \
        if (!(cond)) {                                                                        \
            std::fprintf(stderr, "paged_q8_abi_san: %s:%d: %s\n", __FILE__, __LINE__, #cond); \
            std::exit(1);                                                                     \
        }                                                                                     \
    } while (0)

struct Rng {
    uint64_t s;
    explicit Rng(uint64_t seed) : s(seed * 0x9E3779B97F4A7C15ull + 1) {}
    uint32_t next() { s = s * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(s >> 33); }
    int in(int lo, int hi) { return lo + (int)(next() % (uint32_t)(hi - lo + 1)); }
    template <class T> T pick(std::initializer_list<T> l) { return l.begin()[next() % l.size()]; }
};

void pool_fits(const TrPool& p)
{
    REQUIRE(p.k == g_pages.k && p.v == g_pages.v && p.k_scale == g_pages.k_scale && p.v_scale == g_pages.v_scale);
    REQUIRE(p.n_pages == g_pages.n_pages && 1 << p.page_shift == g_pages.page_size && p.page_shift >= 4 && p.page_shift <= 10);
    REQUIRE(p.page_stride == g_pages.page_stride && p.row_stride == g_pages.row_stride && p.head_stride == g_pages.head_stride);
    REQUIRE(p.page_stride % 16 == 0 && p.row_stride % 16 == 0 && p.head_stride % 16 == 0);
    REQUIRE((uint64_t)63 * p.row_stride + 1024 < (uint64_t)1 << 32); // what a lane adds to a page
}
} // namespace

int tr_launch_paged_append_q8(const TrPagedAppendArgs& a, int dtype, int head_dim, int, hipStream_t)
{
    ++g_launches;
    REQUIRE(a.n_tokens > 0 && (a.n_q_heads > 0 || a.n_kv_heads > 0));
    REQUIRE((a.q != nullptr) == (a.n_q_heads > 0) && (a.q_out != nullptr) == (a.n_q_heads > 0) && (a.k != nullptr) == (a.n_kv_heads > 0));
    REQUIRE(a.rotary_dim % 16 == 0 && a.rotary_dim >= 0 && a.rotary_dim <= head_dim && (a.rotary_dim == 0 || a.pos));
    REQUIRE(a.n_kv_heads == 0 || a.slots);
    const int lanes = head_dim * (dtype == TR_F32 ? 4 : 2) / 16;
    REQUIRE(a.tile_shift >= 0 && 1 << a.tile_shift <= TR_PAGED_APPEND_TOKENS && 256 / lanes >> a.tile_shift >= 1);
    REQUIRE(a.eps > 0.0f && a.q_stride % 16 == 0 && a.k_stride % 16 == 0 && a.v_stride % 16 == 0);
    if (a.n_kv_heads) pool_fits(a.pool);
    return TR_OK;
}

int tr_launch_paged_read_q8(const TrPagedReadArgs& a, int, int, hipStream_t)
{
    ++g_launches;
    pool_fits(a.pool);
    REQUIRE(a.n_rows > 0 && a.n_req > 0 && a.n_req <= 65536 && a.max_blocks > 0 && a.n_kv_heads == g_shape.n_kv_heads);
    REQUIRE((int64_t)a.max_blocks << a.pool.page_shift <= 1 << 30);
    REQUIRE(a.table && a.kv_lens && a.row_start && a.out_k && a.out_v);
    return TR_OK;
}

int tr_launch_paged_decode_q8(const TrPagedDecodeArgs& a, int, int head_dim, int grid, hipStream_t)
{
    ++g_launches;
    pool_fits(a.pool);
    const int rows = std::min(a.group, tr_paged_tile_rows(a.group)), tiles = (a.group + tr_paged_tile_rows(a.group) - 1) / tr_paged_tile_rows(a.group);
    const int64_t items = (int64_t)a.n_req * a.n_kv_heads * tiles, unit = TR_Q8_UNIT, units = std::max<int64_t>((g_keys + unit - 1) / unit, 1);
    const int workers = tr_q8_workers(head_dim);
    REQUIRE(a.ws_rows == rows && a.group == g_shape.n_q_heads / g_shape.n_kv_heads);
    REQUIRE(grid >= 1 && grid <= workers && (grid == workers || grid >= items * units)); // every unit has a wave
    REQUIRE(items * units + workers < INT32_MAX);                                         // the kernel counts them in 32 bits
    REQUIRE((a.cut != 0) == (units > 1));
    if (!a.cut) return TR_OK;
    const char* end = g_ws + g_ws_bytes;
    const int64_t pieces = 2ll * workers * rows, records = a.cut == TR_PAGED_JOIN_BY_WAVE ? grid : items;
    const char *o = (const char*)a.ws_o, *ml = (const char*)a.ws_ml, *it = (const char*)a.ws_items;
    REQUIRE(o >= g_ws && o + pieces * head_dim * 4 <= ml && ml + pieces * 8 <= it && it + records * 8 <= end);
    REQUIRE((uintptr_t)o % 16 == 0 && (uintptr_t)ml % 8 == 0 && (uintptr_t)it % 8 == 0);
    REQUIRE((a.cut == TR_PAGED_JOIN_BY_WAVE ? (int64_t)grid * rows : (int64_t)a.n_req * a.n_q_heads) <= TR_MAX_BLOCKS_256);
    return TR_OK;
}

int main(int argc, char** argv)
{
    const int mixes = argc > 1 ? atoi(argv[1]) : 100;
    char* const base = (char*)0x700000000000ull;
    auto at = [&](int i) { return base + ((int64_t)i << 36); };
    long ok = 0, refused = 0;
    for (int mix = 0; mix < mixes; ++mix) {
        Rng r(mix);
        memset(&g_shape, 0, sizeof g_shape);
        g_shape.n_kv_heads = r.in(1, 9);
        g_shape.n_q_heads = g_shape.n_kv_heads * r.pick({1, 2, 7, 8, 16, 17, 32, 40, 128, 129});
        g_shape.head_dim = r.pick({64, 128, 128, 96});
        g_shape.dtype = r.pick({TR_F32, TR_BF16, TR_BF16});
        g_shape.rope_base = 1e4;
        memset(&g_pages, 0, sizeof g_pages);
        g_pages.k = at(1);
        g_pages.v = at(2);
        g_pages.k_scale = (uint8_t*)at(3) + r.in(0, 3);
        g_pages.v_scale = (uint8_t*)at(r.in(0, 19) ? 900 : 3);
        g_pages.n_pages = r.pick({1, 2, 100, 1 << 20, 1 << 28});
        g_pages.page_size = r.pick({16, 32, 64, 256, 1024, 8, 48});
        g_pages.n_kv_heads = g_shape.n_kv_heads;
        g_pages.head_dim = g_shape.head_dim;
        const int64_t d = g_shape.head_dim, hk = g_shape.n_kv_heads;
        if (r.in(0, 1)) g_pages.row_stride = hk * d, g_pages.head_stride = d, g_pages.page_stride = hk * d * g_pages.page_size;
        else g_pages.row_stride = d, g_pages.head_stride = d * g_pages.page_size, g_pages.page_stride = hk * d * g_pages.page_size * r.in(1, 2);
        if (r.in(0, 19) == 0) g_pages.row_stride = (int64_t)r.next() << r.in(0, 32);
        if (r.in(0, 19) == 0) g_pages.page_stride = (int64_t)r.next() << r.in(0, 33);

        const int n = r.pick({0, 1, 5, 1000, 1 << 20, INT32_MAX});
        const int64_t e = g_shape.dtype == TR_F32 ? 4 : 2, qrow = g_shape.n_q_heads * d, krow = hk * d;
        const bool q = r.in(0, 3), k = r.in(0, 3), packed = r.in(0, 1);
        const int64_t row = qrow + 2 * krow;
        char* const x = at(1004);
        const char *kx = packed ? x + qrow * e : at(1200), *vx = packed ? x + (qrow + krow) * e : at(1400);
        int rc = tr_paged_append_q8(&g_shape, nullptr, q ? x : nullptr, packed ? row : qrow, k ? kx : nullptr, packed ? row : krow, k ? vx : nullptr,
                                    packed ? row : krow, r.in(0, 1) ? at(1600) : nullptr, r.in(0, 1) ? at(1601) : nullptr, 1e-6, (const int32_t*)at(1602),
                                    k ? (const int32_t*)at(1603) : nullptr, n, q ? at(1610) : nullptr, k ? &g_pages : nullptr, nullptr);
        ++(rc == TR_OK ? ok : refused);

        const int req = r.pick({0, 1, 3, 64, 4096, 65536, 65537}), blocks = r.pick({0, 1, 7, 1000, 8192, 1 << 20, 1 << 27});
        rc = tr_paged_read_q8(&g_shape, &g_pages, (const int32_t*)at(1900), blocks, (const int32_t*)at(1901), (const int32_t*)at(1902), req, at(1910), at(2300),
                              r.pick({0, 1, 1000, 1 << 20}), nullptr);
        ++(rc == TR_OK ? ok : refused);

        g_keys = (int64_t)blocks * g_pages.page_size;
        g_ws = at(1800);
        g_ws_bytes = tr_paged_decode_attn_q8_workspace_size(&g_shape, req, blocks, g_pages.page_size);
        auto decode = [&](const char* ws, size_t bytes) {
            return tr_paged_decode_attn_q8(&g_shape, at(1810), &g_pages, (const int32_t*)at(1900), blocks, (const int32_t*)at(1901), req, r.pick({0, 1, INT32_MAX}),
                                           r.pick({0, 4, INT32_MAX}), at(1910), (void*)ws, bytes, nullptr);
        };
        rc = decode(g_ws, g_ws_bytes);
        ++(rc == TR_OK ? ok : refused);
        if (g_ws_bytes && rc == TR_OK) {
            REQUIRE(decode(g_ws, g_ws_bytes - 1) == TR_ERR_WORKSPACE);
            REQUIRE(decode(g_ws + 128, g_ws_bytes) == TR_ERR_WORKSPACE);
            REQUIRE(decode(nullptr, g_ws_bytes) == TR_ERR_WORKSPACE);
        }
    }
    REQUIRE(g_launches > mixes / 2 && refused > mixes / 4);
    std::printf("paged q8 abi sanitizer run ok: %d mixes, %ld calls accepted, %ld refused, %ld launches, %ld checks\n", mixes, ok, refused, g_launches, g_checks);
    return 0;
}
