// The launches of the calls over a paged cache in 8 bits with very many rows, on the CPU: this program defines the runtime's launch entry points
// itself, so the built library's launches end here and only their sizes are looked at.  A launch has fewer than 2^32 threads.
// Argument: path of libturborag_hip.so.  Exit status 0 and "paged q8 launches ok" on stdout mean every launch was legal and its
// workgroups add up.
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../../include/turborag.h"

struct Dim3 {
    uint32_t x, y, z;
};
static uint64_t blocks, launches, largest, lds;
static Dim3 next_grid, next_block;
static size_t next_lds;
extern "C" unsigned __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t bytes, void*)
{
    next_grid = grid;
    next_block = block;
    next_lds = bytes;
    return 0;
}
extern "C" int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* bytes, void** stream)
{
    *grid = next_grid;
    *block = next_block;
    *bytes = next_lds;
    *stream = nullptr;
    return 0;
}
extern "C" int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void**, size_t bytes, void*)
{
    const uint64_t n = (uint64_t)grid.x * grid.y * grid.z, threads = n * block.x * block.y * block.z;
    blocks += n;
    ++launches;
    if (threads > largest) largest = threads;
    if (bytes > lds) lds = bytes;
    return 0;
}
extern "C" int hipGetLastError(void) { return 0; }

static void check(const char* what, int rc, uint64_t want_blocks, uint64_t want_launches)
{
    if (rc != TR_OK || blocks != want_blocks || launches != want_launches || largest >= (uint64_t)1 << 32 || lds > 64 * 1024) {
        fprintf(stderr, "%s: status %d, %llu workgroups (expected %llu) in %llu launches (%llu), largest %llu threads, %llu bytes of LDS\n", what, rc,
                (unsigned long long)blocks, (unsigned long long)want_blocks, (unsigned long long)launches, (unsigned long long)want_launches,
                (unsigned long long)largest, (unsigned long long)lds);
        exit(1);
    }
    blocks = launches = largest = lds = 0;
}

int main(int, char** argv)
{
    void* lib = dlopen(argv[1], RTLD_NOW);
    if (!lib) {
        fprintf(stderr, "%s\n", dlerror());
        return 1;
    }
#define CALL(name) ((decltype(&name))dlsym(lib, #name))
    auto at = [](int i) { return (char*)0x700000000000ull + ((int64_t)i << 44); };
    tr_shape s;
    memset(&s, 0, sizeof s);
    s.n_q_heads = s.n_kv_heads = 32;
    s.head_dim = 128;
    s.rope_base = 1e4;
    s.dtype = TR_BF16;
    tr_pages_q8 p = {at(1), at(2), (uint8_t*)at(5), (uint8_t*)at(6), 16 * 32 * 128, 32 * 128, 128, 1 << 20, 16, 32, 128, 0};
    const int32_t* idx = (const int32_t*)at(3);
    auto append = [&](int32_t n, bool q, bool k) {
        const int64_t row = s.n_q_heads * 128;
        return CALL(tr_paged_append_q8)(&s, nullptr, q ? at(4) : nullptr, row, k ? at(8) : nullptr, row, k ? at(12) : nullptr, row, nullptr, nullptr, 1e-6, idx,
                                        k ? (const int32_t*)at(14) : nullptr, n, q ? at(16) : nullptr, k ? &p : nullptr, nullptr);
    };
    // windows of 1 to 16 tokens, two sides, parts of the 32 heads of two at least, at most 512 workgroups of those if windows of 16 allow
    check("append, one token", append(1, true, true), 2 * 16 + 1, 1);
    check("append, 16 tokens", append(16, false, true), 16 * 2 * 16, 1);
    check("append, 17 tokens", append(17, false, true), 9 * 2 * 16, 1);
    check("append, 300 tokens", append(300, false, true), 19 * 2 * 13, 1);
    check("append, 100000 tokens", append(100000, false, true), 6250 * 2, 1);
    check("append, queries alone, four tokens to a workgroup", append(100000, true, false), 25000, 1);
    check("append, 2^31 - 1 tokens", append(INT32_MAX, true, true), (1ull << 29) + (1ull << 27) * 2, 512);
    s.dtype = TR_F32; // workgroups of 512 threads
    s.n_q_heads = s.n_kv_heads = p.n_kv_heads = 8;
    check("append, 2^31 - 1 tokens of fp32, eight to a workgroup", append(INT32_MAX, true, true), (1ull << 28) + (1ull << 27) * 2, 512);
    s.dtype = TR_BF16;
    s.n_q_heads = s.n_kv_heads = p.n_kv_heads = 1;
    check("append, one head", append(INT32_MAX, true, true), (1ull << 28) + (1ull << 27) * 2, 512);
    auto read = [&](int32_t n_req, int32_t rows) {
        return CALL(tr_paged_read_q8)(&s, &p, idx, 100, (const int32_t*)at(31), (const int32_t*)at(32), n_req, at(34), at(36), rows, nullptr);
    };
    check("read, one row", read(1, 1), 1, 1); // a head of 128 channels: 16 units, 4 rows to a wave
    check("read, 65536 requests", read(65536, 65), 5, 1);
    check("read, 2^31 - 1 rows", read(3, INT32_MAX), 1 << 27, 9);
    s.n_q_heads = s.n_kv_heads = p.n_kv_heads = 32;
    check("read, rows of 512 units", read(3, 1000), 250, 1);
    s.n_q_heads = s.n_kv_heads = p.n_kv_heads = 1;
    auto decode = [&](int32_t n_req, int32_t max_blocks) {
        return CALL(tr_paged_decode_attn_q8)(&s, at(30), &p, idx, max_blocks, (const int32_t*)at(31), n_req, 0, 0, at(32), at(33), (size_t)1 << 40, nullptr);
    };
    check("decode, a unit each", decode(5, 4), 5, 1);
    check("decode, 65536 requests", decode(65536, 4), 1024, 1);
    check("decode, cut", decode(65536, 8), 1024 + 1024, 2);
    check("decode, one row", decode(1, 1000), 250 + 1, 2);
    s.n_q_heads = 128;
    check("decode, 128 heads to one", decode(1000, 100), 1024 + 1024 * 32, 2);
    s.head_dim = p.head_dim = 64;
    check("decode, heads of 64 channels", decode(1000, 100), 2048 + 2048 * 32, 2);
    puts("paged q8 launches ok");
    return 0;
}
