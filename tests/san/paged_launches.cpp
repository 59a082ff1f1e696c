// The launches of the paged cache's calls with very many rows, on the CPU: this program defines the runtime's launch entry points
// itself, so the built library's launches end here and only their sizes are looked at.  A launch has fewer than 2^32 threads.
// Argument: path of libturborag_hip.so.  Exit status 0 and "paged launches ok" on stdout mean every launch was legal and its
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
    tr_pages p = {at(1), at(2), 16 * 32 * 128, 32 * 128, 128, 1 << 20, 16, 32, 128, TR_BF16, 0};
    const int32_t* idx = (const int32_t*)at(3);
    auto append = [&](int32_t n) {
        return CALL(tr_paged_append)(&s, nullptr, at(4), 4096, at(8), 4096, at(12), 4096, nullptr, nullptr, 1e-6, idx, (const int32_t*)at(14), n, at(16), &p, nullptr);
    };
    check("append, one token", append(1), 1, 1);
    check("append, a token to a workgroup: 96 heads", append(100000), 100000, 1);
    check("append, 2^31 - 1 tokens", append(INT32_MAX), (uint64_t)INT32_MAX, 129);
    s.n_q_heads = s.n_kv_heads = p.n_kv_heads = 1;
    check("append, 8 tokens to a workgroup", append(INT32_MAX), ((uint64_t)INT32_MAX + 7) / 8, 17);
    check("append, few tokens", append(2047), 2047, 1);
    int32_t* const o[] = {(int32_t*)at(20), (int32_t*)at(21), (int32_t*)at(22), (int32_t*)at(23), (int32_t*)at(24), (int32_t*)at(25)};
    auto map = [&](int32_t n_req, int32_t slots) {
        return CALL(tr_page_map)(idx, idx, nullptr, n_req, 16, idx, 0, o[0], 100, o[1], o[2], o[3], o[4], slots, o[5], nullptr);
    };
    check("map, no slots", map(4096, 0), 1, 1);
    check("map, 2^31 - 1 slots", map(3, INT32_MAX), 1 << 21, 1);
    auto decode = [&](int32_t n_req, int32_t max_blocks) {
        return CALL(tr_paged_decode_attn)(&s, at(30), &p, idx, max_blocks, (const int32_t*)at(31), n_req, 0, 0, at(32), at(33), (size_t)1 << 40, nullptr);
    };
    check("decode, a unit each", decode(5, 2), 5, 1);
    check("decode, 65536 requests", decode(65536, 2), 1024, 1);
    check("decode, cut", decode(65536, 8), 1024 + 1024, 2);
    check("decode, one row", decode(1, 1000), 500 + 1, 2);
    s.n_q_heads = 128;
    check("decode, 128 heads to one", decode(1000, 100), 1024 + 1024 * 32, 2);
    puts("paged launches ok");
    return 0;
}
